// Adapter gradients of the layer, x as bf16 rows or as an 8-bit checkpoint:
//     u = s x.A^T,  v = s dy.B   (per token, with the token's adapter)        dA_s += v^T x,   dB_s += dy^T u
// Two launches, each over x and dy side by side.
//
// rows_shrink_kernel: u and v.  An item is a piece (up to 128 rows of one segment, counted from the segment's first row: a TMA box
// may begin at any row, so no row of another segment is in it but behind its end) of x or of dy, its work the steps of 128 columns.
// rows_grad_kernel: dA and dB.  An item is (slot, 128 columns of x or dy), its work the slot's pieces.
// A step of either is a tile of 128 rows x 128 columns, which goes through the rings in two halves along what is contracted: 64 columns in the
// first pass, 64 rows in the second: a stage's way through loading, conversion and product takes about as long whatever its size, so
// what counts is how many there are (beside 64 ranks eight and five; with the 8 bits in a place of their own six and four, and 5 % more time
// for 8192 x 11008 in E4M3 and 4096).
// In both the work of all items stands in one line that is cut into equal parts, one per SM; a CTA walks its part without a pause
// between items.  An item that the cuts divide is joined in device memory: every CTA writes its partial result, and the last one to
// arrive adds them in the order of the parts, so the bits do not depend on who that is.  (A form with a cluster per item and an
// exchange through distributed shared memory spent 10 us per CTA on setting up and joining.)
//
// Both are rings of tiles of x or dy as TMA brings them in, multiplied by tcgen05 into one of two accumulators.  Roles: two producers, of
// tiles and of the other operand (one thread for both is the slowest role: a copy costs it a few hundred cycles), the
// first of which tells the others what a stage holds; an issuer; four warps that finish items while the next one is multiplied;
// groups of warps that take 8-bit tiles in turn through their registers and write them back in place as bf16 (exact: the
// scales are powers of two) in the swizzled order of the tensor cores.  The second product contracts over tokens: the tile
// [token][64 columns] is an operand whose contiguous index is the output's (M-major), which the descriptor says; nothing is
// transposed.
//
// dA and dB are fp32 and so are u and v on the way: each goes into the second product as three bf16 values whose sum is the fp32
// value, side by side as 3r columns of one product.  One bf16 value would leave 2^-9, 1e-3 of every gradient, two 3e-6.
//
// x and dy leave HBM once (the second pass finds them in L2 up to about 100 MB), but memory is not what bounds it: 8192 x 11008 in E4M3 and 4096,
// eight adapters of 8 to 64 ranks, take 138 us where the bytes take 28, and nothing is saturated (tensor pipe 5 and 12 %, DRAM 28 %, half of the issue
// slots).  A CTA has about 110 half steps in either pass, some 1100 and 1250 cycles each.  A stage takes 4000 to 6000 from empty to empty.  With five
// of them that is what bounds the second pass; the first has eight, for which half steps of 750 would do: what holds it up has not been found.
// (Without the conversion the call takes 12 % less, without the tiles' loads 5 %, without the other operand 1 %.)  Small calls (100 tokens of one
// adapter 16 us) are made of a dozen latencies in a row.
#include <cstring>

#include "lml_ptx_sm100.cuh"
#include "lml_rows_grad.cuh"

namespace lml {

using namespace ptx;

constexpr int kRgGroups = 4, kRgGroup = 4;      // converting groups, warps of each (8192 tokens, below: 138 us; two of eight 143, one of sixteen 208, eight of two 161)
constexpr int kRgFinish = 4;                    // warps that finish items (warps 2 ... 5: one per quarter of the accumulator's lanes)
constexpr int kRgOther = 2 + kRgFinish;         // the warp that brings in the other operand
constexpr int kRgFirstConv = kRgOther + 1;
constexpr int kRgThreads = 32 * (kRgFirstConv + kRgGroups * kRgGroup);
constexpr int kRgSegs = 320;                    // segments of a launch; a call of more runs in slices
constexpr int kRgTile = 128 * 64 * 2;           // bytes of half a step as it is multiplied: [row][64 columns], or two times [64 rows][64 columns]
constexpr int kRgHalfTile = kRgTile / 2;
constexpr int kRgRaw = 128 * 64;                // ... of the 8 bits that it is made of, [128][64] or [64][128]
constexpr int kRgPiece = 2 * 3 * kRankPad * 128;   // u (or v) of a piece: [64 tokens each][three parts][column][64]
constexpr int kRgPartial = kRankPad * 128;      // floats of a partial result
constexpr int kRgMaxStages = 12;
constexpr int kRgTurns = 16;                    // tiles on their way to and from the converting warps: as many as stages, and an end for each group
static_assert(kRgTurns >= kRgMaxStages + kRgGroups && (kRgTurns & (kRgTurns - 1)) == 0, "a turn's place must have been read before it is used again");
constexpr int kRgChunk = 8;                     // half steps that one accumulator takes; see issue_steps
constexpr int kRgLeast = 2;                     // steps of a CTA's part (of a whole pass, if it has fewer); 100 tokens of 4096 x 4096: 16.1 us, four 17.1

struct alignas(64) RowsGradParams {
    CUtensorMap map[2][2];    // x, dy; first pass: boxes of 64 columns x 128 rows; second: 64 (8-bit x: 128) x 64
    CUtensorMap low[2][kRankPad / kChunk];   // the packed A of the table, B^T of the transposed one: boxes of 64 columns x 16, 32, 48, 64 rows
    SlotSnapshot snap[2];     // table, transposed table
    const uint32_t* scales;   // of x
    const int32_t *seg_offsets, *ids, *ids_T;   // of this slice
    const int* bad;           // or null: not 0 if the arrays of the call do not hold together (calls of several slices)
    uint32_t* status[2];
    uint8_t* pieces[2];       // u, v
    float* partial;           // [CTA][2]: of the item that its part begins in, of the item that its part ends in
    // [CTA], of each pass: of the item that its part ends in and the next one goes on with.  The last to arrive sets it back to 0, so that a call cut
    // off between its launches leaves nothing; and each pass clears the other's, so that calls that overlapped leave nothing to a third.
    unsigned* arrived[2];
    float* out[2];            // dA, dB
    int d[2], tiles[2];       // d_in, d_out; in tiles of 128 columns
    int T, G, num_sms, r16, ring, accumulate, all_tiles, whole_items;
    int check_first, check_last;   // the slice begins, ends the call
    unsigned long long live;  // slots with an adapter
};

// What the producer says about a stage.
constexpr int kRgLast = 1, kRgEnd = 2, kRgTouched = 4;   // last of an item; last of this CTA; goes through the converting warps
struct RgInfo {
    int flags, valid;   // rows
    int r16;            // columns of the other operand (second pass: of each of its three parts)
};
// ... to the converting warps, in 16 bytes.
struct alignas(16) RgTurn {
    int where;                // stage, 256 if its phase is 1, 512 if it is the right half of 128 columns; less than 0: no more
    int valid;                // rows
    const uint32_t* words;    // of an 8-bit tile: its rows' scale words; null: only rows behind the last are cleared
};

// An item that this CTA is to join: all of its threads do, when its part of the line is done.  (Four finishing warps on their own, with two or four
// loads in flight, took up to 9 us.)
struct RgJoin { int job, slot, first, last, at, valid; };   // at: piece (first pass), column (second)

struct RgCtrl {
    unsigned long long full[kRgMaxStages], low_full[kRgMaxStages], empty[kRgMaxStages], turn[kRgTurns], made[kRgTurns], acc_full[2], acc_free[2];
    RgInfo info[kRgMaxStages];
    RgTurn turns[kRgTurns];
    uint32_t used_half[2];   // slots in use
    __device__ unsigned long long used() const { return (unsigned long long)used_half[1] << 32 | used_half[0]; }
    uint32_t tmem_base;
    RgJoin joins[2];   // (a part has at most two items that are not whole)
    int n_joins;
    int abort, count[kRgSegs / 32], units[kMaxSlots], entry[kMaxSlots];
    int first[kRgSegs], len[kRgSegs], piece[kRgSegs], pre[kRgSegs + 1];
    uint8_t slot[2][kRgSegs];
    float4 turned[kRgFinish][32][5];
};

__device__ __forceinline__ uint64_t umma_desc_m128(uint32_t smem_addr)   // 64 contiguous M per 128-byte swizzled row, rows along K
{
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(kRgHalfTile >> 4) << 16;             // to the next 64 of M
    d |= (uint64_t)(1024 >> 4) << 32;                    // to the next 8 of K
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
constexpr uint32_t kIdescMMajorA = 1u << 15;

// 8 columns of 32 lanes
__device__ __forceinline__ void tmem_ld_32x8(uint32_t taddr, uint32_t (&r)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_32x8(uint32_t taddr, const float (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                 :: "r"(__float_as_uint(r[0])), "r"(__float_as_uint(r[1])), "r"(__float_as_uint(r[2])), "r"(__float_as_uint(r[3])),
                    "r"(__float_as_uint(r[4])), "r"(__float_as_uint(r[5])), "r"(__float_as_uint(r[6])), "r"(__float_as_uint(r[7])), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Eight columns of a chunk's accumulator (PARTS: the sums of three that stand r16 apart), plus, if `more`, of the sum of the chunks before at
// `sum`.  By a whole warp.
template <int PARTS>
__device__ __forceinline__ void chunk_sums(uint32_t from, uint32_t r16, uint32_t sum, bool more, float (&s)[8])
{
    uint32_t h[8], m[8], l[8], before[8];
    tmem_ld_32x8(from, h);
    if (PARTS == 3) {
        tmem_ld_32x8(from + r16, m);
        tmem_ld_32x8(from + 2 * r16, l);
    }
    if (more) tmem_ld_32x8(sum, before);
    tmem_ld_wait();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        s[e] = __uint_as_float(h[e]);
        if (PARTS == 3) {
            // A token's Inf times the lower parts may be NaN (they are zero as often as not) or an Inf of the other sign: the first part says it all.
            // (100 tokens: 15.7 -> 16.0 us.  A look at all eight for NaN instead, with what follows apart, spills: 16.3.)
            const float sum = s[e] + (__uint_as_float(m[e]) + __uint_as_float(l[e]));
            s[e] = fabsf(s[e]) < INFINITY ? sum : s[e];
        }
        if (more) s[e] += __uint_as_float(before[e]);
    }
}
// The chunks of an item but its last: waits for each in turn and adds it up at `sum`.  chunk: counted through the items of this CTA.
template <int PARTS>
__device__ __forceinline__ void sum_chunks(RgCtrl* c, uint32_t tmem, uint32_t acc_cols, uint32_t r16, uint32_t sum, int n, uint32_t& chunk, int lane, volatile int* abort)
{
    for (int k = 0; k + 1 < n; ++k, ++chunk) {
        mbar_wait_warp(smem_u32(&c->acc_full[chunk & 1]), (chunk >> 1) & 1, abort);
        __syncwarp();
        tc_fence_after();
#pragma unroll 1
        for (uint32_t j = 0; j < r16; j += 8) {
            float s[8];
            chunk_sums<PARTS>(tmem + (chunk & 1) * acc_cols + j, r16, sum + j, k > 0, s);
            tmem_st_32x8(sum + j, s);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&c->acc_free[chunk & 1]));
    }
    mbar_wait_warp(smem_u32(&c->acc_full[chunk & 1]), (chunk >> 1) & 1, abort);
    __syncwarp();
    tc_fence_after();
}
__device__ __forceinline__ uint4 ld_smem_v4(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void st_smem_v4(uint32_t a, const uint4& v)
{
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ float4 ld_cg_v4(const float* p)   // (written by another CTA of this grid)
{
    float4 v;
    asm volatile("ld.global.cg.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void finish_barrier() { asm volatile("bar.sync 1, %0;" ::"n"(32 * kRgFinish) : "memory"); }
// Of a converting group; whether any thread says so.
__device__ __forceinline__ bool group_any(int group, bool v)
{
    int r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %1, 0;\n\tbar.red.or.pred q, %2, %3, p;\n\tselp.s32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"(v ? 1 : 0), "r"(2 + group), "n"(32 * kRgGroup) : "memory");
    return r != 0;
}

// Whether a segment's two bindings name one adapter in both tables.
__device__ __forceinline__ bool paired(const RowsGradParams& p, int s, int sT)
{
    const int r = slot_rank(p.snap[0], s);
    return r > 0 && r == slot_rank(p.snap[1], sT);
}

__device__ __forceinline__ void rg_setup(RgCtrl* c, int warp, int tid, uint32_t cols)
{
    if (tid == 0) {
        c->abort = 0;
        c->n_joins = 0;
        c->used_half[0] = c->used_half[1] = 0u;
        for (int i = 0; i < kRgMaxStages; ++i) {
            mbar_init(smem_u32(&c->full[i]), 1);
            mbar_init(smem_u32(&c->low_full[i]), 1);
            mbar_init(smem_u32(&c->empty[i]), 1);
        }
        for (int i = 0; i < kRgTurns; ++i) {
            mbar_init(smem_u32(&c->turn[i]), 1);
            mbar_init(smem_u32(&c->made[i]), kRgGroup);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&c->acc_full[i]), 1);
            mbar_init(smem_u32(&c->acc_free[i]), kRgFinish);
        }
        fence_mbar_init();
    }
    if (warp == 1) tmem_alloc(smem_u32(&c->tmem_base), cols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
}
__device__ __forceinline__ uint32_t tmem_cols_for(int n) { return n <= 32 ? 32u : n <= 64 ? 64u : n <= 128 ? 128u : n <= 256 ? 256u : 512u; }

// The ring of a CTA: stages of a tile beside the other operand (of the widest adapter).  A tile's 8 bits come into its second half.  Every role walks
// it with a cursor of its own (a division per step to find the stage costs as much as the step's products).
struct RgRing {
    uint32_t base, stage_bytes;
    int stages;
    __device__ RgRing(uint32_t at, int bytes, uint32_t low) : base(at), stage_bytes(kRgTile + low), stages(min(bytes / (int)(kRgTile + low), kRgMaxStages)) {}
};
struct RgCursor {
    const RgRing& ring;
    int i = 0, stage = 0, turn = 0;   // turn: tiles that the converting warps have had to do with
    uint32_t phase = 0, at;           // of the stage's barriers; its address
    __device__ explicit RgCursor(const RgRing& r) : ring(r), at(r.base) {}
    __device__ void advance()
    {
        ++i;
        at += ring.stage_bytes;
        if (++stage == ring.stages) { stage = 0; phase ^= 1u; at = ring.base; }
    }
};
__device__ __forceinline__ uint32_t turn_phase(int turn) { return (uint32_t)(turn / kRgTurns) & 1u; }

// Producer of tiles (one thread): hands a stage on to the converting warps; stage -1: there is no more.
__device__ __forceinline__ void post_turn(RgCtrl* c, int turn, const RgTurn& what)
{
    c->turns[turn % kRgTurns] = what;
    mbar_arrive(smem_u32(&c->turn[turn % kRgTurns]));   // (releases what was written)
}
// ... the half step at (row, column) into the stage.
template <bool SECOND>
__device__ __forceinline__ void load_tile(RgCtrl* c, const CUtensorMap* map, uint32_t at, int stage, bool raw, int row, int column)
{
    const uint32_t bar = smem_u32(&c->full[stage]);
    mbar_arrive_expect_tx(bar, raw ? kRgRaw : kRgTile);
    tma_load_2d(raw ? at + (kRgTile - kRgRaw) : at, map, bar, raw ? column / 2 : column, row);   // (8-bit columns in pairs)
    if (SECOND && !raw) tma_load_2d(at + kRgHalfTile, map, bar, column + 64, row);
}

// Issuer of both passes: the steps as they come, told apart by what the producer says about them.  The tensor cores cut off what an addition to
// an accumulator loses, always towards zero, so an item's sum goes through the accumulators in chunks of kRgChunk half steps, 32 additions, and
// the finishing warps add those up, rounded, beside them in TMEM.  (Relative errors of dA and dB, 8192 x 11008 and 4096: 5.6e-7; 4.5e-6 in one go, 1.1e-6 with
// twice as long chunks, which take the same time.)  The tile's rows are the product's (first
// pass: K-major) or contracted (second: M-major).
template <bool SECOND>
__device__ __forceinline__ void issue_steps(RgCtrl* c, const RgRing& ring, uint32_t tmem, uint32_t acc_cols, volatile int* abort)   // (one thread)
{
    RgCursor u(ring);
    uint32_t chunks = 0;   // begun
    int flags, in_chunk = 0;
    do {
        if (!mbar_wait(smem_u32(&c->full[u.stage]), u.phase, abort)) return;
        const RgInfo info = c->info[u.stage];
        flags = info.flags;
        const uint32_t buf = chunks & 1u, acc = tmem + buf * acc_cols, fresh = in_chunk == 0 ? 0u : 1u;
        if (!fresh && chunks >= 2 && !mbar_wait(smem_u32(&c->acc_free[buf]), ((chunks >> 1) & 1u) ^ 1u, abort)) return;
        if (flags & kRgTouched) {
            if (!mbar_wait(smem_u32(&c->made[u.turn % kRgTurns]), turn_phase(u.turn), abort)) return;
            ++u.turn;
        }
        if (!mbar_wait(smem_u32(&c->low_full[u.stage]), u.phase, abort)) return;
        tc_fence_after();
        const uint32_t low = u.at + kRgTile;
        const uint64_t bd = umma_desc_k128(low);
        if (SECOND) {
            const uint32_t idesc = umma_idesc_bf16(128, 3 * info.r16) | kIdescMMajorA;
            const uint64_t ad = umma_desc_m128(u.at);
            if (info.valid > 48) {
#pragma unroll
                for (int k = 0; k < 4; ++k) umma_bf16(acc, ad + (uint64_t)(k * (2048 >> 4)), bd + (uint64_t)(k * 2), idesc, k > 0 ? 1u : fresh);
            } else {
                for (int k = 0; k * 16 < info.valid; ++k) umma_bf16(acc, ad + (uint64_t)(k * (2048 >> 4)), bd + (uint64_t)(k * 2), idesc, k > 0 ? 1u : fresh);
            }
        } else {
            const uint32_t idesc = umma_idesc_bf16(128, info.r16);
            const uint64_t ad = umma_desc_k128(u.at);
#pragma unroll
            for (int k = 0; k < 4; ++k) umma_bf16(acc, ad + (uint64_t)(k * 2), bd + (uint64_t)(k * 2), idesc, k > 0 ? 1u : fresh);
        }
        umma_commit(smem_u32(&c->empty[u.stage]));
        if (++in_chunk == kRgChunk || (flags & kRgLast)) {
            umma_commit(smem_u32(&c->acc_full[buf]));
            ++chunks;
            in_chunk = 0;
        }
        u.advance();
    } while (!(flags & kRgEnd));
}

// mbar_wait_warp where the barrier has turned as a rule: the lanes look for themselves first (one of them for all: 151 us for 145).
__device__ __forceinline__ bool mbar_look_warp(uint32_t bar, uint32_t parity, volatile int* abort)
{
    return __all_sync(0xffffffffu, mbar_test_wait(bar, parity)) || mbar_wait_warp(bar, parity, abort);
}

// Converting group of both passes: the half steps that are handed on, in turn.  In the second pass rows behind the last become zeros (in a bf16
// tile those that share a step of 16 with it: another token's values times zero would be NaN where they are not finite).
template <bool E4M3, bool SECOND>
__device__ __forceinline__ void convert_tiles(RgCtrl* c, const RgRing& ring, int group, int wt, int lane, volatile int* abort)
{
    // A thread has 16 values of a row (8-bit: four or eight such to a row) in each of kParts rows, kRows apart, where the swizzle is the same: the
    // 16-byte chunks 2 ch and 2 ch + 1 (of eight) of a row.  In the second pass lanes of the right 64 columns write the odd chunk first, so that
    // the two sides' lanes, which are 8 KB apart, do not meet on a bank.
    constexpr int kRows = (SECOND ? 4 : 8) * kRgGroup, kParts = (SECOND ? 64 : 128) / kRows;
    const int ch = wt & 3, odd = SECOND ? (wt >> 2) & 1 : 0, row0 = SECOND ? wt >> 3 : wt >> 2;
    const uint32_t to0 = (uint32_t)(odd * kRgHalfTile + row0 * 128 + (((2 * ch + odd) ^ (row0 & 7)) * 16));
    // The scale words come straight from memory, and for the tile after this one as soon as it has been handed on, so that they are there with
    // it as a rule.  (Copied into the stage by a producer of their own, 1000 tokens took 36.2 us for 34.8; asked for behind the conversion
    // instead of before it, 8192 take 179 for 144.)
    int where = 0, valid = 0;
    bool raw = false;
    uint32_t word[kParts];
    const auto take = [&](int turn) {
        const uint4 w = ld_smem_v4(smem_u32(&c->turns[turn % kRgTurns]));
        where = (int)w.x;
        valid = (int)w.y;
        const uint32_t* words = reinterpret_cast<const uint32_t*>((uintptr_t)w.w << 32 | w.z);
        raw = words != nullptr;
#pragma unroll
        for (int q = 0; q < kParts; ++q) word[q] = raw && row0 + kRows * q < valid ? ld_after_wait(words + row0 + kRows * q) : 0u;
    };
    bool taken = false;
    for (int turn = group;; turn += kRgGroups) {
        const int k = turn % kRgTurns;
        bool ok = true;
        if (!taken) {
            ok = mbar_look_warp(smem_u32(&c->turn[k]), turn_phase(turn), abort);
            __syncwarp();
            take(turn);
        }
        ok = ok && where >= 0;
        const int stage = where & 255, rows_there = valid;
        const bool kept = raw;
        ok = ok && mbar_look_warp(smem_u32(&c->full[where < 0 ? 0 : stage]), (uint32_t)(where >> 8) & 1u, abort);
        __syncwarp();
        const uint32_t at = ring.base + (where < 0 ? 0u : (uint32_t)stage * ring.stage_bytes);
        const int shift = 8 * (SECOND ? (wt & 7) >> 1 : (ch >> 1) + (where >> 8 & 2));
        uint2 v[kParts][2];
        uint32_t byte[kParts], most = 0;
#pragma unroll
        for (int q = 0; q < kParts; ++q) {
            const uint4 w = ld_smem_v4(at + (uint32_t)(kRgTile - kRgRaw + q * (kRgRaw / kParts) + wt * 16));
            v[q][0] = odd ? make_uint2(w.z, w.w) : make_uint2(w.x, w.y);
            v[q][1] = odd ? make_uint2(w.x, w.y) : make_uint2(w.z, w.w);
            byte[q] = (word[q] >> shift) & 0xffu;
            most = max(most, byte[q]);
        }
        const bool usual = (!SECOND || rows_there == 64) && most <= Decoder<E4M3>::kMost;
        if (group_any(group, !ok)) return;   // (everybody has the tile's values, so their place may be written; or there is no more, or a wait gave up)
        taken = __all_sync(0xffffffffu, mbar_test_wait(smem_u32(&c->turn[(turn + kRgGroups) % kRgTurns]), turn_phase(turn + kRgGroups)));
        if (taken) take(turn + kRgGroups);
        const uint32_t to = at + to0;
        if (kept && usual) {
#pragma unroll
            for (int q = 0; q < kParts; ++q) {
                const Decoder<E4M3> decode(byte[q]);
                st_smem_v4(to + (uint32_t)(q * kRows * 128), decode.eight(v[q][0]));
                st_smem_v4((to ^ 16u) + (uint32_t)(q * kRows * 128), decode.eight(v[q][1]));
            }
        } else if (kept) {
#pragma unroll 1
            for (int q = 0; q < kParts; ++q) {
                const bool there = !SECOND || row0 + kRows * q < rows_there;
                const uint4 zero = make_uint4(0, 0, 0, 0);
                st_smem_v4(to + (uint32_t)(q * kRows * 128), there ? decode8<E4M3>(v[0][0], byte[0]) : zero);
                st_smem_v4((to ^ 16u) + (uint32_t)(q * kRows * 128), there ? decode8<E4M3>(v[0][1], byte[0]) : zero);
#pragma unroll
                for (int i = 0; i + 1 < kParts; ++i) { v[i][0] = v[i + 1][0]; v[i][1] = v[i + 1][1]; byte[i] = byte[i + 1]; }
            }
        } else if (SECOND) {
            const int rows = 16 - (rows_there & 15);
            for (int e = wt; e < rows * 16; e += 32 * kRgGroup) {
                const int row = rows_there + (e >> 4);
                st_smem_v4(at + ((e >> 3) & 1) * kRgHalfTile + row * 128 + (e & 7) * 16, make_uint4(0, 0, 0, 0));
            }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&c->made[k]));
    }
}

// The line of work: W steps, P parts; part k begins at W k / P.  (W: 32 KB of activations each, so 31 bits are enough.)
struct RgLine {
    int W, P;
    __device__ RgLine(int w) : W(w), P(max(1, min((int)gridDim.x, w / kRgLeast))) {}
    __device__ int begin(int k) const { return k < P ? (int)((long long)W * k / P) : W; }
    __device__ int part_of(int w) const { return (int)(((long long)(w + 1) * P - 1) / W); }   // the last part that begins at or before w
};
// An item that several parts share: its first and last part, and where this one leaves its result.
struct RgShare { int first, last, slot; };
__device__ __forceinline__ RgShare share_of(const RgLine& line, int item, int n, int k)
{
    const int first = line.part_of(item);
    return {first, line.part_of(item + n - 1), k == first ? 1 : 0};   // (the others begin behind the item's first step)
}
// After all finishing warps have written this CTA's partial result: if it is the last one of the item's, the CTA joins them later.
__device__ __forceinline__ void arrive(RgCtrl* c, unsigned* arrived, const RgShare& s, int job, int slot, int at, int valid)
{
    __threadfence();
    finish_barrier();
    if (threadIdx.x == 64) {   // (the first of them)
        const unsigned others = (unsigned)(s.last - s.first);
        if (atomicInc(arrived + s.first, others) == others) c->joins[c->n_joins++] = {job, slot, s.first, s.last, at, valid};
        __threadfence();
    }
}
// Four values of the joined result, the parts added in their order, eight of them in flight.
__device__ __forceinline__ float4 joined(const RowsGradParams& p, const RgJoin& s, int at)
{
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k0 = s.first; k0 <= s.last; k0 += 8) {
        float4 w[8];
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (k0 + q <= s.last) w[q] = ld_cg_v4(p.partial + (size_t)(2 * (k0 + q) + (k0 + q == s.first ? 1 : 0)) * kRgPartial + at);
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (k0 + q <= s.last) { v.x += w[q].x; v.y += w[q].y; v.z += w[q].z; v.w += w[q].w; }
    }
    return v;
}

// A segment of the slice, this thread's.  Returns whether the slice's arrays are malformed (the same in all threads).
struct RgSeg { int s0 = 0, s1 = 0, s = -1, sT = -1; bool mine = false; };
__device__ __forceinline__ bool load_segment(const RowsGradParams& p, int g, RgSeg& seg)
{
    int bad = 0;
    if (g < p.G) {
        seg.s0 = ld_after_wait(p.seg_offsets + g);
        seg.s1 = ld_after_wait(p.seg_offsets + g + 1);
        seg.s = ld_after_wait(p.ids + g);
        seg.sT = ld_after_wait(p.ids_T + g);
        if (seg.s1 < seg.s0 || seg.s0 < 0 || seg.s1 > p.T) bad = 1;
        if ((p.check_first && g == 0 && seg.s0 != 0) || (p.check_last && g == p.G - 1 && seg.s1 != p.T)) bad = 1;
        seg.mine = seg.s1 > seg.s0 && paired(p, seg.s, seg.sT);
    }
    if (p.bad && g == 0 && ld_after_wait(p.bad)) bad = 1;
    return __syncthreads_or(bad) != 0;
}
__device__ __forceinline__ void flag_segment(const RowsGradParams& p, const RgSeg& seg)
{
    if (seg.s1 <= seg.s0 || (seg.s == -1 && seg.sT == -1)) return;
    const int r = slot_rank(p.snap[0], seg.s);
    if (r == 0) atomicOr(p.status[0], LML_FLAG_BAD_SLOT);
    if (slot_rank(p.snap[1], seg.sT) != r) atomicOr(p.status[1], LML_FLAG_BAD_SLOT);
}

// Halves of a step with something in them: of its 128 columns (first pass) or rows (second) `from` and more are left of `all`.
__device__ __forceinline__ int halves(int from, int all) { return all - from > 64 ? 2 : 1; }

// ---- first pass ------------------------------------------------------------------------------------------
// This CTA's part of the line, item by item: pieces in order, of each x, then dy.
struct ShrinkTasks {
    const RowsGradParams& p;
    const RgCtrl* c;
    int w, end;
    int e = 0;
    int job = 0, step = 0, n = 0, row = 0, valid = 0, piece = 0, slot = 0;
    __device__ ShrinkTasks(const RowsGradParams& p_, const RgCtrl* c_, int w0, int w1) : p(p_), c(c_), w(w0), end(w1) {}
    __device__ bool next()
    {
        w += n;
        if (w >= end) return false;
        const int both = p.tiles[0] + p.tiles[1], idx = w / both, in = w - idx * both;
        job = in >= p.tiles[0] ? 1 : 0;
        step = in - (job ? p.tiles[0] : 0);
        n = min(p.tiles[job] - step, end - w);
        while (c->pre[e + 1] <= idx) ++e;
        const int i = idx - c->pre[e];
        row = c->first[e] + i * kTileM;
        valid = min(c->len[e] - i * kTileM, kTileM);
        piece = c->piece[e] + i;
        slot = c->slot[job][e];
        return true;
    }
    __device__ bool whole() const { return n == p.tiles[job]; }
    __device__ int item() const { return w - step; }
};

// Three bf16 values whose sum is x, for two x; an x that is not finite stands in the first alone.
__device__ __forceinline__ void split3(float x, float y, uint32_t (&part)[3])
{
    part[0] = pack_bf16(x, y);
    x = fabsf(bf16_lo(part[0])) < INFINITY ? x - bf16_lo(part[0]) : 0.f;
    y = fabsf(bf16_hi(part[0])) < INFINITY ? y - bf16_hi(part[0]) : 0.f;
    part[1] = pack_bf16(x, y);
    part[2] = pack_bf16(x - bf16_lo(part[1]), y - bf16_hi(part[1]));
}

template <int FMT>
__global__ void __launch_bounds__(kRgThreads, 1) rows_shrink_kernel(const __grid_constant__ RowsGradParams p)
{
    extern __shared__ uint8_t rg_smem[];
    __shared__ RgCtrl ctrl;
    RgCtrl* c = &ctrl;
    const uint32_t smem = (smem_u32(rg_smem) + 1023u) & ~1023u;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t cols = tmem_cols_for(3 * p.r16);   // two accumulators, and the sum of the chunks before
    rg_setup(c, warp, tid, cols);
    // (After the allocation: what starts from here on may want TMEM and waits for this grid.  And after the wait: rows_grad_kernel
    // takes it that whatever came before this grid is complete.)
    grid_dependency_wait();
    grid_launch_dependents();
    const uint32_t tmem = c->tmem_base;
    volatile int* abort = &c->abort;

    // The slice's pieces, counted through its segments.
    RgSeg seg;
    const bool bad = load_segment(p, tid, seg);
    if (blockIdx.x == 0) {
        flag_segment(p, seg);
        if (bad && tid == 0) atomicOr(p.status[0], LML_FLAG_BAD_OFFSETS);
        for (int i = tid; i < p.num_sms; i += kRgThreads) p.arrived[1][i] = 0;
    }
    const int mine = seg.mine && !bad ? (seg.s1 - seg.s0 + kTileM - 1) / kTileM : 0;
    int upto = mine;
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, upto, m);
        if (lane >= m) upto += v;
    }
    if (tid < kRgSegs && lane == 31) c->count[warp] = upto;
    __syncthreads();
    if (tid < kRgSegs) {
        for (int k = 0; k < warp; ++k) upto += c->count[k];
        c->first[tid] = seg.s0; c->len[tid] = seg.s1 - seg.s0; c->piece[tid] = seg.s0 / kTileM + tid;
        c->slot[0][tid] = (uint8_t)seg.s; c->slot[1][tid] = (uint8_t)seg.sT;
        c->pre[tid + 1] = upto;
        if (tid == 0) c->pre[0] = 0;
    }
    __syncthreads();
    const RgLine line(c->pre[kRgSegs] * (p.tiles[0] + p.tiles[1]));
    const int w0 = line.begin((int)blockIdx.x), w1 = line.begin((int)blockIdx.x + 1);

    const RgRing ring(smem, p.ring, (uint32_t)p.r16 * 128u);
    // Every half step of this CTA, for a producer: wait for its stage, then `f`.  `item`: what it keeps for an item's.
    auto each = [&](auto&& item, auto&& f) {
        RgCursor u(ring);
        for (ShrinkTasks t(p, c, w0, w1); t.next();) {
            const int d = p.d[t.job];
            const bool end = t.w + t.n == w1;
            item(t);
            int k = t.step * 128;
            for (int left = t.n; left > 0; --left, k += 128) {
                const int n = halves(k, d);
                for (int half = 0; half < n; ++half, u.advance()) {
                    if (!mbar_wait(smem_u32(&c->empty[u.stage]), u.phase ^ 1u, abort)) return u.turn;
                    f(u, k, half, left == 1 && half + 1 == n ? end ? kRgLast | kRgEnd : kRgLast : 0);
                }
            }
        }
        return u.turn;
    };
    if (w0 < w1) {
        if (warp == 0) {
            if (elect_one()) {
                const CUtensorMap* map = nullptr;
                const uint32_t* words = nullptr;
                bool raw = false;
                int r16 = 0, valid = 0, row = 0;
                const int turns = each([&](const ShrinkTasks& t) {
                         map = &p.map[0][t.job]; row = t.row; valid = t.valid;
                         r16 = chunks_of_rank(p.snap[t.job].rank[t.slot]) * kChunk;
                         raw = FMT != kBf16 && t.job == 0;
                         words = p.scales + t.row + (size_t)t.step * p.T;
                     },
                     [&](RgCursor& u, int k, int half, int last) {
                         c->info[u.stage] = {last | (raw ? kRgTouched : 0), valid, r16};
                         load_tile<false>(c, map, u.at, u.stage, raw, row, k + 64 * half);
                         if (raw) {
                             post_turn(c, u.turn, {u.stage | (int)u.phase << 8 | half << 9, valid, words});
                             ++u.turn;
                             if (half) words += p.T;   // (a step with one half is the last)
                         }
                     });
                if (FMT != kBf16)
                    for (int k = 0; k < kRgGroups; ++k) post_turn(c, turns + k, {-1, 0, nullptr});
            }
        } else if (warp == kRgOther) {
            if (elect_one()) {
                const CUtensorMap* map = nullptr;
                uint32_t bytes = 0;
                int row = 0;
                each([&](const ShrinkTasks& t) {
                         const int chunks = chunks_of_rank(p.snap[t.job].rank[t.slot]);
                         map = &p.low[t.job][chunks - 1]; bytes = (uint32_t)chunks * (kChunk * 128u); row = t.slot * kRankPad;
                     },
                     [&](RgCursor& u, int k, int half, int) {
                         const uint32_t bar = smem_u32(&c->low_full[u.stage]);
                         mbar_arrive_expect_tx(bar, bytes);
                         tma_load_2d(u.at + kRgTile, map, bar, k + 64 * half, row);
                     });
            }
        } else if (warp == 1) {
            if (elect_one()) issue_steps<false>(c, ring, tmem, (uint32_t)p.r16, abort);
        } else if (warp < kRgOther) {
            // (After a wait that gave up these warps go through the rest all the same: the counters of shared items come out right.  The
            // status word says that the results do not.)
            uint32_t chunk = 0;
            const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16), sum = lanes + 2 * p.r16;
            for (ShrinkTasks t(p, c, w0, w1); t.next(); ++chunk) {
                const int n_half = 2 * (t.n - 1) + halves((t.step + t.n - 1) * 128, p.d[t.job]), n_chunks = (n_half + kRgChunk - 1) / kRgChunk;
                sum_chunks<1>(c, lanes, (uint32_t)p.r16, (uint32_t)(chunks_of_rank(p.snap[t.job].rank[t.slot]) * kChunk), sum, n_chunks, chunk, lane, abort);
                // The products: lane = token.
                const int r = p.snap[t.job].rank[t.slot], r16 = chunks_of_rank(r) * kChunk, row = (warp & 3) * 32 + lane;
                const float sc = p.snap[t.job].scale[t.slot];
                const bool whole = t.whole();
                const RgShare share = whole ? RgShare{0, 0, 0} : share_of(line, t.item(), p.tiles[t.job], (int)blockIdx.x);
                uint8_t* out = p.pieces[t.job] + (size_t)t.piece * kRgPiece;
                float* mine_at = p.partial + (size_t)(2 * blockIdx.x + share.slot) * kRgPartial;
                // (r16 is a multiple of 16: the swizzle goes by j alone)
                const bool there = row < t.valid;   // (rows behind the segment, columns behind the rank: whatever they hold)
                const uint32_t from = lanes + (chunk & 1) * (uint32_t)p.r16;
                // Two lanes share out two columns, so that each has both tokens of one: 4 bytes per store
                const int odd = lane & 1;
                uint8_t* const pair_at = out + (size_t)(row >> 6) * (r16 * 384) + (row & 6) * 2;
#pragma unroll 1
                for (int j = 0; j < r16; j += 8) {
                    float v[8];
                    chunk_sums<1>(from + (uint32_t)j, 0, sum + (uint32_t)j, n_chunks > 1, v);
                    if (!whole) {
                        float* to = mine_at + j * 128 + row;
#pragma unroll
                        for (int e = 0; e < 8; ++e) to[e * 128] = v[e];
                        continue;
                    }
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        const float x = there && j + e < r ? v[e] * sc : 0.f, y = there && j + e + 1 < r ? v[e + 1] * sc : 0.f;
                        const float got = __shfl_xor_sync(0xffffffffu, odd ? x : y, 1);
                        uint32_t part[3];
                        split3(odd ? got : x, odd ? y : got, part);
                        uint8_t* at = pair_at + (j + e + odd) * 128 + ((((row & 63) >> 3) ^ (e + odd)) * 16);
#pragma unroll
                        for (int k = 0; k < 3; ++k) *reinterpret_cast<uint32_t*>(at + k * r16 * 128) = part[k];
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&c->acc_free[chunk & 1]));
                if (!whole) arrive(c, p.arrived[0], share, t.job, t.slot, t.piece, t.valid);
            }
            fence_proxy_async_all();          // the pieces are read by bulk copies
        } else if (FMT != kBf16) {
            const int group = (warp - kRgFirstConv) / kRgGroup;
            convert_tiles<FMT == kE4m3, false>(c, ring, group, tid - 32 * (kRgFirstConv + group * kRgGroup), lane, abort);
        }
    }
    __syncwarp();
    if (*abort) __nanosleep(50000);   // gave up: let copies still in flight land before the CTA goes away
    __syncthreads();
    for (int i = 0; i < c->n_joins; ++i) {
        const RgJoin s = c->joins[i];
        const int r = p.snap[s.job].rank[s.slot], r16 = chunks_of_rank(r) * kChunk;
        const float sc = p.snap[s.job].scale[s.slot];
        for (int e = tid; e < r16 * 32; e += kRgThreads) {   // four tokens of one column
            const int j = e >> 5, t4 = (e & 31) * 4;
            const float4 v = joined(p, s, e * 4);
            const auto value = [&](float x, int k) { return j < r && t4 + k < s.valid ? x * sc : 0.f; };
            uint32_t part[2][3];
            split3(value(v.x, 0), value(v.y, 1), part[0]);
            split3(value(v.z, 2), value(v.w, 3), part[1]);
            uint8_t* at = p.pieces[s.job] + (size_t)s.at * kRgPiece + (size_t)(t4 >> 6) * (r16 * 384) + j * 128 + ((((t4 & 63) >> 3) ^ (j & 7)) * 16) + (t4 & 4) * 2;
#pragma unroll
            for (int k = 0; k < 3; ++k) *reinterpret_cast<uint2*>(at + k * r16 * 128) = make_uint2(part[0][k], part[1][k]);
        }
        fence_proxy_async_all();
    }
    if (tid == 0 && *abort) atomicOr(p.status[0], LML_FLAG_TIMEOUT);
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, cols);
    }
}

// ---- second pass -----------------------------------------------------------------------------------------
// Items: slots in use in order, of each the column tiles (x first, then dy), of each its units.  A CTA has its part of the line, or, if
// there are few items, whole ones.  In the line an item is as long as it has units, but at least as long as finishing it takes in steps; what is
// behind its units is nobody's work.  (Counted by units alone, the CTAs with the items of an adapter of few tokens and 64 ranks were still at it when
// all others had left: 192 us for 8192 tokens, 114 of them of such a one,
// that take 134 so.)
constexpr int kRgFinishSteps = 2;
__device__ __forceinline__ int item_length(int units, int r16) { return max(units, kRgFinishSteps + r16 / 16); }
struct GradTasks {
    const RowsGradParams& p;
    const RgCtrl* c;
    unsigned long long mask;   // slots from here on
    int w, end, base = 0;   // base: of the slot at hand
    int slot = 0, units = 0, length = 0, tile = 0, a = 0, b = 0;
    __device__ GradTasks(const RowsGradParams& p_, const RgCtrl* c_, int w0, int w1) : p(p_), c(c_), mask(c_->used()), w(w0), end(w1) {}
    __device__ void next_slot()
    {
        base += length * p.all_tiles;
        slot = __ffsll((long long)mask) - 1;
        mask &= mask - 1ull;
        units = c->units[slot];
        length = p.whole_items ? 1 : item_length(units, chunks_of_rank(p.snap[0].rank[slot]) * kChunk);
    }
    __device__ bool next()
    {
        if (b > 0) w = p.whole_items ? w + gridDim.x : base + tile * length + (b < units ? b : length);
        for (;; w = base + (tile + 1) * length) {
            if (w >= end) return false;
            while (w >= base + length * p.all_tiles) next_slot();
            tile = (w - base) / length;
            a = w - base - tile * length;
            if (a < units) break;
        }
        b = p.whole_items ? units : min(units, a + (end - w));
        return true;
    }
    __device__ bool whole() const { return b - a == units; }
    // of this CTA's: what follows is not there, or not its own, or behind an item's units
    __device__ bool last() const { return (p.whole_items ? w + (int)gridDim.x : b < units ? w + (b - a) : base + (tile + 1) * length) >= end; }
    __device__ int item() const { return w - a; }
    __device__ int job() const { return tile < p.tiles[0] ? 0 : 1; }
    __device__ int column() const { return (tile < p.tiles[0] ? tile : tile - p.tiles[0]) * 128; }
};
// The pieces of a task, in the order of the slot's segments.
struct RgPieces {
    const RgCtrl* c;
    int e, k, left, first = 0, len = 0, pieces = 0, at0 = 0;   // of the segment at hand
    __device__ void load()
    {
        first = c->first[e];
        len = c->len[e];
        pieces = (len + kTileM - 1) / kTileM;
        at0 = c->piece[e];
    }
    __device__ RgPieces(const RgCtrl* c_, const GradTasks& t) : c(c_), left(t.b - t.a)
    {
        e = c->entry[t.slot];
        while (c->pre[e] + (c->len[e] + kTileM - 1) / kTileM <= t.a) ++e;
        k = t.a - c->pre[e] - 1;
        load();
    }
    __device__ bool next()
    {
        if (left-- <= 0) return false;
        if (++k >= pieces) { ++e; k = 0; load(); }
        return true;
    }
    __device__ int row() const { return first + k * kTileM; }
    __device__ int valid() const { return min(len - k * kTileM, kTileM); }
    __device__ size_t at() const { return (size_t)(at0 + k) * kRgPiece; }
};

// Half steps of a task: two for every piece, but for those that end a segment with no more than 64 rows.
__device__ __forceinline__ int half_steps(const RgCtrl* c, const GradTasks& t)
{
    int n = 2 * (t.b - t.a);
    for (int e = c->entry[t.slot];; ++e) {
        const int len = c->len[e], end = c->pre[e] + (len + kTileM - 1) / kTileM;
        if (end > t.a && end <= t.b && ((len - 1) & (kTileM - 1)) < 64) --n;
        if (end >= t.b) return n;
    }
}

template <int FMT>
__global__ void __launch_bounds__(kRgThreads, 1) rows_grad_kernel(const __grid_constant__ RowsGradParams p)
{
    extern __shared__ uint8_t rg_smem[];
    __shared__ RgCtrl ctrl;
    RgCtrl* c = &ctrl;
    const uint32_t smem = (smem_u32(rg_smem) + 1023u) & ~1023u;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t cols = tmem_cols_for(7 * p.r16);   // two accumulators of three parts, and the sum of the chunks before
    if (tid < kMaxSlots) c->units[tid] = 0;
    rg_setup(c, warp, tid, cols);
    grid_launch_dependents();   // (after the allocation, see rows_shrink_kernel)
    // rows_shrink_kernel let this grid go after its own wait, so everything but the pieces that it writes is there already; only the
    // producer of the other operand waits for it.  (With no tokens nothing went before.)
    if (p.T == 0) grid_dependency_wait();
    const uint32_t tmem = c->tmem_base;
    volatile int* abort = &c->abort;

    // The slice's segments, by slot.
    RgSeg seg;
    const bool bad = load_segment(p, tid, seg);
    const bool mine = seg.mine && !bad;
    const int mine_units = mine ? (seg.s1 - seg.s0 + kTileM - 1) / kTileM : 0;
    if (tid < kRgSegs) {
        c->slot[0][tid] = mine ? (uint8_t)seg.s : (uint8_t)255;
        c->len[tid] = mine_units;   // (for now)
    }
    if (mine) {
        atomicOr(&c->used_half[seg.s >> 5], 1u << (seg.s & 31));
        atomicAdd(&c->units[seg.s], mine_units);
    }
    __syncthreads();
    int pos = 0, before = 0, same = 0;
    for (int g = 0; g < p.G; ++g) {
        const int s = c->slot[0][g];
        if (s < seg.s || (s == seg.s && g < tid)) ++pos;
        if (s == seg.s && g < tid) { before += c->len[g]; ++same; }
    }
    __syncthreads();
    if (mine) {
        c->first[pos] = seg.s0; c->len[pos] = seg.s1 - seg.s0; c->piece[pos] = seg.s0 / kTileM + tid; c->pre[pos] = before;
        if (same == 0) c->entry[seg.s] = pos;
    }
    __syncthreads();
    int total = 0;
    for (unsigned long long m = c->used(); m; m &= m - 1ull) {
        const int s = __ffsll((long long)m) - 1;
        total += p.whole_items ? 1 : item_length(c->units[s], chunks_of_rank(p.snap[0].rank[s]) * kChunk);
    }
    const RgLine line(total * p.all_tiles);
    const int w0 = p.whole_items ? (int)blockIdx.x : line.begin((int)blockIdx.x), w1 = p.whole_items ? line.W : line.begin((int)blockIdx.x + 1);

    const RgRing ring(smem, p.ring, (uint32_t)p.r16 * 384u);
    auto each = [&](auto&& item, auto&& f) {   // (see rows_shrink_kernel)
        RgCursor u(ring);
        for (GradTasks t(p, c, w0, w1); t.next();) {
            const bool raw = FMT != kBf16 && t.job() == 0, end = t.last();
            item(t, raw);
            for (RgPieces v(c, t); v.next();) {
                const int valid = v.valid(), n = halves(0, valid);
                for (int half = 0; half < n; ++half, u.advance()) {
                    if (!mbar_wait(smem_u32(&c->empty[u.stage]), u.phase ^ 1u, abort)) return u.turn;
                    const int rows = min(valid - 64 * half, 64);
                    const int flags = (raw || (rows & 15) ? kRgTouched : 0) | (v.left == 0 && half + 1 == n ? end ? kRgLast | kRgEnd : kRgLast : 0);
                    f(u, v, half, rows, flags);
                }
            }
        }
        return u.turn;
    };
    if (GradTasks(p, c, w0, w1).next()) {   // (a part can lie behind the units of an item)
        if (warp == 0) {
            if (elect_one()) {
                const CUtensorMap* map = nullptr;
                const uint32_t* words = nullptr;
                bool is_raw = false;
                int column = 0, r16 = 0;
                const int turns = each([&](const GradTasks& t, bool raw) {
                         map = &p.map[1][t.job()]; is_raw = raw; column = t.column();
                         r16 = chunks_of_rank(p.snap[0].rank[t.slot]) * kChunk;
                         words = p.scales + (size_t)t.tile * p.T;
                     },
                     [&](RgCursor& u, const RgPieces& v, int half, int rows, int flags) {
                         const int row = v.row() + 64 * half;
                         c->info[u.stage] = {flags, rows, r16};
                         load_tile<true>(c, map, u.at, u.stage, is_raw, row, column);
                         if (flags & kRgTouched) {
                             post_turn(c, u.turn, {u.stage | (int)u.phase << 8, rows, is_raw ? words + row : nullptr});
                             ++u.turn;
                         }
                     });
                for (int k = 0; k < kRgGroups; ++k) post_turn(c, turns + k, {-1, 0, nullptr});
            }
        } else if (warp == kRgOther) {
            if (elect_one()) {
                grid_dependency_wait();   // (the tiles are on their way meanwhile)
                fence_proxy_async_all();
                uint32_t low = 0;
                const uint8_t* pieces = nullptr;
                each([&](const GradTasks& t, bool) {
                         low = (uint32_t)(chunks_of_rank(p.snap[0].rank[t.slot]) * kChunk) * 384u;
                         pieces = p.pieces[t.job() ^ 1];   // (u for dy, v for x)
                     },
                     [&](RgCursor& u, const RgPieces& v, int half, int, int) {
                         const uint32_t bar = smem_u32(&c->low_full[u.stage]);
                         mbar_arrive_expect_tx(bar, low);
                         bulk_load(u.at + kRgTile, pieces + v.at() + half * low, low, bar);
                     });
            }
        } else if (warp == 1) {
            if (elect_one()) issue_steps<true>(c, ring, tmem, 3u * (uint32_t)p.r16, abort);
        } else if (warp < kRgOther) {
            uint32_t chunk = 0;   // (see rows_shrink_kernel)
            const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16), sum = lanes + 6 * p.r16;
            for (GradTasks t(p, c, w0, w1); t.next(); ++chunk) {
                const int n_chunks = (half_steps(c, t) + kRgChunk - 1) / kRgChunk;
                sum_chunks<3>(c, lanes, 3u * (uint32_t)p.r16, (uint32_t)(chunks_of_rank(p.snap[0].rank[t.slot]) * kChunk), sum, n_chunks, chunk, lane, abort);
                // The sums, 16 columns of the accumulator at a time: lane = column of x or dy.  Partial results: dA [j][column], dB [column][j].
                // dA is written as it stands, 128 bytes of a row per store; dB by way of shared memory, 64 bytes of a column's row.  (Four at a
                // time straight to their places, each asked about: 205 us for the call where this took 176.)
                const int job = t.job(), c0 = t.column();
                const int r = p.snap[0].rank[t.slot], r16 = chunks_of_rank(r) * kChunk, col0 = (warp & 3) * 32, d = p.d[job];
                const bool whole = t.whole(), add = whole && p.accumulate;
                float* dst = p.partial + (size_t)(2 * blockIdx.x + (!whole && line.part_of(t.item()) == (int)blockIdx.x ? 1 : 0)) * kRgPartial;
                if (whole) dst = p.out[job] + (size_t)t.slot * kRankPad * d + (job == 0 ? c0 : c0 * kRankPad);
                const int stride = !whole ? (job == 0 ? 128 : r16) : job == 0 ? d : kRankPad;   // between two j, or two columns
                const int most = whole ? r : r16, columns = whole ? d - c0 : 128;               // of them that there are
                const uint32_t from = lanes + (chunk & 1) * 3u * (uint32_t)p.r16;
#pragma unroll 1
                for (int j = 0; j < r16; j += 16) {
                    float s[16];
#pragma unroll
                    for (int k = 0; k < 16; k += 8) {
                        float v[8];
                        chunk_sums<3>(from + (uint32_t)(j + k), (uint32_t)r16, sum + (uint32_t)(j + k), n_chunks > 1, v);
#pragma unroll
                        for (int e = 0; e < 8; ++e) s[k + e] = v[e];
                    }
                    if (job == 0) {
                        float* to = dst + (size_t)j * stride + col0 + lane;
                        if (!add && j + 16 <= most && col0 + 32 <= columns) {
#pragma unroll
                            for (int e = 0; e < 16; ++e, to += stride) *to = s[e];
                        } else if (col0 + lane < columns) {
                            if (add) {
#pragma unroll
                                for (int e = 0; e < 16; ++e)
                                    if (j + e < most) s[e] += to[(size_t)e * stride];
                            }
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                if (j + e < most) to[(size_t)e * stride] = s[e];
                        }
                        continue;
                    }
                    float4(*turned)[5] = c->turned[warp & 3];   // [column][j / 4], and a place that spreads the columns over the banks
                    __syncwarp();
#pragma unroll
                    for (int e = 0; e < 4; ++e) turned[lane][e] = make_float4(s[4 * e], s[4 * e + 1], s[4 * e + 2], s[4 * e + 3]);
                    __syncwarp();
                    const int j4 = j + (lane & 3) * 4;
                    float* const to0 = dst + (size_t)(col0 + (lane >> 2)) * stride + j4;
                    if (!add && j + 16 <= most && col0 + 32 <= columns) {
                        float* to = to0;
#pragma unroll
                        for (int e = 0; e < 4; ++e, to += 8 * stride) *reinterpret_cast<float4*>(to) = turned[e * 8 + (lane >> 2)][lane & 3];
                        continue;
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int column = e * 8 + (lane >> 2);
                        float4 x = turned[column][lane & 3];
                        float* to = to0 + (size_t)(e * 8) * stride;
                        if (col0 + column >= columns) continue;
                        if (j4 + 4 <= most) {
                            if (add) {
                                const float4 o = *reinterpret_cast<const float4*>(to);
                                x = make_float4(o.x + x.x, o.y + x.y, o.z + x.z, o.w + x.w);
                            }
                            *reinterpret_cast<float4*>(to) = x;
                        } else {
                            const float f[3] = {x.x, x.y, x.z};   // (less than four)
#pragma unroll
                            for (int i = 0; i < 3; ++i)
                                if (j4 + i < most) to[i] = add ? to[i] + f[i] : f[i];
                        }
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&c->acc_free[chunk & 1]));
                if (whole) continue;
                arrive(c, p.arrived[1], share_of(line, t.item(), t.units, (int)blockIdx.x), job, t.slot, c0, 0);
            }
        } else {
            const int group = (warp - kRgFirstConv) / kRgGroup;
            convert_tiles<FMT == kE4m3, true>(c, ring, group, tid - 32 * (kRgFirstConv + group * kRgGroup), lane, abort);
        }
    }
    __syncwarp();
    if (*abort) __nanosleep(50000);
    grid_dependency_wait();   // (a CTA without units too: who waits for this grid has waited for the pieces' writers)
    if (blockIdx.x == 0)
        for (int i = tid; i < p.num_sms; i += kRgThreads) p.arrived[0][i] = 0;
    __syncthreads();
    for (int i = 0; i < c->n_joins; ++i) {
        const RgJoin s = c->joins[i];
        const int r = p.snap[0].rank[s.slot], r16 = chunks_of_rank(r) * kChunk, d = p.d[s.job], per = s.job == 0 ? 32 : r16 / 4;   // float4 per row of the partial results
        float* out = p.out[s.job] + (size_t)s.slot * kRankPad * d;
        for (int e = tid; e < r16 * 32; e += kRgThreads) {
            const int line_at = e / per, col = (e % per) * 4;
            const int j = s.job == 0 ? line_at : col, n = s.at + (s.job == 0 ? col : line_at);
            if (j >= r || n >= d) continue;
            const float4 v = joined(p, s, e * 4);
            float* dst = s.job == 0 ? out + (size_t)j * d + n : out + (size_t)n * kRankPad + j;
            if (s.job == 0 || j + 4 <= r) {   // (d is a multiple of 8)
                const float4 o = p.accumulate ? *reinterpret_cast<const float4*>(dst) : make_float4(0.f, 0.f, 0.f, 0.f);
                *reinterpret_cast<float4*>(dst) = make_float4(o.x + v.x, o.y + v.y, o.z + v.z, o.w + v.w);
            } else {
                const float w[3] = {v.x, v.y, v.z};   // (less than four columns)
#pragma unroll
                for (int k = 0; k < 3; ++k)
                    if (j + k < r) dst[k] = p.accumulate ? dst[k] + w[k] : w[k];
            }
        }
    }
    if (!p.accumulate) {      // adapters without a token
        for (unsigned long long m = p.live & ~c->used(); m; m &= m - 1ull) {
            const int slot = __ffsll((long long)m) - 1, r = p.snap[0].rank[slot];
            const size_t k = (size_t)blockIdx.x * kRgThreads + tid, stride = (size_t)gridDim.x * kRgThreads;
            for (size_t i = k; i < (size_t)r * p.d[0]; i += stride) p.out[0][(size_t)slot * kRankPad * p.d[0] + i] = 0.f;
            for (size_t i = k; i < (size_t)r * p.d[1]; i += stride) p.out[1][((size_t)slot * p.d[1] + i / r) * kRankPad + i % r] = 0.f;
        }
    }
    if (tid == 0 && *abort) atomicOr(p.status[0], LML_FLAG_TIMEOUT);
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, cols);
    }
}

// Calls of several slices: whether their arrays hold together, before any of them adds something.
__global__ void __launch_bounds__(1024) rows_check_kernel(const int32_t* seg_offsets, int G, int T, int* bad_out)
{
    grid_dependency_wait();
    grid_launch_dependents();
    int bad = 0;
    for (int g = threadIdx.x; g < G; g += 1024) {
        const int s0 = ld_after_wait(seg_offsets + g), s1 = ld_after_wait(seg_offsets + g + 1);
        if (s1 < s0 || s0 < 0 || s1 > T || (g == 0 && s0 != 0) || (g == G - 1 && s1 != T)) bad = 1;
    }
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) *bad_out = bad;
}

// ---- host ---------------------------------------------------------------------------------------------
constexpr int kRgRing = 208 * 1024;   // one CTA to an SM

// Workspace: [u][v][partial results of both passes' CTAs][whether the arrays hold together]
struct RgLayout { size_t pieces, partial, bad, total; };
static RgLayout rg_layout(int T, int G, int num_sms)
{
    RgLayout l;
    l.pieces = ((size_t)T / kTileM + (size_t)(G < kRgSegs ? G : kRgSegs)) * kRgPiece;
    l.partial = 2 * l.pieces;
    l.bad = l.partial + (size_t)num_sms * 2 * kRgPartial * sizeof(float);
    l.total = l.bad + 256;
    return l;
}
size_t rows_grad_ws_bytes(int T, int G, int num_sms) { return rg_layout(T, G, num_sms).total; }

template <int FMT> static cudaError_t rg_attributes()
{
    cudaError_t e = cudaFuncSetAttribute(rows_shrink_kernel<FMT>, cudaFuncAttributeMaxDynamicSharedMemorySize, 1024 + kRgRing);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(rows_grad_kernel<FMT>, cudaFuncAttributeMaxDynamicSharedMemorySize, 1024 + kRgRing);
}
cudaError_t rows_grad_init()
{
    cudaError_t e = rg_attributes<kBf16>();
    if (e == cudaSuccess) e = rg_attributes<kInt8>();
    if (e == cudaSuccess) e = rg_attributes<kE4m3>();
    return e;
}

cudaError_t launch_rows_grad(const RowsGradCall& a, cudaStream_t stream, int* launches)
{
    RowsGradParams p;
    *launches = 0;
    int most = 1, live = 0;
    p.live = 0ull;
    p.snap[0] = *a.snap; p.snap[1] = *a.snap_T;
    for (int s = 0; s < a.snap->max_slots; ++s)
        if (a.snap->rank[s]) {
            most = a.snap->rank[s] > most ? a.snap->rank[s] : most;
            p.live |= 1ull << s;
            ++live;
        }
    if (live == 0 && a.T == 0) return cudaSuccess;
    p.r16 = chunks_of_rank(most) * kChunk;
    const RgLayout lay = rg_layout(a.T, a.G, a.num_sms);
    uint8_t* ws = static_cast<uint8_t*>(a.workspace);
    p.d[0] = a.d_in; p.d[1] = a.d_out;
    p.tiles[0] = (a.d_in + 127) / 128; p.tiles[1] = (a.d_out + 127) / 128;
    p.all_tiles = p.tiles[0] + p.tiles[1];
    p.T = a.T; p.ring = kRgRing;
    p.scales = a.x.scales;
    p.status[0] = a.status; p.status[1] = a.status_T;
    p.pieces[0] = ws; p.pieces[1] = ws + lay.pieces;
    p.partial = reinterpret_cast<float*>(ws + lay.partial);
    p.arrived[0] = a.arrived; p.arrived[1] = a.arrived + a.num_sms;
    p.num_sms = a.num_sms;
    p.out[0] = a.dA; p.out[1] = a.dB;
    memset(p.map, 0, sizeof(p.map));
    memset(p.low, 0, sizeof(p.low));
    auto launch = [&](void (*kernel)(RowsGradParams), long long ctas) {
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr[1];
        const long long all = a.num_sms;
        pdl_config(cfg, attr, dim3((unsigned)(ctas < 1 ? 1 : ctas < all ? ctas : all)), dim3(kRgThreads), (size_t)(1024 + kRgRing), stream);
        const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p);
        if (e == cudaSuccess) ++*launches;
        return e;
    };
    const bool e4m3 = a.x.format == kE4m3, bf16 = a.x.format == kBf16;
    const auto shrink = bf16 ? rows_shrink_kernel<kBf16> : e4m3 ? rows_shrink_kernel<kE4m3> : rows_shrink_kernel<kInt8>;
    const auto grad = bf16 ? rows_grad_kernel<kBf16> : e4m3 ? rows_grad_kernel<kE4m3> : rows_grad_kernel<kInt8>;
    p.bad = nullptr;
    if (a.T == 0) {   // adapters' gradients are zero
        p.G = 0; p.seg_offsets = p.ids = p.ids_T = nullptr;
        p.check_first = p.check_last = 0; p.accumulate = 0; p.whole_items = 0;
        return launch(grad, a.num_sms);
    }
    const int pitch = kept_pitch(a.d_in);
    bool ok = true;
    for (int pass = 0; pass < 2; ++pass) {
        const int rows = pass == 0 ? 128 : 64;
        ok = ok && (bf16 ? a.cache->get_2d(&p.map[pass][0], a.x.data, (uint64_t)a.d_in, (uint64_t)a.T, (uint64_t)a.d_in * 2, 64, rows)
                         : a.cache->get_2d(&p.map[pass][0], a.x.data, (uint64_t)pitch / 2, (uint64_t)a.T, (uint64_t)pitch, pass == 0 ? 32 : 64, rows, false));
        ok = ok && a.cache->get_2d(&p.map[pass][1], a.dy, (uint64_t)a.d_out, (uint64_t)a.T, (uint64_t)a.d_out * 2, 64, rows);   // (8-bit rows as pairs)
    }
    for (int k = 0; k < kRankPad / kChunk && k * kChunk < p.r16; ++k)
        for (int i = 0; i < 2; ++i)
            ok = ok && a.cache->get_2d(&p.low[i][k], a.low[i], (uint64_t)p.d[i], (uint64_t)a.slots[i] * kRankPad, (uint64_t)p.d[i] * 2, 64, (k + 1) * kChunk);
    if (!ok) return cudaErrorInvalidValue;
    if (a.G > kRgSegs) {
        p.bad = reinterpret_cast<int*>(ws + lay.bad);
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr[1];
        pdl_config(cfg, attr, dim3(1), dim3(1024), 0, stream);
        const cudaError_t e = cudaLaunchKernelEx(&cfg, rows_check_kernel, a.seg_offsets, a.G, a.T, const_cast<int*>(p.bad));
        if (e != cudaSuccess) return e;
        ++*launches;
    }
    for (int g0 = 0; g0 < a.G; g0 += kRgSegs) {
        p.G = a.G - g0 < kRgSegs ? a.G - g0 : kRgSegs;
        p.seg_offsets = a.seg_offsets + g0; p.ids = a.ids + g0; p.ids_T = a.ids_T + g0;
        p.check_first = g0 == 0; p.check_last = g0 + p.G == a.G;
        p.accumulate = a.accumulate || g0 > 0 ? 1 : 0;
        p.whole_items = 0;
        const long long pieces = a.T / kTileM + p.G;   // at most: every segment can have one that is not full
        cudaError_t e = launch(shrink, pieces * p.all_tiles / kRgLeast);
        if (e != cudaSuccess) return e;
        if (live == 0) continue;   // (nothing to write; the first pass has looked at the segments all the same)
        // Few pieces to an item: whole items, unless there are so many that their number leaves CTAs idle at the end.
        const int slots = p.G < live ? p.G : live;
        const long long items = (long long)p.all_tiles * slots;
        p.whole_items = pieces <= 4ll * slots && items <= a.num_sms;
        e = launch(grad, p.whole_items ? items : pieces * p.all_tiles / kRgLeast);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace lml
