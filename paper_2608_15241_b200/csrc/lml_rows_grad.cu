// Adapter gradients of the layer, x as bf16 rows or as an 8-bit checkpoint:
//     u = s x.A^T,  v = s dy.B   (per token, with the token's adapter)        dA_s += v^T x,   dB_s += dy^T u
// Two launches, each over x and dy side by side.
//
// rows_shrink_kernel: u and v.  An item is a piece (up to 128 rows of one segment, counted from the segment's first row: a TMA box
// may begin at any row, so no row of another segment is in it but behind its end) of x or of dy, its work the steps of 128 columns.
// rows_grad_kernel: dA and dB.  An item is (slot, 128 columns of x or dy), its work the slot's pieces.
// A step of either is a tile of 128 rows x 128 columns.
// In both the work of all items stands in one line that is cut into equal parts, one per SM; a CTA walks its part without a pause
// between items.  An item that the cuts divide is joined in device memory: every CTA writes its partial result, and the last one to
// arrive adds them in the order of the parts, so the bits do not depend on who that is.  (A form with a cluster per item and an
// exchange through distributed shared memory spent 10 us per CTA on setting up and joining.)
//
// Both are rings of tiles of x or dy as TMA brings them in, multiplied by tcgen05 into one of two accumulators.  Roles: a producer of tiles,
// which also tells the others what a stage holds, and one of the other operand (one thread for both would be the slowest role); an issuer; four warps that finish items while the next one is multiplied; two
// groups of eight warps that take 8-bit tiles in turn through their registers and write them back in place as bf16 (exact: the
// scales are powers of two) in the swizzled order of the tensor cores.  The second product contracts over tokens: the tile
// [token][64 columns] is an operand whose contiguous index is the output's (M-major), which the descriptor says; nothing is
// transposed.
//
// dA and dB are fp32 and so are u and v on the way: each goes into the second product as three bf16 values whose sum is the fp32
// value, side by side as 3r columns of one product.  One bf16 value would leave 2^-9, 1e-3 of every gradient, two 3e-6.
//
// Bound by memory: x and dy leave HBM once (the second pass finds them in L2 up to about 100 MB).
#include <cstring>

#include "lml_ptx_sm100.cuh"
#include "lml_rows_grad.cuh"

namespace lml {

using namespace ptx;

constexpr int kRgGroup = 8;                     // warps of a converting group
constexpr int kRgFinish = 4;                    // warps that finish items (warps 2 ... 5: one per quarter of the accumulator's lanes)
constexpr int kRgOther = 2 + kRgFinish;         // the warp that brings in the other operand
constexpr int kRgFirstConv = kRgOther + 1;
constexpr int kRgThreads = 32 * (kRgFirstConv + 2 * kRgGroup);
constexpr int kRgSegs = 320;                    // segments of a launch; a call of more runs in slices
constexpr int kRgTile = 128 * 128 * 2;          // bytes of a tile as it is multiplied: two halves of 64 columns, [half][row][64]
constexpr int kRgHalfTile = kRgTile / 2;
constexpr int kRgRaw = 128 * 128;               // ... of the 8-bit tile it is made of, [row][128]
constexpr int kRgPiece = 2 * 3 * kRankPad * 128;   // u (or v) of a piece: [64 tokens each][three parts][column][64]
constexpr int kRgPartial = kRankPad * 128;      // floats of a partial result
constexpr int kRgMaxStages = 6;
constexpr int kRgTurns = 16;                    // tiles on their way to and from the converting warps: as many as stages, and two ends
static_assert(kRgTurns >= kRgMaxStages + 2 && (kRgTurns & (kRgTurns - 1)) == 0, "a turn's place must have been read before it is used again");
constexpr int kRgWords = 136;                   // scale words of a tile, one per row, brought in from a 16-byte boundary on
constexpr int kRgLeast = 4;                     // steps of a CTA's part (of a whole pass, if it has fewer)

struct alignas(64) RowsGradParams {
    CUtensorMap map[2];       // x, dy: boxes of 64 columns (8-bit x: 128) x 128 rows
    CUtensorMap low[2][kRankPad / kChunk];   // the packed A of the table, B^T of the transposed one: boxes of 64 columns x 16, 32, 48, 64 rows
    SlotSnapshot snap[2];     // table, transposed table
    const uint32_t* scales;   // of x
    const int32_t *seg_offsets, *ids, *ids_T;   // of this slice
    const int* bad;           // or null: not 0 if the arrays of the call do not hold together (calls of several slices)
    uint32_t* status[2];
    uint8_t* pieces[2];       // u, v
    float* partial;           // [CTA][2]: of the item that its part begins in, of the item that its part ends in
    int* arrived;             // [CTA]: of the item that its part ends in and the next one goes on with; zero between calls
    float* out[2];            // dA, dB
    int d[2], tiles[2];       // d_in, d_out; in tiles of 128 columns
    int T, G, r16, ring, accumulate, all_tiles, whole_items;
    int check_first, check_last;   // the slice begins, ends the call
    unsigned long long live;  // slots with an adapter
};

// What the producer says about a stage.
constexpr int kRgFirst = 1, kRgLast = 2, kRgEnd = 4, kRgTouched = 8;   // first, last of an item; last of this CTA; goes through the converting warps
struct RgInfo {
    int flags, valid;   // rows
    int r16;            // columns of the other operand (second pass: of each of its three parts)
    int word;           // of a converted tile: place of its first scale word; -1: only rows behind the last are cleared
};
struct RgTurn { int stage, phase; };   // stage < 0: no more

struct RgCtrl {
    unsigned long long full[kRgMaxStages], empty[kRgMaxStages], turn[kRgTurns], made[kRgTurns], acc_full[2], acc_free[2];
    RgInfo info[kRgMaxStages];
    RgTurn turns[kRgTurns];
    unsigned long long used;
    uint32_t tmem_base;
    int abort, last, count[kRgSegs / 32], units[kMaxSlots], entry[kMaxSlots];
    int first[kRgSegs], len[kRgSegs], piece[kRgSegs], pre[kRgSegs + 1];
    uint8_t slot[2][kRgSegs];
    alignas(16) uint32_t words[kRgMaxStages][kRgWords];
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

// 4 columns of 32 lanes
__device__ __forceinline__ void tmem_ld_32x4(uint32_t taddr, uint32_t (&r)[4])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ uint2 ld_smem_v2(uint32_t a)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
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
        c->used = 0ull;
        for (int i = 0; i < kRgMaxStages; ++i) {
            mbar_init(smem_u32(&c->full[i]), 2);
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

// The ring of a CTA: stages of a tile beside the other operand (of the widest adapter).  Every role walks it with a cursor of its own (a
// division per step to find the stage costs as much as the step's products).
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

// Producer (one thread): hands a stage, what it holds being written, on to the converting warps; stage -1: there is no more.
__device__ __forceinline__ void post_turn(RgCtrl* c, int turn, int stage, uint32_t phase)
{
    c->turns[turn % kRgTurns] = {stage, (int)phase};
    mbar_arrive(smem_u32(&c->turn[turn % kRgTurns]));   // (releases what was written)
}
// Producer of tiles (one thread): the tile at (row, column) into the stage.  `words`: the scale words of the tile's rows.  A bulk copy wants 16-byte boundaries, so theirs begins up to three words early, and takes kRgWords; where that
// would reach behind the array's end, ordinary loads bring the rest.
__device__ __forceinline__ void load_tile(RgCtrl* c, const CUtensorMap* map, uint32_t at, int stage, bool raw, int row, int column, int valid, int flags, int r16,
                                          const uint32_t* words, const uint32_t* words_end)
{
    const uint32_t bar = smem_u32(&c->full[stage]);
    if (raw) {
        const uintptr_t addr = reinterpret_cast<uintptr_t>(words);
        const uint32_t* from = reinterpret_cast<const uint32_t*>(addr & ~(uintptr_t)15);
        c->info[stage] = {flags, valid, r16, (int)(addr >> 2) & 3};
        uint32_t bytes = kRgWords * 4;
        if (words_end - from < kRgWords) {
            bytes = (uint32_t)(words_end - from) * 4u & ~15u;
            for (const uint32_t* w = from + bytes / 4; w < words_end; ++w) c->words[stage][w - from] = ld_after_wait(w);
        }
        mbar_arrive_expect_tx(bar, kRgRaw + bytes);
        tma_load_2d(at, map, bar, column / 2, row);   // (8-bit columns in pairs)
        if (bytes) bulk_load(smem_u32(c->words[stage]), from, bytes, bar);
    } else {
        c->info[stage] = {flags, valid, r16, -1};
        mbar_arrive_expect_tx(bar, kRgTile);
        tma_load_2d(at, map, bar, column, row);
        tma_load_2d(at + kRgHalfTile, map, bar, column + 64, row);
    }
}

// Issuer of both passes: the steps as they come, told apart by what the producer says about them.  The tile's rows are the product's (first
// pass: K-major) or contracted (second: M-major).
template <bool SECOND>
__device__ __forceinline__ void issue_steps(RgCtrl* c, const RgRing& ring, uint32_t tmem, uint32_t acc_cols, volatile int* abort)   // (one thread)
{
    RgCursor u(ring);
    uint32_t items = 0;
    int flags;
    do {
        if (!mbar_wait(smem_u32(&c->full[u.stage]), u.phase, abort)) return;
        const RgInfo info = c->info[u.stage];
        flags = info.flags;
        const uint32_t buf = items & 1u, acc = tmem + buf * acc_cols, fresh = flags & kRgFirst ? 0u : 1u;
        if (!fresh && items >= 2 && !mbar_wait(smem_u32(&c->acc_free[buf]), ((items >> 1) & 1u) ^ 1u, abort)) return;
        if (flags & kRgTouched) {
            if (!mbar_wait(smem_u32(&c->made[u.turn % kRgTurns]), turn_phase(u.turn), abort)) return;
            ++u.turn;
        }
        tc_fence_after();
        const uint32_t low = u.at + kRgTile;
        if (SECOND) {
            const uint32_t idesc = umma_idesc_bf16(128, 3 * info.r16) | kIdescMMajorA;
            const uint64_t ad = umma_desc_m128(u.at), bd = umma_desc_k128(low), bd2 = umma_desc_k128(low + (uint32_t)info.r16 * 384u);
            if (info.valid > kTileM - 16) {
#pragma unroll
                for (int k = 0; k < 8; ++k) umma_bf16(acc, ad + (uint64_t)(k * (2048 >> 4)), (k < 4 ? bd : bd2) + (uint64_t)((k & 3) * 2), idesc, k > 0 ? 1u : fresh);
            } else {
                for (int k = 0; k * 16 < info.valid; ++k) umma_bf16(acc, ad + (uint64_t)(k * (2048 >> 4)), (k < 4 ? bd : bd2) + (uint64_t)((k & 3) * 2), idesc, k > 0 ? 1u : fresh);
            }
        } else {
            const uint32_t idesc = umma_idesc_bf16(128, info.r16);
            const uint64_t ad = umma_desc_k128(u.at), ad2 = umma_desc_k128(u.at + kRgHalfTile);
            const uint64_t bd = umma_desc_k128(low), bd2 = umma_desc_k128(low + (uint32_t)info.r16 * 128u);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                umma_bf16(acc, (k < 4 ? ad : ad2) + (uint64_t)((k & 3) * 2), (k < 4 ? bd : bd2) + (uint64_t)((k & 3) * 2), idesc, k > 0 ? 1u : fresh);
        }
        umma_commit(smem_u32(&c->empty[u.stage]));
        if (flags & kRgLast) {
            umma_commit(smem_u32(&c->acc_full[buf]));
            ++items;
        }
        u.advance();
    } while (!(flags & kRgEnd));
}

// Converting group of both passes: every second tile that is handed on.  Rows behind the last become zeros (in a bf16 tile those that share
// a step of 16 with it: another token's values times zero would be NaN where they are not finite).
template <bool E4M3>
__device__ __forceinline__ void convert_tiles(RgCtrl* c, const RgRing& ring, int group, int wt, int lane, volatile int* abort)
{
    const int ch = wt & 3, odd = (wt >> 2) & 1, row0 = wt >> 3, shift = 8 * ((wt & 7) >> 1);
    const uint32_t to0 = (uint32_t)(odd * kRgHalfTile + row0 * 128 + (((2 * ch + odd) ^ (row0 & 7)) * 16));   // (32 rows on, the swizzle is the same)
    for (int turn = group;; turn += 2) {
        const int k = turn % kRgTurns;
        bool ok = mbar_wait_warp(smem_u32(&c->turn[k]), turn_phase(turn), abort);
        __syncwarp();
        const RgTurn what = c->turns[k];
        if (ok && what.stage < 0) return;
        const int stage = what.stage < 0 ? 0 : what.stage;
        ok = ok && mbar_wait_warp(smem_u32(&c->full[stage]), (uint32_t)what.phase, abort);
        __syncwarp();
        const uint32_t at = ring.base + (uint32_t)stage * ring.stage_bytes;
        const RgInfo info = c->info[stage];
        // 16 values of a row: the 16-byte chunks 2 ch and 2 ch + 1 (of eight) of a half's row, swizzled by the row.  Lanes of the second half
        // take the odd chunk first, so that the two halves' lanes, which are 16 KB apart, do not meet on a bank.
        uint2 v[4][2];
        uint32_t byte[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t from = at + (uint32_t)(q * (kRgRaw / 4) + wt * 16);
            v[q][0] = ld_smem_v2(from + odd * 8);
            v[q][1] = ld_smem_v2(from + 8 - odd * 8);
            byte[q] = (c->words[stage][(info.word & 3) + row0 + 32 * q] >> shift) & 0xffu;
        }
        const bool usual = info.valid == kTileM && max(max(byte[0], byte[1]), max(byte[2], byte[3])) <= Decoder<E4M3>::kMost;
        if (group_any(group, !ok)) return;   // (everybody has the tile's values, so their place may be written; or a wait gave up)
        const uint32_t to = at + to0;
        if (info.word >= 0 && usual) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const Decoder<E4M3> decode(byte[q]);
                st_smem_v4(to + (uint32_t)(q * 32 * 128), decode.eight(v[q][0]));
                st_smem_v4((to ^ 16u) + (uint32_t)(q * 32 * 128), decode.eight(v[q][1]));
            }
        } else if (info.word >= 0) {
#pragma unroll 1
            for (int q = 0; q < 4; ++q) {
                const bool there = row0 + 32 * q < info.valid;
                const uint4 zero = make_uint4(0, 0, 0, 0);
                st_smem_v4(to + (uint32_t)(q * 32 * 128), there ? decode8<E4M3>(v[0][0], byte[0]) : zero);
                st_smem_v4((to ^ 16u) + (uint32_t)(q * 32 * 128), there ? decode8<E4M3>(v[0][1], byte[0]) : zero);
#pragma unroll
                for (int i = 0; i < 3; ++i) { v[i][0] = v[i + 1][0]; v[i][1] = v[i + 1][1]; byte[i] = byte[i + 1]; }
            }
        } else {
            const int rows = 16 - (info.valid & 15);
            for (int e = wt; e < rows * 16; e += 32 * kRgGroup) {
                const int row = info.valid + (e >> 4);
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
// After all finishing warps have written this CTA's partial result: whether it is the last one of the item's.
__device__ __forceinline__ bool arrive_last(RgCtrl* c, const RowsGradParams& p, const RgShare& s)
{
    __threadfence();
    finish_barrier();
    if (threadIdx.x == 64) {   // (the first of them)
        const int n = atomicAdd(p.arrived + s.first, 1);
        c->last = n == s.last - s.first;
        if (c->last) atomicExch(p.arrived + s.first, 0);   // (for the next call)
        __threadfence();
    }
    finish_barrier();
    return c->last != 0;
}
// Four values of the joined result: up to eight parts' loads in flight
__device__ __forceinline__ float4 join(const RowsGradParams& p, const RgShare& s, int at)
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

// Three bf16 values whose sum is x; an x that is not finite stands in the first alone.
__device__ __forceinline__ void split3(float x, float (&part)[3])
{
    part[0] = __bfloat162float(__float2bfloat16_rn(x));
    const float rest = fabsf(part[0]) < INFINITY ? x - part[0] : 0.f;
    part[1] = __bfloat162float(__float2bfloat16_rn(rest));
    part[2] = rest - part[1];
}

template <int FMT>
__global__ void __launch_bounds__(kRgThreads, 1) rows_shrink_kernel(const __grid_constant__ RowsGradParams p)
{
    extern __shared__ uint8_t rg_smem[];
    __shared__ RgCtrl ctrl;
    RgCtrl* c = &ctrl;
    const uint32_t smem = (smem_u32(rg_smem) + 1023u) & ~1023u;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t cols = tmem_cols_for(2 * p.r16);
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

    const RgRing ring(smem, p.ring, (uint32_t)p.r16 * 256u);
    if (w0 < w1) {
        if (warp == 0) {
            if (elect_one()) {
                RgCursor u(ring);
                const uint32_t* words_end = p.scales + (size_t)kept_groups(p.d[0]) * p.T;
                for (ShrinkTasks t(p, c, w0, w1); t.next();) {
                    const bool raw = FMT != kBf16 && t.job == 0;
                    const uint32_t* words = p.scales + (size_t)t.step * p.T + t.row;
                    const CUtensorMap* map = &p.map[t.job];
                    const int r16 = chunks_of_rank(p.snap[t.job].rank[t.slot]) * kChunk, end = t.w + t.n == w1 ? kRgLast | kRgEnd : kRgLast;
                    int flags = kRgFirst | (raw ? kRgTouched : 0), k = t.step * 128;
                    for (int left = t.n; left > 0; --left, k += 128, words += p.T, u.advance()) {
                        if (!mbar_wait(smem_u32(&c->empty[u.stage]), u.phase ^ 1u, abort)) break;
                        if (left == 1) flags |= end;
                        load_tile(c, map, u.at, u.stage, raw, t.row, k, t.valid, flags, r16, words, words_end);
                        if (raw) { post_turn(c, u.turn, u.stage, u.phase); ++u.turn; }
                        flags &= ~kRgFirst;
                    }
                }
                if (FMT != kBf16)
                    for (int k = 0; k < 2; ++k) post_turn(c, u.turn + k, -1, 0);
            }
        } else if (warp == kRgOther) {
            if (elect_one()) {
                RgCursor u(ring);
                for (ShrinkTasks t(p, c, w0, w1); t.next();) {
                    const int chunks = chunks_of_rank(p.snap[t.job].rank[t.slot]), row = t.slot * kRankPad;
                    const uint32_t half = (uint32_t)chunks * kChunk * 128u;
                    const CUtensorMap* low = &p.low[t.job][chunks - 1];
                    int k = t.step * 128;
                    for (int left = t.n; left > 0; --left, k += 128, u.advance()) {
                        if (!mbar_wait(smem_u32(&c->empty[u.stage]), u.phase ^ 1u, abort)) break;
                        const uint32_t bar = smem_u32(&c->full[u.stage]);
                        mbar_arrive_expect_tx(bar, 2 * half);
                        tma_load_2d(u.at + kRgTile, low, bar, k, row);
                        tma_load_2d(u.at + kRgTile + half, low, bar, k + 64, row);
                    }
                }
            }
        } else if (warp == 1) {
            if (elect_one()) issue_steps<false>(c, ring, tmem, (uint32_t)p.r16, abort);
        } else if (warp < kRgOther) {
            // (After a wait that gave up these warps go through the rest all the same: the counters of shared items come out right.  The
            // status word says that the results do not.)
            const int wt = tid - 64;
            uint32_t items = 0;
            for (ShrinkTasks t(p, c, w0, w1); t.next(); ++items) {
                mbar_wait_warp(smem_u32(&c->acc_full[items & 1]), (items >> 1) & 1, abort);
                __syncwarp();
                tc_fence_after();
                // The products: lane = token.
                const int r = p.snap[t.job].rank[t.slot], r16 = chunks_of_rank(r) * kChunk, row = (warp & 3) * 32 + lane;
                const float sc = p.snap[t.job].scale[t.slot];
                const bool whole = t.whole();
                const RgShare share = whole ? RgShare{0, 0, 0} : share_of(line, t.item(), p.tiles[t.job], (int)blockIdx.x);
                uint8_t* out = p.pieces[t.job] + (size_t)t.piece * kRgPiece;
                float* mine_at = p.partial + (size_t)(2 * blockIdx.x + share.slot) * kRgPartial;
                // (r16 is a multiple of 16: the swizzle goes by j alone)
                uint8_t* half = out + (size_t)(row >> 6) * (r16 * 384) + (row & 7) * 2;
                const bool there = row < t.valid;   // (rows behind the segment, columns behind the rank: whatever they hold)
                const uint32_t from = tmem + (items & 1) * (uint32_t)p.r16 + ((uint32_t)((warp & 3) * 32) << 16);
#pragma unroll 1
                for (int j = 0; j < r16; j += 4) {
                    uint32_t v[4];
                    tmem_ld_32x4(from + (uint32_t)j, v);
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (whole) {
                            float part[3];
                            split3(there && j + e < r ? __uint_as_float(v[e]) * sc : 0.f, part);
                            uint8_t* at = half + (j + e) * 128 + ((((row & 63) >> 3) ^ ((j + e) & 7)) * 16);
#pragma unroll
                            for (int k = 0; k < 3; ++k) *reinterpret_cast<__nv_bfloat16*>(at + k * r16 * 128) = __float2bfloat16_rn(part[k]);
                        } else {
                            mine_at[(j + e) * 128 + row] = __uint_as_float(v[e]);
                        }
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&c->acc_free[items & 1]));
                if (!whole && arrive_last(c, p, share)) {
                    for (int e = wt; e < r16 * 32; e += 32 * kRgFinish) {   // four tokens of one column
                        const int j = e >> 5, t4 = (e & 31) * 4;
                        const float4 v = join(p, share, e * 4);
                        const float x[4] = {v.x, v.y, v.z, v.w};
                        float part[4][3];
#pragma unroll
                        for (int i = 0; i < 4; ++i) split3(j < r && t4 + i < t.valid ? x[i] * sc : 0.f, part[i]);
#pragma unroll
                        for (int k = 0; k < 3; ++k) {
                            const int line_at = k * r16 + j;
                            *reinterpret_cast<uint2*>(out + (size_t)(t4 >> 6) * (r16 * 384) + line_at * 128 + ((((t4 & 63) >> 3) ^ (line_at & 7)) * 16) + (t4 & 4) * 2) =
                                make_uint2(pack_bf16(part[0][k], part[1][k]), pack_bf16(part[2][k], part[3][k]));
                        }
                    }
                }
            }
            fence_proxy_async_all();          // the pieces are read by bulk copies
        } else if (FMT != kBf16) {
            const int group = (warp - kRgFirstConv) / kRgGroup;
            convert_tiles<FMT == kE4m3>(c, ring, group, tid - 32 * (kRgFirstConv + group * kRgGroup), lane, abort);
        }
    }
    __syncwarp();
    if (*abort) __nanosleep(50000);   // gave up: let copies still in flight land before the CTA goes away
    __syncthreads();
    if (tid == 0 && *abort) atomicOr(p.status[0], LML_FLAG_TIMEOUT);
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, cols);
    }
}

// ---- second pass -----------------------------------------------------------------------------------------
// Items: slots in use in order, of each the column tiles (x first, then dy), of each its units.  A CTA has its part of the line, or, if
// there are few items, whole ones.
struct GradTasks {
    const RowsGradParams& p;
    const RgCtrl* c;
    unsigned long long mask;   // slots from here on
    int w, end, base = 0;   // base: of the slot at hand
    int slot = 0, units = 0, tile = 0, a = 0, b = 0;
    __device__ GradTasks(const RowsGradParams& p_, const RgCtrl* c_, int w0, int w1) : p(p_), c(c_), mask(c_->used), w(w0), end(w1) {}
    __device__ void next_slot()
    {
        base += units * p.all_tiles;
        slot = __ffsll((long long)mask) - 1;
        mask &= mask - 1ull;
        units = c->units[slot];
    }
    __device__ bool next()
    {
        if (p.whole_items) {   // w, end, base: items here
            if (b > 0) w += gridDim.x;
            if (w >= end) return false;
            while (units == 0 || w >= base + p.all_tiles) {
                if (units) base += p.all_tiles;
                slot = __ffsll((long long)mask) - 1;
                mask &= mask - 1ull;
                units = c->units[slot];
            }
            tile = (int)(w - base);
            a = 0; b = units;
            return true;
        }
        w += b - a;
        if (w >= end) return false;
        while (w >= base + units * p.all_tiles) next_slot();
        const int in = w - base;
        tile = in / units;
        a = in - tile * units;
        b = min(units, a + (end - w));
        return true;
    }
    __device__ bool whole() const { return b - a == units; }
    __device__ bool last() const { return p.whole_items ? w + gridDim.x >= end : w + (b - a) >= end; }   // of this CTA's
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

template <int FMT>
__global__ void __launch_bounds__(kRgThreads, 1) rows_grad_kernel(const __grid_constant__ RowsGradParams p)
{
    extern __shared__ uint8_t rg_smem[];
    __shared__ RgCtrl ctrl;
    RgCtrl* c = &ctrl;
    const uint32_t smem = (smem_u32(rg_smem) + 1023u) & ~1023u;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t cols = tmem_cols_for(6 * p.r16);
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
        atomicOr(&c->used, 1ull << seg.s);
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
    for (unsigned long long m = c->used; m; m &= m - 1ull) total += p.whole_items ? 1 : c->units[__ffsll((long long)m) - 1];
    const RgLine line(total * p.all_tiles);
    const int w0 = p.whole_items ? (int)blockIdx.x : line.begin((int)blockIdx.x), w1 = p.whole_items ? line.W : line.begin((int)blockIdx.x + 1);

    const RgRing ring(smem, p.ring, (uint32_t)p.r16 * 768u);
    if (w0 < w1) {
        if (warp == 0) {
            if (elect_one()) {
                RgCursor u(ring);
                const uint32_t* words_end = p.scales + (size_t)kept_groups(p.d[0]) * p.T;
                for (GradTasks t(p, c, w0, w1); t.next();) {
                    const int job = t.job(), c0 = t.column(), r16 = chunks_of_rank(p.snap[0].rank[t.slot]) * kChunk, end = t.last() ? kRgLast | kRgEnd : kRgLast;
                    const bool raw = FMT != kBf16 && job == 0;
                    const uint32_t* words = p.scales + (size_t)(c0 >> 7) * p.T;
                    const CUtensorMap* map = &p.map[job];
                    int flags = kRgFirst;
                    for (RgPieces v(c, t); v.next(); u.advance()) {
                        const int row = v.row(), valid = v.valid();
                        if (v.left == 0) flags |= end;
                        if (!mbar_wait(smem_u32(&c->empty[u.stage]), u.phase ^ 1u, abort)) break;
                        const bool touched = raw || (valid & 15);
                        load_tile(c, map, u.at, u.stage, raw, row, c0, valid, touched ? flags | kRgTouched : flags, r16, words + row, words_end);
                        if (touched) { post_turn(c, u.turn, u.stage, u.phase); ++u.turn; }
                        flags = 0;
                    }
                }
                for (int k = 0; k < 2; ++k) post_turn(c, u.turn + k, -1, 0);
            }
        } else if (warp == kRgOther) {
            if (elect_one()) {
                grid_dependency_wait();   // (the tiles are on their way meanwhile)
                fence_proxy_async_all();
                RgCursor u(ring);
                for (GradTasks t(p, c, w0, w1); t.next();) {
                    const uint32_t low = (uint32_t)(chunks_of_rank(p.snap[0].rank[t.slot]) * kChunk) * 768u;
                    const uint8_t* pieces = p.pieces[t.job() ^ 1];   // (u for dy, v for x)
                    for (RgPieces v(c, t); v.next(); u.advance()) {
                        if (!mbar_wait(smem_u32(&c->empty[u.stage]), u.phase ^ 1u, abort)) break;
                        const uint32_t bar = smem_u32(&c->full[u.stage]);
                        mbar_arrive_expect_tx(bar, low);
                        bulk_load(u.at + kRgTile, pieces + v.at(), low, bar);
                    }
                }
            }
        } else if (warp == 1) {
            if (elect_one()) issue_steps<true>(c, ring, tmem, 3u * (uint32_t)p.r16, abort);
        } else if (warp < kRgOther) {
            const int wt = tid - 64;   // (see rows_shrink_kernel)
            uint32_t items = 0;
            for (GradTasks t(p, c, w0, w1); t.next(); ++items) {
                mbar_wait_warp(smem_u32(&c->acc_full[items & 1]), (items >> 1) & 1, abort);
                __syncwarp();
                tc_fence_after();
                // The sums: lane = column.  Partial results: dA [j][column], dB [column][j].
                const int job = t.job(), c0 = t.column();
                const int r = p.snap[0].rank[t.slot], r16 = chunks_of_rank(r) * kChunk, row = (warp & 3) * 32 + lane, d = p.d[job];
                const bool whole = t.whole();
                float* dst;   // where (column, j) goes: to a partial result every one of them, to the gradients those that there are
                int stride = 1;   // between two j
                if (!whole) {
                    dst = p.partial + (size_t)(2 * blockIdx.x + (line.part_of(t.item()) == (int)blockIdx.x ? 1 : 0)) * kRgPartial + (job == 0 ? row : row * r16);
                    if (job == 0) stride = 128;
                } else if (job == 0) {
                    dst = p.out[0] + (size_t)t.slot * kRankPad * d + c0 + row;
                    stride = d;
                } else {
                    dst = p.out[1] + ((size_t)t.slot * d + c0 + row) * kRankPad;
                }
                const uint32_t from = tmem + (items & 1) * 3u * (uint32_t)p.r16 + ((uint32_t)((warp & 3) * 32) << 16);
                const bool there = !whole || c0 + row < d, add = whole && p.accumulate;
                const int most = whole ? r : r16;
#pragma unroll 1
                for (int j = 0; j < r16; j += 4) {
                    uint32_t h[4], m[4], l[4];
                    tmem_ld_32x4(from + (uint32_t)j, h);
                    tmem_ld_32x4(from + (uint32_t)(r16 + j), m);
                    tmem_ld_32x4(from + (uint32_t)(2 * r16 + j), l);
                    tmem_ld_wait();
                    float s[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[e] = __uint_as_float(h[e]) + (__uint_as_float(m[e]) + __uint_as_float(l[e]));
                    if (there && job == 1 && j + 4 <= most && !add) {
                        *reinterpret_cast<float4*>(dst) = make_float4(s[0], s[1], s[2], s[3]);
                        dst += 4;
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e, dst += stride)
                            if (there && j + e < most) *dst = add ? *dst + s[e] : s[e];
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&c->acc_free[items & 1]));
                if (whole) continue;
                const RgShare share = share_of(line, t.item(), t.units, (int)blockIdx.x);
                if (arrive_last(c, p, share)) {
                    const int per = job == 0 ? 32 : r16 / 4;   // float4 per row of the partial results
                    float* out = p.out[job] + (size_t)t.slot * kRankPad * d;
                    for (int e = wt; e < r16 * 32; e += 32 * kRgFinish) {
                        const int line_at = e / per, col = (e % per) * 4;
                        const int j = job == 0 ? line_at : col, n = c0 + (job == 0 ? col : line_at);
                        if (j >= r || n >= d) continue;
                        const float4 s = join(p, share, e * 4);
                        float* dst = job == 0 ? out + (size_t)j * d + n : out + (size_t)n * kRankPad + j;
                        if (job == 0 || j + 4 <= r) {   // (d is a multiple of 8)
                            const float4 o = p.accumulate ? *reinterpret_cast<const float4*>(dst) : make_float4(0.f, 0.f, 0.f, 0.f);
                            *reinterpret_cast<float4*>(dst) = make_float4(o.x + s.x, o.y + s.y, o.z + s.z, o.w + s.w);
                        } else {
                            const float w[3] = {s.x, s.y, s.z};   // (less than four columns)
#pragma unroll
                            for (int i = 0; i < 3; ++i)
                                if (j + i < r) dst[i] = p.accumulate ? dst[i] + w[i] : w[i];
                        }
                    }
                }
            }
        } else {
            const int group = (warp - kRgFirstConv) / kRgGroup;
            convert_tiles<FMT == kE4m3>(c, ring, group, tid - 32 * (kRgFirstConv + group * kRgGroup), lane, abort);
        }
    }
    __syncwarp();
    if (*abort) __nanosleep(50000);
    grid_dependency_wait();   // (a CTA without units too: who waits for this grid has waited for the pieces' writers)
    __syncthreads();
    if (!p.accumulate) {      // adapters without a token
        for (unsigned long long m = p.live & ~c->used; m; m &= m - 1ull) {
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
    int most = 0, live = 0;
    p.live = 0ull;
    p.snap[0] = *a.snap; p.snap[1] = *a.snap_T;
    for (int s = 0; s < a.snap->max_slots; ++s)
        if (a.snap->rank[s]) {
            most = a.snap->rank[s] > most ? a.snap->rank[s] : most;
            p.live |= 1ull << s;
            ++live;
        }
    if (live == 0) return cudaSuccess;
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
    p.arrived = a.arrived;
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
    bool ok = bf16 ? a.cache->get_2d(&p.map[0], a.x.data, (uint64_t)a.d_in, (uint64_t)a.T, (uint64_t)a.d_in * 2, 64, kTileM)
                   : a.cache->get_2d(&p.map[0], a.x.data, (uint64_t)pitch / 2, (uint64_t)a.T, (uint64_t)pitch, 64, kTileM, false);   // (8-bit rows as pairs)
    ok = ok && a.cache->get_2d(&p.map[1], a.dy, (uint64_t)a.d_out, (uint64_t)a.T, (uint64_t)a.d_out * 2, 64, kTileM);
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
        const long long pieces = (a.T + kTileM - 1) / kTileM;
        cudaError_t e = launch(shrink, pieces * p.all_tiles / kRgLeast);
        if (e != cudaSuccess) return e;
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
