// Adapter gradients of the layer, x as bf16 rows or as an 8-bit checkpoint:
//     u = s x.A^T,  v = s dy.B   (per token, with the token's adapter)        dA_s += v^T x,   dB_s += dy^T u
// Two launches, each over x and dy side by side.
//
// rows_shrink_kernel: u and v.  A piece is up to 128 rows of one segment, counted from the segment's first row (a TMA box may
// begin at any row), so no row of another segment is in it but behind its end.  A cluster of S CTAs shares the columns; partial
// products meet through distributed shared memory in rank order.
// rows_grad_kernel: a cluster of S CTAs per (128 columns, slot) deals out the slot's units of 64 rows and adds its partial
// sums the same way.
//
// Both are rings of tiles of x or dy as TMA brings them in, multiplied by tcgen05.  8-bit tiles pass through the registers of
// four warps, which write them as bf16 (exact: the scales are powers of two) in the swizzled order of the tensor cores.  The
// second product contracts over tokens: the tile [token][64 columns] is an operand whose contiguous index is the output's
// (M-major), which the descriptor says; nothing is transposed.
//
// dA and dB are fp32 and so are u and v on the way: each goes into the second product as two bf16 values (hi, lo) whose sum is
// the fp32 value to 2^-17, side by side as 2r columns of one product.  One bf16 value would leave 2^-9, 1e-3 of every gradient.
//
// Bound by memory: x and dy leave HBM once (the second pass finds them in L2 up to about 100 MB).
#include <cstring>

#include "lml_ptx_sm100.cuh"
#include "lml_rows_grad.cuh"

namespace lml {

using namespace ptx;

constexpr int kRgThreads = 192;                 // producer, issuer, four warps that convert and finish
constexpr int kRgTile = 128 * 128;              // bytes of a multiplied tile: 128 x 64 bf16 (first pass), 2 x 64 x 64 (second)
constexpr int kRgRaw = 128 * 64;                // ... of the 8-bit tile it is made of
constexpr int kRgHalf = 2 * kRankPad * 128;     // bytes of u (or v) of 64 tokens: hi rows, lo rows, 64 tokens each
constexpr int kRgPiece = 2 * kRgHalf;
constexpr int kRgMaxStages = 4;
constexpr int kRgList = 192;                    // segments of a slot looked at a time

struct alignas(64) RowsGradParams {
    CUtensorMap map[2];       // x, dy: boxes of 64 columns x 64 rows
    CUtensorMap low[2];       // the packed A of the table, B^T of the transposed one
    SlotSnapshot snap[2];     // table, transposed table
    const uint32_t* scales;   // of x
    const int32_t *seg_offsets, *ids, *ids_T;
    uint32_t* status[2];
    uint8_t* pieces[2];       // u, v
    float* out[2];            // dA, dB
    int d[2];                 // d_in, d_out
    int T, G, format, r16, stages, S, accumulate, tiles0;
    unsigned long long live;  // slots with an adapter
};

struct RgCtrl {
    unsigned long long full[kRgMaxStages], made[kRgMaxStages], empty[kRgMaxStages], done;
    unsigned long long used;
    uint32_t tmem_base;
    int abort, count[6], n;
    int first[kRgList], len[kRgList], piece[kRgList];
};

__device__ __forceinline__ uint64_t umma_desc_m128(uint32_t smem_addr)   // 64 contiguous M per 128-byte swizzled row, rows along K
{
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(8192 >> 4) << 16;                    // to the next 64 of M
    d |= (uint64_t)(1024 >> 4) << 32;                    // to the next 8 of K
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
constexpr uint32_t kIdescMMajorA = 1u << 15;

// 16 columns of 32 lanes
__device__ __forceinline__ void tmem_ld_32x16(uint32_t taddr, uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ float4 ld_peer_v4(uint32_t cluster_addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(cluster_addr) : "memory");
    return v;
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
__device__ __forceinline__ void st_smem_f32(uint32_t a, float v) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(a), "f"(v) : "memory"); }

// 16 values of the 8-bit tile at `raw` -> two 16-byte chunks, 2 ch and 2 ch + 1, of the 128-byte row at `row_at` (row: its number, for
// the swizzle)
__device__ __forceinline__ void convert16(uint32_t raw, uint32_t row_at, int row, int ch, float s, bool e4m3, bool keep)
{
    uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
    if (keep) {
        const uint4 q = ld_smem_v4(raw);
        lo = decode8_bf16(make_uint2(q.x, q.y), s, e4m3);
        hi = decode8_bf16(make_uint2(q.z, q.w), s, e4m3);
    }
    st_smem_v4(row_at + (uint32_t)(((2 * ch) ^ (row & 7)) * 16), lo);
    st_smem_v4(row_at + (uint32_t)(((2 * ch + 1) ^ (row & 7)) * 16), hi);
}

// Whether segment g's two bindings name one adapter in both tables.
__device__ __forceinline__ bool paired(const RowsGradParams& p, int s, int sT)
{
    const int r = slot_rank(p.snap[0], s);
    return r > 0 && r == slot_rank(p.snap[1], sT);
}

__device__ __forceinline__ void rg_setup(RgCtrl* c, int stages, int warp, int tid, uint32_t cols)
{
    if (tid == 0) {
        c->abort = 0;
        c->used = 0ull;
        for (int i = 0; i < stages; ++i) {
            mbar_init(smem_u32(&c->full[i]), 1);
            mbar_init(smem_u32(&c->made[i]), 4);
            mbar_init(smem_u32(&c->empty[i]), 1);
        }
        mbar_init(smem_u32(&c->done), 1);
        fence_mbar_init();
    }
    if (warp == 1) tmem_alloc(smem_u32(&c->tmem_base), cols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    grid_launch_dependents();   // (after the allocation: what starts from here on may want TMEM and waits for this grid)
    grid_dependency_wait();
}
__device__ __forceinline__ uint32_t tmem_cols_for(int n) { return n <= 32 ? 32u : n <= 64 ? 64u : 128u; }

__global__ void __launch_bounds__(kRgThreads) rows_shrink_kernel(const __grid_constant__ RowsGradParams p)
{
    extern __shared__ uint8_t rg_smem[];
    __shared__ RgCtrl ctrl;
    RgCtrl* c = &ctrl;
    const uint32_t ring = (smem_u32(rg_smem) + 1023u) & ~1023u;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int job = blockIdx.y, S = p.S, rank = (int)cluster_ctarank();
    const int b = (int)(blockIdx.x / (unsigned)S);
    const uint32_t cols = tmem_cols_for(p.r16);
    rg_setup(c, p.stages, warp, tid, cols);
    const uint32_t tmem = c->tmem_base;
    volatile int* abort = &c->abort;

    // One CTA checks the arrays for the whole call.
    if (blockIdx.x == 0 && job == 0) {
        uint32_t f = 0, fT = 0;
        for (int g = tid; g < p.G; g += kRgThreads) {
            const int s0 = ld_after_wait(p.seg_offsets + g), s1 = ld_after_wait(p.seg_offsets + g + 1);
            if (s1 < s0 || s0 < 0 || s1 > p.T) f |= LML_FLAG_BAD_OFFSETS;
            const int s = ld_after_wait(p.ids + g), sT = ld_after_wait(p.ids_T + g);
            if (s1 <= s0 || (s == -1 && sT == -1)) continue;
            if (slot_rank(p.snap[0], s) == 0) f |= LML_FLAG_BAD_SLOT;
            if (slot_rank(p.snap[1], sT) != slot_rank(p.snap[0], s)) fT |= LML_FLAG_BAD_SLOT;
        }
        if (tid == 0 && (ld_after_wait(p.seg_offsets) != 0 || ld_after_wait(p.seg_offsets + p.G) != p.T)) f |= LML_FLAG_BAD_OFFSETS;
        if (f) atomicOr(p.status[0], f);
        if (fT) atomicOr(p.status[1], fT);
    }

    // Piece b: the largest g whose first piece, s0 / 128 + g, is not behind b.  (Pieces of a segment are never more than lie
    // between its first and the next one's; the arrays may be malformed, so everything is clamped.)
    int p0 = 0, valid = 0, slot = -1;
    {
        int lo = 0, hi = p.G;
        if (p.G <= kRgList) {
            for (int g = tid; g < p.G; g += kRgThreads) c->first[g] = ld_after_wait(p.seg_offsets + g);
            __syncthreads();
        }
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            const int s0 = p.G <= kRgList ? c->first[mid] : ld_after_wait(p.seg_offsets + mid);
            if (mid + s0 / kTileM <= b) lo = mid; else hi = mid;
        }
        const long long s0 = ld_after_wait(p.seg_offsets + lo), s1 = ld_after_wait(p.seg_offsets + lo + 1);
        const long long first = s0 + (b - (s0 / kTileM + lo)) * (long long)kTileM, end = s1 < p.T ? s1 : p.T;
        const int s = ld_after_wait(p.ids + lo), sT = ld_after_wait(p.ids_T + lo);
        if (s0 >= 0 && first >= s0 && first < end && paired(p, s, sT)) {
            p0 = (int)first;
            valid = (int)(end - first < kTileM ? end - first : kTileM);
            slot = job == 0 ? s : sT;
        }
    }
    if (valid > 0) {   // (the same in all CTAs of the cluster)
        const SlotSnapshot& snap = p.snap[job];
        const int r = snap.rank[slot], r16 = chunks_of_rank(r) * kChunk;
        const int nkb = (p.d[job] + 63) / 64, kb0 = nkb * rank / S, n = nkb * (rank + 1) / S - kb0;
        const bool raw = job == 0 && p.format != kBf16;
        const uint32_t low_bytes = (uint32_t)p.r16 * 128u, stage_bytes = kRgTile + low_bytes + (p.format != kBf16 ? kRgRaw : 0);
        if (warp == 0) {
            if (elect_one()) {
                for (int i = 0; i < n; ++i) {
                    const int st = i % p.stages;
                    if (!mbar_wait(smem_u32(&c->empty[st]), ((i / p.stages) & 1) ^ 1, abort)) break;
                    const uint32_t at = ring + st * stage_bytes, bar = smem_u32(&c->full[st]);
                    const int k = (kb0 + i) * 64, boxes = valid > 64 ? 2 : 1;
                    mbar_arrive_expect_tx(bar, (uint32_t)(r16 * 128 + boxes * (raw ? kRgRaw / 2 : kRgTile / 2)));
                    for (int h = 0; h < boxes; ++h) {
                        if (raw) tma_load_2d(at + kRgTile + low_bytes + h * (kRgRaw / 2), &p.map[job], bar, k / 2, p0 + h * 64);
                        else tma_load_2d(at + h * (kRgTile / 2), &p.map[job], bar, k, p0 + h * 64);
                    }
                    for (int j = 0; j < r16; j += kChunk) tma_load_3d(at + kRgTile + j * 128, &p.low[job], bar, k, j, slot);
                }
            }
        } else if (warp == 1) {
            if (elect_one()) {
                const uint32_t idesc = umma_idesc_bf16(128, r16);
                bool ok = true;
                for (int i = 0; i < n; ++i) {
                    const int st = i % p.stages;
                    ok = mbar_wait(smem_u32(&c->full[st]), (i / p.stages) & 1, abort) && (!raw || mbar_wait(smem_u32(&c->made[st]), (i / p.stages) & 1, abort));
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t at = ring + st * stage_bytes;
                    const uint64_t ad = umma_desc_k128(at), bd = umma_desc_k128(at + kRgTile);
#pragma unroll
                    for (int k = 0; k < 4; ++k) umma_bf16(tmem, ad + (uint64_t)(k * 2), bd + (uint64_t)(k * 2), idesc, (i > 0 || k > 0) ? 1u : 0u);
                    umma_commit(smem_u32(&c->empty[st]));
                }
                if (ok && n > 0) umma_commit(smem_u32(&c->done));
            }
        } else if (raw) {
            const int wt = tid - 64, ch = wt & 3;
            const bool e4m3 = p.format == kE4m3;
            uint32_t word[4], next[4];
            auto fetch = [&](int i, uint32_t (&w)[4]) {
                const long long cg = (kb0 + i) >> 1;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int row = q * 32 + (wt >> 2);
                    w[q] = i < n && row < valid ? ld_after_wait(p.scales + cg * p.T + p0 + row) : 0u;
                }
            };
            fetch(0, next);
            for (int i = 0; i < n; ++i) {
                const int st = i % p.stages;
#pragma unroll
                for (int q = 0; q < 4; ++q) word[q] = next[q];
                fetch(i + 1, next);
                if (!mbar_wait_warp(smem_u32(&c->full[st]), (i / p.stages) & 1, abort)) break;
                __syncwarp();
                const uint32_t at = ring + st * stage_bytes;
                const int byte = ((kb0 + i) & 1) * 2 + (ch >> 1);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int row = q * 32 + (wt >> 2);
                    convert16(at + kRgTile + low_bytes + row * 64 + ch * 16, at + row * 128, row, ch,
                              scale_of_byte((word[q] >> (8 * byte)) & 0xffu), e4m3, row < valid);
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&c->made[st]));
            }
        }
        __syncwarp();
        bool ok = true;
        if (warp >= 2 && n > 0) {
            ok = mbar_wait_warp(smem_u32(&c->done), 0, abort);
            if (!ok) __nanosleep(50000);   // gave up: let copies still in flight land before the ring takes the partial sums
            __syncwarp();
            tc_fence_after();
        }
        // partial products [column][token]: the ring is idle in this CTA from here on
        if (warp >= 2) {
            const int row = (warp & 3) * 32 + lane;
            for (int j = 0; j < r16; j += 16) {
                uint32_t v[16];
                tmem_ld_32x16(tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)j, v);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; ++e) st_smem_f32(ring + (uint32_t)(((j + e) * 128 + row) * 4), n > 0 && ok ? __uint_as_float(v[e]) : 0.f);
            }
            tc_fence_before();
        }
        cluster_sync_all();
        const float sc = snap.scale[slot];
        uint8_t* out = p.pieces[job] + (size_t)b * kRgPiece;
        for (int e = rank * kRgThreads + tid; e < r16 * 16; e += S * kRgThreads) {   // eight tokens of one column
            const int j = e >> 4, t8 = e & 15;
            float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            for (int q = 0; q < S; ++q) {   // rank order: the sum does not depend on timing
                const uint32_t from = mapa_shared(ring + (uint32_t)((j * 128 + t8 * 8) * 4), (uint32_t)q);
                const float4 a = ld_peer_v4(from), d = ld_peer_v4(from + 16);
                v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
                v[4] += d.x; v[5] += d.y; v[6] += d.z; v[7] += d.w;
            }
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float x[2], l[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    x[k] = j < r && t8 * 8 + 2 * i + k < valid ? v[2 * i + k] * sc : 0.f;   // (rows behind the segment, columns behind the rank: whatever they hold)
                    const float h = __bfloat162float(__float2bfloat16_rn(x[k]));
                    l[k] = fabsf(h) < INFINITY ? x[k] - h : 0.f;
                }
                hi[i] = pack_bf16(x[0], x[1]);
                lo[i] = pack_bf16(l[0], l[1]);
            }
            uint8_t* half = out + (size_t)(t8 >> 3) * kRgHalf;
            const int jl = r16 + j;
            *reinterpret_cast<uint4*>(half + j * 128 + (((t8 & 7) ^ (j & 7)) * 16)) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            *reinterpret_cast<uint4*>(half + jl * 128 + (((t8 & 7) ^ (jl & 7)) * 16)) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
        fence_proxy_async_all();   // the pieces are read by bulk copies
        if (tid == 0 && *abort) atomicOr(p.status[0], LML_FLAG_TIMEOUT);
        cluster_sync_all();        // peers stay until their partial products have been read
    }
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, cols);
    }
}

__global__ void __launch_bounds__(kRgThreads) rows_grad_kernel(const __grid_constant__ RowsGradParams p)
{
    extern __shared__ uint8_t rg_smem[];
    __shared__ RgCtrl ctrl;
    RgCtrl* c = &ctrl;
    const uint32_t ring = (smem_u32(rg_smem) + 1023u) & ~1023u;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int S = p.S, rank = (int)cluster_ctarank(), tile = (int)(blockIdx.x / (unsigned)S);
    const int job = tile < p.tiles0 ? 0 : 1, c0 = (job == 0 ? tile : tile - p.tiles0) * 128;
    const uint32_t cols = tmem_cols_for(2 * p.r16);
    rg_setup(c, p.stages, warp, tid, cols);
    const uint32_t tmem = c->tmem_base;
    volatile int* abort = &c->abort;

    // The slots in use, and whether the arrays hold together (if not, nothing is added).
    int bad = p.T == 0 ? 1 : 0;
    for (int g = tid; g < p.G && p.T > 0; g += kRgThreads) {
        const int s0 = ld_after_wait(p.seg_offsets + g), s1 = ld_after_wait(p.seg_offsets + g + 1);
        if (s1 < s0 || s0 < 0 || s1 > p.T) bad = 1;
        const int s = ld_after_wait(p.ids + g);
        if (s1 > s0 && paired(p, s, ld_after_wait(p.ids_T + g))) atomicOr(&c->used, 1ull << s);
    }
    if (tid == 0 && p.T > 0 && (ld_after_wait(p.seg_offsets) != 0 || ld_after_wait(p.seg_offsets + p.G) != p.T)) bad = 1;
    bad = __syncthreads_or(bad);
    unsigned long long mask = p.accumulate ? (bad ? 0ull : c->used) : p.live;
    for (int z = blockIdx.y; z > 0 && mask; --z) mask &= mask - 1ull;
    if (mask) {   // (the same in all CTAs of the cluster)
        const int slot = __ffsll((long long)mask) - 1;
        const int r = p.snap[0].rank[slot], r16 = chunks_of_rank(r) * kChunk;
        const bool raw = job == 0 && p.format != kBf16;
        const uint32_t low_bytes = (uint32_t)p.r16 * 256u, stage_bytes = kRgTile + low_bytes + (p.format != kBf16 ? kRgRaw : 0);
        int it = 0;      // units that this CTA has taken; the same in every role
        int unit = 0;    // units of the slot before the list's
        for (int g0 = 0; g0 < p.G && !bad; g0 += kRgThreads) {
            // the slot's segments among the next 192, in order
            const int g = g0 + tid;
            int s0 = 0, s1 = 0;
            bool mine = false;
            if (g < p.G && ld_after_wait(p.ids + g) == slot) {
                s0 = ld_after_wait(p.seg_offsets + g);
                s1 = ld_after_wait(p.seg_offsets + g + 1);
                mine = s1 > s0 && paired(p, slot, ld_after_wait(p.ids_T + g));
            }
            const uint32_t ballot = __ballot_sync(0xffffffffu, mine);
            if (lane == 0) c->count[warp] = __popc(ballot);
            __syncthreads();
            int before = 0, total = 0;
#pragma unroll
            for (int w = 0; w < kRgThreads / 32; ++w) {
                before += w < warp ? c->count[w] : 0;
                total += c->count[w];
            }
            if (mine) {
                const int at = before + __popc(ballot & ((1u << lane) - 1u));
                c->first[at] = s0; c->len[at] = s1 - s0; c->piece[at] = s0 / kTileM + g;
            }
            __syncthreads();
            if (total == 0) continue;
            // Every role walks the same units: f(row, valid rows, piece, half)
            auto walk = [&](auto&& f) {
                int i = it, base = unit;
                for (int e = 0; e < total; ++e) {
                    const int units = (c->len[e] + 63) / 64;
                    int k = rank - base % S;
                    if (k < 0) k += S;
                    for (; k < units; k += S, ++i) {
                        const int left = c->len[e] - k * 64;
                        if (!f(i, c->first[e] + k * 64, left < 64 ? left : 64, c->piece[e] + (k >> 1), k & 1)) return i;
                    }
                    base += units;
                }
                return i;
            };
            if (warp == 0) {
                if (elect_one()) {
                    walk([&](int i, int row, int, int piece, int half) {
                        const int st = i % p.stages;
                        if (!mbar_wait(smem_u32(&c->empty[st]), ((i / p.stages) & 1) ^ 1, abort)) return false;
                        const uint32_t at = ring + st * stage_bytes, bar = smem_u32(&c->full[st]);
                        mbar_arrive_expect_tx(bar, (uint32_t)(r16 * 256 + (raw ? kRgRaw : kRgTile)));
                        for (int h = 0; h < 2; ++h) {
                            if (raw) tma_load_2d(at + kRgTile + low_bytes + h * (kRgRaw / 2), &p.map[job], bar, (c0 + h * 64) / 2, row);
                            else tma_load_2d(at + h * (kRgTile / 2), &p.map[job], bar, c0 + h * 64, row);
                        }
                        // (u for dy, v for x)
                        bulk_load(at + kRgTile, p.pieces[job ^ 1] + (size_t)piece * kRgPiece + (size_t)half * kRgHalf, (uint32_t)(r16 * 256), bar);
                        return true;
                    });
                }
            } else if (warp == 1) {
                if (elect_one()) {
                    const uint32_t idesc = umma_idesc_bf16(128, 2 * r16) | kIdescMMajorA;
                    walk([&](int i, int, int valid, int, int) {
                        const int st = i % p.stages, ph = (i / p.stages) & 1;
                        if (!mbar_wait(smem_u32(&c->full[st]), ph, abort) || !mbar_wait(smem_u32(&c->made[st]), ph, abort)) return false;
                        tc_fence_after();
                        const uint32_t at = ring + st * stage_bytes;
                        const uint64_t ad = umma_desc_m128(at), bd = umma_desc_k128(at + kRgTile);
                        for (int k = 0; k * 16 < valid; ++k)
                            umma_bf16(tmem, ad + (uint64_t)(k * (2048 >> 4)), bd + (uint64_t)(k * 2), idesc, (i > 0 || k > 0) ? 1u : 0u);
                        umma_commit(smem_u32(&c->empty[st]));
                        return true;
                    });
                }
            } else {
                const int wt = tid - 64;
                const bool e4m3 = p.format == kE4m3;
                const uint32_t* scales = p.scales + (size_t)(c0 >> 7) * p.T;
                walk([&](int i, int row0, int valid, int, int) {
                    const int st = i % p.stages;
                    const uint32_t at = ring + st * stage_bytes;
                    uint32_t word[2];
                    if (raw) {
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const int row = q * 32 + (wt >> 2);
                            word[q] = row < valid ? ld_after_wait(scales + row0 + row) : 0u;
                        }
                    }
                    if (!mbar_wait_warp(smem_u32(&c->full[st]), (i / p.stages) & 1, abort)) return false;
                    __syncwarp();
                    if (raw) {
                        const int ch = wt & 3;
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int q = 0; q < 2; ++q) {
                                const int row = q * 32 + (wt >> 2);
                                convert16(at + kRgTile + low_bytes + h * (kRgRaw / 2) + row * 64 + ch * 16, at + h * (kRgTile / 2) + row * 128, row, ch,
                                          scale_of_byte((word[q] >> (8 * (h * 2 + (ch >> 1)))) & 0xffu), e4m3, row < valid);
                            }
                        fence_proxy_async_smem();
                    } else if (valid & 15) {
                        // rows behind the segment's end that share a step of 16 with its last ones: another token's values times
                        // zero would be NaN where they are not finite
                        const int rows = 16 - (valid & 15);
                        for (int e = wt; e < rows * 16; e += 128) {
                            const int row = valid + (e >> 4);
                            st_smem_v4(at + ((e >> 3) & 1) * (kRgTile / 2) + row * 128 + (e & 7) * 16, make_uint4(0, 0, 0, 0));
                        }
                        fence_proxy_async_smem();
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&c->made[st]));
                    return true;
                });
            }
            int base = unit;
            for (int e = 0; e < total; ++e) {   // where everybody stands after this list
                const int units = (c->len[e] + 63) / 64;
                int k = rank - base % S;
                if (k < 0) k += S;
                if (k < units) it += (units - k + S - 1) / S;
                base += units;
            }
            unit = base;
            __syncwarp();
            __syncthreads();   // (the list is written anew)
        }
        if (warp == 1 && it > 0 && !*abort) {
            if (elect_one()) umma_commit(smem_u32(&c->done));
        }
        __syncwarp();
        bool ok = true;
        if (warp >= 2 && it > 0) {
            ok = mbar_wait_warp(smem_u32(&c->done), 0, abort);
            if (!ok) __nanosleep(50000);
            __syncwarp();
            tc_fence_after();
        }
        // partial sums: dA [j][column], dB [column][j]
        const int pitch = job == 0 ? 128 : r16 + 4;
        if (warp >= 2) {
            const int row = (warp & 3) * 32 + lane;
            const uint32_t from = tmem + ((uint32_t)((warp & 3) * 32) << 16);
            for (int j = 0; j < r16; j += 16) {
                uint32_t hi[16], lo[16];
                tmem_ld_32x16(from + (uint32_t)j, hi);
                tmem_ld_32x16(from + (uint32_t)(r16 + j), lo);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float v = it > 0 && ok ? __uint_as_float(hi[e]) + __uint_as_float(lo[e]) : 0.f;
                    st_smem_f32(ring + (uint32_t)((job == 0 ? (j + e) * pitch + row : row * pitch + j + e) * 4), v);
                }
            }
            tc_fence_before();
        }
        cluster_sync_all();
        const int d = p.d[job], per = job == 0 ? 32 : r16 / 4;   // float4 per row of the partial sums
        float* out = p.out[job] + (size_t)slot * kRankPad * d;
        for (int e = rank * kRgThreads + tid; e < (job == 0 ? r16 : 128) * per; e += S * kRgThreads) {
            const int row = e / per, col = (e % per) * 4;
            const int j = job == 0 ? row : col, n = c0 + (job == 0 ? col : row);
            if (j >= r || n >= d) continue;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int q = 0; q < S; ++q) {
                const float4 w = ld_peer_v4(mapa_shared(ring + (uint32_t)((row * pitch + col) * 4), (uint32_t)q));
                v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
            }
            float* dst = job == 0 ? out + (size_t)j * d + n : out + (size_t)n * kRankPad + j;
            if (job == 0 || j + 4 <= r) {   // (d is a multiple of 8)
                if (p.accumulate) {
                    const float4 o = *reinterpret_cast<const float4*>(dst);
                    v = make_float4(o.x + v.x, o.y + v.y, o.z + v.z, o.w + v.w);
                }
                *reinterpret_cast<float4*>(dst) = v;
            } else {
                const float w[4] = {v.x, v.y, v.z, v.w};
                for (int i = 0; j + i < r; ++i) dst[i] = p.accumulate ? dst[i] + w[i] : w[i];
            }
        }
        if (tid == 0 && *abort) atomicOr(p.status[0], LML_FLAG_TIMEOUT);
        cluster_sync_all();
    }
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, cols);
    }
}

// ---- host ---------------------------------------------------------------------------------------------
size_t rows_grad_ws_bytes(int T, int G) { return 2 * ((size_t)T / kTileM + (size_t)G) * kRgPiece; }

constexpr int kRgSmemMax = 1024 + 108 * 1024;   // two CTAs to an SM

cudaError_t rows_grad_init()
{
    cudaError_t e = cudaFuncSetAttribute(rows_shrink_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRgSmemMax);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(rows_grad_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRgSmemMax);
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
    if (live == 0) most = 1;
    p.r16 = chunks_of_rank(most) * kChunk;
    p.d[0] = a.d_in; p.d[1] = a.d_out;
    p.T = a.T; p.G = a.G; p.format = a.x.format; p.accumulate = a.accumulate ? 1 : 0;
    p.scales = a.x.scales;
    p.seg_offsets = a.seg_offsets; p.ids = a.ids; p.ids_T = a.ids_T;
    p.status[0] = a.status; p.status[1] = a.status_T;
    const size_t blocks = (size_t)a.T / kTileM + (size_t)a.G;
    p.pieces[0] = static_cast<uint8_t*>(a.workspace);
    p.pieces[1] = p.pieces[0] + blocks * kRgPiece;
    p.out[0] = a.dA; p.out[1] = a.dB;
    p.tiles0 = (a.d_in + 127) / 128;
    const int tiles = p.tiles0 + (a.d_out + 127) / 128;
    p.low[0] = *a.tmap_A; p.low[1] = *a.tmap_AT;
    if (a.T > 0) {
        const int pitch = kept_pitch(a.d_in);
        const bool ok = a.x.format == kBf16 ? a.cache->get_2d(&p.map[0], a.x.data, (uint64_t)a.d_in, (uint64_t)a.T, (uint64_t)a.d_in * 2, 64, 64)
                                            : a.cache->get_2d(&p.map[0], a.x.data, (uint64_t)pitch / 2, (uint64_t)a.T, (uint64_t)pitch, 32, 64, false);
        if (!ok || !a.cache->get_2d(&p.map[1], a.dy, (uint64_t)a.d_out, (uint64_t)a.T, (uint64_t)a.d_out * 2, 64, 64)) return cudaErrorInvalidValue;
    } else {
        memset(p.map, 0, sizeof(p.map));
    }
    const int raw = a.x.format != kBf16 ? kRgRaw : 0;
    auto config = [&](cudaLaunchConfig_t& cfg, cudaLaunchAttribute (&attr)[2], dim3 grid, int stage) {
        p.stages = (kRgSmemMax - 1024) / stage;
        if (p.stages > kRgMaxStages) p.stages = kRgMaxStages;
        pdl_config(cfg, attr, grid, dim3(kRgThreads), (size_t)(1024 + p.stages * stage), stream);
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)p.S;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    };
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    if (a.T > 0 && live > 0) {
        cfg = {};
        p.S = 8;
        while (p.S > 2 && (long long)blocks * 2 * p.S > 8ll * a.num_sms) p.S >>= 1;
        config(cfg, attr, dim3((unsigned)(blocks * p.S), 2), kRgTile + p.r16 * 128 + raw);
        const cudaError_t e = cudaLaunchKernelEx(&cfg, rows_shrink_kernel, p);
        if (e != cudaSuccess) return e;
        ++*launches;
    }
    const int z = !a.accumulate ? live : (a.G < live ? a.G : live);
    if (z > 0 && (a.T > 0 || !a.accumulate)) {
        cfg = {};
        p.S = 8;
        while (p.S > 1 && ((a.T + 63) / 64 < p.S || (long long)tiles * z * p.S > 8ll * a.num_sms)) p.S >>= 1;
        config(cfg, attr, dim3((unsigned)(tiles * p.S), (unsigned)z), kRgTile + p.r16 * 256 + raw);
        const cudaError_t e = cudaLaunchKernelEx(&cfg, rows_grad_kernel, p);
        if (e != cudaSuccess) return e;
        ++*launches;
    }
    return cudaSuccess;
}

}  // namespace lml
