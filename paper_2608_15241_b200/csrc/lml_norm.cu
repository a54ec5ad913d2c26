// The norms between two blocks, forward and backward.  With o the block's output, h the residual stream, a the residual
// scale and g the gate (one row for all tokens, or a row per token):
//     n = o r w_post,  r = (mean o^2 + eps)^-1/2        h' = h + a g n        x = h' rho w_pre,  rho = (mean h'^2 + eps)^-1/2
// h' is rounded to bf16 once, as it is kept, and normed as it is kept: x is what a call on h' alone gives, bit for bit, and
// what the backward pass differentiates.  Backward, with hh = h' rho, oo = o r and D the whole gradient of h':
//     D = dh' + rho (dx w_pre - hh mean(dx w_pre hh))          dw_pre += sum dx hh
//     dn = a g D                                               dgate += sum a D n  (or a row per token)
//     do = r (dn w_post - oo mean(dn w_post oo))               dw_post += sum dn oo
// Everything is in fp32 between the bf16 of inputs and outputs; sums over tokens are added in an order that the sizes fix.
//
// A group of W warps holds a row in registers, V vectors of eight columns per thread, so every tensor is read and written
// once: bound by memory.
#include <atomic>
#include <cstdlib>
#include <type_traits>

#include "lml_rows.cuh"
#include "lml_ptx_sm100.cuh"

namespace lml {

__device__ __forceinline__ void unpack8(const uint4& v, float (&f)[8])
{
    f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
    f[4] = bf16_lo(v.z); f[5] = bf16_hi(v.z); f[6] = bf16_lo(v.w); f[7] = bf16_hi(v.w);
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8])
{
    return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}
// Sum over the W warps of a row's group; `red` is a slot of W floats that no other sum of the row uses.
template <int W>
__device__ __forceinline__ float group_sum(float v, float* red, int group, int warp, int lane)
{
#pragma unroll
    for (int m = 16; m; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
    if (W == 1) return v;
    if (lane == 0) red[warp] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(W * 32) : "memory");
    v = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) v += red[w];
    return v;
}

template <int W> struct NormShape {
    static constexpr int kGroups = W > 8 ? 1 : 8 / W, kWarps = W * kGroups;
};

// W: warps of a row (a number that the compiler knows takes a tenth less than one that it does not, 8192 x 4096).  AHEAD: the weights are asked for
// along with the row.
// Four vectors per thread: 64 registers at most, 32 warps on an SM.  (Nothing is asked of the other kernels, with one CTA asked for
// they take a third more registers.)
template <int W, int V, bool AHEAD>
__global__ void __launch_bounds__(NormShape<W>::kWarps * 32, V == 4 && !AHEAD ? 32 / NormShape<W>::kWarps : 0) block_norm_kernel(const __grid_constant__ NormForward a)
{
    __shared__ float red[2][NormShape<W>::kWarps];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int T = a.n.T, d = a.n.d, vecs = d >> 3;
    const int group = threadIdx.x / (W * 32), in = threadIdx.x % (W * 32), warp = in >> 5, lane = in & 31;
    const long long t = (long long)blockIdx.x * NormShape<W>::kGroups + group;
    if (t >= T) return;   // (whole groups leave)
    float* red0 = red[0] + group * W;
    float* red1 = red[1] + group * W;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    auto at = [&](const void* p, int vec) { return static_cast<const __nv_bfloat16*>(p) + t * d + vec * 8; };

    uint4 h[V], o[V], w_post[AHEAD ? V : 1], gate[AHEAD ? V : 1], w_pre[AHEAD ? V : 1];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int vec = i * W * 32 + in;
        const bool ok = vec < vecs, ok_o = ok && a.o;
        h[i] = ok ? ld_v4(at(a.h, vec)) : zero;
        o[i] = ok_o ? ld_v4(at(a.o, vec)) : zero;
        if (!AHEAD) continue;
        gate[i] = ok_o && a.n.gate_rows ? ld_v4(at(a.n.gate_rows, vec)) : ok_o && a.n.gate ? ld_weights(a.n.gate, vec) : zero;
        w_post[i] = ok_o && a.n.w_post ? ld_weights(a.n.w_post, vec) : zero;
        w_pre[i] = ok && a.n.w_pre ? ld_weights(a.n.w_pre, vec) : zero;
    }
    if (a.o) {
        float r = 1.f;
        if (a.n.w_post) {
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float f[8];
                unpack8(o[i], f);
#pragma unroll
                for (int e = 0; e < 8; ++e) ss = fmaf(f[e], f[e], ss);
            }
            r = __frsqrt_rn(group_sum<W>(ss, red0, group, warp, lane) / (float)d + a.n.eps);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int vec = i * W * 32 + in;
            if (vec >= vecs) continue;
            float f[8], n[8], w[8];
            unpack8(h[i], f);
            unpack8(o[i], n);
            if (a.n.w_post) {
                unpack8(AHEAD ? w_post[i] : ld_weights(a.n.w_post, vec), w);
#pragma unroll
                for (int e = 0; e < 8; ++e) n[e] *= r * w[e];
            }
            if (a.n.gate || a.n.gate_rows) {
                unpack8(AHEAD ? gate[i] : a.n.gate_rows ? ld_v4(at(a.n.gate_rows, vec)) : ld_weights(a.n.gate, vec), w);
#pragma unroll
                for (int e = 0; e < 8; ++e) n[e] *= w[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = fmaf(a.n.scale, n[e], f[e]);
            h[i] = pack8(f);
            if (a.h_new) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.h_new) + t * d + vec * 8) = h[i];
        }
    }
    if (a.h_kept.data) {
#pragma unroll
        for (int i = 0; i < V; ++i) store_kept(a.h_kept, T, d, t, i * W * 32 + in, h[i]);
    }
    if (!a.n.w_pre) return;
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        float f[8];
        unpack8(h[i], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(f[e], f[e], ss);
    }
    const float rho = __frsqrt_rn(group_sum<W>(ss, red1, group, warp, lane) / (float)d + a.n.eps);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int vec = i * W * 32 + in;
        if (vec < vecs) {
            float f[8], w[8];
            unpack8(h[i], f);
            unpack8(AHEAD ? w_pre[i] : ld_weights(a.n.w_pre, vec), w);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] *= rho * w[e];
            h[i] = pack8(f);
            if (a.x) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.x) + t * d + vec * 8) = h[i];
        }
        if (a.x_kept.data) store_kept(a.x_kept, T, d, t, vec, h[i]);
    }
}

// ---- backward ---------------------------------------------------------------------------------------
// One CTA per SM walks rows with the stride of the grid, groups of W warps taking them in turn.  Every group has a ring in shared memory
// that its warps fill, by bulk copies, with whole rows of all inputs, so that 100 KB and more are in flight whatever the arithmetic does, and
// keeps its share of the sums over tokens in registers: of dx hh, and of D oo (times the token's gate, if it has one of its
// own): dw_post is a times the latter times the channel's gate, dgate a times it times w_post.  The groups of a CTA add
// theirs in shared memory, CTAs write partial sums that a second launch adds up.
// What bounds it next to memory is the number of instructions and the wait at a row's sums.  So a row has one meeting of its warps: with
// z = a g w_post o, the mean that do asks for is that of D z = dh' z + rho dx w_pre z - rho^2 mean(..) h' z, three more sums next to those of
// h'^2, o^2 and dx w_pre h', all six added across the warps in one go.  Arithmetic is on pairs of columns; a thread's columns of the weights and,
// with one vector per thread, of the row stay in registers.  What happens when a wait gives up stands behind the loop over rows, which then needs
// no registers for it.  (8192 x 5120 from E4M3 checkpoints: 96 us, 4.4 TB/s; 110 with a question about the wait at every vector.  On the way there,
// loading into registers 317, with copies ahead but decoding in every phase 185, two meetings per row 150, two rows at a time 153, the
// copies on one thread 141.)
constexpr int kNormSmem = 160 * 1024;   // five rows of 5120; what is left of the SM's is L1, for the spills that there were (224 KB: 117 us where 160 took 111)
constexpr int kNormStages = 64;
__host__ __device__ constexpr int norm_warps(int V) { return V == 1 ? 20 : 16; }   // of a CTA, at most: 96 or 128 registers per thread

struct NormBackwardLaunch {
    NormBackward a;
    int W, G, stages, stage_bytes;       // stages: of a group
    int at_dh, at_h, at_o, at_gate, at_words;   // in a stage; dx comes first
    int waited_for;                      // rows that are: all (with LML_NORM_PATIENCE=0 none)
};

// Arrives at the barrier when the words that this thread has asked for are there.
__device__ __forceinline__ void cp_async_arrive(uint32_t bar)
{
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void cp_async_word(uint32_t* dst, const uint32_t* src)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(ptx::smem_u32(dst)), "l"(src) : "memory");
}
// The eight values of a vector: packed as bf16, or as they are multiplied.
__device__ __forceinline__ void unpack_pairs(const uint4& v, float2 (&f)[4])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = make_float2(bf16_lo(w[e]), bf16_hi(w[e]));
}
__device__ __forceinline__ uint4 pack_pairs(const float2 (&f)[4])
{
    const float g[8] = {f[0].x, f[0].y, f[1].x, f[1].y, f[2].x, f[2].y, f[3].x, f[3].y};
    return pack8(g);
}
template <bool PACKED> struct Eight;
template <> struct Eight<true> {
    uint4 v;
    __device__ __forceinline__ void set(const uint4& x) { v = x; }
    __device__ __forceinline__ void get(float2 (&f)[4]) const { unpack_pairs(v, f); }
};
template <> struct Eight<false> {
    float2 v[4];
    __device__ __forceinline__ void set(const uint4& x) { unpack_pairs(x, v); }
    __device__ __forceinline__ void get(float2 (&f)[4]) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = v[e];
    }
};
// A vector of a row in shared memory; kept rows with their scale words.
__device__ __forceinline__ uint32_t scale_byte(const uint32_t* words, int vec) { return (words[vec >> 4] >> (8 * ((vec >> 2) & 3))) & 0xffu; }
__device__ __forceinline__ void ld_stage(Eight<true>& x, const uint8_t* at, int vec, int format, const uint32_t* words)
{
    if (format == kBf16) return x.set(*reinterpret_cast<const uint4*>(at + vec * 16));
    const uint2 q = *reinterpret_cast<const uint2*>(at + vec * 8);
    const uint32_t byte = scale_byte(words, vec);
    x.set(format == kE4m3 ? decode8<true>(q, byte) : decode8<false>(q, byte));
}
// Straight to fp32, where one multiplication does for every scale: q from e4m3 by way of fp16, from int8 as 2^23 + 128 + q less 2^23 + 128.
__device__ __forceinline__ void ld_stage(Eight<false>& x, const uint8_t* at, int vec, int format, const uint32_t* words)
{
    if (format == kBf16) return x.set(*reinterpret_cast<const uint4*>(at + vec * 16));
    const uint2 q = *reinterpret_cast<const uint2*>(at + vec * 8);
    const uint32_t byte = scale_byte(words, vec);
    const float2 scale = both(__uint_as_float(byte == 255u ? 0x7fc00000u : byte == 0u ? 0x00400000u : byte << 23));
    const uint32_t w[2] = {q.x, q.y};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (format == kE4m3) {
            const __half2_raw v = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
            x.v[i] = __half22float2(__half2(v));
        } else {
            const uint32_t u = w[i >> 1] ^ 0x80808080u;
            const float2 v = make_float2(__uint_as_float(__byte_perm(u, 0x4b000000u, i & 1 ? 0x7442 : 0x7440)),
                                         __uint_as_float(__byte_perm(u, 0x4b000000u, i & 1 ? 0x7443 : 0x7441)));
            x.v[i] = add2(v, both(-8388736.f));
        }
        x.v[i] = mul2(x.v[i], scale);
    }
}
// Six sums over a warp in 26 instructions: a pair of lanes shares the sums out between them as long as there are two and more, so that lane
// 16 (k & 1) + 8 (k >> 1 & 1) + 4 (k >> 2) has the k-th.
__device__ __forceinline__ float warp_sums6(const float (&s)[6], int lane)
{
    const bool up = lane & 16, up8 = lane & 8, up4 = lane & 4;
    float r[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const float mine = up ? s[2 * k + 1] : s[2 * k], other = up ? s[2 * k] : s[2 * k + 1];
        r[k] = mine + __shfl_xor_sync(0xffffffffu, other, 16);
    }
    const float x = (up8 ? r[1] : r[0]) + __shfl_xor_sync(0xffffffffu, up8 ? r[0] : r[1], 8);
    const float y = r[2] + __shfl_xor_sync(0xffffffffu, r[2], 8);
    float z = (up4 ? y : x) + __shfl_xor_sync(0xffffffffu, up4 ? x : y, 4);
    z += __shfl_xor_sync(0xffffffffu, z, 2);
    return z + __shfl_xor_sync(0xffffffffu, z, 1);
}

// V: vectors of a row per thread.  FMT >= 0: the usual call, all of whose inputs and outputs but a gate per token are there, o and h'
// in this format, and whose threads' vectors make up the row: nothing to ask about at every step (8192 x 5120 in bf16 81 us, 6.2 TB/s; the
// others: 8192 x 2880 120 us, 2.4 TB/s, 8192 x 4096 with a gate per token 164 us, 3.3 TB/s).
template <int V, bool SUMS, int FMT>
__global__ void __launch_bounds__(32 * norm_warps(V), 1) block_norm_backward_kernel(const __grid_constant__ NormBackwardLaunch L)
{
    extern __shared__ __align__(16) uint8_t norm_smem[];
    __shared__ unsigned long long full[kNormStages];
    __shared__ float red[2][norm_warps(V) + 4][8];   // (a group reads up to three rows of no warp of its own, and drops them)
    __shared__ int gave_up;
    using namespace ptx;
    constexpr bool kAll = FMT >= 0, kPacked = V > 1;
    const NormBackward& a = L.a;
    const int T = a.n.T, d = a.n.d, vecs = d >> 3, W = L.W, G = L.G;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, group = warp / W, mine = warp % W, in = mine * 32 + lane;
    const bool has_dx = kAll || a.dx, has_dh_new = kAll || a.dh_new, block = kAll || a.o.data, post = kAll || (block && a.n.w_post);
    const bool wants_dh = kAll || a.dh, wants_do = kAll || a.d_o, row_gate = !kAll && block && a.n.gate_rows;
    const int fmt_h = kAll ? FMT : a.h_new.format, fmt_o = kAll ? FMT : a.o.format;
    const bool kept_h = has_dx && fmt_h != kBf16, kept_o = block && fmt_o != kBf16, kept = kept_h || kept_o;
    const int words = kept_groups(d);
    const unsigned step = gridDim.x * G;   // (a row's number and some steps more stay below 2^32)
    if (tid == 0) {
        gave_up = 0;
        for (int i = 0; i < L.stages * G; ++i)
            mbar_init(smem_u32(&full[i]), 2 * has_dx + has_dh_new + block + row_gate + (kept ? 32 : 0));
        fence_mbar_init();
    }
    __syncthreads();
    grid_dependency_wait();
    grid_launch_dependents();

    // This thread's columns: w_pre, and a gate w_post (where there are such)
    Eight<kPacked> w_pre[V];
    float2 w_o[V][4];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int vec = i * W * 32 + in;
        const bool ok = vec < vecs;
        w_pre[i].set(has_dx && ok ? ld_weights(a.n.w_pre, vec) : make_uint4(0, 0, 0, 0));
        float2 f[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w_o[i][e] = both(a.n.scale);
        if (post && ok) {
            unpack_pairs(ld_weights(a.n.w_post, vec), f);
#pragma unroll
            for (int e = 0; e < 4; ++e) w_o[i][e] = mul2(w_o[i][e], f[e]);
        }
        if (block && a.n.gate && ok) {
            unpack_pairs(ld_weights(a.n.gate, vec), f);
#pragma unroll
            for (int e = 0; e < 4; ++e) w_o[i][e] = mul2(w_o[i][e], f[e]);
        }
    }

    float2 s_pre[SUMS ? V : 1][4], s_o[SUMS ? V : 1][4];
    if (SUMS) {
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) s_pre[i][e] = s_o[i][e] = both(0.f);
    }
    const float inv_d = 1.f / (float)d;
    uint8_t* ring = norm_smem + (size_t)group * L.stages * L.stage_bytes;
    unsigned long long* bars = full + group * L.stages;
    auto group_barrier = [&]() {
        if (W > 1) asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(W * 32) : "memory");
        else __syncwarp();
    };
    // The copies of a row: one of the warps asks for the first tensor, the next for the second and so on, and one for the scale words; each
    // arrives at the stage's barrier itself.
    const uint32_t row16 = (uint32_t)d * 2u, h_bytes = kept_h ? (uint32_t)kept_pitch(d) : row16, o_bytes = kept_o ? (uint32_t)kept_pitch(d) : row16;
    unsigned duties = 0;
    for (int k = 0; k < 6; ++k)
        if (k % W == mine && (k == 1 ? has_dh_new : k == 3 ? block : k == 4 ? row_gate : k == 5 ? kept : has_dx)) duties |= 1u << k;
    auto ask = [&](unsigned t, int stage) {
        if (t >= (unsigned)T) return;
        const uint32_t bar = smem_u32(&bars[stage]);
        uint8_t* to = ring + (size_t)stage * L.stage_bytes;
        if ((duties & 31u) && elect_one()) {
            auto copy = [&](int k, const void* src, uint32_t bytes, int place) {
                if (!(duties >> k & 1u)) return;
                mbar_arrive_expect_tx(bar, bytes);
                bulk_load(smem_u32(to) + place, static_cast<const uint8_t*>(src) + (size_t)t * bytes, bytes, bar);
            };
            copy(0, a.dx, row16, 0);
            copy(1, a.dh_new, row16, L.at_dh);
            copy(2, a.h_new.data, h_bytes, L.at_h);
            copy(3, a.o.data, o_bytes, L.at_o);
            copy(4, a.n.gate_rows, row16, L.at_gate);
        }
        if (duties & 32u) {
            uint32_t* w = reinterpret_cast<uint32_t*>(to + L.at_words);
            for (int k = lane; k < words; k += 32) {
                if (kept_h) cp_async_word(w + k, a.h_new.scales + (size_t)k * T + t);
                if (kept_o) cp_async_word(w + words + k, a.o.scales + (size_t)k * T + t);
            }
            cp_async_arrive(bar);
        }
    };
    const unsigned first = blockIdx.x + group * gridDim.x;
    if (duties)
        for (int i = 0; i < L.stages; ++i) ask(first + i * step, i);
    size_t where0 = (size_t)first * d + in * 8;
    const size_t where_step = (size_t)step * d;
    int stage = 0, turn = 0;
    uint32_t phase = 0;
    unsigned t = first;
    for (; t < (unsigned)L.waited_for; t += step, turn ^= 1, where0 += where_step) {
        const uint8_t* at = ring + (size_t)stage * L.stage_bytes;
        const uint32_t* wh = reinterpret_cast<const uint32_t*>(at + L.at_words);
        if (!__all_sync(0xffffffffu, mbar_try_wait(smem_u32(&bars[stage]), phase) || mbar_wait(smem_u32(&bars[stage]), phase, &gave_up))) break;
        // h'^2, o^2, dx w_pre h' (mean(dx w_pre hh) = rho mean(dx w_pre h')), and dh', dx w_pre and h' by z
        Eight<kPacked> hp[V], op[V];
        Eight<true> gp[V], qp[V];
        float2 s2[6];
#pragma unroll
        for (int k = 0; k < 6; ++k) s2[k] = both(0.f);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int vec = i * W * 32 + in;
            const bool ok = kAll || vec < vecs;
            const uint4 zero = make_uint4(0, 0, 0, 0);
            if (has_dx && ok) {
                ld_stage(hp[i], at + L.at_h, vec, fmt_h, wh);
                ld_stage(gp[i], at, vec, kBf16, nullptr);
            } else {
                hp[i].set(zero);
                gp[i].set(zero);
            }
            if (block && ok) ld_stage(op[i], at + L.at_o, vec, fmt_o, wh + words);
            else op[i].set(zero);
            if (has_dh_new && ok) ld_stage(qp[i], at + L.at_dh, vec, kBf16, nullptr);
            else qp[i].set(zero);
            float2 h[4], g[4], o[4], q[4], w[4], gate[4];
            hp[i].get(h); gp[i].get(g); op[i].get(o); qp[i].get(q); w_pre[i].get(w);
            if (row_gate) unpack_pairs(ok ? *reinterpret_cast<const uint4*>(at + L.at_gate + vec * 16) : zero, gate);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 gw = mul2(g[e], w[e]);
                s2[0] = fma2(h[e], h[e], s2[0]);
                s2[1] = fma2(gw, h[e], s2[1]);
                if (post) {
                    float2 z = mul2(o[e], w_o[i][e]);
                    if (row_gate) z = mul2(z, gate[e]);
                    s2[2] = fma2(o[e], o[e], s2[2]);
                    s2[3] = fma2(q[e], z, s2[3]);
                    s2[4] = fma2(gw, z, s2[4]);
                    s2[5] = fma2(h[e], z, s2[5]);
                }
            }
        }
        float s[6];
#pragma unroll
        for (int k = 0; k < 6; ++k) s[k] = s2[k].x + s2[k].y;
        float(*const my_red)[8] = red[turn] + group * W;
        const float sum = warp_sums6(s, lane);
        if ((lane & 3) == 0 && (lane & 12) != 12) my_red[mine][(lane >> 4) + (lane >> 2 & 2) + (lane & 4)] = sum;
        group_barrier();
        if (!row_gate && duties) ask(t + L.stages * step, stage);   // (all of the row is in registers)
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < norm_warps(V); k += 4) {
            if (k >= W) break;
            const float x = my_red[k + (lane >> 3)][lane & 7];
            v += k + (lane >> 3) < W ? x : 0.f;
        }
        v += __shfl_xor_sync(0xffffffffu, v, 8);
        v += __shfl_xor_sync(0xffffffffu, v, 16);
#pragma unroll
        for (int k = 0; k < 6; ++k) s[k] = __shfl_sync(0xffffffffu, v, k);
        const float rho = has_dx ? rsqrtf(s[0] * inv_d + a.n.eps) : 0.f, mean_gh = s[1] * inv_d * rho;
        const float r_o = post ? rsqrtf(s[2] * inv_d + a.n.eps) : 1.f;
        const float mean_dz = fmaf(-rho * mean_gh, rho * s[5], fmaf(rho, s[4], s[3])) * inv_d * r_o;   // of D z r
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int vec = i * W * 32 + in;
            if (!kAll && vec >= vecs) continue;
            const size_t where = where0 + i * W * 256;
            float2 h[4], g[4], o[4], q[4], w[4];
            hp[i].get(h); gp[i].get(g); op[i].get(o); qp[i].get(q); w_pre[i].get(w);
            if (has_dx) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 x = mul2(h[e], both(rho));
                    if (SUMS) s_pre[i][e] = fma2(g[e], x, s_pre[i][e]);
                    q[e] = fma2(mul2(g[e], w[e]), both(rho), fma2(x, both(-rho * mean_gh), q[e]));   // D
                }
            }
            if (wants_dh) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.dh) + where) = pack_pairs(q);
            if (!block) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = mul2(o[e], both(r_o));   // oo
            if (row_gate) {
                if (a.dgate_rows) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) g[e] = mul2(mul2(q[e], o[e]), w_o[i][e]);
                    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.dgate_rows) + where) = pack_pairs(g);
                }
                unpack_pairs(*reinterpret_cast<const uint4*>(at + L.at_gate + vec * 16), g);
#pragma unroll
                for (int e = 0; e < 4; ++e) q[e] = mul2(q[e], g[e]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (SUMS) s_o[i][e] = fma2(q[e], o[e], s_o[i][e]);
                q[e] = mul2(q[e], w_o[i][e]);
                if (post) q[e] = mul2(fma2(o[e], both(-mean_dz), q[e]), both(r_o));
            }
            if (wants_do) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.d_o) + where) = pack_pairs(q);
        }
        if (row_gate) {
            group_barrier();
            if (duties) ask(t + L.stages * step, stage);
        }
        if (++stage == L.stages) { stage = 0; phase ^= 1u; }
    }
    if (t < (unsigned)T) {
        // A wait gave up.  Of this row and all that follow this warp makes NaN, of the sums too, and through the meeting the others do.  It asks for
        // no more rows: copies that have not landed may still count on the stages' barriers, whose phases nobody knows any more.
        const float nan = __uint_as_float(0x7fc00000u);
        const uint4 nans = make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
#pragma unroll 1
        for (; t < (unsigned)T; t += step, turn ^= 1, where0 += where_step) {
            if (lane < 6) red[turn][group * W + mine][lane] = nan;
            group_barrier();
            for (int i = 0; i < V; ++i) {
                const int vec = i * W * 32 + in;
                const size_t where = where0 + i * W * 256;
                if (!kAll && vec >= vecs) continue;
                if (wants_dh) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.dh) + where) = nans;
                if (wants_do) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.d_o) + where) = nans;
                if (row_gate && a.dgate_rows) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.dgate_rows) + where) = nans;
            }
            if (row_gate) group_barrier();
        }
        if (SUMS) {
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) s_pre[i][e] = s_o[i][e] = both(nan);
        }
        __nanosleep(50000);   // let copies still in flight land before their place is used again, by this CTA or the next
    }
    if (!SUMS) return;
    // this CTA's partial sums, groups added in order, where the ring was
    __syncthreads();
    float* sums = reinterpret_cast<float*>(norm_smem);
    float* out = a.partial + (size_t)blockIdx.x * 2 * d;
#pragma unroll 1
    for (int g = 0; g < G; ++g) {
        if (g == group) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int vec = i * W * 32 + in;
                if (!kAll && vec >= vecs) continue;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float2(&s)[4] = k == 0 ? s_pre[i] : s_o[i];
                    float4* acc = reinterpret_cast<float4*>(sums + (size_t)k * d + vec * 8);
                    float4 lo = make_float4(s[0].x, s[0].y, s[1].x, s[1].y), hi = make_float4(s[2].x, s[2].y, s[3].x, s[3].y);
                    if (g > 0) {
                        const float4 l = acc[0], h = acc[1];
                        lo = make_float4(l.x + lo.x, l.y + lo.y, l.z + lo.z, l.w + lo.w);
                        hi = make_float4(h.x + hi.x, h.y + hi.y, h.z + hi.z, h.w + hi.w);
                    }
                    float4* dst = g < G - 1 ? acc : reinterpret_cast<float4*>(out + (size_t)k * d + vec * 8);
                    dst[0] = lo; dst[1] = hi;
                }
            }
        }
        __syncthreads();
    }
}

// Adds up partial[0..P)[2][d]: 32 float4 columns by 16 slices of the partial sums per CTA.  The first of the two goes onto dw_pre, a times the
// second times the channel's gate onto dw_post, and times w_post onto dgate.
constexpr int kSumSlices = 16;
__global__ void __launch_bounds__(32 * kSumSlices) norm_sums_kernel(const __grid_constant__ NormBackward a, int P)
{
    __shared__ float4 part[kSumSlices][32];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int d = a.n.d;
    if (blockIdx.y == 0 ? !a.dw_pre : !a.dw_post && !a.dgate) return;
    const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5, c = (blockIdx.x * 32 + lane) * 4;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < d) {
        const float* src = a.partial + ((size_t)slice * 2 + blockIdx.y) * d + c;
        const size_t stride = (size_t)kSumSlices * 2 * d;
#pragma unroll 1
        for (int p = slice; p < P; p += 5 * kSumSlices, src += 5 * stride) {
            float4 v[5];
#pragma unroll
            for (int k = 0; k < 5; ++k)
                if (p + k * kSumSlices < P)
                    asm volatile("ld.global.cg.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v[k].x), "=f"(v[k].y), "=f"(v[k].z), "=f"(v[k].w) : "l"(src + k * stride) : "memory");
#pragma unroll
            for (int k = 0; k < 5; ++k)
                if (p + k * kSumSlices < P) { s.x += v[k].x; s.y += v[k].y; s.z += v[k].z; s.w += v[k].w; }
        }
    }
    part[slice][lane] = s;
    __syncthreads();
    if (slice == 0 && c < d) {
#pragma unroll
        for (int k = 1; k < kSumSlices; ++k) {
            const float4 v = part[k][lane];
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        auto add = [&](float* out, const void* times) {
            if (!out) return;
            const float m = blockIdx.y == 0 ? 1.f : a.n.scale;
            float4 f = make_float4(m, m, m, m);
            if (times) {
                const uint2 w = ld_v2(static_cast<const __nv_bfloat16*>(times) + c);
                f = make_float4(m * bf16_lo(w.x), m * bf16_hi(w.x), m * bf16_lo(w.y), m * bf16_hi(w.y));
            }
            float4* dst = reinterpret_cast<float4*>(out + c);
            const float4 v = *dst;
            *dst = make_float4(fmaf(s.x, f.x, v.x), fmaf(s.y, f.y, v.y), fmaf(s.z, f.z, v.z), fmaf(s.w, f.w, v.w));
        };
        if (blockIdx.y == 0) {
            add(a.dw_pre, nullptr);
        } else {
            add(a.dw_post, a.n.gate);
            add(a.dgate, a.n.w_post);
        }
    }
}

// ---- launches ----------------------------------------------------------------------------------------
cudaError_t launch_block_norm(const NormForward& a, int num_sms, cudaStream_t stream)
{
    // As few vectors per thread as the warps allow where there are rows for one wave at most: what counts is one row's time.  Two for more, to
    // some 40 rows per SM (2000 x 4096 with a block before: 14.9 us, four 17.1; 5000 x 4096 30.4 and 32.0), four beyond, where what counts is
    // loads in flight (8192 x 4096 without o: 24.2 us, 5.6 TB/s, two 27.1; 16384 x 2048 23.2 and 29.4; 8192 x 4096 with a block before the same).
    // The weights are asked for ahead of the sums up to a few waves (40 x 4096 with a gate per token: 2.4 us, 2.8 behind them; 1000 x 4096 8.8 and
    // 10.0); beyond they come from L1, and the registers are better used for more rows (8192 x 4096 without o: 24.2 us, 41 ahead).  T and d decide
    // and nothing else: a call on h' alone gives the same bits.
    const int vecs = a.n.d / 8;
    const bool ahead = a.n.T <= 8 * num_sms;
    int V = a.n.T <= num_sms ? 1 : a.n.T <= 40 * num_sms ? 2 : 4;
    while (V > 1 && 16 * V >= vecs) V /= 2;                 // (not more than the row has)
    while (32 * 16 * V < vecs) V *= 2;
    const int needs = (vecs + 32 * V - 1) / (32 * V);
    const auto launch = [&](auto w, auto v) {
        constexpr int W = decltype(w)::value, V = decltype(v)::value, kGroups = NormShape<W>::kGroups;
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr[1];
        pdl_config(cfg, attr, dim3((unsigned)(((long long)a.n.T + kGroups - 1) / kGroups)), dim3(NormShape<W>::kWarps * 32), 0, stream);
        return cudaLaunchKernelEx(&cfg, ahead ? block_norm_kernel<W, V, true> : block_norm_kernel<W, V, false>, a);
    };
    // Numbers of warps that there are kernels for: powers of two, and 5 and 10 in their widest gaps, so that a third of a row's threads at most have
    // nothing to do (11 warps' columns on 16).
    const auto widths = [&](auto v) {
        const auto fits = [&](auto w) { return needs <= decltype(w)::value; };
        using std::integral_constant;
        if (fits(integral_constant<int, 1>())) return launch(integral_constant<int, 1>(), v);
        if (fits(integral_constant<int, 2>())) return launch(integral_constant<int, 2>(), v);
        if (fits(integral_constant<int, 4>())) return launch(integral_constant<int, 4>(), v);
        if (fits(integral_constant<int, 5>())) return launch(integral_constant<int, 5>(), v);
        if (fits(integral_constant<int, 8>())) return launch(integral_constant<int, 8>(), v);
        if (fits(integral_constant<int, 10>())) return launch(integral_constant<int, 10>(), v);
        return launch(integral_constant<int, 16>(), v);
    };
    return V == 1 ? widths(std::integral_constant<int, 1>()) : V == 2 ? widths(std::integral_constant<int, 2>()) : widths(std::integral_constant<int, 4>());
}

static int norm_backward_ctas(int T, int num_sms) { return T < num_sms ? T : num_sms; }
size_t norm_backward_ws_bytes(int T, int d, int num_sms) { return (size_t)norm_backward_ctas(T, num_sms) * 2 * d * sizeof(float); }

using NormBackwardKernel = void (*)(NormBackwardLaunch);
template <int V, int FMT> static NormBackwardKernel norm_backward_kernel(bool sums)
{
    return sums ? block_norm_backward_kernel<V, true, FMT> : block_norm_backward_kernel<V, false, FMT>;
}
static NormBackwardKernel norm_backward_kernel(int V, int fmt, bool sums)
{
    switch (V * 4 + fmt) {
        case 4 + kBf16: return norm_backward_kernel<1, kBf16>(sums);
        case 4 + kInt8: return norm_backward_kernel<1, kInt8>(sums);
        case 4 + kE4m3: return norm_backward_kernel<1, kE4m3>(sums);
        case 8 + kBf16: return norm_backward_kernel<2, kBf16>(sums);
        case 8 + kInt8: return norm_backward_kernel<2, kInt8>(sums);
        case 8 + kE4m3: return norm_backward_kernel<2, kE4m3>(sums);
    }
    return V == 1 ? norm_backward_kernel<1, -1>(sums) : V == 2 ? norm_backward_kernel<2, -1>(sums) : norm_backward_kernel<4, -1>(sums);
}
static cudaError_t norm_init()   // once per device
{
    static std::atomic<unsigned long long> done;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (dev < 64 && (done.load(std::memory_order_acquire) >> dev & 1ull))) return e;
    for (int V = 1; V <= 4; V *= 2)
        for (int fmt = -1; fmt <= kE4m3; ++fmt)
            for (int sums = 0; sums < 2 && e == cudaSuccess; ++sums)
                e = cudaFuncSetAttribute(norm_backward_kernel(V, fmt, sums), cudaFuncAttributeMaxDynamicSharedMemorySize, kNormSmem);
    if (e == cudaSuccess && dev < 64) done.fetch_or(1ull << dev, std::memory_order_release);
    return e;
}

// LML_NORM_PATIENCE=0 (as it stands at the first call; a test knob): no row is waited for, as if every wait had given up.
static bool norm_waits()
{
    static const bool waits = [] {
        const char* e = getenv("LML_NORM_PATIENCE");
        return !e || atoi(e) > 0;
    }();
    return waits;
}

cudaError_t launch_block_norm_backward(const NormBackward& a, int num_sms, cudaStream_t stream)
{
    cudaError_t e = norm_init();
    if (e != cudaSuccess) return e;
    const bool sums = a.dw_pre || a.dw_post || a.dgate;
    const int d = a.n.d, vecs = d / 8, ctas = norm_backward_ctas(a.n.T, num_sms), rows = (a.n.T + ctas - 1) / ctas;   // of a CTA
    NormBackwardLaunch L;
    L.a = a;
    L.waited_for = norm_waits() ? a.n.T : 0;
    // One vector per thread up to the width that the warps allow; two or four where a row is wider.
    const int V = vecs <= 32 * norm_warps(1) ? 1 : vecs <= 2 * 32 * norm_warps(2) ? 2 : 4;
    L.W = (vecs + 32 * V - 1) / (32 * V);
    L.G = norm_warps(V) / L.W < rows ? norm_warps(V) / L.W : rows;
    const int row16 = d * 2, row8 = kept_pitch(d);
    int at = a.dx ? row16 : 0;
    L.at_dh = at;
    at += a.dh_new ? row16 : 0;
    L.at_h = at;
    at += !a.dx ? 0 : a.h_new.format == kBf16 ? row16 : row8;
    L.at_o = at;
    at += !a.o.data ? 0 : a.o.format == kBf16 ? row16 : row8;
    L.at_gate = at;
    at += a.n.gate_rows && a.o.data ? row16 : 0;
    L.at_words = at;
    const bool kept = (a.dx && a.h_new.format != kBf16) || (a.o.data && a.o.format != kBf16);
    if (kept) at += 2 * kept_groups(d) * (int)sizeof(uint32_t);
    at = (at + 15) / 16 * 16;
    L.stage_bytes = at;
    for (;; --L.G) {   // (one group has room: a row of all inputs of 16384 columns is 160 KB)
        L.stages = kNormSmem / (L.G * at);
        if (L.stages >= 2 || L.G == 1) break;
    }
    if (L.stages * L.G > kNormStages) L.stages = kNormStages / L.G;
    const int each = (rows + L.G - 1) / L.G;
    if (L.stages > each) L.stages = each;
    const size_t used = (size_t)L.G * L.stages * at, needed = (size_t)2 * d * sizeof(float);
    const size_t smem = used > needed ? used : needed;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    pdl_config(cfg, attr, dim3((unsigned)ctas), dim3((unsigned)(32 * L.W * L.G)), smem, stream);
    const bool all = a.dx && a.dh_new && a.dh && a.d_o && a.o.data && a.n.w_post && !a.n.gate_rows && a.o.format == a.h_new.format && L.W * V * 32 == vecs;
    e = cudaLaunchKernelEx(&cfg, norm_backward_kernel(V, all ? a.o.format : -1, sums), L);
    if (e != cudaSuccess || !sums) return e;
    pdl_config(cfg, attr, dim3((unsigned)((d + 127) / 128), 2), dim3(32 * kSumSlices), 0, stream);
    return cudaLaunchKernelEx(&cfg, norm_sums_kernel, a, ctas);
}

}  // namespace lml
