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
    static constexpr int kWarps = W > 8 ? W : 8;
    static constexpr int kGroups = kWarps / W;
};

template <int W, int V>
__global__ void __launch_bounds__(NormShape<W>::kWarps * 32) block_norm_kernel(const __grid_constant__ NormForward a)
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
    const float inv_d = 1.f / (float)d;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    auto at = [&](const void* p, int vec) { return static_cast<const __nv_bfloat16*>(p) + t * d + vec * 8; };

    uint4 h[V], o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int vec = i * W * 32 + in;
        h[i] = vec < vecs ? ld_v4(at(a.h, vec)) : zero;
        o[i] = a.o && vec < vecs ? ld_v4(at(a.o, vec)) : zero;
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
            r = rsqrtf(group_sum<W>(ss, red0, group, warp, lane) * inv_d + a.n.eps);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int vec = i * W * 32 + in;
            if (vec >= vecs) continue;
            float f[8], n[8], w[8];
            unpack8(h[i], f);
            unpack8(o[i], n);
            if (a.n.w_post) {
                unpack8(ld_weights(a.n.w_post, vec), w);
#pragma unroll
                for (int e = 0; e < 8; ++e) n[e] *= r * w[e];
            }
            if (a.n.gate || a.n.gate_rows) {
                unpack8(a.n.gate_rows ? ld_v4(at(a.n.gate_rows, vec)) : ld_weights(a.n.gate, vec), w);
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
    const float rho = rsqrtf(group_sum<W>(ss, red1, group, warp, lane) * inv_d + a.n.eps);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int vec = i * W * 32 + in;
        if (vec < vecs) {
            float f[8], w[8];
            unpack8(h[i], f);
            unpack8(ld_weights(a.n.w_pre, vec), w);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] *= rho * w[e];
            h[i] = pack8(f);
            if (a.x) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.x) + t * d + vec * 8) = h[i];
        }
        if (a.x_kept.data) store_kept(a.x_kept, T, d, t, vec, h[i]);
    }
}

// ---- backward ---------------------------------------------------------------------------------------
// Persistent: a group walks rows with a stride of all groups and keeps its share of the three sums over tokens in
// registers; the groups of a CTA add theirs in shared memory, CTAs write partial sums that a second launch adds up.
template <int W, int V, bool SUMS>
__global__ void __launch_bounds__(NormShape<W>::kWarps * 32) block_norm_backward_kernel(const __grid_constant__ NormBackward a)
{
    __shared__ float red[2][NormShape<W>::kWarps];
    __shared__ float3 red3[2][NormShape<W>::kWarps];
    extern __shared__ float sums[];   // [3][d], where a CTA has several groups
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    constexpr int kGroups = NormShape<W>::kGroups;
    const int T = a.n.T, d = a.n.d, vecs = d >> 3;
    const int group = threadIdx.x / (W * 32), in = threadIdx.x % (W * 32), warp = in >> 5, lane = in & 31;
    const float inv_d = 1.f / (float)d;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    const bool block = a.o.data != nullptr, post = block && a.n.w_post, gated = block && (a.n.gate || a.n.gate_rows);

    float s_pre[SUMS ? V : 1][8], s_post[SUMS ? V : 1][8], s_gate[SUMS ? V : 1][8];
    if (SUMS) {
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) s_pre[i][e] = s_post[i][e] = s_gate[i][e] = 0.f;
    }
    int phase = 0;
    for (long long t = (long long)blockIdx.x * kGroups + group; t < T; t += (long long)gridDim.x * kGroups, phase ^= 1) {
        float* red1 = red[phase] + group * W;
        auto at = [&](const void* p, int vec) { return static_cast<const __nv_bfloat16*>(p) + t * d + vec * 8; };
        uint4 h[V], o[V], dx[V], dd[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int vec = i * W * 32 + in;
            const bool ok = vec < vecs;
            h[i] = ok && a.dx ? load_rows(a.h_new, T, d, t, vec) : zero;
            dx[i] = ok && a.dx ? ld_v4(at(a.dx, vec)) : zero;
            dd[i] = ok && a.dh_new ? ld_v4(at(a.dh_new, vec)) : zero;
            o[i] = ok && block ? load_rows(a.o, T, d, t, vec) : zero;
        }
        // sums over the row: h'^2, o^2 and g.h' (mean(g hh) = rho mean(g h'))
        float rho = 0.f, mean_gh = 0.f, r = 1.f;
        {
            float hh = 0.f, gh = 0.f, oo = 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int vec = i * W * 32 + in;
                float f[8], g[8], w[8];
                if (a.dx && vec < vecs) {
                    unpack8(h[i], f);
                    unpack8(dx[i], g);
                    unpack8(ld_weights(a.n.w_pre, vec), w);
#pragma unroll
                    for (int e = 0; e < 8; ++e) { hh = fmaf(f[e], f[e], hh); gh = fmaf(g[e] * w[e], f[e], gh); }
                }
                if (post) {
                    unpack8(o[i], f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) oo = fmaf(f[e], f[e], oo);
                }
            }
#pragma unroll
            for (int m = 16; m; m >>= 1) {
                hh += __shfl_xor_sync(0xffffffffu, hh, m);
                gh += __shfl_xor_sync(0xffffffffu, gh, m);
                oo += __shfl_xor_sync(0xffffffffu, oo, m);
            }
            if (W > 1) {
                if (lane == 0) red3[phase][group * W + warp] = make_float3(hh, gh, oo);
                asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(W * 32) : "memory");
                hh = gh = oo = 0.f;
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const float3 v = red3[phase][group * W + w];
                    hh += v.x; gh += v.y; oo += v.z;
                }
            }
            if (a.dx) rho = rsqrtf(hh * inv_d + a.n.eps);
            mean_gh = gh * inv_d * rho;
            if (post) r = rsqrtf(oo * inv_d + a.n.eps);
        }
        // D, in fp32 (held in place of what it was made from); dn w_post . o for the second mean
        float D[V][8], go = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int vec = i * W * 32 + in;
            if (vec >= vecs) continue;
            float f[8], g[8], w[8];
            unpack8(dd[i], D[i]);
            if (a.dx) {
                unpack8(h[i], f);
                unpack8(dx[i], g);
                unpack8(ld_weights(a.n.w_pre, vec), w);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float hh = f[e] * rho;
                    if (SUMS) s_pre[i][e] = fmaf(g[e], hh, s_pre[i][e]);
                    D[i][e] = fmaf(rho, fmaf(-hh, mean_gh, g[e] * w[e]), D[i][e]);
                }
            }
            if (a.dh) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.dh) + t * d + vec * 8) = pack8(D[i]);
            if (!block) continue;
            unpack8(o[i], f);
            if (post) {
                unpack8(ld_weights(a.n.w_post, vec), w);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = 1.f;
            }
            float gt[8];
            if (gated) unpack8(a.n.gate_rows ? ld_v4(at(a.n.gate_rows, vec)) : ld_weights(a.n.gate, vec), gt);
            float dg[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float oo = f[e] * r, aD = a.n.scale * D[i][e];
                dg[e] = aD * oo * w[e];
                if (SUMS && gated) s_gate[i][e] += dg[e];
                const float dn = gated ? aD * gt[e] : aD;
                if (SUMS) s_post[i][e] = fmaf(dn, oo, s_post[i][e]);
                D[i][e] = dn * w[e];          // the gradient of oo from here on
                go = fmaf(D[i][e], oo, go);
            }
            if (a.dgate_rows) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.dgate_rows) + t * d + vec * 8) = pack8(dg);
        }
        if (!block) continue;
        float mean_go = 0.f;
        if (post) mean_go = group_sum<W>(go, red1, group, warp, lane) * inv_d;
        if (a.d_o) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int vec = i * W * 32 + in;
                if (vec >= vecs) continue;
                float f[8];
                if (post) {
                    unpack8(o[i], f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) D[i][e] = r * fmaf(-f[e] * r, mean_go, D[i][e]);
                }
                *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.d_o) + t * d + vec * 8) = pack8(D[i]);
            }
        }
    }
    if (!SUMS) return;
    // this CTA's partial sums, groups added in order
    float* out = a.partial + (size_t)blockIdx.x * 3 * d;
#pragma unroll 1
    for (int g = 0; g < kGroups; ++g) {
        if (g == group) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int vec = i * W * 32 + in;
                if (vec >= vecs) continue;
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    float(&s)[8] = k == 0 ? s_pre[i] : k == 1 ? s_post[i] : s_gate[i];
                    float4* acc = reinterpret_cast<float4*>(sums + (size_t)k * d + vec * 8);
                    float4 lo = make_float4(s[0], s[1], s[2], s[3]), hi = make_float4(s[4], s[5], s[6], s[7]);
                    if (kGroups > 1 && g > 0) {
                        const float4 l = acc[0], h = acc[1];
                        lo = make_float4(l.x + lo.x, l.y + lo.y, l.z + lo.z, l.w + lo.w);
                        hi = make_float4(h.x + hi.x, h.y + hi.y, h.z + hi.z, h.w + hi.w);
                    }
                    if (g < kGroups - 1) {
                        acc[0] = lo; acc[1] = hi;
                    } else {
                        float4* dst = reinterpret_cast<float4*>(out + (size_t)k * d + vec * 8);
                        dst[0] = lo; dst[1] = hi;
                    }
                }
            }
        }
        if (kGroups > 1) __syncthreads();
    }
}

// sums[k][c] += partial[0..P)[k][c]: 32 float4 columns by 8 slices of the partial sums per CTA
__global__ void __launch_bounds__(256) norm_sums_kernel(const float* __restrict__ partial, int P, int d, float* __restrict__ dw_pre,
                                                        float* __restrict__ dw_post, float* __restrict__ dgate)
{
    __shared__ float4 part[8][32];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    float* out = blockIdx.y == 0 ? dw_pre : blockIdx.y == 1 ? dw_post : dgate;
    if (!out) return;
    const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5, c = (blockIdx.x * 32 + lane) * 4;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < d) {
#pragma unroll 8
        for (int p = slice; p < P; p += 8) {
            float4 v;
            const float* src = partial + ((size_t)p * 3 + blockIdx.y) * d + c;
            asm volatile("ld.global.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(src) : "memory");
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
    }
    part[slice][lane] = s;
    __syncthreads();
    if (slice == 0 && c < d) {
#pragma unroll
        for (int k = 1; k < 8; ++k) {
            const float4 v = part[k][lane];
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        float4* dst = reinterpret_cast<float4*>(out + c);
        const float4 v = *dst;
        *dst = make_float4(v.x + s.x, v.y + s.y, v.z + s.z, v.w + s.w);
    }
}

// ---- launches ----------------------------------------------------------------------------------------
struct NormPick { int W, V; };
// vectors per thread: as few as 16 warps allow where there are few rows (latency), else up to `most`
static NormPick norm_pick(int T, int d, int num_sms, int most)
{
    const int vecs = d / 8;
    int V = 1, W = 1;
    const int want = T <= num_sms ? 1 : most;
    for (V = 1; V <= 4; V *= 2) {
        for (W = 1; W < 16 && W * V * 32 < vecs; W *= 2) {}
        if (W * V * 32 >= vecs && (V >= want || W == 1)) break;
    }
    if (V > 4) V = 4;
    return {W, V};
}

template <typename F> static cudaError_t norm_dispatch(const NormPick& p, F&& f)
{
#define LML_NORM_CASE(w, v) if (p.W == w && p.V == v) return f(std::integral_constant<int, w>(), std::integral_constant<int, v>())
    LML_NORM_CASE(1, 1); LML_NORM_CASE(2, 1); LML_NORM_CASE(4, 1); LML_NORM_CASE(8, 1); LML_NORM_CASE(16, 1);
    LML_NORM_CASE(1, 2); LML_NORM_CASE(2, 2); LML_NORM_CASE(4, 2); LML_NORM_CASE(8, 2); LML_NORM_CASE(16, 2);
    LML_NORM_CASE(1, 4); LML_NORM_CASE(2, 4); LML_NORM_CASE(4, 4); LML_NORM_CASE(8, 4); LML_NORM_CASE(16, 4);
#undef LML_NORM_CASE
    return cudaErrorInvalidValue;
}

cudaError_t launch_block_norm(const NormForward& a, int num_sms, cudaStream_t stream)
{
    return norm_dispatch(norm_pick(a.n.T, a.n.d, num_sms, 2), [&](auto w, auto v) {
        constexpr int W = decltype(w)::value, V = decltype(v)::value;
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr[1];
        const int groups = NormShape<W>::kGroups;
        pdl_config(cfg, attr, dim3((unsigned)((a.n.T + groups - 1) / groups)), dim3(NormShape<W>::kWarps * 32), 0, stream);
        return cudaLaunchKernelEx(&cfg, block_norm_kernel<W, V>, a);
    });
}

static int norm_backward_ctas(int T, int groups, int num_sms)
{
    const int need = (T + groups - 1) / groups;
    return need < 2 * num_sms ? need : 2 * num_sms;
}
size_t norm_backward_ws_bytes(int T, int d, int num_sms)
{
    return (size_t)norm_backward_ctas(T, 1, num_sms) * 3 * d * sizeof(float);
}

cudaError_t launch_block_norm_backward(const NormBackward& a, int num_sms, cudaStream_t stream)
{
    const bool sums = a.dw_pre || a.dw_post || a.dgate;
    return norm_dispatch(norm_pick(a.n.T, a.n.d, num_sms, 2), [&](auto w, auto v) -> cudaError_t {
        constexpr int W = decltype(w)::value, V = decltype(v)::value;
        constexpr int groups = NormShape<W>::kGroups;
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr[1];
        const int ctas = sums ? norm_backward_ctas(a.n.T, groups, num_sms) : (a.n.T + groups - 1) / groups;
        const size_t smem = sums && groups > 1 ? (size_t)3 * a.n.d * sizeof(float) : 0;   // (W < 8: d <= 4 * 32 * 4 * 8)
        pdl_config(cfg, attr, dim3((unsigned)ctas), dim3(NormShape<W>::kWarps * 32), smem, stream);
        if (!sums) return cudaLaunchKernelEx(&cfg, block_norm_backward_kernel<W, V, false>, a);
        cudaError_t e = cudaLaunchKernelEx(&cfg, block_norm_backward_kernel<W, V, true>, a);
        if (e != cudaSuccess) return e;
        pdl_config(cfg, attr, dim3((unsigned)((a.n.d + 127) / 128), 3), dim3(256), 0, stream);
        return cudaLaunchKernelEx(&cfg, norm_sums_kernel, (const float*)a.partial, ctas, a.n.d, a.dw_pre, a.dw_post, a.dgate);
    });
}

}  // namespace lml
