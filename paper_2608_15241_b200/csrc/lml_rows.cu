// 8-bit checkpoints of activations: store and load (the format stands in lml_rows.cuh).
#include "lml_rows.cuh"
#include "lml_ptx_sm100.cuh"

namespace lml {

// A warp has 1024 columns of a row, asked for all at once, 256 of them per step: a lane has eight, one 16-byte access on the bf16 side, one of 8
// bytes on the other, a word of scales per 16 lanes.  The warps of a CTA have consecutive rows, whose words of scales share a sector.
// Bound by memory: 2 + 1 + 1/32 bytes per value.  (8192 x 11008 stored and loaded: 91 us, 6.0 TB/s; a loop over 256 columns at a time 136.)
constexpr int kKeptWarps = 8, kKeptSteps = 4;

template <bool STORE, bool E4M3>
__global__ void __launch_bounds__(32 * kKeptWarps) kept_kernel(const void* x_in, void* x_out, const Rows rows, int T, int d)
{
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const long long t = (long long)blockIdx.x * kKeptWarps + (threadIdx.x >> 5);
    const int vec0 = blockIdx.y * 32 * kKeptSteps + (threadIdx.x & 31), pitch = kept_pitch(d);
    if (t >= T) return;
    uint8_t* kept = static_cast<uint8_t*>(rows.data) + t * pitch + vec0 * 8;
    uint32_t* word_at = rows.scales + (long long)(vec0 >> 4) * T + t;
    const size_t two = (size_t)T * 2;   // words of 256 columns on
    if (STORE) {
        const __nv_bfloat16* from = static_cast<const __nv_bfloat16*>(x_in) + t * d + vec0 * 8;
        uint4 v[kKeptSteps];
#pragma unroll
        for (int k = 0; k < kKeptSteps; ++k) v[k] = (vec0 + 32 * k) * 8 < d ? ld_v4(from + k * 256) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int k = 0; k < kKeptSteps; ++k)
            if ((blockIdx.y * kKeptSteps + k) * 256 < d)
                store_vector<E4M3>(kept + k * 256, word_at + k * two, (vec0 + 32 * k) * 8 < pitch, vec0, v[k]);
    } else {
        __nv_bfloat16* to = static_cast<__nv_bfloat16*>(x_out) + t * d + vec0 * 8;
        uint2 q[kKeptSteps];
        uint32_t word[kKeptSteps];
#pragma unroll
        for (int k = 0; k < kKeptSteps; ++k) {
            q[k] = make_uint2(0, 0);
            word[k] = 0;
            if ((vec0 + 32 * k) * 8 < d) {
                q[k] = ld_v2(kept + k * 256);
                word[k] = ld_after_wait(word_at + k * two);
            }
        }
        const int shift = 8 * ((vec0 >> 2) & 3);
#pragma unroll
        for (int k = 0; k < kKeptSteps; ++k)
            if ((vec0 + 32 * k) * 8 < d) *reinterpret_cast<uint4*>(to + k * 256) = decode8<E4M3>(q[k], (word[k] >> shift) & 0xffu);
    }
}

static cudaError_t launch_kept(bool store, const void* x_in, void* x_out, const Rows& rows, int T, int d, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    const int columns = 256 * kKeptSteps;
    pdl_config(cfg, attr, dim3((unsigned)(((long long)T + kKeptWarps - 1) / kKeptWarps), (unsigned)((d + columns - 1) / columns)), dim3(32 * kKeptWarps), 0, stream);
    const bool e4m3 = rows.format == kE4m3;
    const auto kernel = store ? (e4m3 ? kept_kernel<true, true> : kept_kernel<true, false>) : e4m3 ? kept_kernel<false, true> : kept_kernel<false, false>;
    return cudaLaunchKernelEx(&cfg, kernel, x_in, x_out, rows, T, d);
}
cudaError_t launch_kept_store(const void* x, int T, int d, const Rows& out, cudaStream_t stream)
{
    return launch_kept(true, x, nullptr, out, T, d, stream);
}
cudaError_t launch_kept_load(const Rows& in, int T, int d, void* x, cudaStream_t stream)
{
    return launch_kept(false, nullptr, x, in, T, d, stream);
}

}  // namespace lml
