// 8-bit checkpoints of activations: store and load (the format stands in lml_rows.cuh).
#include "lml_rows.cuh"
#include "lml_ptx_sm100.cuh"

namespace lml {

// A warp takes 256 columns of a row at a time, a lane eight of them: one 16-byte access on the bf16 side, one of 8 bytes on
// the other, a word of scales per 16 lanes.  Bound by memory: 2 + 1 + 1/32 bytes per value.
constexpr int kKeptThreads = 256;

template <bool STORE>
__global__ void __launch_bounds__(kKeptThreads) kept_kernel(const void* x_in, void* x_out, const Rows rows, int T, int d)
{
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int lane = threadIdx.x & 31, chunks = (d + 255) / 256;
    const long long work = (long long)T * chunks, stride = (long long)gridDim.x * (kKeptThreads / 32);
    for (long long w = (long long)blockIdx.x * (kKeptThreads / 32) + (threadIdx.x >> 5); w < work; w += stride) {
        const long long t = w / chunks;
        const int vec = (int)(w - t * chunks) * 32 + lane;
        const bool valid = vec * 8 < d;
        if (STORE) {
            const uint4 v = valid ? ld_v4(static_cast<const __nv_bfloat16*>(x_in) + t * d + vec * 8) : make_uint4(0, 0, 0, 0);
            store_kept(rows, T, d, t, vec, v);
        } else if (valid) {
            *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(x_out) + t * d + vec * 8) = load_rows(rows, T, d, t, vec);
        }
    }
}

static cudaError_t launch_kept(bool store, const void* x_in, void* x_out, const Rows& rows, int T, int d, cudaStream_t stream)
{
    const long long work = (long long)T * ((d + 255) / 256), per = kKeptThreads / 32;
    const long long blocks = (work + per - 1) / per;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    pdl_config(cfg, attr, dim3((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20))), dim3(kKeptThreads), 0, stream);
    return store ? cudaLaunchKernelEx(&cfg, kept_kernel<true>, x_in, x_out, rows, T, d)
                 : cudaLaunchKernelEx(&cfg, kept_kernel<false>, x_in, x_out, rows, T, d);
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
