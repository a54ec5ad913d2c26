// Rows of activations as the training calls take them: bf16, or an 8-bit checkpoint.
//
// A checkpoint holds, per row and 32 columns, 8-bit values q and one power of two 2^(b - 127) (the OCP Microscaling
// formats MXINT8, its steps counted as integers, and MXFP8 E4M3); a value is q * 2^(b - 127).  Powers of two, because a
// decoded value then is exact in bf16 (q has at most 7 significant bits): what the tensor cores multiply is what the
// checkpoint stands for, and the only rounding of the whole path is that of q, half a step at most.
//   int8: b = E + 121 with E the binade of the block's largest value, |q| <= 127: the largest bf16 value of a binade is
//         127.5 steps, so the clamp is half a step as well.
//   e4m3: the least b with amax <= 448 * 2^(b - 127).  (Values of 1.9375 * 2^127 and more, 3.3e38, become 1.875 * 2^127.)
// b = 0 (2^-127) at least, 3 for e4m3 (its smallest step is then 2^-133, bf16's); a block that holds Inf or NaN has
// b = 255 and reads back as NaN throughout.
//
// Layout: q [T][pitch], pitch = d up to a multiple of 32, zeros behind column d; b in words of four blocks (128 columns),
// [column group][T]: a tile of 128 columns reads its scales as one contiguous piece, a row writes one word per 128 columns.
#pragma once
#include <cuda_fp8.h>

#include "lml_internal.cuh"

namespace lml {

enum RowFormat { kBf16 = LML_ROWS_BF16, kInt8 = LML_ROWS_INT8, kE4m3 = LML_ROWS_E4M3 };

__host__ __device__ __forceinline__ int kept_pitch(int d) { return (d + 31) / 32 * 32; }
__host__ __device__ __forceinline__ int kept_groups(int d) { return (d + 127) / 128; }

// Rows as a kernel reads or writes them.
struct Rows {
    void* data;
    uint32_t* scales;   // word [column group][T]
    int format;
};

// scale byte of a block from the largest |value| of it, as the bits of a bf16
__device__ __forceinline__ uint32_t byte_of_amax(uint32_t amax, bool e4m3)
{
    const uint32_t ef = amax >> 7, mant = amax & 0x7fu;
    if (ef == 255u) return 255u;
    const int b = e4m3 ? (int)ef - 8 + (mant > 0x60u ? 1 : 0) : (int)ef - 6;
    return (uint32_t)max(b, e4m3 ? 3 : 0);
}

// The scale byte of e4m3 blocks whose largest value is beyond 1.75 * 2^127: 248 units and more would round to 2^128, which bf16 does not
// have, so they become 240 units (1.875 * 2^127).
constexpr uint32_t kTopByte = 247u;

// Arithmetic on pairs of fp32 values.
__device__ __forceinline__ float2 fma2(const float2& x, const float2& y, const float2& z)
{
    float2 d;
    asm("{.reg .b64 x, y, z, d;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n mov.b64 z, {%6, %7};\n"
        " fma.rn.f32x2 d, x, y, z;\n mov.b64 {%0, %1}, d;}"
        : "=f"(d.x), "=f"(d.y) : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y), "f"(z.x), "f"(z.y));
    return d;
}
__device__ __forceinline__ float2 mul2(const float2& x, const float2& y)
{
    float2 d;
    asm("{.reg .b64 x, y, d;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n mul.rn.f32x2 d, x, y;\n mov.b64 {%0, %1}, d;}"
        : "=f"(d.x), "=f"(d.y) : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y));
    return d;
}
__device__ __forceinline__ float2 add2(const float2& x, const float2& y)
{
    float2 d;
    asm("{.reg .b64 x, y, d;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n add.rn.f32x2 d, x, y;\n mov.b64 {%0, %1}, d;}"
        : "=f"(d.x), "=f"(d.y) : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y));
    return d;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// Eight consecutive values, packed bf16 -> 8 bits; byte: their block's scale byte.
__device__ __forceinline__ uint2 encode8(const uint4& v, uint32_t byte, bool e4m3)
{
    const float2 inv = both(byte == 255u ? 0.f : __uint_as_float((254u - byte) << 23));   // 2^(127 - byte)
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t out[4];   // of two values each
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 x = make_float2(bf16_lo(w[i]), bf16_hi(w[i]));
        if (e4m3) {
            float2 q = mul2(x, inv);
            if (byte == kTopByte) q = make_float2(fminf(fmaxf(q.x, -240.f), 240.f), fminf(fmaxf(q.y, -240.f), 240.f));
            out[i] = __nv_cvt_float2_to_fp8x2(q, __NV_SATFINITE, __NV_E4M3);
        } else {
            // rounding to an integer by adding 1.5 * 2^23: the low 16 bits of the sum's are q in two's complement (the product is exact)
            const float2 q = fma2(x, inv, both(12582912.f));
            out[i] = __vmins2(__vmaxs2(__byte_perm(__float_as_uint(q.x), __float_as_uint(q.y), 0x5410), 0xff81ff81u), 0x007f007fu);
        }
    }
    if (e4m3) return make_uint2(out[0] | out[1] << 16, out[2] | out[3] << 16);
    return make_uint2(__byte_perm(out[0], out[1], 0x6420), __byte_perm(out[2], out[3], 0x6420));
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// Decoding, two values at a time, in integer and packed bf16 arithmetic, exact in every step.  What a block's scale byte b becomes for it:
//   int8: 2^(b - 120), which is 128 units.  With q's low seven bits as mantissa it is 128 + q units, or 256 + q where q is negative; 128 or, one
//         binade up, 256 units are taken off again.
//   e4m3: sign, exponent and mantissa put in their places in bf16 are the value times 2^-120; the factor is 2^(b - 7).
// Factors beyond the format (and NaN, b = 255) are the rare case: the value is made at scale 1 and multiplied.
// (us for 8 KB by 256 threads: 0.21, and 0.34 with a subtraction and a multiplication each, 0.48 through fp32.)
template <bool E4M3> struct Decoder {
    uint32_t base;
    static constexpr uint32_t kMost = E4M3 ? 134u : 246u;   // scale bytes of the usual case
    __device__ __forceinline__ explicit Decoder(uint32_t b) : base((b + (E4M3 ? 120u : 7u)) * 0x00800080u) {}
    __device__ __forceinline__ uint32_t pair(uint32_t q, int i) const   // bytes 2 i and 2 i + 1
    {
        if (E4M3) {
            const uint32_t w = __byte_perm(q, 0u, i ? 0x3424 : 0x1404);
            return mul_bf16x2((w & 0x80008000u) | ((w >> 4) & 0x07f007f0u), base);
        }
        const uint32_t w = __byte_perm(q, 0u, i ? 0x4342 : 0x4140);
        return sub_bf16x2((w & 0x007f007fu) | base, (w & 0x00800080u) + base);
    }
    __device__ __forceinline__ uint4 eight(const uint2& q) const { return make_uint4(pair(q.x, 0), pair(q.x, 1), pair(q.y, 0), pair(q.y, 1)); }
};
// ... of a block with any scale byte
template <bool E4M3>
__device__ __forceinline__ uint4 decode8(const uint2& q, uint32_t b)
{
    if (b <= Decoder<E4M3>::kMost) return Decoder<E4M3>(b).eight(q);
    const uint4 v = Decoder<E4M3>(127u).eight(q);
    const uint32_t s = (b == 255u ? 0x7fc0u : b << 7) * 0x10001u;
    return make_uint4(mul_bf16x2(v.x, s), mul_bf16x2(v.y, s), mul_bf16x2(v.z, s), mul_bf16x2(v.w, s));
}

__device__ __forceinline__ uint32_t amax_bits(const uint4& v)   // largest |value| of eight, as bf16 bits
{
    const uint32_t m = 0x7fff7fffu;
    const uint32_t a = __vmaxu2(__vmaxu2(v.x & m, v.y & m), __vmaxu2(v.z & m, v.w & m));
    return max(a & 0xffffu, a >> 16);
}

// Vector `vec` (columns 8 vec ...) of a row of a checkpoint, by the 32 lanes of a converged warp that hold consecutive vectors, the first a multiple
// of 32.  to: where the vector's bytes go; word_to: the row's scale word of these columns (what of them is behind the row is not written).  Lanes
// behind the last column pass zeros.
template <bool E4M3>
__device__ __forceinline__ void store_vector(uint8_t* to, uint32_t* word_to, bool there, int vec, const uint4& v)
{
    uint32_t amax = amax_bits(v);
    amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    const uint32_t byte = byte_of_amax(amax, E4M3);
    if (there) *reinterpret_cast<uint2*>(to) = encode8(v, byte, E4M3);
    uint32_t word = there ? byte << (8 * ((vec >> 2) & 3)) : 0u;   // (blocks behind the last have scale byte 0)
    word |= __shfl_xor_sync(0xffffffffu, word, 4);
    word |= __shfl_xor_sync(0xffffffffu, word, 8);
    if ((vec & 15) == 0 && there) *word_to = word;
}
__device__ __forceinline__ void store_kept(const Rows& r, int T, int d, long long t, int vec, const uint4& v)
{
    const int pitch = kept_pitch(d);
    const bool there = vec * 8 < pitch;
    uint8_t* to = static_cast<uint8_t*>(r.data) + t * pitch + vec * 8;
    uint32_t* word_to = r.scales + (long long)(vec >> 4) * T + t;
    if (r.format == kE4m3) store_vector<true>(to, word_to, there, vec, v);
    else store_vector<false>(to, word_to, there, vec, v);
}
// Ordinary loads, not through the non-coherent path: the kernels start while the work that writes their inputs still runs, and
// an output may be the buffer of an input.
__device__ __forceinline__ uint4 ld_v4(const void* p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint2 ld_v2(const void* p)
{
    uint2 v;
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint4 ld_weights(const void* p, int vec)   // (kept in L1: read for every row)
{
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(static_cast<const uint4*>(p) + vec) : "memory");
    return v;
}
// ---- launchers ------------------------------------------------------------------------------------
cudaError_t launch_kept_store(const void* x, int T, int d, const Rows& out, cudaStream_t stream);
cudaError_t launch_kept_load(const Rows& in, int T, int d, void* x, cudaStream_t stream);

constexpr int kMaxNormWidth = LML_MAX_NORM_WIDTH;
struct NormArgs {
    int T, d;
    float eps, scale;
    const void *w_post, *w_pre, *gate, *gate_rows;
};
struct NormForward {
    NormArgs n;
    const void *h, *o;
    void *h_new, *x;
    Rows x_kept, h_kept;   // data null: not wanted
};
struct NormBackward {
    NormArgs n;
    Rows h_new, o;         // data null: not there
    const void *dx, *dh_new;
    void *dh, *d_o, *dgate_rows;
    float *dw_pre, *dw_post, *dgate;
    float* partial;        // workspace
};
cudaError_t launch_block_norm(const NormForward& a, int num_sms, cudaStream_t stream);
cudaError_t launch_block_norm_backward(const NormBackward& a, int num_sms, cudaStream_t stream);
size_t norm_backward_ws_bytes(int T, int d, int num_sms);

}  // namespace lml
