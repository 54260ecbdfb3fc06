// 8-bit rows: e4m3 values with a power of two as the scale of every block of 128.
//
// Block exponent e: the smallest integer >= -126 with (largest finite magnitude of the block) <= 448 2^e; 0 for a block of zeros.  The
// stored value is x 2^-e rounded to e4m3 once, to nearest even (448 is the largest e4m3 value, so nothing saturates; the product with a power
// of two is exact).  A value that is not finite is stored as NaN.  Scales are kept as E8M0 bytes, e + 127: what the scaled MFMA takes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "row_math.h"

namespace rapid {

constexpr int FP8_BLOCK = 128;
// bytes of a row of values, and of its scales (whole 32-bit words, for loads of four)
__host__ __device__ inline int64_t fp8_row(int64_t d) { return (d + FP8_BLOCK - 1) / FP8_BLOCK * FP8_BLOCK; }
__host__ __device__ inline int64_t fp8_scale_row(int64_t d) { return (fp8_row(d) / FP8_BLOCK + 3) / 4 * 4; }

constexpr uint32_t INFINITY_BITS = 0x7f800000u;
__device__ __forceinline__ uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t finite_magnitude(float x) { return magnitude(x) < INFINITY_BITS ? magnitude(x) : 0u; }
// E8M0 byte of a block whose largest finite magnitude has the bits `most` (1.75 2^8 = 448)
__device__ __forceinline__ uint32_t block_scale(uint32_t most) {
    if (most == 0u) return 127u;
    const int e = (int)(most >> 23) - 8 + ((most & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)(e < 1 ? 1 : e);
}
__device__ __forceinline__ float scale_inverse(uint32_t byte) { return __builtin_bit_cast(float, (254u - byte) << 23); }

// 4 values, scaled and rounded
__device__ __forceinline__ uint32_t to_fp8x4(float a, float b, float c, float d, float inverse) {
    int v = 0;
    v = __builtin_amdgcn_cvt_pk_fp8_f32(a * inverse, b * inverse, v, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inverse, d * inverse, v, true);
}
__device__ __forceinline__ float not_finite_is_nan(float x) { return magnitude(x) < INFINITY_BITS ? x : __builtin_nanf(""); }
__device__ __forceinline__ void from_fp8x4(uint32_t v, float (&f)[4]) {
    f[0] = __builtin_amdgcn_cvt_f32_fp8((int)v, 0);
    f[1] = __builtin_amdgcn_cvt_f32_fp8((int)v, 1);
    f[2] = __builtin_amdgcn_cvt_f32_fp8((int)v, 2);
    f[3] = __builtin_amdgcn_cvt_f32_fp8((int)v, 3);
}

// 8 consecutive elements as they are stored
template <class T> struct Raw8;
template <> struct Raw8<unsigned short> {
    uint4 v;
    __device__ __forceinline__ void clear() { v = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ float operator[](int e) const {
        const uint32_t w = e < 2 ? v.x : e < 4 ? v.y : e < 6 ? v.z : v.w;
        return __builtin_bit_cast(float, e % 2 ? w & 0xffff0000u : w << 16);
    }
};
template <> struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void clear() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ float operator[](int e) const {
        const float4 q = e < 4 ? a : b;
        return e % 4 == 0 ? q.x : e % 4 == 1 ? q.y : e % 4 == 2 ? q.z : q.w;
    }
};
// from column c on of a row of d: bf16 (d % 8 == 0) or fp32; zeros behind the end
__device__ __forceinline__ Raw8<unsigned short> load8(const unsigned short* row, int64_t c, int64_t d) {
    Raw8<unsigned short> r;
    r.clear();
    if (c < d) r.v = *(const uint4*)(row + c);
    return r;
}
__device__ __forceinline__ Raw8<float> load8(const float* row, int64_t c, int64_t d) {
    Raw8<float> r;
    r.clear();
    if (d % 4 == 0) {
        if (c < d) r.a = *(const float4*)(row + c);
        if (c + 4 < d) r.b = *(const float4*)(row + c + 4);
    } else if (c + 8 <= d) {            // (16-byte loads take any address that is a multiple of 4)
        typedef float any4 __attribute__((ext_vector_type(4), aligned(4)));
        r.a = __builtin_bit_cast(float4, *(const any4*)(row + c));
        r.b = __builtin_bit_cast(float4, *(const any4*)(row + c + 4));
    } else {
        float* p[8] = {&r.a.x, &r.a.y, &r.a.z, &r.a.w, &r.b.x, &r.b.y, &r.b.z, &r.b.w};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < d) *p[e] = row[c + e];
    }
    return r;
}
template <class T>
__device__ __forceinline__ void load8(const T* row, int64_t c, int64_t d, float (&x)[8]) {
    const Raw8<T> r = load8(row, c, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = r[e];
}
// the block that 16 lanes hold 8 elements each of: its scale, and the lane's elements rounded
__device__ __forceinline__ uint2 quantize_block(float (&x)[8], uint32_t& scale, bool& bad) {
    uint32_t most = 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, magnitude(x[e]));
    if (most >= INFINITY_BITS) {        // rare: the largest finite one instead, NaN for the others
        bad = true;
        most = 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            most = max(most, finite_magnitude(x[e]));
            x[e] = not_finite_is_nan(x[e]);
        }
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o, 64));
    scale = block_scale(most);
    const float inv = scale_inverse(scale);
    return make_uint2(to_fp8x4(x[0], x[1], x[2], x[3], inv), to_fp8x4(x[4], x[5], x[6], x[7], inv));
}

// the scales of the four blocks that a wave holds, as a word
__device__ __forceinline__ uint32_t scale_word(uint32_t s) {
    return (uint32_t)__shfl((int)s, 0, 64) | (uint32_t)__shfl((int)s, 16, 64) << 8 | (uint32_t)__shfl((int)s, 32, 64) << 16 |
           (uint32_t)__shfl((int)s, 48, 64) << 24;
}

}  // namespace rapid
