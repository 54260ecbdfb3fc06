// The head to 8 bits (fp8.h), once per update of W: one pass over W, bound by memory.
#include "rapid_internal.h"
#include "fp8.h"

namespace rapid {

namespace {

// W stored [V, d]: a wave takes four consecutive blocks of a row at a time, 16 lanes with 8 elements each per block.
template <class T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T* __restrict__ W, int64_t V, int64_t d, int64_t quads, uint8_t* __restrict__ values,
                                                            uint32_t* __restrict__ scales, int32_t* __restrict__ dev_status) {
    const int64_t row_bytes = fp8_row(d);
    const int lane = threadIdx.x & 63;
    bool bad = false;
    for (int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); i < V * quads; i += (int64_t)gridDim.x * 4) {
        const int64_t v = i / quads, q = i - v * quads, c = q * 512 + lane * 8;
        float x[8];
        load8(W + v * d, c, d, x);
        uint32_t s;
        const uint2 out = quantize_block(x, s, bad);
        if (c < row_bytes) *(uint2*)(values + v * row_bytes + c) = out;
        const uint32_t word = scale_word(s);
        if (lane == 0) scales[i] = word;
    }
    if (bad && dev_status) atomicOr(dev_status, RAPID_STATUS_NONFINITE_VALUE);
}

// rows that do not begin on 16 bytes (a type's vectors of any alignment are loaded as the chip allows it)
__device__ __forceinline__ Raw8<bf16_t> load8_any(const bf16_t* row, int64_t c, int64_t n) {
    typedef unsigned any4 __attribute__((ext_vector_type(4), aligned(2)));
    if (c + 8 <= n) return Raw8<bf16_t>{__builtin_bit_cast(uint4, *(const any4*)(row + c))};
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
        w[e] = (c + 2 * e < n ? (uint32_t)row[c + 2 * e] : 0u) | (c + 2 * e + 1 < n ? (uint32_t)row[c + 2 * e + 1] << 16 : 0u);
    return Raw8<bf16_t>{make_uint4(w[0], w[1], w[2], w[3])};
}
__device__ __forceinline__ Raw8<float> load8_any(const float* row, int64_t c, int64_t n) {
    typedef float any4 __attribute__((ext_vector_type(4), aligned(4)));
    if (c + 8 <= n) return Raw8<float>{__builtin_bit_cast(float4, *(const any4*)(row + c)), __builtin_bit_cast(float4, *(const any4*)(row + c + 4))};
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = c + e < n ? row[c + e] : 0.f;
    return Raw8<float>{make_float4(f[0], f[1], f[2], f[3]), make_float4(f[4], f[5], f[6], f[7])};
}

// W stored [d, V]: a block takes the 128 rows of one block index and 128 columns.  A thread holds 8 x 8 elements (rows 8 (tid / 16) on, columns
// 8 (tid % 16) on); the columns' largest magnitudes meet in the LDS, and so do the rounded values, which leave as whole 128-byte rows.
template <class T, bool WHOLE>
__global__ __launch_bounds__(256) void quantize_columns_kernel(const T* __restrict__ W, int64_t V, int64_t d, uint8_t* __restrict__ values,
                                                               uint8_t* __restrict__ scales, int32_t* __restrict__ dev_status) {
    __shared__ uint32_t s_most[16][128];
    __shared__ uint2 s_out[128][17];
    const int64_t row_bytes = fp8_row(d), scale_row = (row_bytes / FP8_BLOCK + 3) / 4 * 4;
    const int64_t v0 = (int64_t)blockIdx.x * 128, b = blockIdx.y, k0 = b * FP8_BLOCK;
    const int tc = threadIdx.x & 15, tr = threadIdx.x >> 4;
    const int64_t c = v0 + tc * 8;
    Raw8<T> x[8];                   // as stored: half the registers of floats
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const int64_t k = k0 + tr * 8 + r;
        x[r].clear();
        if (k >= d) continue;
        if (WHOLE) x[r] = load8(W + k * V, c, V);
        else x[r] = load8_any(W + k * V, c, V);
    }
    uint32_t top = 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        uint32_t most = 0u;
#pragma unroll
        for (int r = 0; r < 8; ++r) most = max(most, magnitude(x[r][e]));
        s_most[tr][tc * 8 + e] = most;
        top = max(top, most);
    }
    const bool bad = top >= INFINITY_BITS;
    if (bad) {                      // rare: the largest finite ones instead
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            uint32_t most = 0u;
#pragma unroll
            for (int r = 0; r < 8; ++r) most = max(most, finite_magnitude(x[r][e]));
            s_most[tr][tc * 8 + e] = most;
        }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        uint32_t most = 0u;
#pragma unroll
        for (int g = 0; g < 16; ++g) most = max(most, s_most[g][tc * 8 + e]);
        const uint32_t s = block_scale(most);
        const float inv = scale_inverse(s);
        float f[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) f[r] = x[r][e];
        if (bad)
#pragma unroll
            for (int r = 0; r < 8; ++r) f[r] = not_finite_is_nan(f[r]);
        s_out[tc * 8 + e][tr] = make_uint2(to_fp8x4(f[0], f[1], f[2], f[3], inv), to_fp8x4(f[4], f[5], f[6], f[7], inv));
        if (tr == 0 && c + e < V) scales[(c + e) * scale_row + b] = (uint8_t)s;
    }
    // the bytes that fill a row of scales up to whole words
    if (b == gridDim.y - 1)
        for (int64_t i = b + 1 + tr; i < scale_row; i += 16)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e < V) scales[(c + e) * scale_row + i] = 127;
    __syncthreads();
    for (int i = threadIdx.x; i < 128 * 16; i += 256) {
        const int64_t v = v0 + (i >> 4);
        if (v < V) *(uint2*)(values + v * row_bytes + k0 + (i & 15) * 8) = s_out[i >> 4][i & 15];
    }
    if (bad && dev_status) atomicOr(dev_status, RAPID_STATUS_NONFINITE_VALUE);
}

template <class T>
void quantize_t(const T* W, int64_t V, int64_t d, int w_layout, uint8_t* values, uint8_t* scales, int32_t* dev_status, hipStream_t st) {
    if (w_layout == RAPID_W_VD) {
        const int64_t quads = fp8_scale_row(d) / 4, waves = V * quads;
        const int64_t blocks = (waves + 3) / 4 < 65536 ? (waves + 3) / 4 : 65536;
        quantize_rows_kernel<T><<<(unsigned)blocks, 256, 0, st>>>(W, V, d, quads, values, (uint32_t*)scales, dev_status);
        return;
    }
    const dim3 grid((unsigned)((V + 127) / 128), (unsigned)(fp8_row(d) / FP8_BLOCK));
    if (V % 8 == 0) quantize_columns_kernel<T, true><<<grid, 256, 0, st>>>(W, V, d, values, scales, dev_status);
    else quantize_columns_kernel<T, false><<<grid, 256, 0, st>>>(W, V, d, values, scales, dev_status);
}

}  // namespace

void launch_quantize_fp8(const void* W, int64_t V, int64_t d, int dtype, int w_layout, uint8_t* values, uint8_t* scales, int32_t* dev_status, hipStream_t st) {
    if (dtype == RAPID_DTYPE_BF16) quantize_t((const bf16_t*)W, V, d, w_layout, values, scales, dev_status, st);
    else quantize_t((const float*)W, V, d, w_layout, values, scales, dev_status, st);
}

}  // namespace rapid
