// Quantisation to 8-bit floating point (e4m3) with one scale for each block
// of 128 values of a row, or of 128 x 128 values.
//
// With amax the largest magnitude among a block's finite values, the scale is
// the least power of two 2^e (e >= -126) with amax <= 448 * 2^e, and 1 for a
// block without one; q = e4m3(x / scale), to nearest, ties to even.  Dividing
// by a power of two is exact, so each value is rounded once, and the result
// depends on no order of evaluation.  The exponent comes from amax's own bits:
// 448 = 1.75 * 2^8, so the mantissa either fits (<= 1.75) or one more is needed.
// A power of two costs no precision: e4m3 keeps 3 mantissa bits wherever in
// its range the block lies, and the block's largest value is in [224, 448].
// e4m3 has no infinity: a non-finite value becomes NaN, so that a corrupted
// activation still reaches the outputs instead of being clipped to 448.
#include "ops_common.cuh"

namespace ct {
namespace ops {
namespace {

struct QuantArgs {
    const void *x;
    int64_t m, k, ldx;
    uint8_t *q;
    int64_t ldq;
    float *scale;
    int64_t srow, sblk;
    int64_t kb;                // blocks of 128 columns
    int xvec, qvec;            // rows of x / q may be read 16 / written 8 (4 for FP32) bytes at a time
};

__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u; }

// magnitude bits of a finite value, 0 for a non-finite one: ordered like the magnitudes
__device__ __forceinline__ uint32_t mag_bits(float v) {
    const uint32_t b = __float_as_uint(v) & 0x7FFFFFFFu;
    return b < 0x7F800000u ? b : 0u;
}

// (scale, 1 / scale), both exact
__device__ __forceinline__ void block_scale(uint32_t amax, float &scale, float &inv) {
    // exponent field, one more when the mantissa exceeds 1.75, less the 8 of 448's exponent
    const int f = max((int)((amax + 0x1FFFFFu) >> 23) - 8, 1);
    scale = amax == 0u ? 1.f : __uint_as_float((uint32_t)f << 23);
    inv = amax == 0u ? 1.f : __uint_as_float((uint32_t)(254 - f) << 23);
}

// two e4m3 values, `lo` in the low byte; NaN for a non-finite input
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi, float inv) {
    lo = finite(lo) ? lo * inv : __uint_as_float(0x7FC00000u);
    hi = finite(hi) ? hi * inv : __uint_as_float(0x7FC00000u);
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

template <typename T, int V>
__device__ __forceinline__ uint32_t load_values(const QuantArgs &a, int64_t row, int64_t c0, bool vec, float *v) {
    const T *p = static_cast<const T *>(a.x) + row * a.ldx + c0;
    if (vec) {
        unpack16<T>(__ldg(reinterpret_cast<const uint4 *>(p)), v);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = c0 + i < a.k ? to_f32(p[i]) : 0.f;
    }
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) amax = max(amax, mag_bits(v[i]));
    return amax;
}

template <int V>
__device__ __forceinline__ void store_values(const QuantArgs &a, int64_t row, int64_t c0, bool vec, const float *v,
                                             float inv) {
    uint32_t w[V / 4];
#pragma unroll
    for (int i = 0; i < V / 4; ++i)
        w[i] = e4m3x2(v[4 * i], v[4 * i + 1], inv) | (e4m3x2(v[4 * i + 2], v[4 * i + 3], inv) << 16);
    uint8_t *p = a.q + row * a.ldq + c0;
    if (vec) {
        if constexpr (V == 8) *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t *>(p) = w[0];
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (c0 + i < a.k) p[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
    }
}

constexpr int THREADS = 256;

// One block of 128 values of a row for each group of 128 / V lanes.
template <typename T>
__global__ void __launch_bounds__(THREADS) quantize_rows_kernel(const QuantArgs a) {
    constexpr int V = Vec16<T>::N;
    constexpr int G = 128 / V;               // lanes of a block: 32 (FP32) or 16
    pdl_wait();
    pdl_trigger();
    const int64_t blocks = a.m * a.kb;
    const int g = threadIdx.x / G, l = threadIdx.x % G;
    const int64_t at = (int64_t)blockIdx.x * (THREADS / G) + g;
    const bool live = at < blocks;
    const int64_t row = live ? at / a.kb : 0, b = live ? at % a.kb : 0;
    const int64_t c0 = b * 128 + l * V;
    const bool whole = c0 + V <= a.k;
    float v[V] = {};
    uint32_t amax = live ? load_values<T, V>(a, row, c0, a.xvec && whole, v) : 0u;
#pragma unroll
    for (int d = G / 2; d > 0; d >>= 1) amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, d));
    if (!live) return;
    float s, inv;
    block_scale(amax, s, inv);
    store_values<V>(a, row, c0, a.qvec && whole, v, inv);
    if (l == 0) a.scale[row * a.srow + b * a.sblk] = s;
}

// One CTA per 128 x 128 block: its values stay in registers between the
// maximum and the rounding.
template <typename T>
__global__ void __launch_bounds__(THREADS) quantize_blocks_kernel(const QuantArgs a) {
    constexpr int V = Vec16<T>::N;
    constexpr int G = 128 / V;
    constexpr int ROWS = THREADS / G;        // rows of one step
    constexpr int STEPS = 128 / ROWS;
    __shared__ uint32_t part[THREADS / 32];
    pdl_wait();
    pdl_trigger();
    const int64_t br = blockIdx.x / a.kb, b = blockIdx.x % a.kb;
    const int g = threadIdx.x / G, l = threadIdx.x % G;
    const int64_t c0 = b * 128 + l * V;
    const bool whole = c0 + V <= a.k;
    float v[STEPS][V];
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int64_t row = br * 128 + i * ROWS + g;
        if (row < a.m) {
            amax = max(amax, load_values<T, V>(a, row, c0, a.xvec && whole, v[i]));
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) v[i][j] = 0.f;
        }
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, d));
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = amax;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) amax = max(amax, part[i]);
    float s, inv;
    block_scale(amax, s, inv);
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int64_t row = br * 128 + i * ROWS + g;
        if (row < a.m) store_values<V>(a, row, c0, a.qvec && whole, v[i], inv);
    }
    if (threadIdx.x == 0) a.scale[br * a.srow + b * a.sblk] = s;
}

template <typename T>
cudaError_t launch(const QuantArgs &a, int block_rows, int64_t grid, cudaStream_t st) {
    return block_rows == 1 ? pdl_launch(quantize_rows_kernel<T>, dim3((unsigned)grid), dim3(THREADS), 0, st, a)
                           : pdl_launch(quantize_blocks_kernel<T>, dim3((unsigned)grid), dim3(THREADS), 0, st, a);
}

}  // namespace

ct_status quantize(const void *x, int dtype, int64_t m, int64_t k, int64_t ldx, int block_rows, uint8_t *q, int64_t ldq,
                   float *scale, int64_t srow, int64_t sblk, cudaStream_t st) {
    const int es = dtype_size(dtype), per16 = 16 / es;
    QuantArgs a = {x, m, k, ldx, q, ldq, scale, srow, sblk, (k + 127) / 128, 0, 0};
    a.xvec = aligned(x, 16) && ldx % per16 == 0;
    a.qvec = aligned(q, per16) && ldq % per16 == 0;
    const int64_t rows = (m + block_rows - 1) / block_rows;
    if (a.kb > INT64_MAX / 2 / rows) return CT_ERANGE;
    int64_t grid = rows * a.kb;
    if (block_rows == 1) grid = (grid + THREADS / (128 / per16) - 1) / (THREADS / (128 / per16));
    if (grid > INT32_MAX) return CT_ERANGE;
    cudaError_t e = dtype == CT_DT_F32   ? launch<float>(a, block_rows, grid, st)
                    : dtype == CT_DT_F16 ? launch<__half>(a, block_rows, grid, st)
                                         : launch<__nv_bfloat16>(a, block_rows, grid, st);
    return e == cudaSuccess ? CT_OK : CT_ECUDA;
}

}  // namespace ops
}  // namespace ct

extern "C" ct_status ct_fp8_quantize(const void *x_dev, int32_t dtype, int64_t m, int64_t k, int64_t ldx,
                                     int32_t block_rows, uint8_t *q_dev, int64_t ldq, float *scale_dev,
                                     int64_t scale_row, int64_t scale_blk, void *stream) {
    using namespace ct::ops;
    if (!dtype_ok(dtype) || (block_rows != 1 && block_rows != 128)) return CT_EINVAL;
    if (m < 0 || k < 0) return CT_ERANGE;
    if (m == 0 || k == 0) return CT_OK;
    if (x_dev == nullptr || q_dev == nullptr || scale_dev == nullptr || ldx < k || ldq < k) return CT_EINVAL;
    if (!aligned(x_dev, dtype_size(dtype)) || !aligned(scale_dev, 4)) return CT_EINVAL;
    return quantize(x_dev, dtype, m, k, ldx, block_rows, q_dev, ldq, scale_dev, scale_row, scale_blk,
                    static_cast<cudaStream_t>(stream));
}
