// Quantisation to 8-bit floating point (e4m3) with one scale for each block
// of 128 values of a row, or of 128 x 128 values.  fp8_quantize.cuh has the
// definition of a block's scale and values.
#include "fp8_quantize.cuh"

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

// 16 bytes of values, of which the first `have` are the row's, from wherever
// they start, of N rows `step` apart (none from row `rows` on): the 16-byte
// units that hold one of them, all in flight before the first is looked at;
// zeros for the others
template <typename T, int N>
__device__ __forceinline__ void load_any(const QuantArgs &a, int64_t r0, int64_t c0, int64_t step, int rows, int have,
                                         uint4 (&u)[N]) {
    constexpr int BATCH = N < 4 ? N : 4;     // registers of 8 units
    static_assert(N % BATCH == 0, "batches");
    const uintptr_t p0 = reinterpret_cast<uintptr_t>(static_cast<const T *>(a.x) + r0 * a.ldx + c0);
    const int64_t pitch = step * a.ldx * (int)sizeof(T);
    const int bytes = have * (int)sizeof(T);
#pragma unroll
    for (int h = 0; h < N; h += BATCH) {
        uint4 first[BATCH], second[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const uintptr_t p = p0 + (h + i) * pitch;
            const uint4 *at = reinterpret_cast<const uint4 *>(p & ~(uintptr_t)15);
            const bool any = h + i < rows && have > 0;
            first[i] = second[i] = make_uint4(0, 0, 0, 0);
            if (any) first[i] = __ldg(at);
            if (any && (int)(p & 15u) + bytes > 16) second[i] = __ldg(at + 1);
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i)
            u[h + i] = first_bytes(shifted(first[i], second[i], (uint32_t)(p0 + (h + i) * pitch) & 15u), bytes);
    }
}

template <typename T, int V> __device__ __forceinline__ void store_whole(uint8_t *p, const uint4 &u, float inv) {
    uint32_t w[V / 4];
    convert<T, V>(u, inv, w);
    if constexpr (V == 8) *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t *>(p) = w[0];
}

template <typename T, int V>
__device__ __forceinline__ void store_values(const QuantArgs &a, int64_t row, int64_t c0, bool vec, const uint4 &u,
                                             float inv) {
    uint8_t *p = a.q + row * a.ldq + c0;
    if (vec) {
        store_whole<T, V>(p, u, inv);
    } else {
        uint32_t w[V / 4];
        convert<T, V>(u, inv, w);
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (c0 + i < a.k) p[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
    }
}

constexpr int ROW_THREADS = 256;

// One block of 128 values of ROWS (1 or 8) consecutive rows for each group of
// 128 / V lanes: ROWS loads in flight.  With 8 rows the maxima are reduced by
// an exchange that halves the rows a lane keeps with each of its first three
// steps, so that each lane ends with one row's, makes that row's scale, and
// passes it round (8 + 8 shuffles and one scale a lane; row by row it was 32 to
// 40 and 8, 107 instructions for 128 FP32 values).  Where the scales lie block
// by block, the 8 are one 32-byte sector.
// Bound by HBM: 8192 x 4096 BF16 in 14.9 us, 6.8 TB/s.  Rows that start inside
// a 16-byte unit cost instructions: 5000 x 3001 BF16 in 13.2 us, 3.4 TB/s.
template <typename T, int ROWS>
__global__ void __launch_bounds__(ROW_THREADS, 4) quantize_rows_kernel(const QuantArgs a) {
    static_assert(ROWS == 1 || ROWS == 8, "one row, or the exchange's 8");
    constexpr int V = Vec16<T>::N;
    constexpr int G = 128 / V;               // lanes of a block: 32 (FP32) or 16
    constexpr int GROUPS = ROW_THREADS / G;
    constexpr uint32_t ALL = 0xFFFFFFFFu;
    pdl_wait();
    pdl_trigger();
    const int64_t blocks = (a.m + ROWS - 1) / ROWS * a.kb;
    const int g = threadIdx.x / G, l = threadIdx.x % G;
    const int64_t at = (int64_t)blockIdx.x * GROUPS + g;
    const bool live = at < blocks;
    int64_t r0 = 0, b = 0;
    if (live) {
        if (blocks <= UINT32_MAX) {          // a 32-bit division where it is enough
            r0 = (int64_t)((uint32_t)at / (uint32_t)a.kb) * ROWS;
            b = (uint32_t)at % (uint32_t)a.kb;
        } else {
            r0 = at / a.kb * ROWS;
            b = at % a.kb;
        }
    }
    const int64_t c0 = b * 128 + l * V;
    const bool whole = c0 + V <= a.k;
    const int rows = live ? (int)min((int64_t)ROWS, a.m - r0) : 0;
    const bool plain = rows == ROWS && whole && a.xvec && a.qvec;      // all of it, in whole accesses
    uint4 u[ROWS];
    if (plain) {
        const T *p = static_cast<const T *>(a.x) + r0 * a.ldx + c0;
#pragma unroll
        for (int i = 0; i < ROWS; ++i, p += a.ldx) u[i] = __ldcs(reinterpret_cast<const uint4 *>(p));
    } else {
        load_any<T, ROWS>(a, r0, c0, 1, rows, (int)max((int64_t)0, min((int64_t)V, a.k - c0)), u);
    }
    uint32_t mx[ROWS];
    bool odd = false;                        // something that is not finite
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        mx[i] = largest_any<T>(u[i]);
        odd |= mx[i] >= 0x7F800000u;
    }
    if (__any_sync(ALL, odd)) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) mx[i] = largest<T, V>(u[i]);
    }
    float s, inv;
    if constexpr (ROWS == 8) {
#pragma unroll
        for (int n = 4, d = G / 2; n > 0; n /= 2, d /= 2) {
            const bool upper = l & d;        // keeps the upper half of the rows
#pragma unroll
            for (int i = 0; i < n; ++i) {
                const uint32_t give = upper ? mx[i] : mx[i + n], keep = upper ? mx[i + n] : mx[i];
                mx[i] = max(keep, __shfl_xor_sync(ALL, give, d));
            }
        }
    }
#pragma unroll
    for (int d = ROWS == 8 ? G / 16 : G / 2; d > 0; d /= 2) mx[0] = max(mx[0], __shfl_xor_sync(ALL, mx[0], d));
    block_scale(mx[0], s, inv);              // of row l / (G / ROWS)
    float f[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) f[i] = ROWS == 1 ? inv : __shfl_sync(ALL, inv, i * (G / ROWS), G);
    if (plain) {
        uint8_t *p = a.q + r0 * a.ldq + c0;
#pragma unroll
        for (int i = 0; i < ROWS; ++i, p += a.ldq) store_whole<T, V>(p, u[i], f[i]);
    } else {
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
            if (i < rows) store_values<T, V>(a, r0 + i, c0, a.qvec && whole, u[i], f[i]);
    }
    const int mine = l / (G / ROWS);
    if (l % (G / ROWS) == 0 && mine < rows) a.scale[(r0 + mine) * a.srow + b * a.sblk] = s;
}

constexpr int BLOCK_THREADS = 512;

// One CTA per 128 x 128 block: its values stay in registers between the
// maximum and the rounding, so that HBM is read once and bounds it:
// 4096 x 25088 FP32 in 78.3 us, 6.6 TB/s.
template <typename T>
__global__ void __launch_bounds__(BLOCK_THREADS, 2) quantize_blocks_kernel(const QuantArgs a) {
    constexpr int V = Vec16<T>::N;
    constexpr int G = 128 / V;
    constexpr int ROWS = BLOCK_THREADS / G;  // rows of one step
    constexpr int STEPS = 128 / ROWS;
    __shared__ uint32_t part[BLOCK_THREADS / 32];
    pdl_wait();
    pdl_trigger();
    const int64_t br = blockIdx.x / a.kb, b = blockIdx.x % a.kb;
    const int g = threadIdx.x / G, l = threadIdx.x % G;
    const int64_t c0 = b * 128 + l * V, r0 = br * 128 + g;
    const bool inside = b * 128 + 128 <= a.k && br * 128 + 128 <= a.m;
    uint4 u[STEPS];
    if (inside && a.xvec) {                  // all loads in flight at once
        const T *p = static_cast<const T *>(a.x) + r0 * a.ldx + c0;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) u[i] = __ldg(reinterpret_cast<const uint4 *>(p + i * ROWS * a.ldx));
    } else {
        const int64_t left = a.m - r0;       // a row in ROWS is this thread's
        load_any<T, STEPS>(a, r0, c0, ROWS, left <= 0 ? 0 : (int)min((int64_t)STEPS, (left + ROWS - 1) / ROWS),
                           (int)max((int64_t)0, min((int64_t)V, a.k - c0)), u);
    }
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) amax = max(amax, largest<T, V>(u[i]));
    amax = __reduce_max_sync(0xFFFFFFFFu, amax);
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = amax;
    __syncthreads();
    amax = __reduce_max_sync(0xFFFFFFFFu, part[threadIdx.x % (BLOCK_THREADS / 32)]);
    float s, inv;
    block_scale(amax, s, inv);
#pragma unroll
    for (int i = 0; i < STEPS; ++i)
        if (r0 + i * ROWS < a.m) store_values<T, V>(a, r0 + i * ROWS, c0, a.qvec && c0 + V <= a.k, u[i], inv);
    if (threadIdx.x == 0) a.scale[br * a.srow + b * a.sblk] = s;
}

// rows that a group of the row kernel takes: 8, or one where there are fewer
int row_step(int64_t m) { return m >= 8 ? 8 : 1; }

template <typename T>
cudaError_t launch(const QuantArgs &a, int block_rows, int64_t grid, cudaStream_t st) {
    if (block_rows != 1)
        return pdl_launch(quantize_blocks_kernel<T>, dim3((unsigned)grid), dim3(BLOCK_THREADS), 0, st, a);
    return row_step(a.m) == 8 ? pdl_launch(quantize_rows_kernel<T, 8>, dim3((unsigned)grid), dim3(ROW_THREADS), 0, st, a)
                              : pdl_launch(quantize_rows_kernel<T, 1>, dim3((unsigned)grid), dim3(ROW_THREADS), 0, st, a);
}

}  // namespace

ct_status quantize(const void *x, int dtype, int64_t m, int64_t k, int64_t ldx, int block_rows, uint8_t *q, int64_t ldq,
                   float *scale, int64_t srow, int64_t sblk, cudaStream_t st) {
    const int es = dtype_size(dtype), per16 = 16 / es;
    QuantArgs a = {x, m, k, ldx, q, ldq, scale, srow, sblk, (k + 127) / 128, 0, 0};
    a.xvec = aligned(x, 16) && ldx % per16 == 0;
    a.qvec = aligned(q, per16) && ldq % per16 == 0;
    const int step = block_rows == 1 ? row_step(m) : block_rows;
    const int64_t rows = (m + step - 1) / step, groups = ROW_THREADS / (128 / per16);
    if (a.kb > INT64_MAX / 2 / rows) return CT_ERANGE;
    int64_t grid = rows * a.kb;
    if (block_rows == 1) grid = (grid + groups - 1) / groups;
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
