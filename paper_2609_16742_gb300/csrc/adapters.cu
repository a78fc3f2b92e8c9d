// Low-rank adapters of many requests beside a shared projection, and their
// gradients.
//
//   v[t] = scale[i] A[i] x[t],  y[t] = act(y[t] + B[i] v[t]),  i = ids[t]
//   u[t] = scale[i] B[i]^T dy[t],  dx[t] += A[i]^T u[t],
//   dA[i] = sum_t u[t] x[t]^T,  dB[i] = sum_t dy[t] v[t]^T
//
// v and u are FP32: they are short, and rounding them to 16 bits would cost the
// result as much as its own rounding does.
#include "ops_common.cuh"

namespace ct {
namespace ops {
namespace {

constexpr int THREADS = 256;

// a tensor of one of the three types
struct Any {
    const void *p;
    int64_t ld;                                   // of rows
    int64_t la;                                   // of adapters
    int32_t dtype;
    __device__ __forceinline__ float at(int64_t i) const {
        return dtype == CT_DT_F32   ? static_cast<const float *>(p)[i]
               : dtype == CT_DT_F16 ? to_f32(static_cast<const __half *>(p)[i])
                                    : to_f32(static_cast<const __nv_bfloat16 *>(p)[i]);
    }
};

__device__ __forceinline__ void put(void *p, int32_t dtype, int64_t i, float v) {
    if (dtype == CT_DT_F32) static_cast<float *>(p)[i] = v;
    else if (dtype == CT_DT_F16) static_cast<__half *>(p)[i] = __float2half_rn(v);
    else static_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(v);
}

__device__ __forceinline__ int64_t adapter_of(const int64_t *ids, int64_t t) { return ids != nullptr ? ids[t] : 0; }

// v[t][j] = scale sum_c m[i](j, c) x[t][c]; m(j, c) at j * sj + c * sc.  A warp for each j, a block for each row.
__global__ void __launch_bounds__(THREADS) shrink_kernel(Any x, Any m, int64_t sj, int64_t sc, const int64_t *ids, const float *scale,
                                                         int64_t adapters, int rank, int64_t cols, float *v) {
    pdl_wait();
    pdl_trigger();
    const int64_t t = blockIdx.x, i = adapter_of(ids, t);
    if (i < 0 || i >= adapters) return;
    const int lane = threadIdx.x & 31;
    const float s = scale != nullptr ? scale[i] : 1.f;
    for (int j = threadIdx.x >> 5; j < rank; j += THREADS / 32) {
        double sum = 0.0;
        for (int64_t c0 = 0; c0 < cols; c0 += 1024) {
            float part = 0.f;
            for (int64_t c = c0 + lane; c < min(c0 + 1024, cols); c += 32) part = fmaf(x.at(t * x.ld + c), m.at(i * m.la + j * sj + c * sc), part);
            sum += part;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) v[t * rank + j] = (float)(sum * s);
    }
}

// y[t][c] = act(y[t][c] + sum_j m[i](c, j) v[t][j]); m(c, j) at c * sc + j * sj
__global__ void __launch_bounds__(THREADS) expand_kernel(void *y, int32_t y_dtype, int64_t ldy, Any m, int64_t sc, int64_t sj,
                                                         const int64_t *ids, int64_t adapters, int rank, int64_t cols, int relu,
                                                         const float *v) {
    pdl_wait();
    pdl_trigger();
    const int64_t t = blockIdx.x, i = adapter_of(ids, t);
    if (i == -1 && !relu) return;
    const bool out = i < -1 || i >= adapters;
    const Any yv = {y, ldy, 0, y_dtype};
    for (int64_t c = blockIdx.y * (int64_t)THREADS + threadIdx.x; c < cols; c += (int64_t)gridDim.y * THREADS) {
        float s = 0.f;
        if (i >= 0 && !out)
            for (int j = 0; j < rank; ++j) s = fmaf(m.at(i * m.la + c * sc + j * sj), v[t * rank + j], s);
        s += yv.at(t * ldy + c);
        if (relu) s = s < 0.f ? 0.f : s;
        put(y, y_dtype, t * ldy + c, out ? __uint_as_float(0x7FC00000u) : s);
    }
}

// g[i](j, c) = sum over the rows t of adapter i of v[t][j] x[t][c]; a block: 256 c of one j of one adapter.  g at j * gj + c * gc.
__global__ void __launch_bounds__(THREADS) outer_kernel(Any x, const float *v, const int64_t *ids, int64_t rows, int rank, int64_t cols,
                                                        void *g, int32_t g_dtype, int64_t gj, int64_t gc) {
    pdl_wait();
    pdl_trigger();
    const int64_t i = blockIdx.z, c = blockIdx.x * (int64_t)THREADS + threadIdx.x;
    const int j = blockIdx.y;
    if (c >= cols) return;
    double sum = 0.0;
    for (int64_t t0 = 0; t0 < rows; t0 += 64) {
        float part = 0.f;
        for (int64_t t = t0; t < min(t0 + 64, rows); ++t)
            if (adapter_of(ids, t) == i) part = fmaf(v[t * rank + j], x.at(t * x.ld + c), part);
        sum += part;
    }
    put(g, g_dtype, i * rank * cols + j * gj + c * gc, (float)sum);
}

inline bool adapter_matrix_ok(const void *p, int64_t sa, int64_t sr, int64_t adapters, int64_t rows, int64_t cols, int es) {
    if (adapters == 0 || rows == 0 || cols == 0) return true;
    return p != nullptr && aligned(p, es) && sa >= 0 && sr >= 0 && (rows == 1 || sr >= cols || sr == 0);
}
inline bool matrix_ok(const void *p, int64_t ld, int64_t rows, int64_t cols, int es) {
    if (rows == 0 || cols == 0) return true;
    return p != nullptr && aligned(p, es) && (rows == 1 || ld >= cols);
}
inline bool sizes_ok(int64_t t, int64_t adapters, int64_t rank, int64_t k, int64_t n) {
    return t >= 0 && t <= INT32_MAX && adapters >= 0 && adapters <= 65535 && rank >= 0 && rank <= CT_MAX_RANK && k >= 0 && k <= INT32_MAX &&
           n >= 0 && n <= INT32_MAX;
}
inline size_t part_bytes(int64_t t, int64_t rank) { return ((size_t)t * (size_t)rank * 4 + 15) / 16 * 16; }

cudaError_t shrink(const Any &x, const Any &m, int64_t sj, int64_t sc, const int64_t *ids, const float *scale, int64_t t, int64_t adapters,
                   int rank, int64_t cols, float *v, cudaStream_t st) {
    return pdl_launch(shrink_kernel, dim3((unsigned)t), dim3(THREADS), 0, st, x, m, sj, sc, ids, scale, adapters, rank, cols, v);
}
cudaError_t expand(void *y, int32_t y_dtype, int64_t ldy, const Any &m, int64_t sc, int64_t sj, const int64_t *ids, int64_t t,
                   int64_t adapters, int rank, int64_t cols, int relu, const float *v, cudaStream_t st) {
    const int64_t by = (cols + THREADS - 1) / THREADS;
    return pdl_launch(expand_kernel, dim3((unsigned)t, (unsigned)(by < 256 ? by : 256)), dim3(THREADS), 0, st, y, y_dtype, ldy, m, sc, sj,
                      ids, adapters, rank, cols, relu, v);
}
cudaError_t outer(const Any &x, const float *v, const int64_t *ids, int64_t t, int64_t adapters, int rank, int64_t cols, void *g,
                  int32_t g_dtype, int64_t gj, int64_t gc, cudaStream_t st) {
    return pdl_launch(outer_kernel, dim3((unsigned)((cols + THREADS - 1) / THREADS), (unsigned)rank, (unsigned)adapters), dim3(THREADS), 0,
                      st, x, v, ids, t, rank, cols, g, g_dtype, gj, gc);
}
}  // namespace
}  // namespace ops
}  // namespace ct

extern "C" ct_status ct_adapters_workspace(int64_t t, int64_t adapters, int64_t rank, int64_t k, int64_t n, size_t *bytes) {
    using namespace ct::ops;
    if (bytes == nullptr) return CT_EINVAL;
    if (!sizes_ok(t, adapters, rank, k, n)) return CT_ERANGE;
    *bytes = part_bytes(t, rank);
    return CT_OK;
}

extern "C" ct_status ct_adapters(void *y_dev, int32_t y_dtype, int64_t ldy, const void *x_dev, int32_t x_dtype, int64_t ldx,
                                 const void *a_dev, int64_t a_adapter, int64_t a_row, const void *b_dev, int64_t b_adapter,
                                 int64_t b_row, int32_t dtype, const int64_t *ids_dev, const float *scale_dev, int64_t t,
                                 int64_t adapters, int64_t rank, int64_t k, int64_t n, int32_t relu, void *workspace_dev,
                                 size_t workspace_bytes, void *stream) {
    using namespace ct::ops;
    if (!dtype_ok(y_dtype) || !dtype_ok(dtype) || (x_dtype != dtype && x_dtype != CT_DT_F32)) return CT_EINVAL;
    if (!sizes_ok(t, adapters, rank, k, n)) return CT_ERANGE;
    if (t == 0 || n == 0) return CT_OK;
    const int es = dtype_size(dtype);
    if (!matrix_ok(y_dev, ldy, t, n, dtype_size(y_dtype)) || !matrix_ok(x_dev, ldx, t, k, dtype_size(x_dtype)) ||
        !adapter_matrix_ok(a_dev, a_adapter, a_row, adapters, rank, k, es) ||
        !adapter_matrix_ok(b_dev, b_adapter, b_row, adapters, n, rank, es) || !aligned(ids_dev, 8) || !aligned(scale_dev, 4))
        return CT_EINVAL;
    if (ids_dev == nullptr && adapters == 0) return CT_EINVAL;
    if (part_bytes(t, rank) > 0 && (workspace_dev == nullptr || !aligned(workspace_dev, 16))) return CT_EINVAL;
    if (workspace_bytes < part_bytes(t, rank)) return CT_ENOMEM;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    float *v = static_cast<float *>(workspace_dev);
    cudaError_t e = cudaSuccess;
    if (rank > 0) e = shrink({x_dev, ldx, 0, x_dtype}, {a_dev, 0, a_adapter, dtype}, a_row, 1, ids_dev, scale_dev, t, adapters, (int)rank, k, v, st);
    if (e == cudaSuccess) e = expand(y_dev, y_dtype, ldy, {b_dev, 0, b_adapter, dtype}, b_row, 1, ids_dev, t, adapters, (int)rank, n, relu != 0, v, st);
    return e == cudaSuccess ? CT_OK : CT_ECUDA;
}

extern "C" ct_status ct_adapters_grad_workspace(int64_t t, int64_t adapters, int64_t rank, int64_t k, int64_t n, size_t *bytes) {
    using namespace ct::ops;
    if (bytes == nullptr) return CT_EINVAL;
    if (!sizes_ok(t, adapters, rank, k, n)) return CT_ERANGE;
    *bytes = 2 * part_bytes(t, rank);
    return CT_OK;
}

extern "C" ct_status ct_adapters_grad(const void *dy_dev, int32_t dy_dtype, int64_t lddy, const void *x_dev, int32_t x_dtype,
                                      int64_t ldx, const void *a_dev, int64_t a_adapter, int64_t a_row, const void *b_dev,
                                      int64_t b_adapter, int64_t b_row, int32_t dtype, const int64_t *ids_dev,
                                      const float *scale_dev, int64_t t, int64_t adapters, int64_t rank, int64_t k, int64_t n,
                                      void *dx_dev, int32_t dx_dtype, int64_t lddx, void *da_dev, void *db_dev, int32_t grad_dtype,
                                      void *workspace_dev, size_t workspace_bytes, void *stream) {
    using namespace ct::ops;
    if (!dtype_ok(dtype) || (x_dtype != dtype && x_dtype != CT_DT_F32) || (dy_dtype != dtype && dy_dtype != CT_DT_F32) ||
        (grad_dtype != dtype && grad_dtype != CT_DT_F32) || (dx_dev != nullptr && !dtype_ok(dx_dtype)))
        return CT_EINVAL;
    if (!sizes_ok(t, adapters, rank, k, n)) return CT_ERANGE;
    const int es = dtype_size(dtype), ges = dtype_size(grad_dtype);
    if (!matrix_ok(dy_dev, lddy, t, n, dtype_size(dy_dtype)) || !matrix_ok(x_dev, ldx, t, k, dtype_size(x_dtype)) ||
        !adapter_matrix_ok(a_dev, a_adapter, a_row, adapters, rank, k, es) ||
        !adapter_matrix_ok(b_dev, b_adapter, b_row, adapters, n, rank, es) || !aligned(ids_dev, 8) || !aligned(scale_dev, 4) ||
        (dx_dev != nullptr && !matrix_ok(dx_dev, lddx, t, k, dtype_size(dx_dtype))) ||
        (adapters * rank * k > 0 && (da_dev == nullptr || !aligned(da_dev, ges))) ||
        (adapters * rank * n > 0 && (db_dev == nullptr || !aligned(db_dev, ges))))
        return CT_EINVAL;
    if (ids_dev == nullptr && adapters == 0 && t > 0) return CT_EINVAL;
    const size_t part = part_bytes(t, rank);
    if (part > 0 && (workspace_dev == nullptr || !aligned(workspace_dev, 16))) return CT_EINVAL;
    if (workspace_bytes < 2 * part) return CT_ENOMEM;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    float *v = static_cast<float *>(workspace_dev), *u = v + part / 4;
    const Any x = {x_dev, ldx, 0, x_dtype}, dy = {dy_dev, lddy, 0, dy_dtype}, a = {a_dev, 0, a_adapter, dtype}, b = {b_dev, 0, b_adapter, dtype};
    const int r = (int)rank;
    cudaError_t e = cudaSuccess;
    if (t > 0 && rank > 0) {
        e = shrink(x, a, a_row, 1, ids_dev, scale_dev, t, adapters, r, k, v, st);
        if (e == cudaSuccess) e = shrink(dy, b, 1, b_row, ids_dev, scale_dev, t, adapters, r, n, u, st);
    }
    if (e == cudaSuccess && t > 0 && k > 0 && dx_dev != nullptr)
        e = expand(dx_dev, dx_dtype, lddx, a, 1, a_row, ids_dev, t, adapters, r, k, 0, u, st);
    if (e == cudaSuccess && adapters * rank * k > 0) e = outer(x, u, ids_dev, t, adapters, r, k, da_dev, grad_dtype, k, 1, st);
    if (e == cudaSuccess && adapters * rank * n > 0) e = outer(dy, v, ids_dev, t, adapters, r, n, db_dev, grad_dtype, 1, rank, st);
    return e == cudaSuccess ? CT_OK : CT_ECUDA;
}
