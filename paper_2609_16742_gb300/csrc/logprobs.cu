// Log probability of a given token, entropy, log normaliser and the most
// probable tokens of each row of logits, and the gradient of the first two.
//
// With m the row's maximum, Z = sum e^(x - m) and T = sum e^(x - m) (x - m):
//   lse = m + log Z,   log p[j] = x[j] - lse,   entropy = log Z - T / Z
// (both terms of the entropy are >= 0: nothing cancels).  A forbidden token
// (logit -inf) has probability 0 and adds nothing; where e^(x - m) is 0 the
// product with x - m is taken as 0, also when x - m overflows to -inf (a mask
// of the type's lowest value).  Sums are held in FP32.
#include "ops_common.cuh"

namespace ct {
namespace ops {
namespace {

constexpr float INF = __builtin_huge_valf();
__device__ __forceinline__ float nan_f() { return __uint_as_float(0x7FC00000u); }

struct LpArgs {
    const void *x;
    int64_t ldx;
    const int64_t *ids;
    int64_t rows;
    int64_t vocab;
    int top_k;
    float *lp, *entropy, *lse;
    float *top_lp;
    int64_t *top_id;
};

constexpr int THREADS = 256;

// running (m, Z, T) of a set of logits
struct Stat {
    float m, z, t;
};

__device__ __forceinline__ Stat merge(const Stat &a, const Stat &b) {
    Stat r;
    r.m = fmaxf(a.m, b.m);
    const float da = a.m == r.m ? 0.f : a.m - r.m, db = b.m == r.m ? 0.f : b.m - r.m;
    const float fa = expf(da), fb = expf(db);
    r.z = fa * a.z + fb * b.z;
    r.t = (fa == 0.f ? 0.f : fa * (a.t + da * a.z)) + (fb == 0.f ? 0.f : fb * (b.t + db * b.z));
    return r;
}

// order of the top tokens: the larger logit first, the lower index among equals; a key of 0 is no token
__device__ __forceinline__ uint64_t order_key(float x, int64_t j) {
    if (!(x > -INF)) return 0;
    const uint32_t b = __float_as_uint(x + 0.f);           // -0 and +0 are equal
    const uint32_t o = (b & 0x80000000u) ? ~b : (b | 0x80000000u);
    return ((uint64_t)o << 32) | (uint32_t)(0xFFFFFFFFu - (uint32_t)j);
}

template <typename T>
__global__ void __launch_bounds__(THREADS) logprobs_kernel(const LpArgs a) {
    __shared__ Stat part[THREADS / 32];
    __shared__ uint64_t best[THREADS / 32];
    __shared__ int bad_s;
    pdl_wait();
    pdl_trigger();
    const int64_t r = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + r * a.ldx;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    if (threadIdx.x == 0) bad_s = 0;
    __syncthreads();
    Stat s = {-INF, 0.f, 0.f};
    bool bad = false;
    for (int64_t j = threadIdx.x; j < a.vocab; j += THREADS) {
        const float v = to_f32(x[j]);
        bad |= !(v < INF);
        if (v > -INF) s = merge(s, Stat{v, 1.f, 0.f});
    }
    if (bad) bad_s = 1;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1)
        s = merge(s, Stat{__shfl_xor_sync(~0u, s.m, d), __shfl_xor_sync(~0u, s.z, d), __shfl_xor_sync(~0u, s.t, d)});
    if (lane == 0) part[warp] = s;
    __syncthreads();
    s = part[0];
    for (int w = 1; w < THREADS / 32; ++w) s = merge(s, part[w]);
    bad = bad_s != 0;
    const bool none = s.m == -INF;
    const float lz = logf(s.z);
    const float lse = bad ? nan_f() : none ? -INF : s.m + lz;
    if (threadIdx.x == 0) {
        a.lse[r] = lse;
        a.entropy[r] = bad ? nan_f() : none ? 0.f : lz - s.t / s.z;
        if (a.lp != nullptr) {
            const int64_t id = a.ids[r];
            float lp = nan_f();
            if (!bad && id == -1) lp = 0.f;
            else if (!bad && id >= 0 && id < a.vocab) {
                const float v = to_f32(x[id]);
                lp = v == -INF ? -INF : v - lse;
            }
            a.lp[r] = lp;
        }
    }
    uint64_t last = ~0ull;
    for (int k = 0; k < a.top_k; ++k) {
        uint64_t b = 0;
        if (!bad && last != 0)
            for (int64_t j = threadIdx.x; j < a.vocab; j += THREADS) {
                const uint64_t key = order_key(to_f32(x[j]), j);
                if (key < last && key > b) b = key;
            }
        for (int d = 16; d > 0; d >>= 1) b = max(b, __shfl_xor_sync(~0u, b, d));
        __syncthreads();
        if (lane == 0) best[warp] = b;
        __syncthreads();
        for (int w = 0; w < THREADS / 32; ++w) b = max(b, best[w]);
        last = b;
        if (threadIdx.x == 0) {
            const int64_t j = b == 0 ? -1 : (int64_t)(0xFFFFFFFFu - (uint32_t)b);
            a.top_id[r * a.top_k + k] = j;
            a.top_lp[r * a.top_k + k] = bad ? nan_f() : b == 0 ? -INF : to_f32(x[j]) - lse;
        }
    }
}

struct GradArgs {
    const void *x;
    int64_t ldx;
    const int64_t *ids;
    const float *lse, *entropy, *g_lp, *g_h;
    void *dx;
    int64_t lddx;
    int64_t rows, vocab;
    int vec;
};

template <typename T>
__global__ void __launch_bounds__(THREADS) logprobs_grad_kernel(const GradArgs a, int chunks, int64_t chunk) {
    pdl_wait();
    pdl_trigger();
    const int64_t r = blockIdx.x / chunks;
    const int64_t j0 = blockIdx.x % chunks * chunk, j1 = min(j0 + chunk, a.vocab);
    const T *x = static_cast<const T *>(a.x) + r * a.ldx;
    T *dx = static_cast<T *>(a.dx) + r * a.lddx;
    const float lse = a.lse[r];
    const int64_t id = a.g_lp != nullptr ? a.ids[r] : -1;
    const float g = id == -1 ? 0.f : id >= 0 && id < a.vocab ? a.g_lp[r] : nan_f();
    const float gh = a.g_h != nullptr ? a.g_h[r] : 0.f;
    const float h = a.g_h != nullptr ? a.entropy[r] : 0.f;
    for (int64_t j = j0 + threadIdx.x; j < j1; j += THREADS) {
        const float v = to_f32(x[j]);
        const float lp = v - lse;
        float p = v == -INF ? 0.f : expf(lp);
        float d = p == 0.f ? 0.f : -p * (g + gh * (lp + h));
        if (j == id) d += g;
        if (lse != lse || g != g) d = nan_f();
        dx[j] = from_f32<T>(d);
    }
}

}  // namespace
}  // namespace ops
}  // namespace ct

extern "C" ct_status ct_logprobs(const void *logits_dev, int32_t dtype, int64_t ld, const int64_t *ids_dev,
                                 int64_t rows, int64_t vocab, int32_t top_k, float *logprob_dev, float *entropy_dev,
                                 float *lse_dev, float *top_logprob_dev, int64_t *top_id_dev, void *stream) {
    using namespace ct::ops;
    if (!dtype_ok(dtype)) return CT_EINVAL;
    if (rows < 0 || vocab < 0 || rows > INT32_MAX || vocab > INT32_MAX || top_k < 0 || top_k > CT_MAX_TOP_K)
        return CT_ERANGE;
    if (rows == 0) return CT_OK;
    if (entropy_dev == nullptr || lse_dev == nullptr || (logprob_dev != nullptr && ids_dev == nullptr)) return CT_EINVAL;
    if (top_k > 0 && (top_logprob_dev == nullptr || top_id_dev == nullptr)) return CT_EINVAL;
    if (vocab > 0 && (logits_dev == nullptr || (ld < vocab && rows > 1) || !ct::ops::aligned(logits_dev, dtype_size(dtype))))
        return CT_EINVAL;
    if (!ct::ops::aligned(ids_dev, 8) || !ct::ops::aligned(logprob_dev, 4) || !ct::ops::aligned(entropy_dev, 4) ||
        !ct::ops::aligned(lse_dev, 4) || !ct::ops::aligned(top_logprob_dev, 4) || !ct::ops::aligned(top_id_dev, 8))
        return CT_EINVAL;
    const LpArgs a = {logits_dev, ld, ids_dev, rows, vocab, top_k, logprob_dev, entropy_dev, lse_dev, top_logprob_dev,
                      top_id_dev};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const dim3 grid((unsigned)rows), block(THREADS);
    const cudaError_t e = dtype == CT_DT_F32   ? ct::pdl_launch(logprobs_kernel<float>, grid, block, 0, st, a)
                          : dtype == CT_DT_F16 ? ct::pdl_launch(logprobs_kernel<__half>, grid, block, 0, st, a)
                                               : ct::pdl_launch(logprobs_kernel<__nv_bfloat16>, grid, block, 0, st, a);
    return e == cudaSuccess ? CT_OK : CT_ECUDA;
}

extern "C" ct_status ct_logprobs_grad(const void *logits_dev, int32_t dtype, int64_t ld, const int64_t *ids_dev,
                                      int64_t rows, int64_t vocab, const float *lse_dev, const float *entropy_dev,
                                      const float *g_logprob_dev, const float *g_entropy_dev, void *dlogits_dev,
                                      int64_t ld_d, void *stream) {
    using namespace ct::ops;
    if (!dtype_ok(dtype)) return CT_EINVAL;
    if (rows < 0 || vocab < 0 || rows > INT32_MAX || vocab > INT32_MAX) return CT_ERANGE;
    if (rows == 0 || vocab == 0) return CT_OK;
    if (logits_dev == nullptr || dlogits_dev == nullptr || lse_dev == nullptr) return CT_EINVAL;
    if (rows > 1 && (ld < vocab || ld_d < vocab)) return CT_EINVAL;
    if ((g_logprob_dev != nullptr && ids_dev == nullptr) || (g_entropy_dev != nullptr && entropy_dev == nullptr))
        return CT_EINVAL;
    const int es = dtype_size(dtype);
    if (!ct::ops::aligned(logits_dev, es) || !ct::ops::aligned(dlogits_dev, es) || !ct::ops::aligned(ids_dev, 8) ||
        !ct::ops::aligned(lse_dev, 4) || !ct::ops::aligned(entropy_dev, 4) || !ct::ops::aligned(g_logprob_dev, 4) ||
        !ct::ops::aligned(g_entropy_dev, 4))
        return CT_EINVAL;
    const GradArgs a = {logits_dev, ld, ids_dev, lse_dev, entropy_dev, g_logprob_dev, g_entropy_dev, dlogits_dev, ld_d,
                        rows, vocab, 0};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int64_t chunk = 8192, chunks = (vocab + chunk - 1) / chunk;
    if (rows > INT32_MAX / chunks) return CT_ERANGE;
    const dim3 grid((unsigned)(rows * chunks)), block(THREADS);
    const cudaError_t e =
        dtype == CT_DT_F32   ? ct::pdl_launch(logprobs_grad_kernel<float>, grid, block, 0, st, a, (int)chunks, chunk)
        : dtype == CT_DT_F16 ? ct::pdl_launch(logprobs_grad_kernel<__half>, grid, block, 0, st, a, (int)chunks, chunk)
                             : ct::pdl_launch(logprobs_grad_kernel<__nv_bfloat16>, grid, block, 0, st, a, (int)chunks,
                                              chunk);
    return e == cudaSuccess ? CT_OK : CT_ECUDA;
}
