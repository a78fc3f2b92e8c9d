// The norm of many tensors together, the norm of each, and their values scaled
// so that the norm is at most a given one.
//
//   norm_i = sqrt(sum g^2) or max |g|,  norm = the same over the norm_i,
//   g' = g c,  c = min(1, max_norm / norm)
//
// A thread sums the squares of at most 1024 values in FP32; what it found goes on
// in FP64, joined in a fixed order, so that long sums lose nothing and
// the result does not depend on the run.  Squares leave FP32's range long before the
// values do: a thread whose largest magnitude is outside [2^-50, 2^55] sums again
// with its values scaled by a power of two.
#include <algorithm>
#include <vector>

#include "ops_common.cuh"

namespace ct {
namespace ops {
namespace {

constexpr int THREADS = 256;
constexpr int64_t LEAST = 4096, MOST = 1024 * THREADS;   // values of a block

struct ClipTensor {
    const void *src;
    void *dst;
    int64_t rows, cols, ld_src, ld_dst;
    int32_t dtype;
    int32_t block0;                               // its first block, of the launch
};

// tensors of one launch: passed by value, so that a captured launch holds them
template <int N> struct Table {
    ClipTensor t[N];
    int n;                                        // tensors here
    int base;                                     // blocks of the launches before
    int first;                                    // tensors of the launches before
    int64_t chunk;                                // values of a block
};
constexpr int SMALL = 48, LARGE = 480;            // 2.7 and 27 KB of arguments (at most 32,764 bytes)

struct Part {
    double sum;                                   // of the squares
    float top;                                    // largest magnitude, or NaN
    float pad;
};

__device__ __forceinline__ float load(const ClipTensor &t, int64_t i) {
    const int64_t r = t.rows == 1 ? 0 : i / t.cols, at = r * t.ld_src + (i - r * t.cols);
    return t.dtype == CT_DT_F32   ? static_cast<const float *>(t.src)[at]
           : t.dtype == CT_DT_F16 ? to_f32(static_cast<const __half *>(t.src)[at])
                                  : to_f32(static_cast<const __nv_bfloat16 *>(t.src)[at]);
}

__device__ __forceinline__ float join_top(float a, float b) { return a != a ? a : (b != b ? b : fmaxf(a, b)); }

template <typename TAB> __device__ __forceinline__ int find(const TAB &tab, int block) {
    int lo = 0, hi = tab.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (tab.t[mid].block0 <= block) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

template <int N> __global__ void __launch_bounds__(THREADS) clip_parts_kernel(const __grid_constant__ Table<N> tab, Part *parts) {
    pdl_wait();
    pdl_trigger();
    const ClipTensor &t = tab.t[find(tab, (int)blockIdx.x)];
    const int64_t total = t.rows * t.cols, i0 = (int64_t)((int)blockIdx.x - t.block0) * tab.chunk, i1 = min(i0 + tab.chunk, total);
    float s = 0.f, m = 0.f;
    for (int64_t i = i0 + threadIdx.x; i < i1; i += THREADS) {
        const float v = load(t, i);
        s = fmaf(v, v, s);
        m = fmaxf(m, fabsf(v));
    }
    double sum = s;
    if (s == s && m > 0.f && m < __builtin_huge_valf() && (m > 0x1p55f || m < 0x1p-50f)) {
        const int e = ilogbf(m);
        s = 0.f;
        for (int64_t i = i0 + threadIdx.x; i < i1; i += THREADS) {
            const float v = ldexpf(load(t, i), -e);
            s = fmaf(v, v, s);
        }
        sum = ldexp((double)s, 2 * e);
    }
    if (s != s) m = s;
    __shared__ double ss[THREADS / 32];
    __shared__ float sm[THREADS / 32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
        m = join_top(m, __shfl_xor_sync(0xffffffffu, m, o));
    }
    if ((threadIdx.x & 31) == 0) {
        ss[threadIdx.x >> 5] = sum;
        sm[threadIdx.x >> 5] = m;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < THREADS / 32; ++w) {
            sum += ss[w];
            m = join_top(m, sm[w]);
        }
        parts[tab.base + blockIdx.x] = {sum, m, 0.f};
    }
}

// What the launches hand on: sums over the tensors so far, then the factor.
struct Found {
    double sum;
    float top;
    float factor;
};

// One block: the norms of a launch's tensors from their blocks' parts, a warp a
// tensor, each in the order of its values; after the last launch's the factor.
constexpr int JOIN_WARPS = 32;
template <int N> __global__ void __launch_bounds__(32 * JOIN_WARPS)
clip_join_kernel(const __grid_constant__ Table<N> tab, const Part *parts, int blocks, Found *found, float *norms, int kind,
                 double max_norm, float *norm, int last) {
    pdl_wait();
    pdl_trigger();
    __shared__ double ss[N];
    __shared__ float sm[N];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int i = warp; i < tab.n; i += JOIN_WARPS) {
        const int p0 = tab.t[i].block0, p1 = i + 1 < tab.n ? tab.t[i + 1].block0 : blocks;
        double sum = 0.0;
        float m = 0.f;
        for (int p = p0 + lane; p < p1; p += 32) {
            sum += parts[tab.base + p].sum;
            m = join_top(m, parts[tab.base + p].top);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            sum += __shfl_xor_sync(0xffffffffu, sum, o);
            m = join_top(m, __shfl_xor_sync(0xffffffffu, m, o));
        }
        if (lane == 0) {
            ss[i] = sum;
            sm[i] = m;
            norms[tab.first + i] = kind == CT_NORM_2 ? (float)sqrt(sum) : m;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        Found f = tab.first > 0 ? *found : Found{0.0, 0.f, 1.f};
        for (int i = 0; i < tab.n; ++i) {
            f.sum += ss[i];
            f.top = join_top(f.top, sm[i]);
        }
        if (last) {
            const double v = kind == CT_NORM_2 ? sqrt(f.sum) : (double)f.top;
            *norm = (float)v;
            f.factor = isfinite((float)v) && v > max_norm ? (float)(max_norm / v) : 1.f;
        }
        *found = f;
    }
}

template <int N> __global__ void __launch_bounds__(THREADS) clip_scale_kernel(const __grid_constant__ Table<N> tab, const Found *found) {
    pdl_wait();
    pdl_trigger();
    const ClipTensor &t = tab.t[find(tab, (int)blockIdx.x)];
    const float c = found->factor;
    if (c == 1.f && t.src == t.dst) return;
    const int64_t total = t.rows * t.cols, i0 = (int64_t)((int)blockIdx.x - t.block0) * tab.chunk, i1 = min(i0 + tab.chunk, total);
    for (int64_t i = i0 + threadIdx.x; i < i1; i += THREADS) {
        const float v = load(t, i);
        const int64_t r = t.rows == 1 ? 0 : i / t.cols, at = r * t.ld_dst + (i - r * t.cols);
        const float o = c == 1.f ? v : v * c;
        if (t.dtype == CT_DT_F32) static_cast<float *>(t.dst)[at] = o;
        else if (t.dtype == CT_DT_F16) static_cast<__half *>(t.dst)[at] = __float2half_rn(o);
        else static_cast<__nv_bfloat16 *>(t.dst)[at] = __float2bfloat16_rn(o);
    }
}

inline bool tensor_ok(const ct_tensor &t) {
    if (t.rows == 0 || t.cols == 0) return true;
    const int size = dtype_size((int)t.dtype);
    return t.src != nullptr && t.dst != nullptr && aligned(t.src, size) && aligned(t.dst, size) &&
           (t.rows == 1 || (t.ld_src >= t.cols && t.ld_dst >= t.cols));
}

// bytes from a tensor's first value to behind its last
struct Range {
    uintptr_t from, to;
    int64_t row, pitch;                           // bytes
};

// whether two ranges touch: side by side as columns of one matrix is fine
bool overlap(std::vector<Range> &v) {
    std::sort(v.begin(), v.end(), [](const Range &a, const Range &b) { return a.from < b.from; });
    for (size_t i = 0; i < v.size(); ++i)
        for (size_t j = i + 1; j < v.size() && v[j].from < v[i].to; ++j) {
            const int64_t pitch = v[i].pitch, off = (int64_t)((v[j].from - v[i].from) % (uintptr_t)(pitch > 0 ? pitch : 1));
            if (pitch == 0 || pitch != v[j].pitch || off < v[i].row || off + v[j].row > pitch) return true;
        }
    return false;
}

// values of a block: blocks enough for the whole GPU, with something to do for each
int64_t chunk_of(int64_t total) {
    const int64_t want = (total + 1215) / 1216;   // 8 blocks of each of 152 SMs
    const int64_t c = (want + 1023) / 1024 * 1024;
    return c < LEAST ? LEAST : c > MOST ? MOST : c;
}

ct_status measure(const ct_tensor *t, int64_t n, int64_t *total, int64_t *blocks) {
    if (n < 0 || n > INT32_MAX) return CT_ERANGE;
    if (n > 0 && t == nullptr) return CT_EINVAL;
    *total = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (t[i].rows < 0 || t[i].cols < 0 || (t[i].rows > 0 && t[i].cols > (INT64_MAX >> 8) / t[i].rows)) return CT_ERANGE;
        *total += t[i].rows * t[i].cols;
        if (*total > INT64_MAX >> 8) return CT_ERANGE;
    }
    const int64_t chunk = chunk_of(*total);
    *blocks = 0;
    for (int64_t i = 0; i < n; ++i) *blocks += (t[i].rows * t[i].cols + chunk - 1) / chunk;
    return *blocks > INT32_MAX ? CT_ERANGE : CT_OK;
}

template <int N>
cudaError_t launch(const ct_tensor *t, int64_t n, int64_t chunk, int kind, double max_norm, float *norms, float *norm, Part *parts,
                   Found *found, cudaStream_t st) {
    Table<N> tab;
    tab.chunk = chunk;
    for (int pass = 0; pass < 2; ++pass) {
        tab.base = 0;
        for (int64_t first = 0; first < n || first == 0; first += N) {
            tab.first = (int)first;
            tab.n = (int)std::min<int64_t>(N, n - first);
            int64_t blocks = 0;
            for (int i = 0; i < tab.n; ++i) {
                const ct_tensor &q = t[first + i];
                const bool flat = q.rows <= 1 || (q.ld_src == q.cols && q.ld_dst == q.cols);
                tab.t[i] = {q.src, q.dst, flat ? 1 : q.rows, flat ? q.rows * q.cols : q.cols, q.ld_src, q.ld_dst, (int32_t)q.dtype,
                            (int32_t)blocks};
                blocks += (q.rows * q.cols + chunk - 1) / chunk;
            }
            cudaError_t e = cudaSuccess;
            const dim3 grid((unsigned)blocks), block(THREADS);
            if (pass == 0) {
                if (blocks > 0) e = pdl_launch(clip_parts_kernel<N>, grid, block, 0, st, tab, parts);
                if (e == cudaSuccess)
                    e = pdl_launch(clip_join_kernel<N>, dim3(1), dim3(32 * JOIN_WARPS), 0, st, tab, (const Part *)parts, (int)blocks,
                                   found, norms, kind, max_norm, norm, (int)(first + N >= n));
            } else if (blocks > 0) {
                e = pdl_launch(clip_scale_kernel<N>, grid, block, 0, st, tab, (const Found *)found);
            }
            if (e != cudaSuccess) return e;
            tab.base += (int)blocks;
        }
    }
    return cudaSuccess;
}
}  // namespace
}  // namespace ops
}  // namespace ct

extern "C" ct_status ct_clip_grads_workspace(const ct_tensor *tensors, int64_t n, size_t *bytes) {
    using namespace ct::ops;
    if (bytes == nullptr) return CT_EINVAL;
    int64_t total, blocks;
    const ct_status s = measure(tensors, n, &total, &blocks);
    if (s == CT_OK) *bytes = sizeof(Found) + sizeof(Part) * (size_t)blocks;
    return s;
}

extern "C" ct_status ct_clip_grads(const ct_tensor *tensors, int64_t n, int32_t kind, double max_norm, float *norms_dev,
                                   float *norm_dev, void *workspace_dev, size_t workspace_bytes, void *stream) {
    using namespace ct::ops;
    if ((kind != CT_NORM_2 && kind != CT_NORM_INF) || !(max_norm >= 0.0)) return CT_EINVAL;
    int64_t total, blocks;
    const ct_status s = measure(tensors, n, &total, &blocks);
    if (s != CT_OK) return s;
    if (norm_dev == nullptr || !aligned(norm_dev, 4) || (n > 0 && (norms_dev == nullptr || !aligned(norms_dev, 4)))) return CT_EINVAL;
    for (int64_t i = 0; i < n; ++i)
        if (tensors[i].dtype < CT_DT_F32 || tensors[i].dtype > CT_DT_BF16 || !tensor_ok(tensors[i])) return CT_EINVAL;
    if (workspace_dev == nullptr || !aligned(workspace_dev, 16)) return CT_EINVAL;
    if (workspace_bytes < sizeof(Found) + sizeof(Part) * (size_t)blocks) return CT_ENOMEM;
    try {
        std::vector<Range> v;
        v.reserve(2 * (size_t)n);
        for (int64_t i = 0; i < n; ++i) {
            const ct_tensor &t = tensors[i];
            if (t.rows == 0 || t.cols == 0) continue;
            const int64_t size = dtype_size((int)t.dtype), rows = t.rows - 1;
            const auto range = [&](const void *p, int64_t ld) {
                const uintptr_t at = (uintptr_t)p;
                v.push_back({at, at + (uintptr_t)((rows * ld + t.cols) * size), t.cols * size, rows > 0 ? ld * size : 0});
            };
            range(t.dst, t.ld_dst);
            if (t.src != t.dst) range(t.src, t.ld_src);
            else if (rows > 0 && t.ld_src != t.ld_dst) return CT_EINVAL;
        }
        if (overlap(v)) return CT_EINVAL;
    } catch (const std::exception &) {
        return CT_ENOMEM;
    }
    Found *found = static_cast<Found *>(workspace_dev);
    Part *parts = reinterpret_cast<Part *>(found + 1);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int64_t chunk = chunk_of(total);
    const cudaError_t e = n <= SMALL ? launch<SMALL>(tensors, n, chunk, kind, max_norm, norms_dev, norm_dev, parts, found, st)
                                     : launch<LARGE>(tensors, n, chunk, kind, max_norm, norms_dev, norm_dev, parts, found, st);
    return e == cudaSuccess ? CT_OK : CT_ECUDA;
}
