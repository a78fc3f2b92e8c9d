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
//
// Two launches, bound by HBM where there is much to read: every block of the second joins all blocks' parts itself, which costs it 2 us and
// saves a launch.  138 million FP32 values: 96 us for the norms (5.8 TB/s), 166 us for scaled copies (6.7 TB/s).  The second goes from the last
// block and its last values on, of which L2 still holds some: 264.4 us in all, 265.9 forwards; loads that ask L2 to keep them added nothing.
#include <algorithm>
#include <vector>

#include "ops_common.cuh"

namespace ct {
namespace ops {
namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
// values of a block; at most as many as leave a thread 1024 with its value before the first 16-byte unit and its one behind the last
constexpr int64_t LEAST = 4096, MOST = 1016 * THREADS;
constexpr int64_t BLOCKS = 1216;                  // wanted: 8 for each of a GB300's 152 SMs; the workspace's size hangs on no device
constexpr int UNROLL = 4;                         // 16-byte loads of a thread on their way together

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
    int blocks;                                   // blocks here
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
__device__ __forceinline__ void store(const ClipTensor &t, int64_t i, float v) {
    const int64_t r = t.rows == 1 ? 0 : i / t.cols, at = r * t.ld_dst + (i - r * t.cols);
    if (t.dtype == CT_DT_F32) static_cast<float *>(t.dst)[at] = v;
    else if (t.dtype == CT_DT_F16) static_cast<__half *>(t.dst)[at] = __float2half_rn(v);
    else static_cast<__nv_bfloat16 *>(t.dst)[at] = __float2bfloat16_rn(v);
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

// A block's run of a dense tensor: values before the first 16-byte boundary, 16-byte vectors, values behind them.
struct Run {
    int64_t i0, i1, head, vecs;
    __device__ __forceinline__ Run(const void *src, int size, int64_t from, int64_t to) : i0(from), i1(to) {
        const int64_t off = (int64_t)((16 - ((uintptr_t)src + (uintptr_t)(from * size)) % 16) % 16) / size;
        head = off < to - from ? off : to - from;
        vecs = (to - from - head) * size / 16;
    }
};

struct Found {
    float s, m;
};
__device__ __forceinline__ void see(Found &f, float v) {
    f.s = fmaf(v, v, f.s);
    f.m = fmaxf(f.m, fabsf(v));
}
// f(v) for every value of the thread's share of a run
template <typename T, typename F> __device__ __forceinline__ void each_value(const T *src, const Run &r, F f) {
    constexpr int E = 16 / (int)sizeof(T);
    const T *p = src + r.i0;
    const int tid = threadIdx.x;
    if (tid < r.head) f(to_f32(p[tid]));
    const int64_t tail = r.head + r.vecs * E;
    if (tail + tid < r.i1 - r.i0) f(to_f32(p[tail + tid]));
    const uint4 *q = reinterpret_cast<const uint4 *>(p + r.head);
    int64_t v = tid;
    for (; v + (UNROLL - 1) * THREADS < r.vecs; v += (int64_t)THREADS * UNROLL) {
        uint4 u[UNROLL];
#pragma unroll
        for (int i = 0; i < UNROLL; ++i) u[i] = q[v + i * THREADS];
#pragma unroll
        for (int i = 0; i < UNROLL; ++i) {
            float x[E];
            unpack16<T>(u[i], x);
#pragma unroll
            for (int e = 0; e < E; ++e) f(x[e]);
        }
    }
    for (; v < r.vecs; v += THREADS) {
        float x[E];
        unpack16<T>(q[v], x);
#pragma unroll
        for (int e = 0; e < E; ++e) f(x[e]);
    }
}
template <typename F> __device__ __forceinline__ void each_value(const ClipTensor &t, int64_t i0, int64_t i1, F f) {
    if (t.rows > 1) {
        for (int64_t i = i0 + threadIdx.x; i < i1; i += THREADS) f(load(t, i));
    } else if (t.dtype == CT_DT_F32) {
        each_value(static_cast<const float *>(t.src), Run(t.src, 4, i0, i1), f);
    } else if (t.dtype == CT_DT_F16) {
        each_value(static_cast<const __half *>(t.src), Run(t.src, 2, i0, i1), f);
    } else {
        each_value(static_cast<const __nv_bfloat16 *>(t.src), Run(t.src, 2, i0, i1), f);
    }
}

template <int N> __global__ void __launch_bounds__(THREADS) clip_parts_kernel(const __grid_constant__ Table<N> tab, Part *parts) {
    pdl_wait();
    pdl_trigger();
    const ClipTensor &t = tab.t[find(tab, (int)blockIdx.x)];
    const int64_t total = t.rows * t.cols, i0 = (int64_t)((int)blockIdx.x - t.block0) * tab.chunk, i1 = min(i0 + tab.chunk, total);
    Found f = {0.f, 0.f};
    each_value(t, i0, i1, [&](float v) { see(f, v); });
    double sum = f.s;
    float m = f.m;
    if (f.s == f.s && m > 0.f && m < __builtin_huge_valf() && (m > 0x1p55f || m < 0x1p-50f)) {
        const int e = ilogbf(m);
        f.s = 0.f;
        each_value(t, i0, i1, [&](float v) { see(f, ldexpf(v, -e)); });
        sum = ldexp((double)f.s, 2 * e);
    }
    if (f.s != f.s) m = f.s;
    __shared__ double ss[WARPS];
    __shared__ float sm[WARPS];
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
        for (int w = 1; w < WARPS; ++w) {
            sum += ss[w];
            m = join_top(m, sm[w]);
        }
        parts[tab.base + blockIdx.x] = {sum, m, 0.f};
    }
}

// values of a run times c into dst, whose run starts at the same place of a 16-byte unit; from its end on, which was read last
template <typename T> __device__ __forceinline__ void scale_run(const T *src, T *dst, const Run &r, float c) {
    constexpr int E = 16 / (int)sizeof(T);
    const T *p = src + r.i0;
    T *d = dst + r.i0;
    const int tid = threadIdx.x;
    if (tid < r.head) d[tid] = from_f32<T>(to_f32(p[tid]) * c);
    const int64_t tail = r.head + r.vecs * E;
    if (tail + tid < r.i1 - r.i0) d[tail + tid] = from_f32<T>(to_f32(p[tail + tid]) * c);
    const uint4 *q = reinterpret_cast<const uint4 *>(p + r.head);
    uint4 *w = reinterpret_cast<uint4 *>(d + r.head);
    int64_t v = r.vecs - 1 - tid;
    for (; v - (UNROLL - 1) * THREADS >= 0; v -= (int64_t)THREADS * UNROLL) {
        uint4 u[UNROLL];
#pragma unroll
        for (int i = 0; i < UNROLL; ++i) u[i] = __ldcs(q + v - i * THREADS);
#pragma unroll
        for (int i = 0; i < UNROLL; ++i) {
            float x[E];
            unpack16<T>(u[i], x);
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] *= c;
            __stcs(w + v - i * THREADS, pack16<T>(x));
        }
    }
    for (; v >= 0; v -= THREADS) {
        float x[E];
        unpack16<T>(__ldcs(q + v), x);
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] *= c;
        __stcs(w + v, pack16<T>(x));
    }
}
template <typename T> __device__ __forceinline__ bool scale_dense(const ClipTensor &t, int64_t i0, int64_t i1, float c) {
    if (((uintptr_t)t.src - (uintptr_t)t.dst) % 16 != 0) return false;
    scale_run(static_cast<const T *>(t.src), static_cast<T *>(t.dst), Run(t.src, (int)sizeof(T), i0, i1), c);
    return true;
}

// Every block joins the parts of all blocks, in one order, to the factor; the blocks share the tensors' own norms among them.  Then
// each scales its run.
template <int N> __global__ void __launch_bounds__(THREADS)
clip_scale_kernel(const __grid_constant__ Table<N> tab, const Part *parts, int all, int kind, double max_norm, float *norms, float *norm) {
    pdl_wait();
    pdl_trigger();
    __shared__ double ss[WARPS], factor;
    __shared__ float sm[WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    double sum = 0.0;
    float m = 0.f;
    for (int i = threadIdx.x; i < all; i += THREADS) {
        const Part p = parts[i];
        sum += p.sum;
        m = join_top(m, p.top);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
        m = join_top(m, __shfl_xor_sync(0xffffffffu, m, o));
    }
    if (lane == 0) {
        ss[warp] = sum;
        sm[warp] = m;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < WARPS; ++w) {
            sum += ss[w];
            m = join_top(m, sm[w]);
        }
        const double v = kind == CT_NORM_2 ? sqrt(sum) : (double)m;
        factor = isfinite((float)v) && v > max_norm ? max_norm / v : 1.0;
        if (blockIdx.x == 0 && tab.first == 0) *norm = (float)v;
    }
    for (int i = (int)blockIdx.x + (int)gridDim.x * warp; i < tab.n; i += (int)gridDim.x * WARPS) {
        const int p0 = tab.t[i].block0, p1 = i + 1 < tab.n ? tab.t[i + 1].block0 : tab.blocks;
        sum = 0.0;
        m = 0.f;
        for (int p = p0 + lane; p < p1; p += 32) {
            sum += parts[tab.base + p].sum;
            m = join_top(m, parts[tab.base + p].top);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            sum += __shfl_xor_sync(0xffffffffu, sum, o);
            m = join_top(m, __shfl_xor_sync(0xffffffffu, m, o));
        }
        if (lane == 0) norms[tab.first + i] = kind == CT_NORM_2 ? (float)sqrt(sum) : m;
    }
    __syncthreads();
    const double whole = factor;
    const float c = (float)whole;
    const int block = tab.blocks - 1 - (int)blockIdx.x;
    if (block < 0) return;
    const ClipTensor &t = tab.t[find(tab, block)];
    if (c == 1.f && t.src == t.dst) return;
    const int64_t i0 = (int64_t)(block - t.block0) * tab.chunk, i1 = min(i0 + tab.chunk, t.rows * t.cols);
    if (whole != 0.0 && c < 0x1p-126f) {
        // A factor below the normal 32-bit numbers, of a norm that is large next to max_norm: its products with the largest values are in
        // their range, and are taken in FP64 (slow here, and rare).
        for (int64_t i = i0 + threadIdx.x; i < i1; i += THREADS) store(t, i, (float)(load(t, i) * whole));
        return;
    }
    if (t.rows == 1) {
        // 1 times a value is the value, but for a NaN, whose bits need not stay: it stays one
        if (t.dtype == CT_DT_F32 ? scale_dense<float>(t, i0, i1, c)
            : t.dtype == CT_DT_F16 ? scale_dense<__half>(t, i0, i1, c)
                                   : scale_dense<__nv_bfloat16>(t, i0, i1, c))
            return;
    }
    for (int64_t i = i0 + threadIdx.x; i < i1; i += THREADS) store(t, i, load(t, i) * c);
}

inline bool tensor_ok(const ct_tensor &t) {
    if (t.rows == 0 || t.cols == 0) return true;
    const int size = dtype_size((int)t.dtype);
    return t.src != nullptr && t.dst != nullptr && aligned(t.src, size) && aligned(t.dst, size) &&
           (t.rows == 1 || (t.ld_src >= t.cols && t.ld_dst >= t.cols));
}

// whether two tensors have a value in common: side by side as columns of one matrix, which many may be, is seen without a look at their rows
bool overlap(std::vector<Span> &v) {
    std::sort(v.begin(), v.end(), [](const Span &a, const Span &b) { return a.at < b.at; });
    for (size_t i = 0; i < v.size(); ++i) {
        const uintptr_t end = v[i].end();
        for (size_t j = i + 1; j < v.size() && v[j].at < end; ++j) {
            const int64_t pitch = v[i].pitch, off = (int64_t)((v[j].at - v[i].at) % (uintptr_t)(pitch > 0 ? pitch : 1));
            if (pitch > 0 && pitch == v[j].pitch && off >= v[i].width && off + v[j].width <= pitch) continue;
            if (share(v[i], v[j])) return true;
        }
    }
    return false;
}

// values of a block: blocks enough for the whole GPU, with something to do for each
int64_t chunk_of(int64_t total) {
    const int64_t c = ((total + BLOCKS - 1) / BLOCKS + 1023) / 1024 * 1024;
    return c < LEAST ? LEAST : c > MOST ? MOST : c;
}
// at most so many blocks: each tensor may end with a part of one
inline int64_t blocks_most(int64_t n, int64_t total) { return total / chunk_of(total) + n; }

ct_status sizes(int64_t n, int64_t total) {
    return n < 0 || total < 0 || n > INT32_MAX / 2 || total > INT64_MAX >> 8 || blocks_most(n, total) > INT32_MAX ? CT_ERANGE : CT_OK;
}

template <int N>
cudaError_t launch(const ct_tensor *t, int64_t n, int64_t total, int kind, double max_norm, float *norms, float *norm,
                   Part *parts, cudaStream_t st) {
    Table<N> tab;
    tab.chunk = chunk_of(total);
    int all = 0;
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
                blocks += (q.rows * q.cols + tab.chunk - 1) / tab.chunk;
            }
            tab.blocks = (int)blocks;
            cudaError_t e = cudaSuccess;
            const dim3 block(THREADS);
            if (pass == 0) {
                all += (int)blocks;
                if (blocks > 0) e = pdl_launch(clip_parts_kernel<N>, dim3((unsigned)blocks), block, 0, st, tab, parts);
            } else {
                e = pdl_launch(clip_scale_kernel<N>, dim3((unsigned)(blocks > 0 ? blocks : 1)), block, 0, st, tab, (const Part *)parts, all,
                               kind, max_norm, norms, norm);
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

extern "C" ct_status ct_clip_grads_workspace(int64_t n, int64_t values, size_t *bytes) {
    using namespace ct::ops;
    if (bytes == nullptr) return CT_EINVAL;
    const ct_status s = sizes(n, values);
    if (s == CT_OK) *bytes = sizeof(Part) * (size_t)(blocks_most(n, values) + 1);
    return s;
}

extern "C" ct_status ct_clip_grads(const ct_tensor *tensors, int64_t n, int32_t kind, double max_norm, float *norms_dev,
                                   float *norm_dev, void *workspace_dev, size_t workspace_bytes, void *stream) {
    using namespace ct::ops;
    if ((kind != CT_NORM_2 && kind != CT_NORM_INF) || !(max_norm >= 0.0)) return CT_EINVAL;
    if (n < 0 || n > INT32_MAX / 2) return CT_ERANGE;
    if (norm_dev == nullptr || !aligned(norm_dev, 4) || (n > 0 && (tensors == nullptr || norms_dev == nullptr || !aligned(norms_dev, 4))))
        return CT_EINVAL;
    int64_t total = 0;
    for (int64_t i = 0; i < n; ++i) {
        const ct_tensor &t = tensors[i];
        if (t.rows < 0 || t.cols < 0 || (t.rows > 0 && t.cols > (INT64_MAX >> 8) / t.rows)) return CT_ERANGE;
        if (t.dtype < CT_DT_F32 || t.dtype > CT_DT_BF16 || !tensor_ok(t)) return CT_EINVAL;
        total += t.rows * t.cols;
        if (total > INT64_MAX >> 8) return CT_ERANGE;
    }
    if (sizes(n, total) != CT_OK) return CT_ERANGE;
    if (workspace_dev == nullptr || !aligned(workspace_dev, 16)) return CT_EINVAL;
    if (workspace_bytes < sizeof(Part) * (size_t)(blocks_most(n, total) + 1)) return CT_ENOMEM;
    try {
        std::vector<Span> v;
        v.reserve(2 * (size_t)n);
        for (int64_t i = 0; i < n; ++i) {
            const ct_tensor &t = tensors[i];
            if (t.rows == 0 || t.cols == 0) continue;
            const int size = dtype_size((int)t.dtype);
            v.push_back(span(t.dst, t.rows, t.cols, t.ld_dst, size));
            if (t.src != t.dst) v.push_back(span(t.src, t.rows, t.cols, t.ld_src, size));
            else if (t.rows > 1 && t.ld_src != t.ld_dst) return CT_EINVAL;
        }
        if (overlap(v)) return CT_EINVAL;
    } catch (const std::exception &) {
        return CT_ENOMEM;
    }
    Part *parts = static_cast<Part *>(workspace_dev);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = n <= SMALL ? launch<SMALL>(tensors, n, total, kind, max_norm, norms_dev, norm_dev, parts, st)
                                     : launch<LARGE>(tensors, n, total, kind, max_norm, norms_dev, norm_dev, parts, st);
    return e == cudaSuccess ? CT_OK : CT_ECUDA;
}
