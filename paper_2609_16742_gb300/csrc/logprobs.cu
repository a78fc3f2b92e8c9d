// Log probability of a given token, entropy, log normaliser and the most
// probable tokens of each row of logits, and the gradient of the first two.
//
// With m the row's maximum, Z = sum e^(x - m) and T = sum e^(x - m) (x - m):
//   lse = m + log Z,   log p[j] = x[j] - lse,   entropy = log Z - T / Z
// (both terms of the entropy are >= 0: nothing cancels).  A forbidden token
// (logit -inf) has probability 0 and adds nothing; where e^(x - m) is 0 the
// product with x - m is taken as 0, also when x - m overflows to -inf (a mask
// of the type's lowest value).  Sums are held in FP32.
#include <atomic>

#include "ops_common.cuh"
#include "tc_common.cuh"

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
    uint32_t *err;
};

constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ float ld_cluster_f32(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint64_t ld_cluster_u64(uint32_t addr) {
    uint64_t v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
    return v;
}

__device__ __forceinline__ float ex2(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// Running sums of a set of logits relative to m, one of its logits near the
// largest: z = sum e^(x - m), t = sum e^(x - m) (x - m).  m = -inf: nothing but
// -inf so far.
struct Stat {
    float m, z, t;
};

__device__ __forceinline__ Stat merge(const Stat &a, const Stat &b) {
    Stat r;
    r.m = fmaxf(a.m, b.m);
    const float da = a.m - r.m, db = b.m - r.m;
    const float fa = a.m == -INF ? 0.f : ex2(da * LOG2E), fb = b.m == -INF ? 0.f : ex2(db * LOG2E);
    r.z = fa * a.z + fb * b.z;                 // a NaN or +inf stays one
    r.t = (fa == 0.f ? 0.f : fa * (a.t + da * a.z)) + (fb == 0.f ? 0.f : fb * (b.t + db * b.z));
    return r;
}

// order of the top tokens: the larger logit first, the lower index among equals; a key of 0 is no token
__device__ __forceinline__ uint64_t order_key(float x, uint32_t j) {
    if (!(x > -INF)) return 0;
    const uint32_t b = __float_as_uint(x + 0.f);           // -0 and +0 are equal
    const uint32_t o = (b & 0x80000000u) ? ~b : (b | 0x80000000u);
    return ((uint64_t)o << 32) | (0xFFFFFFFFu - j);
}
__device__ __forceinline__ float key_value(uint64_t key) {
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float((o & 0x80000000u) ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ int64_t key_index(uint64_t key) { return (int64_t)(0xFFFFFFFFu - (uint32_t)key); }

// 32-bit words of logits: one FP32 value or two 16-bit ones
template <typename T> struct Words;
template <> struct Words<float> {
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    }
    static __device__ __forceinline__ float largest(uint32_t a) { return __uint_as_float(a); }
    static __device__ __forceinline__ float value(uint32_t w, int) { return __uint_as_float(w); }
    static __device__ __forceinline__ uint32_t mask(uint32_t w, int valid) { return valid > 0 ? w : 0xFF800000u; }
};
template <> struct Words<__half> {
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ float value(uint32_t w, int i) {
        return __half2float(__ushort_as_half((unsigned short)(i ? w >> 16 : w & 0xFFFFu)));
    }
    static __device__ __forceinline__ float largest(uint32_t a) { return fmaxf(value(a, 0), value(a, 1)); }
    static __device__ __forceinline__ uint32_t mask(uint32_t w, int valid) {
        return valid >= 2 ? w : valid == 1 ? (w & 0xFFFFu) | 0xFC000000u : 0xFC00FC00u;
    }
};
template <> struct Words<__nv_bfloat16> {
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ float value(uint32_t w, int i) { return __uint_as_float(i ? w & 0xFFFF0000u : w << 16); }
    static __device__ __forceinline__ float largest(uint32_t a) { return fmaxf(value(a, 0), value(a, 1)); }
    static __device__ __forceinline__ uint32_t mask(uint32_t w, int valid) {
        return valid >= 2 ? w : valid == 1 ? (w & 0xFFFFu) | 0xFF800000u : 0xFF80FF80u;
    }
};

// x - m kept away from -inf (a forbidden token, or a mask of the type's lowest
// value below a large m), where e^(x - m) (x - m) would be NaN instead of 0;
// keeps NaN
__device__ __forceinline__ float below(float x, float m) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x - m), "f"(-1e30f));
    return r;
}

// Sums of one thread.  A logit more than 8 above the reference moves it.
template <typename T> struct Sums {
    float m, lim;              // reference; the largest logit it stands for (-inf: none yet)
    float z0, z1, t0, t1;

    __device__ __forceinline__ void start() {
        m = 0.f; lim = -INF;
        z0 = z1 = t0 = t1 = 0.f;
    }
    __device__ __forceinline__ void raise(float top) {     // top > lim: the largest logit so far
        if (lim > -INF) {
            const float d = m - top, f = ex2(d * LOG2E);
            t0 = f == 0.f ? 0.f : f * (t0 + d * z0);
            t1 = f == 0.f ? 0.f : f * (t1 + d * z1);
            z0 *= f; z1 *= f;
        }
        m = top;
        lim = top + 8.f;
    }
    // N words; `top`: their largest value
    template <int N> __device__ __forceinline__ void add(const uint32_t (&w)[N], float top) {
        if (top > lim) raise(top);
#pragma unroll
        for (int i = 0; i < N; i += sizeof(T) == 4 ? 2 : 1) {
            const float a = Words<T>::value(w[i], 0);
            const float b = sizeof(T) == 4 ? Words<T>::value(w[sizeof(T) == 4 ? i + 1 : i], 0) : Words<T>::value(w[i], 1);
            const float d0 = below(a, m), d1 = below(b, m);
            const float e0 = ex2(d0 * LOG2E), e1 = ex2(d1 * LOG2E);
            z0 += e0; z1 += e1;
            t0 = fmaf(e0, d0, t0); t1 = fmaf(e1, d1, t1);
        }
    }
    __device__ __forceinline__ Stat stat() const {
        // the reference of a thread that saw only -inf is -inf; a NaN among them stays in z
        return Stat{lim > -INF ? m : -INF, z0 + z1, t0 + t1};
    }
};

__device__ __forceinline__ Stat warp_merge(Stat s) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1)
        s = merge(s, Stat{__shfl_xor_sync(~0u, s.m, d), __shfl_xor_sync(~0u, s.z, d), __shfl_xor_sync(~0u, s.t, d)});
    return s;
}

// what a row's merged sums say
struct RowResult {
    bool bad, none;
    float lse, entropy;
};
__device__ __forceinline__ RowResult row_result(const Stat &s) {
    RowResult r;
    r.bad = !(s.z < INF);
    r.none = s.m == -INF;
    const float lz = logf(s.z);
    r.lse = r.bad ? nan_f() : r.none ? -INF : s.m + lz;
    r.entropy = r.bad ? nan_f() : r.none ? 0.f : lz - s.t / s.z;
    return r;
}

__device__ __forceinline__ void write_row(const LpArgs &a, int64_t r, const RowResult &q, int64_t id, float given) {
    a.lse[r] = q.lse;
    a.entropy[r] = q.entropy;
    if (a.lp == nullptr) return;
    float lp = nan_f();
    if (!q.bad && id == -1) lp = 0.f;
    else if (!q.bad && id >= 0 && id < a.vocab) lp = given == -INF ? -INF : given - q.lse;
    a.lp[r] = lp;
}

__device__ __forceinline__ void write_top(const LpArgs &a, int64_t r, int i, uint64_t key, const RowResult &q) {
    if (q.bad) key = 0;
    a.top_id[r * a.top_k + i] = key == 0 ? -1 : key_index(key);
    a.top_lp[r * a.top_k + i] = q.bad ? nan_f() : key == 0 ? -INF : key_value(key) - q.lse;
}

// the row's given token and its logit (thread 0 fetches them while the row streams)
template <typename T> __device__ __forceinline__ float given_logit(const LpArgs &a, int64_t r, int64_t &id) {
    id = a.lp != nullptr ? a.ids[r] : -1;
    return id >= 0 && id < a.vocab ? to_f32(static_cast<const T *>(a.x)[r * a.ldx + id]) : 0.f;
}

// ---------------------------------------------------------------------------
// Short rows: one warp each, the whole row in registers.  The next top token
// is the warp's largest key below the last one.
// ---------------------------------------------------------------------------
constexpr int SHORT = 1024;
constexpr int SHORT_WARPS = 4;

template <typename T>
__global__ void __launch_bounds__(32 * SHORT_WARPS) logprobs_short_kernel(const LpArgs a, int vec) {
    constexpr int E = Vec16<T>::N;                         // values of 16 bytes
    constexpr int NW = SHORT / 32 * (int)sizeof(T) / 4;    // words of a lane
    constexpr int W2 = 4 / (int)sizeof(T);                 // values of a word
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x % 32;
    const int64_t r = (int64_t)blockIdx.x * SHORT_WARPS + threadIdx.x / 32;
    if (r >= a.rows) return;
    const T *x = static_cast<const T *>(a.x) + r * a.ldx;
    const int vocab = (int)a.vocab;
    int64_t id = -1;
    const float given = lane == 0 ? given_logit<T>(a, r, id) : 0.f;
    uint32_t w[NW];
#pragma unroll
    for (int i = 0; i < NW; i += 4) {
        const int j = (i / 4 * 32 + lane) * E;
        if (vec && j + E <= vocab) {
            const uint4 u = __ldg(reinterpret_cast<const uint4 *>(x + j));
            w[i] = u.x; w[i + 1] = u.y; w[i + 2] = u.z; w[i + 3] = u.w;
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float v[2];
#pragma unroll
                for (int e = 0; e < W2; ++e) v[e] = j + q * W2 + e < vocab ? to_f32(x[j + q * W2 + e]) : -INF;
                if constexpr (sizeof(T) == 4) w[i + q] = __float_as_uint(v[0]);
                else w[i + q] = pack2<T>(v[0], v[1]);
            }
        }
    }
    Sums<T> sums;
    sums.start();
#pragma unroll
    for (int i = 0; i < NW; i += 4) {
        if (i / 4 * 32 * E >= vocab) break;
        uint32_t part[4] = {w[i], w[i + 1], w[i + 2], w[i + 3]};
        sums.add(part, Words<T>::largest(Words<T>::max2(Words<T>::max2(w[i], w[i + 1]), Words<T>::max2(w[i + 2], w[i + 3]))));
    }
    const RowResult q = row_result(warp_merge(sums.stat()));
    if (lane == 0) write_row(a, r, q, id, given);
    uint64_t last = ~0ull, mine = ~0ull;                   // mine: this lane's largest key below `last`
    uint64_t out = 0;                                      // lane i keeps the i-th token
    for (int k = 0; k < a.top_k && !q.bad; ++k) {
        if (mine >= last) {
            mine = 0;
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                if (i / 4 * 32 * E >= vocab) break;
#pragma unroll
                for (int e = 0; e < W2; ++e) {
                    const uint32_t j = (uint32_t)((i / 4 * 32 + lane) * E + i % 4 * W2 + e);
                    const uint64_t key = order_key(Words<T>::value(w[i], e), j);
                    if (key < last && key > mine) mine = key;
                }
            }
        }
        uint64_t b = mine;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) b = max(b, __shfl_xor_sync(~0u, b, d));
        if (lane == k) out = b;
        last = b;
        if (b == 0) break;
    }
    if (lane < a.top_k) write_top(a, r, lane, out, q);
}

// ---------------------------------------------------------------------------
// Long rows: a row, or a share of it, streams through shared memory in chunks
// of 128 bytes a thread, copied by the bulk engine STAGES ahead (of the next
// row too, while this one is finished).
//
// Top tokens: `thr` is a logit that at least top_k of the row's tokens reach.
// A thread that meets a logit >= thr writes its key to a candidate list; the
// list's best top_k are the answer.  The first chunk (every chunk, until one
// has enough tokens) sets thr to the top_k-th largest of 64 group maxima and is
// looked over again by the threads whose maximum reaches it: some 1.1 top_k
// candidates, and about as many from each later chunk.  A chunk that overflows
// the list is looked over again with a threshold of its own, and if that fails
// too (its best tokens all in a few threads' hands) its best are picked one by
// one.  The list's order varies, the set and its sorted best do not.
// ---------------------------------------------------------------------------
constexpr int STAGES = 3;
constexpr int THREAD_VECS = 8;                             // 16-byte vectors of a thread in a chunk
constexpr int BATCH = 4;                                   // ... examined together
constexpr int GROUPS = 64;                                 // of threads, for the threshold; > CT_MAX_TOP_K

template <int NT> struct Long {
    static constexpr int CHUNK = NT * THREAD_VECS * 16;    // bytes
    static constexpr int STAGE = CHUNK + 128;              // a row may start anywhere in its first 16 bytes
    static constexpr int CTAS = NT == 256 ? 2 : 7;         // on an SM: what its shared memory holds
    static constexpr int CAP = NT == 256 ? 2048 : 512;     // candidates
    struct Shared {
        uint64_t full[STAGES];
        uint64_t cand[CAP];
        uint64_t best[CT_MAX_TOP_K];
        uint64_t pick[NT / 32];
        Stat part[NT / 32];
        Stat total;
        float group[GROUPS];
        float thr;
        int count;
    };
    static constexpr size_t SMEM = (size_t)STAGES * STAGE + sizeof(Shared) + 16;
};

template <typename T, int NT> struct LongRow {
    using L = Long<NT>;
    static constexpr int E = Vec16<T>::N;
    static constexpr int W2 = 4 / (int)sizeof(T);
    static constexpr int CE = L::CHUNK / (int)sizeof(T);   // values of a chunk

    // the 4 words of 16-byte vector v of a chunk whose first value lies `shift` bytes into the stage
    static __device__ __forceinline__ void load(const uint8_t *stage, int v, int shift, uint32_t *w) {
        const uint4 p = *reinterpret_cast<const uint4 *>(stage + v * 16);
        if (shift == 0) {
            w[0] = p.x; w[1] = p.y; w[2] = p.z; w[3] = p.w;
            return;
        }
        const uint4 n = *reinterpret_cast<const uint4 *>(stage + v * 16 + 16);
        const uint32_t bits = (uint32_t)(shift & 3) * 8;
        uint32_t s[5];
        switch (shift >> 2) {
            case 0: s[0] = p.x; s[1] = p.y; s[2] = p.z; s[3] = p.w; s[4] = n.x; break;
            case 1: s[0] = p.y; s[1] = p.z; s[2] = p.w; s[3] = n.x; s[4] = n.y; break;
            case 2: s[0] = p.z; s[1] = p.w; s[2] = n.x; s[3] = n.y; s[4] = n.z; break;
            default: s[0] = p.w; s[1] = n.x; s[2] = n.y; s[3] = n.z; s[4] = n.w; break;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(s[i], s[i + 1], bits);
    }
    // ... with the values from n_valid on replaced by -inf
    static __device__ __forceinline__ void load_masked(const uint8_t *stage, int v, int shift, int n_valid, uint32_t *w) {
        load(stage, v, shift, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = Words<T>::mask(w[i], n_valid - v * E - i * W2);
    }
    // writes the keys of a thread's values in vectors [i0, i1) that reach thr
    static __device__ __noinline__ void push(const uint8_t *stage, int shift, int n_valid, int i0, int i1, float thr,
                                             uint32_t j0, uint64_t *cand, int *count) {
#pragma unroll 1
        for (int i = i0; i < i1; ++i) {
            const int v = i * NT + (int)threadIdx.x;
            if (v * E >= n_valid) break;
            uint32_t w[4];
            load_masked(stage, v, shift, n_valid, w);
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int e = 0; e < W2; ++e) {
                    const float x = Words<T>::value(w[q], e);
                    if (x >= thr && x > -INF) {
                        const int at = atomicAdd(count, 1);
                        if (at < L::CAP) cand[at] = order_key(x, j0 + (uint32_t)(v * E + q * W2 + e));
                    }
                }
        }
    }
    // the top_k-th largest of the groups' maxima (all threads)
    static __device__ __forceinline__ float threshold(typename L::Shared &sh, float mx, int k) {
        constexpr int LANES = NT / GROUPS;
#pragma unroll
        for (int d = LANES / 2; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, d));
        if (threadIdx.x % LANES == 0) sh.group[threadIdx.x / LANES] = mx;
        __syncthreads();
        if (threadIdx.x < GROUPS) {
            const float g = sh.group[threadIdx.x];
            int rank = 0;
            for (int i = 0; i < GROUPS; ++i) {
                const float o = sh.group[i];
                rank += o > g || (o == g && i < (int)threadIdx.x);
            }
            if (rank == k - 1) sh.thr = g;
        }
        __syncthreads();
        return sh.thr;
    }
    // sorts the list's best top_k into sh.best (all threads)
    static __device__ __forceinline__ void select(typename L::Shared &sh, int n, int k) {
        if ((int)threadIdx.x < k) sh.best[threadIdx.x] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += NT) {
            const uint64_t key = sh.cand[i];
            int rank = 0;
            for (int j = 0; j < n && rank < k; ++j) rank += sh.cand[j] > key;
            if (rank < k) sh.best[rank] = key;
        }
        __syncthreads();
    }
    // keeps only the list's best top_k; the new threshold
    static __device__ __noinline__ float compact(typename L::Shared &sh, int n, int k, float thr) {
        select(sh, n, k);
        if ((int)threadIdx.x < k) sh.cand[threadIdx.x] = sh.best[threadIdx.x];
        if (threadIdx.x == 0) sh.count = min(n, k);
        __syncthreads();
        return n >= k ? fmaxf(thr, key_value(sh.best[k - 1])) : thr;
    }
    // the best top_k of the list's first n and the whole chunk, one by one
    static __device__ __noinline__ float pick(typename L::Shared &sh, int n, int k, float thr, const uint8_t *stage,
                                              int shift, int n_valid, uint32_t j0) {
        uint64_t last = ~0ull;
        int found = 0;
        for (; found < k && last != 0; ++found) {
            uint64_t b = 0;
            for (int i = threadIdx.x; i < n; i += NT) {
                const uint64_t key = sh.cand[i];
                if (key < last && key > b) b = key;
            }
#pragma unroll 1
            for (int i = 0; i < THREAD_VECS; ++i) {
                const int v = i * NT + (int)threadIdx.x;
                if (v * E >= n_valid) break;
                uint32_t w[4];
                load_masked(stage, v, shift, n_valid, w);
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int e = 0; e < W2; ++e) {
                        const uint64_t key = order_key(Words<T>::value(w[q], e), j0 + (uint32_t)(v * E + q * W2 + e));
                        if (key < last && key > b) b = key;
                    }
            }
            for (int d = 16; d > 0; d >>= 1) b = max(b, __shfl_xor_sync(~0u, b, d));
            if (threadIdx.x % 32 == 0) sh.pick[threadIdx.x / 32] = b;
            __syncthreads();
            for (int i = 0; i < NT / 32; ++i) b = max(b, sh.pick[i]);
            if (threadIdx.x == 0) sh.best[found] = b;
            last = b;
            __syncthreads();
        }
        if (last == 0) --found;
        if ((int)threadIdx.x < found) sh.cand[threadIdx.x] = sh.best[threadIdx.x];
        if (threadIdx.x == 0) sh.count = found;
        __syncthreads();
        return found == k ? fmaxf(thr, key_value(last)) : thr;
    }
};

template <typename T, int NT>
__global__ void __launch_bounds__(NT, Long<NT>::CTAS) logprobs_long_kernel(const LpArgs a, int splits) {
    using L = Long<NT>;
    using R = LongRow<T, NT>;
    extern __shared__ __align__(128) uint8_t smem[];
    typename L::Shared &sh = *reinterpret_cast<typename L::Shared *>(smem + STAGES * L::STAGE);
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int rank = (int)(blockIdx.x % (unsigned)splits);
    const int64_t cid = blockIdx.x / (unsigned)splits, ncl = gridDim.x / (unsigned)splits;
    const int chunks = (int)((a.vocab + R::CE - 1) / R::CE);
    const int ch0 = (int)((int64_t)chunks * rank / splits), ch1 = (int)((int64_t)chunks * (rank + 1) / splits);
    const int k = a.top_k;

    if (tid == 0) {
        for (int s = 0; s < STAGES; ++s) tc::mbar_init(tc::smem_u32(&sh.full[s]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    pdl_wait();
    pdl_trigger();

    // thread 0: the next chunk to copy
    int64_t next_row = cid;
    int next_ch = ch0;
    const auto copy_next = [&](int s) {
        if (next_row >= a.rows) return;
        const uint8_t *row = reinterpret_cast<const uint8_t *>(static_cast<const T *>(a.x) + next_row * a.ldx);
        const int64_t end = min((int64_t)(next_ch + 1) * L::CHUNK, a.vocab * (int64_t)sizeof(T));
        // whole 16-byte units that hold a value of the chunk
        const uintptr_t from = (uintptr_t)(row + (int64_t)next_ch * L::CHUNK) & ~(uintptr_t)15;
        const uintptr_t to = ((uintptr_t)(row + end) + 15) & ~(uintptr_t)15;
        const uint32_t bar = tc::smem_u32(&sh.full[s]);
        tc::mbar_arrive_expect_tx(bar, (uint32_t)(to - from));
        tc::bulk_load(tc::smem_u32(smem + s * L::STAGE), reinterpret_cast<const void *>(from), (uint32_t)(to - from), bar);
        if (++next_ch == ch1) { next_ch = ch0; next_row += ncl; }
    };
    if (tid == 0)
        for (int s = 0; s < STAGES; ++s) copy_next(s);

    int it = 0;
    for (int64_t r = cid; r < a.rows; r += ncl) {
        const int shift = (int)((uintptr_t)(static_cast<const T *>(a.x) + r * a.ldx) & 15);
        int64_t id = -1;
        const float given = tid == 0 && rank == 0 ? given_logit<T>(a, r, id) : 0.f;
        Sums<T> sums;
        sums.start();
        float thr = k > 0 ? -INF : INF;
        if (tid == 0) sh.count = 0;
        __syncthreads();
        for (int ch = ch0; ch < ch1; ++ch, ++it) {
            const int s = it % STAGES;
            const uint8_t *stage = smem + s * L::STAGE;
            const uint32_t j0 = (uint32_t)ch * R::CE;
            const int n_valid = (int)min((int64_t)R::CE, a.vocab - (int64_t)ch * R::CE);
            const int before = k > 0 ? sh.count : 0;       // the same for all threads: between two barriers
            const bool first = thr == -INF;                // no threshold yet
            const float limit = first ? INF : thr;
            // a wait that runs out leaves the results invalid; it is reported
            tc::mbar_wait(tc::smem_u32(&sh.full[s]), (uint32_t)(it / STAGES) & 1u, a.err, 0x2000u);
            __syncthreads();
            float mx = -INF;
#pragma unroll 1
            for (int i = 0; i < THREAD_VECS; i += BATCH) {
                if ((i * NT + (tid & ~31)) * R::E >= n_valid) break;
                uint32_t w[4 * BATCH];
                if (n_valid == R::CE) {
#pragma unroll
                    for (int b = 0; b < BATCH; ++b) R::load(stage, (i + b) * NT + tid, shift, w + 4 * b);
                } else {
#pragma unroll
                    for (int b = 0; b < BATCH; ++b) R::load_masked(stage, (i + b) * NT + tid, shift, n_valid, w + 4 * b);
                }
                uint32_t m2 = w[0];
#pragma unroll
                for (int b = 1; b < 4 * BATCH; ++b) m2 = Words<T>::max2(m2, w[b]);
                const float top = Words<T>::largest(m2);
                sums.add(w, top);
                mx = fmaxf(mx, top);
                if (top >= limit) R::push(stage, shift, n_valid, i, i + BATCH, thr, j0, sh.cand, &sh.count);
            }
            if (k > 0) {
                if (first) {
                    thr = R::threshold(sh, mx, k);
                    if (mx >= thr && mx > -INF) R::push(stage, shift, n_valid, 0, THREAD_VECS, thr, j0, sh.cand, &sh.count);
                }
                __syncthreads();
                int n = sh.count;
                if (n > L::CAP) {
                    __syncthreads();
                    if (tid == 0) sh.count = before;
                    const float own = fmaxf(thr, R::threshold(sh, mx, k));
                    if (mx >= own && mx > -INF) R::push(stage, shift, n_valid, 0, THREAD_VECS, own, j0, sh.cand, &sh.count);
                    __syncthreads();
                    n = sh.count;
                    if (n > L::CAP) {
                        __syncthreads();
                        thr = R::pick(sh, before, k, thr, stage, shift, n_valid, j0);
                        n = 0;
                    } else {
                        thr = own;
                    }
                }
                if (n > L::CAP / 2) {
                    __syncthreads();
                    thr = R::compact(sh, n, k, thr);
                }
            }
            __syncthreads();                               // the chunk has been read
            if (tid == 0) copy_next(s);
        }
        // the row
        Stat st = warp_merge(sums.stat());
        if (lane == 0) sh.part[warp] = st;
        if (k > 0) R::select(sh, sh.count, k);
        else __syncthreads();
        st = sh.part[0];
#pragma unroll
        for (int i = 1; i < NT / 32; ++i) st = merge(st, sh.part[i]);
        if (splits == 1) {
            const RowResult q = row_result(st);
            if (tid == 0) write_row(a, r, q, id, given);
            if (tid < k) write_top(a, r, tid, sh.best[tid], q);
        } else {
            // rank 0 joins the shares, in rank order
            if (tid == 0) sh.total = st;
            tc::cluster_sync();
            if (rank == 0) {
                for (int p = 1; p < splits; ++p) {
                    const uint32_t at = tc::mapa_shared(tc::smem_u32(&sh.total), (uint32_t)p);
                    st = merge(st, Stat{ld_cluster_f32(at), ld_cluster_f32(at + 4), ld_cluster_f32(at + 8)});
                }
                const RowResult q = row_result(st);
                if (tid == 0) write_row(a, r, q, id, given);
                if (k > 0) {
                    for (int i = tid; i < splits * k; i += NT)
                        sh.cand[i] = ld_cluster_u64(tc::mapa_shared(tc::smem_u32(&sh.best[i % k]), (uint32_t)(i / k)));
                    __syncthreads();
                    R::select(sh, splits * k, k);
                    if (tid < k) write_top(a, r, tid, sh.best[tid], q);
                }
            }
            tc::cluster_sync();
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// Gradient: each CTA a piece of one row, GRAD_VECS 16-byte vectors a thread.
// ---------------------------------------------------------------------------
constexpr int GRAD_THREADS = 256;
constexpr int GRAD_VECS = 4;

struct GradArgs {
    const void *x;
    int64_t ldx;
    const int64_t *ids;
    const float *lse, *entropy, *g_lp, *g_h;
    void *dx;
    int64_t lddx;
    int64_t rows, vocab;
};

// what a row's gradient needs
struct GradRow {
    float lse, g, gh, h;
    int64_t id;
    bool bad;
};

// d = -p (g + gh (log p + h)), without the given token's own g
__device__ __forceinline__ float grad_value(const GradRow &q, float x) {
    const float lp = x - q.lse;
    const float p = ex2(lp * LOG2E);
    const float d = -p * fmaf(q.gh, lp + q.h, q.g);
    return p == 0.f ? 0.f : d;                             // also where lp is -inf
}

template <typename T>
__device__ __forceinline__ void grad_one(const GradRow &q, const T *x, T *dx, int64_t j) {
    float d = grad_value(q, to_f32(x[j]));
    if (j == q.id) d += q.g;
    dx[j] = from_f32<T>(q.bad ? nan_f() : d);
}

template <typename T>
__global__ void __launch_bounds__(GRAD_THREADS) logprobs_grad_kernel(const GradArgs a, int pieces) {
    constexpr int E = Vec16<T>::N;
    pdl_wait();
    pdl_trigger();
    const int64_t r = blockIdx.x / (unsigned)pieces;
    const int piece = (int)(blockIdx.x % (unsigned)pieces);
    const T *x = static_cast<const T *>(a.x) + r * a.ldx;
    T *dx = static_cast<T *>(a.dx) + r * a.lddx;
    GradRow q;
    q.lse = a.lse[r];
    q.id = a.g_lp != nullptr ? a.ids[r] : -1;
    q.g = q.id == -1 ? 0.f : q.id >= 0 && q.id < a.vocab ? a.g_lp[r] : nan_f();
    q.gh = a.g_h != nullptr ? a.g_h[r] : 0.f;
    q.h = a.g_h != nullptr ? a.entropy[r] : 0.f;
    q.bad = q.lse != q.lse || q.g != q.g;
    if (q.lse == -INF) q.lse = 0.f;                        // nothing can occur: every p is 0
    // values before the first 16-byte boundary, and the vectors after it
    const int64_t head = min((int64_t)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(T), a.vocab);
    const bool same = (((uintptr_t)x ^ (uintptr_t)dx) & 15) == 0;
    const int64_t vecs = (a.vocab - head) / E, per = GRAD_THREADS * GRAD_VECS;
    const int64_t v0 = piece * per + threadIdx.x;
    uint4 u[GRAD_VECS];
#pragma unroll
    for (int i = 0; i < GRAD_VECS; ++i) {
        const int64_t v = v0 + i * GRAD_THREADS;
        if (v < vecs) u[i] = __ldcs(reinterpret_cast<const uint4 *>(x + head + v * E));
    }
    // the ends of the row: its first piece's threads
    if (piece == 0) {
        const int64_t tail = head + vecs * E;
        if ((int64_t)threadIdx.x < head) grad_one(q, x, dx, (int64_t)threadIdx.x);
        if (tail + (int64_t)threadIdx.x < a.vocab) grad_one(q, x, dx, tail + (int64_t)threadIdx.x);
    }
#pragma unroll
    for (int i = 0; i < GRAD_VECS; ++i) {
        const int64_t v = v0 + i * GRAD_THREADS;
        if (v >= vecs) break;
        const int64_t j = head + v * E;
        float d[E];
        unpack16<T>(u[i], d);
#pragma unroll
        for (int e = 0; e < E; ++e) d[e] = grad_value(q, d[e]);
        if (q.id >= j && q.id < j + E) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (q.id == j + e) d[e] += q.g;
        }
        if (q.bad) {
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] = nan_f();
        }
        if (same) {
            __stcs(reinterpret_cast<uint4 *>(dx + j), pack16<T>(d));
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) dx[j + e] = from_f32<T>(d[e]);
        }
    }
}

template <typename T, int NT> cudaError_t launch_long(const LpArgs &a, cudaStream_t st) {
    using L = Long<NT>;
    static std::atomic<bool> sized[MAX_DEVICES];
    cudaError_t e = allow_smem(logprobs_long_kernel<T, NT>, sized, L::SMEM);
    if (e != cudaSuccess) return e;
    const int64_t slots = (int64_t)sm_count() * L::CTAS;
    const int64_t chunks = (a.vocab * (int64_t)sizeof(T) + L::CHUNK - 1) / L::CHUNK;
    // few rows: each is shared by a cluster, so that the whole GPU reads
    int splits = 1;
    while (splits < 8 && a.rows * splits * 2 <= slots && splits * 2 <= chunks) splits *= 2;
    const int64_t clusters = a.rows < slots / splits ? a.rows : slots / splits;
    if (splits == 1)
        return pdl_launch(logprobs_long_kernel<T, NT>, dim3((unsigned)clusters), dim3(NT), L::SMEM, st, a, splits);
    return pdl_launch_cluster(logprobs_long_kernel<T, NT>, dim3((unsigned)(clusters * splits)), dim3(NT), L::SMEM, st,
                              splits, a, splits);
}

template <typename T> cudaError_t launch_logprobs(const LpArgs &a, cudaStream_t st) {
    if (a.vocab <= SHORT) {
        const int vec = aligned(a.x, 16) && (a.rows == 1 || a.ldx % Vec16<T>::N == 0);
        return pdl_launch(logprobs_short_kernel<T>, dim3((unsigned)((a.rows + SHORT_WARPS - 1) / SHORT_WARPS)),
                          dim3(32 * SHORT_WARPS), 0, st, a, vec);
    }
    return a.vocab * (int64_t)sizeof(T) <= 4 * Long<64>::CHUNK ? launch_long<T, 64>(a, st) : launch_long<T, 256>(a, st);
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
                      top_id_dev, device_error_word()};
    if (a.err == nullptr) return CT_ECUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == CT_DT_F32   ? launch_logprobs<float>(a, st)
                          : dtype == CT_DT_F16 ? launch_logprobs<__half>(a, st)
                                               : launch_logprobs<__nv_bfloat16>(a, st);
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
                        rows, vocab};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int64_t per = (int64_t)GRAD_THREADS * GRAD_VECS * (16 / es), pieces = (vocab + per - 1) / per;
    if (rows > INT32_MAX / pieces) return CT_ERANGE;
    const dim3 grid((unsigned)(rows * pieces)), block(GRAD_THREADS);
    const cudaError_t e =
        dtype == CT_DT_F32   ? ct::pdl_launch(logprobs_grad_kernel<float>, grid, block, 0, st, a, (int)pieces)
        : dtype == CT_DT_F16 ? ct::pdl_launch(logprobs_grad_kernel<__half>, grid, block, 0, st, a, (int)pieces)
                             : ct::pdl_launch(logprobs_grad_kernel<__nv_bfloat16>, grid, block, 0, st, a, (int)pieces);
    return e == cudaSuccess ? CT_OK : CT_ECUDA;
}
