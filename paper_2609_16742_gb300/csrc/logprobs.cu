// Log probability of a given token, entropy, log normaliser and the most
// probable tokens of each row of logits, and the gradient of the first two.
//
// With m the row's maximum, Z = sum e^(x - m) and T = sum e^(x - m) (x - m):
//   lse = m + log Z,   log p[j] = x[j] - lse,   entropy = log Z - T / Z
// (both terms of the entropy are >= 0: nothing cancels, so a confident row's
// entropy, next to 0, keeps its digits).  A running m is a warp's largest logit
// so far, the same for its lanes; warps' sums are joined relative to the
// largest of theirs, which is the row's.  A forbidden token
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

constexpr uint32_t E_LOGPROBS = 0x2000, E_DRAIN = 0x4000;      // error codes of the bounded waits

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
constexpr float LN2 = 0.6931471805599453f;

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

// Running sums of a set of logits relative to m, the largest of them, in units of
// log 2: z = sum 2^u, t = sum 2^u u, u = (x - m) log2(e).
// m = -inf: nothing but -inf so far.
struct Stat {
    float m, z, t;
};

__device__ __forceinline__ Stat merge(const Stat &a, const Stat &b) {
    Stat r;
    r.m = fmaxf(a.m, b.m);
    const float da = (a.m - r.m) * LOG2E, db = (b.m - r.m) * LOG2E;
    const float fa = a.m == -INF ? 0.f : ex2(da), fb = b.m == -INF ? 0.f : ex2(db);
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
    static __device__ __forceinline__ uint32_t dup(float v) { return __float_as_uint(v); }
    static __device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.NaN.f32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static constexpr float MODERATE = 1e6f;
    static __device__ __forceinline__ float value(uint32_t w, int) { return __uint_as_float(w); }
    static __device__ __forceinline__ uint32_t mask(uint32_t w, int valid) { return valid > 0 ? w : 0xFF800000u; }
};
template <> struct Words<__half> {
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ uint32_t dup(float v) { return pack2<__half>(v, v); }
    static constexpr float MODERATE = 6e4f;
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
    static __device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ uint32_t dup(float v) { return pack2<__nv_bfloat16>(v, v); }
    static constexpr float MODERATE = 1e6f;
    static __device__ __forceinline__ float value(uint32_t w, int i) { return __uint_as_float(i ? w & 0xFFFF0000u : w << 16); }
    static __device__ __forceinline__ float largest(uint32_t a) { return fmaxf(value(a, 0), value(a, 1)); }
    static __device__ __forceinline__ uint32_t mask(uint32_t w, int valid) {
        return valid >= 2 ? w : valid == 1 ? (w & 0xFFFFu) | 0xFF800000u : 0xFF80FF80u;
    }
};

// two FP32 values at once
__device__ __forceinline__ uint64_t pair(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float &a, float &b) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// sums of (2^u, 2^u u) over 4 words, with u kept above -inf
template <typename T> __device__ __noinline__ float2 slow_terms(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3, float m) {
    float2 r = make_float2(0.f, 0.f);
    for (int i = 0; i < 4; ++i)
        for (int h = 0; h < 4 / (int)sizeof(T); ++h) {
            const float x = Words<T>::value(i == 0 ? w0 : i == 1 ? w1 : i == 2 ? w2 : w3, h);
            const float u = fmaxf((x - m) * LOG2E, -1e30f), e = x != x ? x : ex2(u);
            r.x += e;
            r.y += e * u;
        }
    return r;
}

// Sums of one thread, relative to the largest logit that its warp has met so
// far, m: a larger one takes its place, once for all lanes.  (With a reference for
// each lane some lane's changes at nearly every step, and the warp waits for it.)
//
// The sums are taken with v = x log2(e) - c, c = m log2(e) rounded: one
// instruction.  v differs from u by what c was rounded by, the same for every
// x, and stat() takes that out.  Logits that vanish next to m are raised to
// `low`, a value some 160 or more below it, so that -inf (a forbidden token)
// and masks of the type's lowest value add 2^v v = 0 * finite and not 0 * inf.
// Where |m| > MODERATE the rounding of c would matter or the type has no such
// value; there c is 0 and the terms are taken one by one from x - m.
template <typename T> struct Sums {
    float m, lim;              // reference (0: none yet); the largest logit so far (-inf: none yet)
    float c;
    uint32_t low;
    uint64_t z, t;             // even and odd values'

    __device__ __forceinline__ void start() {
        m = c = 0.f;
        lim = -INF;
        low = Words<T>::dup(-160.f);
        z = t = 0;
    }
    static __device__ __forceinline__ bool moderate(float m) { return fabsf(m) <= Words<T>::MODERATE; }
    // v - u
    __device__ __forceinline__ float rounded() const { return moderate(m) ? fmaf(m, LOG2E, -c) : 0.f; }
    __device__ __forceinline__ void raise(float top) {     // top > lim
        const float cn = moderate(top) ? top * LOG2E : 0.f;
        if (lim > -INF) {
            const float d = (m - top) * LOG2E - rounded() + (moderate(top) ? fmaf(top, LOG2E, -cn) : 0.f), f = ex2(d);
            t = f == 0.f ? 0 : mul2(pair(f, f), fma2(pair(d, d), z, t));
            z = mul2(pair(f, f), z);
        }
        m = top;
        c = cn;
        lim = top;
        low = Words<T>::dup(top - fmaxf(160.f, fabsf(top) * 0.03125f));
    }
    // all lanes together, before they add words whose largest value is `top`
    __device__ __forceinline__ void reference(float top) {
        if (!__any_sync(~0u, top > lim)) return;
        float most;
        asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(most) : "f"(top));   // (past NaN)
        raise(most);
    }
    // N words
    template <int N> __device__ __forceinline__ void add(const uint32_t (&w)[N]) {
        if (!moderate(m)) {
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                const float2 q = slow_terms<T>(w[i], w[i + 1], w[i + 2], w[i + 3], m);
                z = add2(z, pair(q.x, 0.f));
                t = add2(t, pair(q.y, 0.f));
            }
            return;
        }
        const uint64_t minus_c = pair(-c, -c), log2e = pair(LOG2E, LOG2E);
#pragma unroll
        for (int i = 0; i < N; i += sizeof(T) == 4 ? 2 : 1) {
            const uint32_t x = Words<T>::max2_nan(w[i], low);
            const float a = Words<T>::value(x, 0);
            const float b = sizeof(T) == 4 ? Words<T>::value(Words<T>::max2_nan(w[sizeof(T) == 4 ? i + 1 : i], low), 0)
                                           : Words<T>::value(x, 1);
            const uint64_t v = fma2(pair(a, b), log2e, minus_c);
            float v0, v1;
            unpair(v, v0, v1);
            const uint64_t e = pair(ex2(v0), ex2(v1));
            z = add2(z, e);
            t = fma2(e, v, t);
        }
    }
    __device__ __forceinline__ Stat stat() const {
        float z0, z1, t0, t1;
        unpair(z, z0, z1);
        unpair(t, t0, t1);
        const float d = -rounded(), f = ex2(d), zs = z0 + z1, ts = t0 + t1;
        // the reference of a warp that saw only -inf is -inf; a NaN among them stays in z
        return Stat{lim > -INF ? m : -INF, f * zs, f * fmaf(d, zs, ts)};
    }
};

// over the warp, whose lanes have the same reference
__device__ __forceinline__ Stat warp_sum(Stat s) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        s.z += __shfl_xor_sync(~0u, s.z, d);
        s.t += __shfl_xor_sync(~0u, s.t, d);
    }
    return s;
}
// over the warp: the largest reference first, then plain sums relative to it
__device__ __forceinline__ Stat warp_merge(Stat s) {
    float m = s.m;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
    return warp_sum(merge(s, Stat{m, 0.f, 0.f}));
}

// what a row's merged sums say
struct RowResult {
    bool bad, none;
    float lse, entropy;
};
__device__ __forceinline__ RowResult row_result(const Stat &s) {
    RowResult r;
    r.bad = !(s.z < INF && s.m < INF);
    r.none = s.m == -INF;
    const float lz = log2f(s.z);
    r.lse = r.bad ? nan_f() : r.none ? -INF : fmaf(lz, LN2, s.m);
    // (Z of one token can round to just below 1)
    r.entropy = r.bad ? nan_f() : r.none ? 0.f : fmaxf(lz - s.t / s.z, 0.f) * LN2;
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
// Short rows: one warp each, the whole row in registers.  Top tokens: at least
// top_k logits reach the top_k-th largest of the lanes' maxima; those that do
// are listed in shared memory and sorted by counting.  Where ties overflow
// the list, the next token is the warp's largest key below the last one.
// One warp because a row is 2 to 4 KB: no exchange through shared memory, no
// barrier.  Bound by latency for few rows (256 x 1000 FP32, 5 tokens: 4.3 us,
// of which the row's load and the launch are half), by instructions for many
// (8192 x 1000 FP16: 7.4 us without tokens, 14.2 us with 5).
// ---------------------------------------------------------------------------
constexpr int SHORT = 1024;
constexpr int SHORT_WARPS = 4;
constexpr int SHORT_CAP = 192;                             // candidates of a warp

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
    float ga = -INF, gb = -INF;                            // this lane's largest logits, of even and of odd words
#pragma unroll
    for (int i = 0; i < NW; i += 4) {
        if (i / 4 * 32 * E >= vocab) break;
        ga = fmaxf(ga, Words<T>::largest(Words<T>::max2(w[i], w[i + 2])));
        gb = fmaxf(gb, Words<T>::largest(Words<T>::max2(w[i + 1], w[i + 3])));
    }
    const float mx = fmaxf(ga, gb);
    Sums<T> sums;
    sums.start();
    sums.reference(mx);
#pragma unroll
    for (int i = 0; i < NW; i += 4) {
        if (i / 4 * 32 * E >= vocab) break;
        const uint32_t part[4] = {w[i], w[i + 1], w[i + 2], w[i + 3]};
        sums.add(part);
    }
    const RowResult q = row_result(warp_sum(sums.stat()));
    if (lane == 0) write_row(a, r, q, id, given);
    if (a.top_k == 0) return;
    __shared__ __align__(16) uint64_t lists[SHORT_WARPS][SHORT_CAP];
    uint64_t *list = lists[threadIdx.x / 32];
    const int k = a.top_k;
    // The k-th largest of the lanes' maxima, the least of those that fewer than k
    // exceed: one a lane for few tokens, two where the 32nd of 32 would list too
    // much (8192 x 1000 FP16, 5 and 32 tokens: 14 and 73 us with one, 16 and 26 us
    // with two).
    const bool few = k <= 16;
    float *groups = reinterpret_cast<float *>(list);
    if (few) ga = mx;
    groups[lane] = ga;
    groups[32 + lane] = gb;
    __syncwarp();
    const auto above = [&](int from, float v) {
        int n = 0;
#pragma unroll
        for (int i = from; i < from + 32; i += 4) {
            const float4 o = *reinterpret_cast<const float4 *>(groups + i);
            n += (o.x > v) + (o.y > v) + (o.z > v) + (o.w > v);
        }
        return n;
    };
    const int ca = above(0, ga) + (few ? 0 : above(32, ga)), cb = few ? k : above(0, gb) + above(32, gb);
    __syncwarp();
    const uint32_t oa = (uint32_t)(order_key(ga, 0) >> 32), ob = (uint32_t)(order_key(gb, 0) >> 32);
    const uint32_t ot = __reduce_min_sync(~0u, min(ca < k ? oa : ~0u, cb < k ? ob : ~0u));
    const float thr = ot == 0 ? -INF : key_value((uint64_t)ot << 32);
    // how many of this lane's logits reach it, and where they go in the list
    int have = 0;
    if (mx >= thr && mx > -INF) {
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            if (i / 4 * 32 * E >= vocab) break;
#pragma unroll
            for (int e = 0; e < W2; ++e) {
                const float v = Words<T>::value(w[i], e);
                have += v >= thr && v > -INF;
            }
        }
    }
    int at = have;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(~0u, at, d);
        if (lane >= d) at += o;
    }
    const int n = __shfl_sync(~0u, at, 31);
    at -= have;
    uint64_t out = 0;                                      // lane i: the i-th token
    if (n <= SHORT_CAP) {
        if (have > 0) {
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                if (i / 4 * 32 * E >= vocab) break;
#pragma unroll
                for (int e = 0; e < W2; ++e) {
                    const float v = Words<T>::value(w[i], e);
                    if (v >= thr && v > -INF)
                        list[at++] = order_key(v, (uint32_t)((i / 4 * 32 + lane) * E + i % 4 * W2 + e));
                }
            }
        }
        __syncwarp();
        uint64_t keys[SHORT_CAP / 32];
        int ranks[SHORT_CAP / 32];
#pragma unroll
        for (int q = 0; q < SHORT_CAP / 32; ++q) {
            ranks[q] = 0;
            keys[q] = q * 32 + lane < n ? list[q * 32 + lane] : 0;
        }
        for (int j = 0; j < n; ++j) {
            const uint64_t o = list[j];
#pragma unroll
            for (int q = 0; q < SHORT_CAP / 32; ++q)
                if (q * 32 < n) ranks[q] += o > keys[q];
        }
        __syncwarp();
#pragma unroll
        for (int q = 0; q < SHORT_CAP / 32; ++q)
            if (q * 32 + lane < n && ranks[q] < k) list[ranks[q]] = keys[q];
        __syncwarp();
        if (lane < min(n, k)) out = list[lane];
    } else {
        uint64_t last = ~0ull, mine = ~0ull;               // mine: this lane's largest key below `last`
        for (int t = 0; t < k; ++t) {
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
            if (lane == t) out = b;
            last = b;
            if (b == 0) break;
        }
    }
    if (lane < k) write_top(a, r, lane, out, q);
}

// ---------------------------------------------------------------------------
// Top tokens of a row, or of a share of it, that NT threads read in vectors of
// 16 bytes, thread t vectors t, t + NT, ...  Each thread leaves its largest logit of
// the row and of each of up to 8 segments of it.  thr, the top_k-th largest of
// (up to) 64 group maxima, is reached by at least top_k tokens, but by few
// threads in few segments (little more than top_k): one warp looks over those
// threads' logits of those segments again, lists the keys that reach thr, and
// sorts the list by counting.  Where ties overflow the list it lists what
// exceeds thr and then the first tokens of the row that equal it; where that
// overflows too (the best tokens all in a few threads' hands) it picks the
// best one by one.  The list's order varies, the set and its sorted best do not.
// ---------------------------------------------------------------------------
constexpr int VECS = 4;                                    // 16-byte vectors that a thread examines together
constexpr int SEGMENTS = 8;                                // of a row, for a thread's maxima

template <typename T, int NT> struct Top {
    static constexpr int E = Vec16<T>::N;                  // values of a vector
    static constexpr int W2 = 4 / (int)sizeof(T);          // values of a word
    static constexpr int CAP = 8 * CT_MAX_TOP_K;           // candidates
    static constexpr int HITS = 8 * (NT < 64 ? NT : 64);   // thread segments looked over again
    struct Scratch {                                       // a finishing warp's
        alignas(16) uint64_t cand[CAP];
        uint64_t best[CT_MAX_TOP_K];
        uint8_t thread[NT];                                // threads, and
        uint16_t hit[HITS];                                // thread segments (thread * SEGMENTS + segment) with top tokens
    };
    struct Left {                                          // what the threads leave of a row
        float mx[NT];
        T seg[SEGMENTS][NT];
    };
    // a row's share in global memory: n values from x on, whose first has index j0 in the row
    struct Share {
        const T *x;
        int64_t n;
        uint32_t j0;
        uint32_t shift;                                    // bytes by which x misses a 16-byte boundary
        int seg_vecs;                                      // vectors of a thread in a segment
        int segs;
    };
    // the one or two 16-byte units that hold values of vector v, and its words, -inf past the end: apart, so that
    // several loads are in flight before the first is looked at
    struct Units {
        uint4 p, n;
    };
    static __device__ __forceinline__ Units fetch(const Share &q, int64_t v) {
        const int64_t left = (q.n - v * E) * (int)sizeof(T);
        const uint4 *at = reinterpret_cast<const uint4 *>((uintptr_t)q.x & ~(uintptr_t)15) + v;
        Units u = {};
        if (left > 0) u.p = __ldg(at);
        if (left > 0 && q.shift > 0 && (int64_t)q.shift + left > 16) u.n = __ldg(at + 1);
        return u;
    }
    static __device__ __forceinline__ uint4 words(const Share &q, int64_t v, const Units &u) {
        uint4 w = shifted(u.p, u.n, q.shift);
        const int have = (int)max((int64_t)0, min((int64_t)E, q.n - v * E));
        if (have < E) {
            w.x = Words<T>::mask(w.x, have);
            w.y = Words<T>::mask(w.y, have - W2);
            w.z = Words<T>::mask(w.z, have - 2 * W2);
            w.w = Words<T>::mask(w.w, have - 3 * W2);
        }
        return w;
    }
    // 32 bits ordered like the logits, 0 for none; and the least logit of that order
    static __device__ __forceinline__ uint32_t order(float x) { return (uint32_t)(order_key(x, 0) >> 32); }
    static __device__ __forceinline__ float order_value(uint32_t o) {
        // below every order: the lowest finite number's is the least that a token has
        return o <= order(-3.402823466e+38f) ? -3.402823466e+38f : key_value((uint64_t)o << 32);
    }

    // lists the keys of the logits whose order is at least `from` (> 0), looking at the thread segments that have
    // any; the list's length, or CAP + 1 where something overflowed
    static __device__ __forceinline__ int collect(Scratch &sh, const Left &left, const Share &q, uint32_t from) {
        const int lane = threadIdx.x % 32;
        const uint32_t below = (1u << lane) - 1u;
        const float least = order_value(from);
        // threads
        float mx[NT / 32];
#pragma unroll
        for (int i = 0; i < NT / 32; ++i) mx[i] = left.mx[i * 32 + lane];
        int threads = 0;
#pragma unroll
        for (int i = 0; i < NT / 32; ++i) {
            const uint32_t b = __ballot_sync(~0u, mx[i] >= least);
            if (mx[i] >= least) sh.thread[threads + __popc(b & below)] = (uint8_t)(i * 32 + lane);
            threads += __popc(b);
        }
        __syncwarp();
        // their segments: a thread for each lane
        int hits = 0;
        for (int i = 0; i < threads; i += 32) {
            const bool live = i + lane < threads;
            const int t = live ? sh.thread[i + lane] : 0;
            uint32_t b[SEGMENTS];
            int n = 0;
#pragma unroll
            for (int g = 0; g < SEGMENTS; ++g) {
                b[g] = __ballot_sync(~0u, live && g < q.segs && to_f32(left.seg[g][t]) >= least);
                n += __popc(b[g]);
            }
            if (hits + n > HITS) return CAP + 1;
#pragma unroll
            for (int g = 0; g < SEGMENTS; ++g) {
                if (b[g] >> lane & 1u) sh.hit[hits + __popc(b[g] & below)] = (uint16_t)(t * SEGMENTS + g);
                hits += __popc(b[g]);
            }
        }
        __syncwarp();
        // their vectors
        int count = 0;
        constexpr int AHEAD = 2;                           // loads in flight together
        const int all = hits * q.seg_vecs;
        for (int i = lane; i - lane < all; i += 32 * AHEAD) {
            Units x[AHEAD];
            uint32_t v[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const uint32_t at = (uint32_t)(i + 32 * u), h = at / (uint32_t)q.seg_vecs, o = at % (uint32_t)q.seg_vecs;
                const uint32_t hit = at < (uint32_t)all ? sh.hit[h] : 0;
                v[u] = (hit % SEGMENTS * (uint32_t)q.seg_vecs + o) * NT + hit / SEGMENTS;
                x[u] = Units{};
                if (at < (uint32_t)all) x[u] = fetch(q, v[u]);
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (i - lane + 32 * u >= all) break;
                uint4 w = words(q, v[u], x[u]);
                if (i + 32 * u >= all) w.x = w.y = w.z = w.w = Words<T>::dup(-INF);
                const float top = Words<T>::largest(Words<T>::max2(Words<T>::max2(w.x, w.y), Words<T>::max2(w.z, w.w)));
                if (__ballot_sync(~0u, top >= least) == 0) continue;
                float f[E];
                unpack16<T>(w, f);
                uint32_t mine = 0;                         // values that reach it, mostly one or none
#pragma unroll
                for (int e = 0; e < E; ++e) mine |= f[e] >= least ? 1u << e : 0u;
                for (uint32_t b; (b = __ballot_sync(~0u, mine != 0)) != 0; mine &= mine - 1, count += __popc(b)) {
                    const int at = count + __popc(b & below), e = __ffs(mine) - 1;
                    float x = f[0];
#pragma unroll
                    for (int n = 1; n < E; ++n) x = e == n ? f[n] : x;
                    if (mine != 0 && at < CAP) sh.cand[at] = order_key(x, q.j0 + v[u] * E + (uint32_t)e);
                }
            }
        }
        __syncwarp();
        return min(count, CAP + 1);
    }
    // sorts the list's best k into sh.best
    static __device__ __forceinline__ void select(Scratch &sh, int n, int k) {
        const int lane = threadIdx.x % 32;
        if (lane < k) sh.best[lane] = 0;
        __syncwarp();
        for (int i = lane; i < n; i += 32) {
            const uint64_t key = sh.cand[i];
            int rank = 0;
#pragma unroll 4
            for (int j = 0; j < n; ++j) rank += sh.cand[j] > key;
            if (rank < k) sh.best[rank] = key;
        }
        __syncwarp();
    }
    // the share's best k into sh.best
    static __device__ __forceinline__ void top(Scratch &sh, const Left &left, const Share &q, int k) {
        const int lane = threadIdx.x % 32;
        // up to 64 groups of threads, two for each lane
        uint32_t g0 = 0, g1 = 0;
        if constexpr (NT > 32) {
#pragma unroll
            for (int i = 0; i < NT / 32; i += 2) {
                g0 = max(g0, order(left.mx[i * 32 + lane]));
                g1 = max(g1, order(left.mx[i * 32 + 32 + lane]));
            }
        } else {                                           // each thread's, of either half of the segments
            for (int g = 0; g < q.segs; ++g) {
                const uint32_t o = order(to_f32(left.seg[g][lane]));
                if (2 * g < q.segs) g0 = max(g0, o);
                else g1 = max(g1, o);
            }
        }
        // the k-th largest: the least of those that fewer than k exceed
        uint32_t *all = reinterpret_cast<uint32_t *>(sh.cand);
        all[lane] = g0;
        all[32 + lane] = g1;
        __syncwarp();
        int c0 = 0, c1 = 0;
#pragma unroll
        for (int i = 0; i < 64; i += 4) {
            const uint4 o = *reinterpret_cast<const uint4 *>(all + i);
            c0 += (o.x > g0) + (o.y > g0) + (o.z > g0) + (o.w > g0);
            c1 += (o.x > g1) + (o.y > g1) + (o.z > g1) + (o.w > g1);
        }
        const uint32_t thr = __reduce_min_sync(~0u, min(c0 < k ? g0 : ~0u, c1 < k ? g1 : ~0u));   // k <= 32
        __syncwarp();
        const int n = collect(sh, left, q, max(thr, 1u));
        if (n <= CAP) select(sh, n, k);
        else top_ties(sh, q, left, k, thr);
    }
    // the same where more logits reach thr than the list holds
    static __device__ __noinline__ void top_ties(Scratch &sh, const Share &q, const Left &left, int k, uint32_t thr) {
        const int lane = threadIdx.x % 32;
        const int64_t vecs = (q.n + E - 1) / E;
        int n = thr == 0 ? CAP + 1 : collect(sh, left, q, thr + 1);
        if (n <= CAP) {
            select(sh, n, k);
            // ... and the first that equal it, in the row's order
            for (int64_t v0 = 0; n < k && v0 < vecs; v0 += 32) {
                float x[E];
                unpack16<T>(words(q, v0 + lane, fetch(q, v0 + lane)), x);
                int have = 0;
#pragma unroll
                for (int e = 0; e < E; ++e) have += order(x[e]) == thr;
                int at = have;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int u = __shfl_up_sync(~0u, at, d);
                    if (lane >= d) at += u;
                }
                const int found = __shfl_sync(~0u, at, 31);
                at += n - have;
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (order(x[e]) == thr) {
                        if (at < k) sh.best[at] = order_key(x[e], q.j0 + (uint32_t)((v0 + lane) * E + e));
                        ++at;
                    }
                n += found;
            }
            __syncwarp();
            return;
        }
        if (lane < k) sh.best[lane] = 0;
        __syncwarp();
        uint64_t last = ~0ull;
        for (int i = 0; i < k && last != 0; ++i) {
            uint64_t b = 0;
#pragma unroll 2
            for (int64_t v = lane; v < vecs; v += 32) {
                float x[E];
                unpack16<T>(words(q, v, fetch(q, v)), x);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const uint64_t key = order_key(x[e], q.j0 + (uint32_t)(v * E + e));
                    if (key < last && key > b) b = key;
                }
            }
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) b = max(b, __shfl_xor_sync(~0u, b, d));
            if (lane == 0) sh.best[i] = b;
            last = b;
        }
        __syncwarp();
    }
};

// ---------------------------------------------------------------------------
// Many rows of moderate length: one warp each, straight from global memory,
// VECS vectors a lane on their way while VECS are added.  A row of the kernel
// below would fill its last chunk badly and meet its barriers too often.
// Bound by waiting: 26 of the 32 warps that an SM holds are active, and a warp has
// no load on its way while it finishes a row (issue slots are 67% busy, DRAM 61%,
// the exponentials' pipe 27%): 8192 x 16000 BF16 with 8 tokens in 58.7 us, 4.5
// TB/s; 5696 x 5714 FP16 without tokens in 16.7 us, 3.9 TB/s.  ANY: rows that may start inside a
// 16-byte unit (96 registers a thread, not 64).
// ---------------------------------------------------------------------------
constexpr int ROW_WARPS = 4;

// VECS vectors that start `shift` (1 to 15) bytes into their first unit
template <int WS>
__device__ __forceinline__ void shift_words(const uint4 (&x)[VECS], const uint4 (&next)[VECS], uint32_t bits,
                                            uint32_t (&w)[4 * VECS]) {
#pragma unroll
    for (int u = 0; u < VECS; ++u) {
        const uint32_t s[8] = {x[u].x, x[u].y, x[u].z, x[u].w, next[u].x, next[u].y, next[u].z, next[u].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) w[4 * u + i] = __funnelshift_r(s[WS + i], s[WS + i + 1], bits);
    }
}
__device__ __forceinline__ void shift_all(const uint4 (&x)[VECS], const uint4 (&next)[VECS], uint32_t shift,
                                          uint32_t (&w)[4 * VECS]) {
    const uint32_t bits = (shift & 3u) * 8u;
    if (shift < 4) shift_words<0>(x, next, bits, w);
    else if (shift < 8) shift_words<1>(x, next, bits, w);
    else if (shift < 12) shift_words<2>(x, next, bits, w);
    else shift_words<3>(x, next, bits, w);
}

template <typename T, bool ANY>
__global__ void __launch_bounds__(32 * ROW_WARPS, ANY ? 5 : 8) logprobs_warp_kernel(const LpArgs a) {
    using P = Top<T, 32>;
    __shared__ typename P::Scratch scratch[ROW_WARPS];
    __shared__ typename P::Left lefts[ROW_WARPS];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int64_t r = (int64_t)blockIdx.x * ROW_WARPS + warp;
    if (r >= a.rows) return;
    const T *row = static_cast<const T *>(a.x) + r * a.ldx;
    int64_t id = -1;
    const float given = lane == 0 ? given_logit<T>(a, r, id) : 0.f;
    const int batches = (int)((a.vocab + 32 * VECS * P::E - 1) / (32 * VECS * P::E));
    const int seg_batches = (batches + SEGMENTS - 1) / SEGMENTS;
    const typename P::Share q = {row, a.vocab, 0u, (uint32_t)((uintptr_t)row & 15), seg_batches * VECS,
                                 (batches + seg_batches - 1) / seg_batches};
    typename P::Left &left = lefts[warp];
    Sums<T> sums;
    sums.start();
    float mx = -INF, seg_mx = -INF;
    const uint4 *units = reinterpret_cast<const uint4 *>((uintptr_t)row & ~(uintptr_t)15);
    const int vocab = (int)a.vocab;
    // batch b's 16-byte units that hold one of its values (with `next`, the second ones of rows that start inside one)
    uint4 x[VECS], next[VECS];
    const auto load = [&](int b) {
#pragma unroll
        for (int u = 0; u < VECS; ++u) {
            const int v = (b * VECS + u) * 32 + lane, bytes = (vocab - v * P::E) * (int)sizeof(T);
            if (bytes > 0) x[u] = __ldg(units + v);
            if (ANY && q.shift > 0 && (int)q.shift + bytes > 16 && bytes > 0) next[u] = __ldg(units + v + 1);
        }
    };
    load(0);
    int seg = 0, seg_left = seg_batches;
    for (int b = 0; b < batches; ++b) {
        uint32_t w[4 * VECS];
        if (!ANY || q.shift == 0) {
#pragma unroll
            for (int u = 0; u < VECS; ++u) {
                w[4 * u] = x[u].x; w[4 * u + 1] = x[u].y; w[4 * u + 2] = x[u].z; w[4 * u + 3] = x[u].w;
            }
        } else {
            shift_all(x, next, q.shift, w);
        }
        if (b + 1 < batches) {
            load(b + 1);
        } else {
#pragma unroll
            for (int i = 0; i < 4 * VECS; ++i)
                w[i] = Words<T>::mask(w[i], vocab - ((b * VECS + i / 4) * 32 + lane) * P::E - i % 4 * P::W2);
        }
        uint32_t m2 = w[0];
#pragma unroll
        for (int i = 1; i < 4 * VECS; ++i) m2 = Words<T>::max2(m2, w[i]);
        const float top = Words<T>::largest(m2);
        sums.reference(top);
        sums.add(w);
        seg_mx = fmaxf(seg_mx, top);
        if (--seg_left == 0 || b + 1 == batches) {
            left.seg[seg++][lane] = from_f32<T>(seg_mx);   // exact: a value of this type
            mx = fmaxf(mx, seg_mx);
            seg_mx = -INF;
            seg_left = seg_batches;
        }
    }
    left.mx[lane] = mx;
    const RowResult res = row_result(warp_sum(sums.stat()));
    if (lane == 0) write_row(a, r, res, id, given);
    if (a.top_k > 0) {
        __syncwarp();
        P::top(scratch[warp], left, q, a.top_k);
        if (lane < a.top_k) write_top(a, r, lane, scratch[warp].best[lane], res);
    }
}

// ---------------------------------------------------------------------------
// Long rows.  A row, or a share of it, streams through shared memory in chunks
// of 64 bytes a thread.  A producer warp has the bulk engine copy STAGES chunks
// ahead, the consumer warps take each chunk at their own pace and go on with
// the next row, and finisher warps, in turn, make a row's results of what they
// leave of it meanwhile.  Where there are fewer rows than CTAs a cluster of up to
// 8 shares a row and one warp joins the shares, in their order.
// Bound by HBM where rows abound (2048 x 131072 BF16 with 8 tokens in 88 us, 6.1
// TB/s, without tokens 6.5), by the way from the last value to the result where
// they do not: 1 x 131072 FP16 takes 3.5 us, with 20 tokens 7.8 us.
// ---------------------------------------------------------------------------

constexpr int MAX_SPLITS = 8;                              // CTAs that share a row

// A thread's wait for a barrier's phase, at most `limit` x 2^32 cycles.  Its first
// wait in vain takes the limit away, so that they do not add up, one for each
// chunk: each later one ends after 256 polls, 0.3 ms.  (A vote of the warp, or a flag
// that all threads see, costs every chunk 1 to 2%.)
__device__ __forceinline__ bool wait_for(uint64_t *bar, uint32_t parity, uint32_t *err, int &limit) {
    const uint32_t b = tc::smem_u32(bar);
    if (tc::mbar_try_wait(b, parity)) return true;
    const long long t0 = clock64();
    for (uint32_t it = 1;; ++it) {
        if (tc::mbar_try_wait(b, parity)) return true;
        if ((it & 255) == 0 && (int)((clock64() - t0) >> 32) >= limit) {
            atomicOr(err, E_LOGPROBS);
            limit = 0;
            return false;
        }
    }
}

// the 32 best keys of two lists, each sorted over the lanes from the best on
__device__ __forceinline__ uint64_t best32(uint64_t a, uint64_t b) {
    const int lane = threadIdx.x % 32;
    a = max(a, __shfl_sync(~0u, b, 31 - lane));            // rises, then falls
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        const uint64_t o = __shfl_xor_sync(~0u, a, d);
        a = (lane & d) == 0 ? max(a, o) : min(a, o);
    }
    return a;
}

// NT consumer threads, a producer warp and FIN finisher warps
template <typename T, int NT> struct Long : Top<T, NT> {
    using P = Top<T, NT>;
    using P::E;
    using P::W2;
    static constexpr int CHUNK = NT * VECS * 16;           // bytes
    static constexpr int CE = CHUNK / (int)sizeof(T);      // values
    static constexpr int STAGE = CHUNK + 128;              // a row may start anywhere in its first 16 bytes
    static constexpr int FIN = NT == 256 ? 2 : 4;
    static constexpr int THREADS = NT + 32 + 32 * FIN;
    static constexpr int CTAS = NT == 256 ? 2 : 3;         // on an SM
    static constexpr int STAGES = 3;
    struct Left : P::Left {
        Stat part[NT / 32];
    };
    struct Shared {
        uint64_t full[STAGES], empty[STAGES];
        uint64_t left_full[FIN], left_free[FIN];
        typename P::Scratch scratch[FIN];
        Left left[FIN];
        Stat total;                                        // a split row's
        float given;
        int64_t id;
    };
    static constexpr size_t SMEM = (size_t)STAGES * STAGE + sizeof(Shared) + 16;
    static_assert(CTAS * (SMEM + 1024) <= 228 * 1024, "shared memory of an SM");

    // The 4 words of 16-byte vector v of a chunk whose first value lies WS words and `bits` bits into the stage
    // (WS = -1: at its start).  Which values a thread takes does not depend on where the row starts, so neither do
    // the sums.
    template <int WS> static __device__ __forceinline__ void load(const uint8_t *stage, int v, uint32_t bits, uint32_t *w) {
        const uint4 p = *reinterpret_cast<const uint4 *>(stage + v * 16);
        if constexpr (WS < 0) {
            w[0] = p.x; w[1] = p.y; w[2] = p.z; w[3] = p.w;
        } else {
            const uint4 n = *reinterpret_cast<const uint4 *>(stage + v * 16 + 16);
            const uint32_t s[8] = {p.x, p.y, p.z, p.w, n.x, n.y, n.z, n.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(s[WS + i], s[WS + i + 1], bits);
        }
    }
    template <int WS> static __device__ __forceinline__ void load_all(const uint8_t *stage, uint32_t bits, uint32_t *w) {
#pragma unroll
        for (int b = 0; b < VECS; ++b) load<WS>(stage, b * NT + (int)threadIdx.x, bits, w + 4 * b);
    }
    // adds a chunk's first n_valid values to the thread's sums, releases the stage as soon as it is read; the
    // thread's largest
    static __device__ __forceinline__ float chunk(const uint8_t *stage, uint32_t shift, int n_valid, uint64_t *empty,
                                                  Sums<T> &sums) {
        uint32_t w[4 * VECS];
        const uint32_t bits = (shift & 3u) * 8u;
        if (shift == 0) load_all<-1>(stage, 0, w);
        else if (shift < 4) load_all<0>(stage, bits, w);
        else if (shift < 8) load_all<1>(stage, bits, w);
        else if (shift < 12) load_all<2>(stage, bits, w);
        else load_all<3>(stage, bits, w);
        __syncwarp();
        if (threadIdx.x % 32 == 0) tc::mbar_arrive(tc::smem_u32(empty));
        if (n_valid < CE) {
#pragma unroll
            for (int b = 0; b < 4 * VECS; ++b)
                w[b] = Words<T>::mask(w[b], n_valid - (b / 4 * NT + (int)threadIdx.x) * E - b % 4 * W2);
        }
        uint32_t m2 = w[0];
#pragma unroll
        for (int b = 1; b < 4 * VECS; ++b) m2 = Words<T>::max2(m2, w[b]);
        const float top = Words<T>::largest(m2);
        sums.reference(top);
        sums.add(w);
        return top;
    }
};

template <typename T, int NT>
__global__ void __launch_bounds__(Long<T, NT>::THREADS, Long<T, NT>::CTAS) logprobs_long_kernel(const LpArgs a, int splits) {
    using L = Long<T, NT>;
    constexpr int STAGES = L::STAGES, FIN = L::FIN;
    extern __shared__ __align__(128) uint8_t smem[];
    typename L::Shared &sh = *reinterpret_cast<typename L::Shared *>(smem + STAGES * L::STAGE);
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int rank = (int)(blockIdx.x % (unsigned)splits);
    const int64_t cid = blockIdx.x / (unsigned)splits, ncl = gridDim.x / (unsigned)splits;
    const int chunks = (int)((a.vocab + L::CE - 1) / L::CE);
    const int ch0 = (int)((int64_t)chunks * rank / splits), ch1 = (int)((int64_t)chunks * (rank + 1) / splits);
    const int seg_chunks = (ch1 - ch0 + SEGMENTS - 1) / SEGMENTS;
    const int k = a.top_k;

    if (tid == 0) {
        for (int s = 0; s < STAGES; ++s) {
            tc::mbar_init(tc::smem_u32(&sh.full[s]), 1);
            tc::mbar_init(tc::smem_u32(&sh.empty[s]), NT / 32);
        }
        for (int b = 0; b < FIN; ++b) {
            tc::mbar_init(tc::smem_u32(&sh.left_full[b]), NT / 32);
            tc::mbar_init(tc::smem_u32(&sh.left_free[b]), 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    pdl_wait();
    pdl_trigger();

    // A wait that runs out is reported: the results are invalid.  The producer and the
    // finishers stop then, consumers run through to the end with next to no more waits.
    if (warp == NT / 32) {
        if (lane == 0) {
            int it = 0;
            bool ok = true;
            for (int64_t r = cid; r < a.rows && ok; r += ncl) {
                const uint8_t *row = reinterpret_cast<const uint8_t *>(static_cast<const T *>(a.x) + r * a.ldx);
                const int64_t row_bytes = a.vocab * (int64_t)sizeof(T);
                for (int ch = ch0; ch < ch1; ++ch, ++it) {
                    const int s = it % STAGES;
                    ok = tc::mbar_wait(tc::smem_u32(&sh.empty[s]), ((uint32_t)(it / STAGES) & 1u) ^ 1u, a.err, E_LOGPROBS);
                    if (!ok) break;
                    // whole 16-byte units that hold a value of the chunk
                    const int64_t end = min((int64_t)(ch + 1) * L::CHUNK, row_bytes);
                    const uintptr_t from = (uintptr_t)(row + (int64_t)ch * L::CHUNK) & ~(uintptr_t)15;
                    const uintptr_t to = ((uintptr_t)(row + end) + 15) & ~(uintptr_t)15;
                    const uint32_t bar = tc::smem_u32(&sh.full[s]);
                    tc::mbar_arrive_expect_tx(bar, (uint32_t)(to - from));
                    tc::bulk_load(tc::smem_u32(smem + s * L::STAGE), reinterpret_cast<const void *>(from),
                                  (uint32_t)(to - from), bar);
                }
            }
            // no copy is under way when the CTA ends, whoever gave up
            for (int j = max(0, it - STAGES); j < it; ++j)
                tc::mbar_wait(tc::smem_u32(&sh.full[j % STAGES]), (uint32_t)(j / STAGES) & 1u, a.err, E_DRAIN);
        }
        __syncwarp();
    } else if (warp > NT / 32) {
        const int f = warp - NT / 32 - 1;                  // rows f, f + FIN, ... of this CTA's
        typename L::Scratch &scratch = sh.scratch[f];
        const typename L::Left &left = sh.left[f];
        uint32_t phase = 0;
        for (int64_t r = cid + f * ncl; r < a.rows; r += FIN * ncl, phase ^= 1u) {
            const T *row = static_cast<const T *>(a.x) + r * a.ldx;
            int64_t id = -1;
            const float given = lane == 0 && rank == 0 ? given_logit<T>(a, r, id) : 0.f;
            if (!tc::warp_wait(tc::smem_u32(&sh.left_full[f]), phase, a.err, E_LOGPROBS)) break;
            const Stat st = warp_merge(lane < NT / 32 ? left.part[lane] : Stat{-INF, 0.f, 0.f});
            if (k > 0) {
                const int64_t v0 = (int64_t)ch0 * L::CE;
                const typename L::Share q = {row + v0, min((int64_t)ch1 * L::CE, a.vocab) - v0, (uint32_t)v0,
                                             (uint32_t)((uintptr_t)(row + v0) & 15), seg_chunks * VECS,
                                             (ch1 - ch0 + seg_chunks - 1) / seg_chunks};
                L::top(scratch, left, q, k);
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(tc::smem_u32(&sh.left_free[f]));
            if (splits == 1) {
                const RowResult q = row_result(st);
                if (lane == 0) write_row(a, r, q, id, given);
                if (lane < k) write_top(a, r, lane, scratch.best[lane], q);
            } else if (lane == 0) {
                sh.total = st;
                sh.id = id;
                sh.given = given;
            }
            __syncwarp();
        }
    } else {
        int limit = 1;
        int it = 0, f = 0;                                 // f: whose turn it is to finish the row
        uint32_t phase = 0;
        for (int64_t r = cid; r < a.rows; r += ncl) {
            const uint32_t shift = (uint32_t)((uintptr_t)(static_cast<const T *>(a.x) + r * a.ldx) & 15);
            typename L::Left &left = sh.left[f];
            Sums<T> sums;
            sums.start();
            float mx = -INF, seg_mx = -INF;
            int seg = 0, seg_left = seg_chunks;
            for (int ch = ch0; ch < ch1; ++ch, ++it) {
                const int s = it % STAGES;
                const uint8_t *stage = smem + s * L::STAGE;
                const int n_valid = (int)min((int64_t)L::CE, a.vocab - (int64_t)ch * L::CE);
                wait_for(&sh.full[s], (uint32_t)(it / STAGES) & 1u, a.err, limit);
                const float top = L::chunk(stage, shift, n_valid, &sh.empty[s], sums);
                seg_mx = fmaxf(seg_mx, top);
                if (--seg_left == 0 || ch + 1 == ch1) {
                    if (seg == 0)                          // the row FIN before is finished
                        wait_for(&sh.left_free[f], phase ^ 1u, a.err, limit);
                    left.seg[seg++][tid] = from_f32<T>(seg_mx);        // exact: a value of this type
                    mx = fmaxf(mx, seg_mx);
                    seg_mx = -INF;
                    seg_left = seg_chunks;
                }
            }
            left.mx[tid] = mx;
            const Stat st = warp_sum(sums.stat());
            if (lane == 0) left.part[warp] = st;
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(tc::smem_u32(&sh.left_full[f]));
            if (++f == FIN) {
                f = 0;
                phase ^= 1u;
            }
        }
    }
    __syncwarp();
    if (splits > 1) {
        // one row for each cluster: rank 0's consumer threads join the shares, in rank order
        tc::cluster_sync();
        if (rank == 0 && warp == 0) {
            // lane p: share p's sums; lane i: each share's i-th best token
            Stat st = {-INF, 0.f, 0.f};
            if (lane < splits) {
                const uint32_t at = tc::mapa_shared(tc::smem_u32(&sh.total), (uint32_t)lane);
                st = Stat{ld_cluster_f32(at), ld_cluster_f32(at + 4), ld_cluster_f32(at + 8)};
            }
            uint64_t best[MAX_SPLITS];
#pragma unroll
            for (int p = 0; p < MAX_SPLITS; ++p)
                best[p] = p < splits && lane < k
                              ? ld_cluster_u64(tc::mapa_shared(tc::smem_u32(&sh.scratch[0].best[lane]), (uint32_t)p))
                              : 0;
            const RowResult q = row_result(warp_merge(st));
            if (lane == 0) write_row(a, cid, q, sh.id, sh.given);
            if (k > 0) {
#pragma unroll
                for (int n = MAX_SPLITS / 2; n > 0; n /= 2)
#pragma unroll
                    for (int p = 0; p < n; ++p) best[p] = best32(best[p], best[p + n]);
                if (lane < k) write_top(a, cid, lane, best[0], q);
            }
        }
        tc::cluster_sync();
    }
}

// ---------------------------------------------------------------------------
// Gradient: each CTA a piece of one row, GRAD_VECS 16-byte vectors a thread, or
// short rows side by side, a power of two of threads each (8 to 256).  The
// vectors are those of dx, so that every store is whole wherever the rows of x
// start.  LONG: rows of 256 threads or more that start as those of dx do, in
// fewer registers (32 and not 59: 2048 x 131072 BF16 153 us and not 170).
// Bound by HBM, each logit read and each gradient written once: 7.0 TB/s there;
// short rows by latency (6476 x 15 BF16 in 2.1 us; a CTA a row took 11.6).
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

template <typename T, bool LONG>
__global__ void __launch_bounds__(GRAD_THREADS) logprobs_grad_kernel(const GradArgs a, int pieces, int row_lanes) {
    constexpr int E = Vec16<T>::N;
    const int lanes = LONG ? GRAD_THREADS : row_lanes;
    pdl_wait();
    pdl_trigger();
    const int64_t r = LONG || pieces > 1 ? (int64_t)(blockIdx.x / (unsigned)pieces)
                                 : (int64_t)blockIdx.x * (GRAD_THREADS / (unsigned)lanes) + threadIdx.x / (unsigned)lanes;
    if (r >= a.rows) return;
    const int piece = (int)(blockIdx.x % (unsigned)pieces), lane = (int)threadIdx.x & (lanes - 1);
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
    // values before dx's first 16-byte boundary, and the vectors after it
    const int64_t head = min((int64_t)((16 - ((uintptr_t)dx & 15)) & 15) / (int)sizeof(T), a.vocab);
    const uint32_t shift = LONG ? 0u : (uint32_t)(uintptr_t)(x + head) & 15u;
    const int64_t vecs = (a.vocab - head) / E, per = GRAD_THREADS * GRAD_VECS;
    const int64_t v0 = piece * per + lane;
    const uint4 *units = reinterpret_cast<const uint4 *>((uintptr_t)(x + head) - shift);
    uint4 u[GRAD_VECS];
#pragma unroll
    for (int i = 0; i < GRAD_VECS; ++i)
        if (v0 + i * lanes < vecs) u[i] = __ldcs(units + v0 + i * lanes);
    if (!LONG && shift != 0) {
        uint4 n[GRAD_VECS];
#pragma unroll
        for (int i = 0; i < GRAD_VECS; ++i)
            if (v0 + i * lanes < vecs) n[i] = __ldg(units + v0 + i * lanes + 1);
#pragma unroll
        for (int i = 0; i < GRAD_VECS; ++i) u[i] = shifted(u[i], n[i], shift);
    }
    // the ends of the row: its first piece's threads
    if (piece == 0) {
        const int64_t tail = head + vecs * E;
        if (lane < head) grad_one(q, x, dx, (int64_t)lane);
        if (tail + lane < a.vocab) grad_one(q, x, dx, tail + lane);
    }
#pragma unroll
    for (int i = 0; i < GRAD_VECS; ++i) {
        const int64_t v = v0 + i * lanes;
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
        __stcs(reinterpret_cast<uint4 *>(dx + j), pack16<T>(d));
    }
}

template <typename T, int NT> cudaError_t launch_long(const LpArgs &a, cudaStream_t st) {
    using L = Long<T, NT>;
    static std::atomic<bool> sized[MAX_DEVICES];
    cudaError_t e = allow_smem(logprobs_long_kernel<T, NT>, sized, L::SMEM);
    if (e != cudaSuccess) return e;
    const int64_t slots = (int64_t)sm_count() * L::CTAS;
    const int64_t chunks = (a.vocab + L::CE - 1) / L::CE;
    // few rows: each is shared by a cluster (one row each), so that the whole GPU reads
    int splits = 1;
    while (splits < MAX_SPLITS && a.rows * splits * 2 <= slots && splits * 2 <= chunks) splits *= 2;
    const dim3 block(L::THREADS);
    if (splits > 1)
        return pdl_launch_cluster(logprobs_long_kernel<T, NT>, dim3((unsigned)(a.rows * splits)), block, L::SMEM, st,
                                  splits, a, splits);
    return pdl_launch(logprobs_long_kernel<T, NT>, dim3((unsigned)(a.rows < slots ? a.rows : slots)), block, L::SMEM, st,
                      a, splits);
}

template <typename T> cudaError_t launch_logprobs(const LpArgs &a, cudaStream_t st) {
    if (a.vocab <= SHORT) {
        const int vec = aligned(a.x, 16) && (a.rows == 1 || a.ldx % Vec16<T>::N == 0);
        return pdl_launch(logprobs_short_kernel<T>, dim3((unsigned)((a.rows + SHORT_WARPS - 1) / SHORT_WARPS)),
                          dim3(32 * SHORT_WARPS), 0, st, a, vec);
    }
    const int64_t row_bytes = a.vocab * (int64_t)sizeof(T);
    if (row_bytes <= 32768 && a.rows >= 8 * (int64_t)sm_count()) {
        const dim3 grid((unsigned)((a.rows + ROW_WARPS - 1) / ROW_WARPS)), block(32 * ROW_WARPS);
        return aligned(a.x, 16) && a.ldx % Vec16<T>::N == 0 ? pdl_launch(logprobs_warp_kernel<T, false>, grid, block, 0, st, a)
                                                            : pdl_launch(logprobs_warp_kernel<T, true>, grid, block, 0, st, a);
    }
    return row_bytes < 98304 ? launch_long<T, 128>(a, st) : launch_long<T, 256>(a, st);
}

template <typename T>
cudaError_t launch_grad(const GradArgs &a, dim3 grid, int pieces, int lanes, bool shifted, cudaStream_t st) {
    return lanes < GRAD_THREADS || shifted
               ? pdl_launch(logprobs_grad_kernel<T, false>, grid, dim3(GRAD_THREADS), 0, st, a, pieces, lanes)
               : pdl_launch(logprobs_grad_kernel<T, true>, grid, dim3(GRAD_THREADS), 0, st, a, pieces, lanes);
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
    // short rows: two vectors a thread, and threads enough for the values at a row's ends
    int lanes = 8;
    while (lanes < GRAD_THREADS && (int64_t)lanes * 2 * (16 / es) < vocab) lanes *= 2;
    const int64_t side = GRAD_THREADS / lanes;
    const dim3 grid((unsigned)(pieces > 1 ? rows * pieces : (rows + side - 1) / side));
    const bool shifted = (((uintptr_t)logits_dev ^ (uintptr_t)dlogits_dev) & 15) != 0 ||
                         (rows > 1 && (ld - ld_d) % (16 / es) != 0);
    const cudaError_t e = dtype == CT_DT_F32   ? launch_grad<float>(a, grid, (int)pieces, lanes, shifted, st)
                          : dtype == CT_DT_F16 ? launch_grad<__half>(a, grid, (int)pieces, lanes, shifted, st)
                                               : launch_grad<__nv_bfloat16>(a, grid, (int)pieces, lanes, shifted, st);
    return e == cudaSuccess ? CT_OK : CT_ECUDA;
}
