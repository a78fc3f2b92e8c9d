// Drafted tokens held against the target's probabilities.
//
// Draft x_j stands while those before it do and u_j q_j(x_j) < p_j(x_j), with p and q
// the softmaxes of the target's and the draft's row at the sequence's temperature.
// After the last that stands one token is drawn from max(p - q, 0), normalised, at the
// draft that fell (which makes the whole distributed as p), or from p after all of
// them.  The draw is a race: of independent exponentials E_i the one with the least
// E_i / w_i is i with probability w_i / sum w.  It needs no normaliser and no running
// sum, so its outcome hangs on no order of addition; ties go to the lower index.
//
// A row's maximum m and Z = sum e^((x - m) / T) come from parts of the row, each held
// in FP32 relative to its own maximum; comparisons that are close are made in FP64.
//
// Two launches.  The first reads every row once, a warp for each piece of a row, and is bound by HBM (it has about the
// least time that one exponential for each value leaves, too).  The second decides, a cluster for each sequence, and reads
// the row of the draft that fell, the draft's, and the noise: the rows mostly from L2.  Measured alone, 64 sequences of 5 drafts over
// 131072 BF16 logits: 33 us (5.6 TB/s) and 18 us; in a row, as the second begins early, 50 us.
#include "ops_common.cuh"
#include "tc_common.cuh"

namespace ct {
namespace ops {
namespace {

constexpr float INF = __builtin_huge_valf();
__device__ __forceinline__ float nan_f() { return __uint_as_float(0x7FC00000u); }
constexpr float LOG2E = 1.4426950408889634f;

struct VerifyArgs {
    const void *x, *q;
    int64_t ldx, ldq;
    const int64_t *drafts, *offsets;
    const float *uniform, *noise, *temperature;
    int64_t ld_noise;
    int64_t sequences, count, vocab;
    int most;
    int64_t *accepted, *token;
    float *logprob;
};

// What a piece of a row holds: its largest logit, sum e^((x - m) / T) (NaN where a NaN or +inf is in it), and, for greedy sequences, the
// lowest index that has the largest.
struct Piece {
    float m, z;
    int32_t at, pad;
};

struct Sequence {
    int64_t from;                                 // its first draft
    int d;                                        // drafts looked at
    float heat;                                   // 1 / T; 1 where greedy
    bool greedy, bad;
};

__device__ __forceinline__ Sequence sequence(const VerifyArgs &a, int64_t b) {
    Sequence s;
    s.from = min(max(a.offsets[b], (int64_t)0), a.count);
    const int64_t to = min(max(a.offsets[b + 1], s.from), a.count);
    s.d = (int)min(to - s.from, (int64_t)a.most);
    const float t = a.temperature != nullptr ? a.temperature[b] : 1.f;
    s.bad = !(t >= 0.f && t < INF);
    s.greedy = t < 1e-30f;
    s.heat = s.greedy || s.bad ? 1.f : 1.f / t;
    return s;
}

__device__ __forceinline__ float ex2(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// ---------------------------------------------------------------- rows

constexpr int ROW_WARPS = 4;
constexpr int BATCH = 4;                          // vectors of 16 bytes that a lane takes at a time

struct Stat {
    float m, z;
    int32_t at;
};

// N values and their indices, in any order (ARG: the lowest index of the largest is wanted)
template <int N, bool ARG> __device__ __forceinline__ void see(Stat &s, const float (&v)[N], float c, const int32_t (&at)[N]) {
    float top = v[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, v[i]);
    const float m = fmaxf(s.m, top), ref = m == -INF ? 0.f : m;
    if (ARG && top >= s.m) {
        // a lane's values behind a piece's last 16-byte unit come before those of the units, so that an equal one may have a lower index
        int32_t first = top > s.m ? INT32_MAX : s.at;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (v[i] == top && at[i] < first) first = at[i];
        s.at = first;
    }
    float z = s.z * ex2((s.m - ref) * c);         // s.m = -inf: s.z is 0, and stays it
#pragma unroll
    for (int i = 0; i < N; ++i) z += ex2((v[i] - ref) * c);                     // +inf and NaN give NaN
    s.m = m;
    s.z = z;
}

__device__ __forceinline__ Stat join(const Stat &a, const Stat &b, float c) {
    Stat r;
    r.m = fmaxf(a.m, b.m);
    const float ref = r.m == -INF ? 0.f : r.m;
    r.z = a.z * ex2((a.m - ref) * c) + b.z * ex2((b.m - ref) * c);
    r.at = a.m > b.m || (a.m == b.m && a.at < b.at) ? a.at : b.at;
    return r;
}

// values j0 to j1 - 1 of a row, by a warp
template <typename T, bool ARG> __device__ __forceinline__ Stat scan(const T *x, int64_t j0, int64_t j1, float c) {
    constexpr int E = 16 / (int)sizeof(T);
    const int lane = threadIdx.x & 31;
    Stat s = {-INF, 0.f, INT32_MAX};
    const T *p = x + j0;
    const int n = (int)(j1 - j0), off = (int)((16 - (uintptr_t)p % 16) % 16) / (int)sizeof(T), head = off < n ? off : n;
    const int vecs = (n - head) / E, tail = head + vecs * E;
    if (lane < head || lane < n - tail) {
        const float v[2] = {lane < head ? to_f32(p[lane]) : -INF, lane < n - tail ? to_f32(p[tail + lane]) : -INF};
        const int32_t at[2] = {(int32_t)j0 + lane, (int32_t)j0 + tail + lane};
        see<2, ARG>(s, v, c, at);
    }
    const uint4 *q = reinterpret_cast<const uint4 *>(p + head);
    int v0 = lane;
    if (v0 + 32 * (BATCH - 1) < vecs) {
        uint4 u[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) u[i] = q[v0 + 32 * i];
        while (true) {
            // the next batch is on its way while this one is worked on; behind the end, the last one again
            const int next = v0 + 32 * BATCH, safe = next + 32 * (BATCH - 1) < vecs ? next : v0;
            uint4 w[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) w[i] = q[safe + 32 * i];
            float v[BATCH * E];
            int32_t at[BATCH * E];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                unpack16<T>(u[i], v + i * E);
                if (ARG)
#pragma unroll
                    for (int e = 0; e < E; ++e) at[i * E + e] = (int32_t)j0 + head + (v0 + 32 * i) * E + e;
            }
            see<BATCH * E, ARG>(s, v, c, at);
            v0 = next;
            if (safe != next) break;
#pragma unroll
            for (int i = 0; i < BATCH; ++i) u[i] = w[i];
        }
    }
    for (; v0 < vecs; v0 += 32) {
        float v[E];
        int32_t at[E];
        unpack16<T>(q[v0], v);
#pragma unroll
        for (int e = 0; e < E; ++e) at[e] = (int32_t)j0 + head + v0 * E + e;
        see<E, ARG>(s, v, c, at);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const Stat b = {__shfl_xor_sync(0xffffffffu, s.m, o), __shfl_xor_sync(0xffffffffu, s.z, o), __shfl_xor_sync(0xffffffffu, s.at, o)};
        s = join(s, b, c);
    }
    return s;
}

// pieces of rows, a warp for each: the target's rows of all sequences, then the drafts'
template <typename T>
__global__ void __launch_bounds__(32 * ROW_WARPS) verify_rows_kernel(const VerifyArgs a, int pieces, int per, int64_t all, Piece *out) {
    pdl_wait();
    pdl_trigger();
    const int64_t unit = (int64_t)blockIdx.x * ROW_WARPS + (threadIdx.x >> 5);
    if (unit >= all) return;
    const int64_t row = unit / pieces, targets = a.count + a.sequences;
    const int piece = (int)(unit - row * pieces);
    const bool draft = row >= targets;
    const int64_t at = draft ? row - targets : row;
    // the sequence of the row: the last whose rows begin at or before it
    int64_t lo = 0, hi = a.sequences - 1;
    while (lo < hi) {
        const int64_t mid = (lo + hi + 1) / 2;
        if (min(max(a.offsets[mid], (int64_t)0), a.count) + (draft ? 0 : mid) <= at) lo = mid;
        else hi = mid - 1;
    }
    const Sequence s = sequence(a, lo);
    const T *x = draft ? static_cast<const T *>(a.q) + at * a.ldq : static_cast<const T *>(a.x) + at * a.ldx;
    const int64_t j0 = (int64_t)piece * per, j1 = min(j0 + per, a.vocab);
    const float c = s.heat * LOG2E;
    const Stat r = s.greedy ? scan<T, true>(x, j0, j1, c) : scan<T, false>(x, j0, j1, c);
    if ((threadIdx.x & 31) == 0) out[unit] = {r.m, r.z, r.at, 0};
}

// ---------------------------------------------------------------- sequences

constexpr int THREADS = 512, WARPS = THREADS / 32;

// a whole row: its largest logit and sum e^((x - m) / T); bad: a NaN or +inf in it
struct Row {
    float m, z;
    int32_t at;
    bool bad;
};

// by a warp
__device__ __forceinline__ Row row_of(const Piece *p, int pieces, float c) {
    const int lane = threadIdx.x & 31;
    Row r = {-INF, 0.f, INT32_MAX, false};
    for (int i = lane; i < pieces; i += 32) {
        const Piece q = p[i];
        if (q.m > r.m || (q.m == r.m && q.at < r.at)) {
            r.m = q.m;
            r.at = q.at;
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float m = __shfl_xor_sync(0xffffffffu, r.m, o);
        const int32_t at = __shfl_xor_sync(0xffffffffu, r.at, o);
        if (m > r.m || (m == r.m && at < r.at)) {
            r.m = m;
            r.at = at;
        }
    }
    const float ref = r.m == -INF ? 0.f : r.m;
    for (int i = lane; i < pieces; i += 32) r.z += p[i].z * exp2f((p[i].m - ref) * c);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) r.z += __shfl_xor_sync(0xffffffffu, r.z, o);
    r.bad = !(r.z < INF) || r.m == INF;
    // INT32_MAX: a row that offsets which descend give to two sequences, the other one not greedy
    if (r.m == -INF || r.at == INT32_MAX) r.at = -1;
    return r;
}

// whether u q < p:  log(u zp / zq) + (xq - mq) / T < (x - m) / T.  In FP32 where that is clear (each term's error is a few 2^-23 of it);
// FP64 is slow here (two operations a cycle for an SM) and left to what is close.
__device__ __forceinline__ bool stands(float u, const Row &p, float x, bool have, const Row &q, float xq, float heat) {
    if (have && !(xq > -INF)) return true;        // q is 0, p is not
    const float l0 = logf(u), l1 = have ? logf(p.z) - logf(q.z) : logf(p.z), l2 = (x - p.m) * heat, l3 = have ? (xq - q.m) * heat : 0.f;
    const float far = l0 + l1 + l3 - l2;
    if (fabsf(far) > 1e-5f * (1.f + fabsf(l0) + fabsf(l2) + fabsf(l3) + 32.f)) return far < 0.f;
    if (!(u > 0.f)) return u == 0.f;              // a NaN stands for nothing
    double ratio = (double)u * (double)p.z, lq = 0.0;
    if (have) {
        ratio /= (double)q.z;
        lq = ((double)xq - (double)q.m) * (double)heat;
    }
    return log(ratio) + lq < ((double)x - (double)p.m) * (double)heat;
}

struct Best {
    float score;
    int32_t at;                                   // -1: none
};
__device__ __forceinline__ bool better(float s, int32_t at, const Best &b) {
    return at >= 0 && (b.at < 0 || s > b.score || (s == b.score && at < b.at));
}

// p, or p - q, from logits: each an exponential times the reciprocal of its row's sum, so that equal logits of equal rows come out at
// most a few 2^-24 apart (sums of the same numbers in two orders).  A difference below 2^-20 of p is none: equal rows leave nothing,
// and not what rounding leaves.
struct Weigh {
    float pm, pz, qm, qz, c;
    int32_t out;                                  // the token that does not count, or -1
};
// The quotient's 2^-22 next to w's own error is nothing.  A weight of 0, and a NaN, win nothing.
template <bool REST> __device__ __forceinline__ void race(Best &b, const Weigh &w, float x, float q, float e, int32_t j) {
    float p = ex2((x - w.pm) * w.c) * w.pz;
    if (REST) {
        const float r = fmaf(-ex2((q - w.qm) * w.c), w.qz, p);
        p = r > p * 0x1p-20f ? r : 0.f;
    } else {
        p = j == w.out ? 0.f : p;
    }
    const float s = __fdividef(p, e);
    if (s > b.score) b = {s, j};
}

// the best of values j0 to j1 - 1, a thread's: each thread's values come in ascending order
template <typename T, bool REST>
__device__ __forceinline__ Best run_race(const T *x, const T *q, const float *e, int64_t j0, int64_t j1, const Weigh &w) {
    constexpr int E = 16 / (int)sizeof(T);
    Best b = {0.f, -1};
    if (((uintptr_t)(x + j0) | (uintptr_t)(e + j0) | (REST ? (uintptr_t)(q + j0) : 0)) % 16 == 0) {
        const int vecs = (int)((j1 - j0) / E);
        const uint4 *px = reinterpret_cast<const uint4 *>(x + j0), *pq = reinterpret_cast<const uint4 *>(REST ? q + j0 : x + j0);
        const uint4 *pe = reinterpret_cast<const uint4 *>(e + j0);
        constexpr int G = 2;                      // vectors whose loads are on their way together
        for (int v0 = threadIdx.x; v0 < vecs; v0 += G * THREADS) {
            uint4 ux[G], uq[G], ue[G][E / 4];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int v = v0 + g * THREADS < vecs ? v0 + g * THREADS : v0;  // the same again behind the end: it wins nothing more
                ux[g] = px[v];
                if (REST) uq[g] = pq[v];
#pragma unroll
                for (int i = 0; i < E / 4; ++i) ue[g][i] = __ldcs(pe + v * (E / 4) + i);
            }
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int v = v0 + g * THREADS < vecs ? v0 + g * THREADS : v0;
                float fx[E], fq[E] = {}, fe[E];
                unpack16<T>(ux[g], fx);
                if (REST) unpack16<T>(uq[g], fq);
#pragma unroll
                for (int i = 0; i < E / 4; ++i) unpack16<float>(ue[g][i], fe + 4 * i);
#pragma unroll
                for (int i = 0; i < E; ++i) race<REST>(b, w, fx[i], fq[i], fe[i], (int32_t)j0 + v * E + i);
            }
        }
        for (int64_t j = j0 + (int64_t)vecs * E + threadIdx.x; j < j1; j += THREADS)
            race<REST>(b, w, to_f32(x[j]), REST ? to_f32(q[j]) : 0.f, e[j], (int32_t)j);
        return b;
    }
    int64_t j = j0 + threadIdx.x;
    for (; j + 3 * THREADS < j1; j += 4 * THREADS) {
        float fx[4], fq[4] = {}, fe[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            fx[i] = to_f32(x[j + i * THREADS]);
            if (REST) fq[i] = to_f32(q[j + i * THREADS]);
            fe[i] = __ldcs(e + j + i * THREADS);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) race<REST>(b, w, fx[i], fq[i], fe[i], (int32_t)j + i * THREADS);
    }
    for (; j < j1; j += THREADS) race<REST>(b, w, to_f32(x[j]), REST ? to_f32(q[j]) : 0.f, e[j], (int32_t)j);
    return b;
}

enum { STANDS = 0, FALLS = 1, BAD = 2 };

template <typename T>
__global__ void __launch_bounds__(THREADS, 2) verify_draw_kernel(const VerifyArgs a, int pieces, const Piece *parts, int splits) {
    __shared__ int verdict[CT_MAX_DRAFTS + 1];
    __shared__ Row target[CT_MAX_DRAFTS + 1], draft[CT_MAX_DRAFTS + 1];
    __shared__ Best found[WARPS];
    __shared__ Best mine;                         // this CTA's, read by the others
    pdl_wait();
    pdl_trigger();
    const int rank = splits > 1 ? (int)tc::cluster_ctarank() : 0, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t b = blockIdx.x / (unsigned)splits;
    const Sequence s = sequence(a, b);
    const int64_t row0 = s.from + b, targets = a.count + a.sequences;
    const T *tx = static_cast<const T *>(a.x), *tq = static_cast<const T *>(a.q);
    const float c = s.heat * LOG2E;
    // the rows, a warp for each: the target's d + 1, the draft's d
    const int rows = s.d + 1 + (tq != nullptr && !s.greedy ? s.d : 0);
    for (int i = warp; i < rows; i += WARPS) {
        const bool t = i <= s.d;
        const Row r = row_of(parts + (t ? row0 + i : targets + s.from + i - s.d - 1) * pieces, pieces, c);
        if (lane == 0) (t ? target[i] : draft[i - s.d - 1]) = r;
    }
    __syncthreads();
    if ((int)threadIdx.x <= s.d) {
        const int j = threadIdx.x;
        const Row p = target[j];
        int v = BAD;
        if (!s.bad && !p.bad) {
            v = FALLS;
            if (j < s.d) {
                const int64_t id = a.drafts[s.from + j];
                const bool there = id >= 0 && id < a.vocab;
                const float x = there ? to_f32(tx[(row0 + j) * a.ldx + id]) : -INF;
                if (s.greedy) {
                    v = there && id == p.at ? STANDS : FALLS;
                } else if (tq != nullptr && draft[j].bad) {
                    v = BAD;
                } else if (x > -INF) {
                    const float xq = tq != nullptr ? to_f32(tq[(s.from + j) * a.ldq + id]) : 0.f;
                    v = stands(a.uniform[s.from + j], p, x, tq != nullptr, draft[j], xq, s.heat) ? STANDS : FALLS;
                }
            }
        }
        verdict[j] = v;
    }
    __syncthreads();
    int n = 0;
    while (n < s.d && verdict[n] == STANDS) ++n;
    const bool bad = verdict[n] == BAD, fell = n < s.d;
    int64_t token = -1;
    if (!bad && s.greedy) {
        token = target[n].at;
    } else if (!bad) {
        const T *x = tx + (row0 + n) * a.ldx, *q = fell && tq != nullptr ? tq + (s.from + n) * a.ldq : nullptr;
        const float *e = a.noise + b * a.ld_noise;
        const int64_t id = fell && q == nullptr ? a.drafts[s.from + n] : -1;
        const Row p = target[n];
        // the draft's part: its row, or all of its token
        bool rest = fell && tq != nullptr && draft[n].m > -INF;
        const Weigh w = {p.m, 1.f / p.z, rest ? draft[n].m : 0.f, rest ? 1.f / draft[n].z : 0.f, c, -1};
        Weigh w0 = w;
        if (id >= 0 && id < a.vocab) w0.out = (int32_t)id;
        const bool empty = p.m == -INF;
        // pieces that start on 16 bytes wherever the rows do
        const int64_t per = (a.vocab + 8 * splits - 1) / (8 * splits) * 8, j0 = min(per * rank, a.vocab), j1 = min(j0 + per, a.vocab);
        // once with the draft's part taken out; where that leaves nothing, without
        for (int round = 0; round < 2; ++round) {
            Best m = {0.f, -1};
            if (!empty) m = rest ? run_race<T, true>(x, q, e, j0, j1, w) : run_race<T, false>(x, q, e, j0, j1, round == 0 ? w0 : w);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                const float sc = __shfl_xor_sync(0xffffffffu, m.score, o);
                const int32_t at = __shfl_xor_sync(0xffffffffu, m.at, o);
                if (better(sc, at, m)) m = {sc, at};
            }
            if (lane == 0) found[warp] = m;
            __syncthreads();
            if (threadIdx.x == 0) {
                for (int i = 1; i < WARPS; ++i)
                    if (better(found[i].score, found[i].at, m)) m = found[i];
                mine = m;
            }
            __syncthreads();
            m = mine;
            if (splits > 1) {
                tc::cluster_sync();
                m = {0.f, -1};
                for (int r = 0; r < splits; ++r) {
                    const uint32_t at = tc::mapa_shared(tc::smem_u32(&mine), (uint32_t)r);
                    float sc;
                    int32_t i;
                    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(sc) : "r"(at) : "memory");
                    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(i) : "r"(at + 4) : "memory");
                    if (better(sc, i, m)) m = {sc, i};
                }
                tc::cluster_sync();               // all have read, before a CTA leaves or goes round again
            } else {
                __syncthreads();
            }
            token = m.at;
            if (token >= 0 || empty || (!rest && w0.out < 0)) break;            // the whole cluster alike
            rest = false;
        }
    }
    if (rank != 0) return;
    if (threadIdx.x == 0) a.accepted[b] = n;
    if ((int)threadIdx.x <= a.most) {
        const int j = threadIdx.x;
        const int64_t id = j < n ? a.drafts[s.from + j] : j == n ? token : -1;
        float lp = 0.f;
        if (j <= n) lp = j == n && bad ? nan_f() : id < 0 ? -INF : (to_f32(tx[(row0 + j) * a.ldx + id]) - target[j].m) * s.heat - logf(target[j].z);
        a.token[b * (a.most + 1) + j] = id;
        a.logprob[b * (a.most + 1) + j] = lp;
    }
}

// ---------------------------------------------------------------- host

inline int64_t rows_of(int64_t sequences, int64_t drafts) { return 2 * drafts + sequences; }
// Values of a piece: the warps of a few rows share them in pieces of 2048 (two batches of 16-bit values); where there are many rows, longer
// pieces leave less to join.  (152: a GB300's SMs; the workspace's size hangs on no device.)
inline int64_t per_of(int64_t rows, int64_t vocab) {
    int64_t per = 2048;
    while (per < 8192 && rows * ((vocab + per - 1) / per) > 32 * 152) per *= 2;
    return per;
}
inline int64_t pieces_of(int64_t rows, int64_t vocab) {
    const int64_t per = per_of(rows, vocab);
    return vocab > per ? (vocab + per - 1) / per : 1;
}

template <typename T> cudaError_t launch(const VerifyArgs &a, Piece *parts, cudaStream_t st) {
    const int64_t most = rows_of(a.sequences, a.count), rows = a.q != nullptr ? most : a.count + a.sequences;
    const int pieces = (int)pieces_of(most, a.vocab), per = (int)per_of(most, a.vocab);
    const int64_t all = rows * pieces;
    const cudaError_t e = pdl_launch(verify_rows_kernel<T>, dim3((unsigned)((all + ROW_WARPS - 1) / ROW_WARPS)), dim3(32 * ROW_WARPS), 0, st, a,
                                     pieces, per, all, parts);
    if (e != cudaSuccess) return e;
    // few sequences: clusters share a sequence's row, as many CTAs as are resident together (two for each SM)
    int splits = 1;
    while (splits < 8 && a.sequences * splits <= sm_count() && a.vocab >= 4096 * splits) splits *= 2;
    if (splits == 1) return pdl_launch(verify_draw_kernel<T>, dim3((unsigned)a.sequences), dim3(THREADS), 0, st, a, pieces, (const Piece *)parts, splits);
    return pdl_launch_cluster(verify_draw_kernel<T>, dim3((unsigned)(a.sequences * splits)), dim3(THREADS), 0, st, splits, a, pieces,
                              (const Piece *)parts, splits);
}
}  // namespace
}  // namespace ops
}  // namespace ct

extern "C" ct_status ct_verify_drafts_workspace(int64_t sequences, int64_t drafts, int64_t vocab, int64_t max_drafts, size_t *bytes) {
    using namespace ct::ops;
    if (bytes == nullptr) return CT_EINVAL;
    if (sequences < 0 || drafts < 0 || vocab < 0 || sequences > INT32_MAX / 8 || drafts > INT32_MAX / 2 || vocab > INT32_MAX ||
        max_drafts < 0 || max_drafts > CT_MAX_DRAFTS || rows_of(sequences, drafts) * pieces_of(rows_of(sequences, drafts), vocab) > INT32_MAX)
        return CT_ERANGE;
    *bytes = sizeof(Piece) * (size_t)(rows_of(sequences, drafts) * pieces_of(rows_of(sequences, drafts), vocab));
    return CT_OK;
}

extern "C" ct_status ct_verify_drafts(const void *logits_dev, int32_t dtype, int64_t ld, const void *draft_logits_dev,
                                      int64_t ld_draft, const int64_t *drafts_dev, const int64_t *offsets_dev,
                                      const float *uniform_dev, const float *noise_dev, int64_t ld_noise,
                                      const float *temperature_dev, int64_t sequences, int64_t drafts, int64_t vocab,
                                      int64_t max_drafts, int64_t *accepted_dev, int64_t *token_dev, float *logprob_dev,
                                      void *workspace_dev, size_t workspace_bytes, void *stream) {
    using namespace ct::ops;
    if (!dtype_ok(dtype)) return CT_EINVAL;
    size_t need;
    const ct_status s = ct_verify_drafts_workspace(sequences, drafts, vocab, max_drafts, &need);
    if (s != CT_OK) return s;
    if (sequences == 0) return CT_OK;
    const int es = dtype_size(dtype);
    if (offsets_dev == nullptr || accepted_dev == nullptr || token_dev == nullptr || logprob_dev == nullptr) return CT_EINVAL;
    if (drafts > 0 && (drafts_dev == nullptr || uniform_dev == nullptr)) return CT_EINVAL;
    if (vocab > 0 && (logits_dev == nullptr || noise_dev == nullptr || (ld < vocab && drafts + sequences > 1) ||
                      (ld_noise < vocab && sequences > 1) || (draft_logits_dev != nullptr && ld_draft < vocab && drafts > 1)))
        return CT_EINVAL;
    if (!ct::ops::aligned(logits_dev, es) || !ct::ops::aligned(draft_logits_dev, es) || !ct::ops::aligned(drafts_dev, 8) ||
        !ct::ops::aligned(offsets_dev, 8) || !ct::ops::aligned(uniform_dev, 4) || !ct::ops::aligned(noise_dev, 4) ||
        !ct::ops::aligned(temperature_dev, 4) || !ct::ops::aligned(accepted_dev, 8) || !ct::ops::aligned(token_dev, 8) ||
        !ct::ops::aligned(logprob_dev, 4))
        return CT_EINVAL;
    if (workspace_dev == nullptr || !ct::ops::aligned(workspace_dev, 16)) return CT_EINVAL;
    if (workspace_bytes < need) return CT_ENOMEM;
    const VerifyArgs a = {logits_dev, draft_logits_dev, ld, ld_draft, drafts_dev, offsets_dev, uniform_dev, noise_dev,
                          temperature_dev, ld_noise, sequences, drafts, vocab, (int)max_drafts, accepted_dev, token_dev, logprob_dev};
    Piece *parts = static_cast<Piece *>(workspace_dev);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == CT_DT_F32   ? launch<float>(a, parts, st)
                          : dtype == CT_DT_F16 ? launch<__half>(a, parts, st)
                                               : launch<__nv_bfloat16>(a, parts, st);
    return e == cudaSuccess ? CT_OK : CT_ECUDA;
}
