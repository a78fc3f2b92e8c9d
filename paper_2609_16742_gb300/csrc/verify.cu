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
// in FP32 relative to its own maximum and joined in FP64; the comparisons that decide
// are made in FP64.
#include "ops_common.cuh"

namespace ct {
namespace ops {
namespace {

constexpr float INF = __builtin_huge_valf();
__device__ __forceinline__ float nan_f() { return __uint_as_float(0x7FC00000u); }
constexpr float LOG2E = 1.4426950408889634f;

constexpr int THREADS = 512;
constexpr int64_t PIECE = 16384;                  // values of a row that a block looks at

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

// what a piece of a row holds: its largest logit (NaN for a NaN or +inf in it), the lowest index that has it, and sum e^((x - m) / T)
struct Piece {
    float m, z;
    int64_t at;
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

template <typename T> __device__ __forceinline__ Piece scan(const T *x, int64_t j0, int64_t j1, float heat) {
    Piece p = {-INF, 0.f, -1};
    bool bad = false;
    const float c = heat * LOG2E;
    for (int64_t j = j0 + threadIdx.x; j < j1; j += THREADS) {
        const float v = to_f32(x[j]);
        bad |= !(v < INF);
        if (v > p.m) {
            p.z = p.z * exp2f((p.m - v) * c) + 1.f;
            p.m = v;
            p.at = j;
        } else if (v > -INF) {
            p.z += exp2f((v - p.m) * c);
        }
    }
    if (bad) p.m = nan_f();
    return p;
}

__device__ __forceinline__ Piece join(const Piece &a, const Piece &b, float heat) {
    if (a.m != a.m) return a;
    if (b.m != b.m) return b;
    Piece r;
    r.m = fmaxf(a.m, b.m);
    const float c = heat * LOG2E;
    r.z = (a.m == -INF ? 0.f : a.z * exp2f((a.m - r.m) * c)) + (b.m == -INF ? 0.f : b.z * exp2f((b.m - r.m) * c));
    r.at = a.m > b.m || (a.m == b.m && (uint64_t)a.at < (uint64_t)b.at) ? a.at : b.at;
    return r;
}

// pieces of rows: a block's row is blockIdx.x / pieces; the target's rows of all sequences, then the drafts'
template <typename T>
__global__ void __launch_bounds__(THREADS) verify_rows_kernel(VerifyArgs a, int pieces, Piece *out) {
    pdl_wait();
    pdl_trigger();
    const int64_t row = blockIdx.x / (unsigned)pieces, targets = a.count + a.sequences;
    const int piece = (int)(blockIdx.x % (unsigned)pieces);
    const bool draft = row >= targets;
    const int64_t at = draft ? row - targets : row;
    // the sequence of the row: the last whose rows begin at or before it
    int64_t lo = 0, hi = a.sequences - 1;
    while (lo < hi) {
        const int64_t mid = (lo + hi + 1) / 2;
        if (a.offsets[mid] + (draft ? 0 : mid) <= at) lo = mid;
        else hi = mid - 1;
    }
    const Sequence s = sequence(a, lo);
    const T *x = draft ? static_cast<const T *>(a.q) + at * a.ldq : static_cast<const T *>(a.x) + at * a.ldx;
    const int64_t j0 = piece * PIECE, j1 = min(j0 + PIECE, a.vocab);
    Piece p = scan(x, j0, j1, s.heat);
    __shared__ Piece sp[THREADS];
    sp[threadIdx.x] = p;
    __syncthreads();
    for (int o = THREADS / 2; o > 0; o >>= 1) {
        if ((int)threadIdx.x < o) sp[threadIdx.x] = join(sp[threadIdx.x], sp[threadIdx.x + o], s.heat);
        __syncthreads();
    }
    if (threadIdx.x == 0) out[blockIdx.x] = sp[0];
}

// a whole row: lse relative to its maximum, in FP64 (log sum e^((x - m) / T))
struct Row {
    float m;
    double logz;
    int64_t at;
};

__device__ __forceinline__ Row row_of(const Piece *p, int pieces, float heat) {
    Row r = {-INF, 0.0, -1};
    double z = 0.0;
    for (int i = 0; i < pieces; ++i) {
        if (p[i].m != p[i].m) return {p[i].m, 0.0, -1};
        if (p[i].m > r.m) {
            r.m = p[i].m;
            r.at = p[i].at;
        }
    }
    if (r.m == -INF) return r;
    for (int i = 0; i < pieces; ++i)
        if (p[i].m > -INF) z += (double)p[i].z * exp((double)(p[i].m - r.m) * (double)heat);
    r.logz = log(z);
    return r;
}

// log probability of a logit, in FP64
__device__ __forceinline__ double logp_of(const Row &r, float x, float heat) {
    return x == -INF ? -(double)INF : ((double)x - (double)r.m) * (double)heat - r.logz;
}

enum { STANDS = 0, FALLS = 1, BAD = 2 };

template <typename T>
__global__ void __launch_bounds__(THREADS) verify_draw_kernel(VerifyArgs a, int pieces, const Piece *parts) {
    pdl_wait();
    pdl_trigger();
    const int64_t b = blockIdx.x;
    const Sequence s = sequence(a, b);
    const int64_t row0 = s.from + b, targets = a.count + a.sequences;
    const T *tx = static_cast<const T *>(a.x), *tq = static_cast<const T *>(a.q);
    __shared__ int verdict[CT_MAX_DRAFTS + 1];
    __shared__ double lps[CT_MAX_DRAFTS + 1];
    __shared__ Row target, draft;
    if ((int)threadIdx.x <= s.d) {
        const int j = threadIdx.x;
        const Row p = row_of(parts + (row0 + j) * pieces, pieces, s.heat);
        int v = BAD;
        double lp = 0.0;
        if (!s.bad && p.m == p.m) {
            v = FALLS;
            if (j < s.d) {
                const int64_t id = a.drafts[s.from + j];
                const bool there = id >= 0 && id < a.vocab;
                lp = there ? logp_of(p, to_f32(tx[(row0 + j) * a.ldx + id]), s.heat) : -(double)INF;
                if (s.greedy) {
                    v = there && id == p.at ? STANDS : FALLS;
                } else {
                    double lq = 0.0;
                    bool fine = true;
                    if (tq != nullptr) {
                        const Row q = row_of(parts + (targets + s.from + j) * pieces, pieces, s.heat);
                        fine = q.m == q.m;
                        lq = there && q.m > -INF ? logp_of(q, to_f32(tq[(s.from + j) * a.ldq + id]), s.heat) : -(double)INF;
                    }
                    v = !fine ? BAD : there && lp > -(double)INF && log((double)a.uniform[s.from + j]) + lq < lp ? STANDS : FALLS;
                }
            }
        }
        verdict[j] = v;
        lps[j] = lp;
    }
    __syncthreads();
    int n = 0;
    while (n < s.d && verdict[n] == STANDS) ++n;
    const bool bad = verdict[n] == BAD, fell = n < s.d;
    if (threadIdx.x == 0) {
        target = row_of(parts + (row0 + n) * pieces, pieces, s.heat);
        if (fell && tq != nullptr) draft = row_of(parts + (targets + s.from + n) * pieces, pieces, s.heat);
    }
    __syncthreads();
    int64_t token = -1;
    if (!bad && s.greedy) {
        token = target.at;
    } else if (!bad) {
        const T *x = tx + (row0 + n) * a.ldx, *q = fell && tq != nullptr ? tq + (s.from + n) * a.ldq : nullptr;
        const float *e = a.noise + b * a.ld_noise;
        const int64_t id = fell ? a.drafts[s.from + n] : -1;
        // the best of w / E with the draft's part taken out, and without
        float best[2] = {0.f, 0.f};
        int64_t at[2] = {-1, -1};
        const float c = s.heat * LOG2E, pz = (float)(-target.logz * 1.4426950408889634), qz = (float)(-draft.logz * 1.4426950408889634);
        for (int64_t j = threadIdx.x; j < a.vocab; j += THREADS) {
            const float v = to_f32(x[j]);
            if (!(v > -INF)) continue;
            const float p = exp2f(fmaf(v - target.m, c, pz)), w = to_f32(q != nullptr ? q[j] : T());
            const float r = !fell             ? p
                            : q != nullptr    ? p - (w > -INF ? exp2f(fmaf(w - draft.m, c, qz)) : 0.f)
                            : j == id         ? 0.f
                                              : p;
            const float s0 = r / e[j], s1 = p / e[j];
            if (r > 0.f && s0 > best[0]) { best[0] = s0; at[0] = j; }
            if (p > 0.f && s1 > best[1]) { best[1] = s1; at[1] = j; }
        }
        __shared__ float sb[2][THREADS];
        __shared__ int64_t sa[2][THREADS];
        for (int k = 0; k < 2; ++k) {
            sb[k][threadIdx.x] = best[k];
            sa[k][threadIdx.x] = at[k];
        }
        __syncthreads();
        for (int o = THREADS / 2; o > 0; o >>= 1) {
            if ((int)threadIdx.x < o)
                for (int k = 0; k < 2; ++k) {
                    const float v = sb[k][threadIdx.x + o];
                    const int64_t i = sa[k][threadIdx.x + o];
                    if (v > sb[k][threadIdx.x] || (v == sb[k][threadIdx.x] && (uint64_t)i < (uint64_t)sa[k][threadIdx.x])) {
                        sb[k][threadIdx.x] = v;
                        sa[k][threadIdx.x] = i;
                    }
                }
            __syncthreads();
        }
        token = sa[0][0] >= 0 ? sa[0][0] : sa[1][0];
    }
    if (threadIdx.x == 0) a.accepted[b] = n;
    if ((int)threadIdx.x <= a.most) {
        const int j = threadIdx.x;
        int64_t id = -1;
        float lp = 0.f;
        if (j < n) {
            id = a.drafts[s.from + j];
            lp = (float)lps[j];
        } else if (j == n) {
            id = token;
            lp = bad ? nan_f() : token < 0 ? -INF : (float)logp_of(target, to_f32(tx[(row0 + n) * a.ldx + token]), s.heat);
        }
        a.token[b * (a.most + 1) + j] = id;
        a.logprob[b * (a.most + 1) + j] = lp;
    }
}

inline int64_t rows_of(int64_t sequences, int64_t drafts) { return 2 * drafts + sequences; }
inline int64_t pieces_of(int64_t vocab) { return vocab > PIECE ? (vocab + PIECE - 1) / PIECE : 1; }

template <typename T> cudaError_t launch(const VerifyArgs &a, Piece *parts, cudaStream_t st) {
    const int pieces = (int)pieces_of(a.vocab);
    const int64_t rows = a.count + a.sequences + (a.q != nullptr ? a.count : 0);
    const cudaError_t e = pdl_launch(verify_rows_kernel<T>, dim3((unsigned)(rows * pieces)), dim3(THREADS), 0, st, a, pieces, parts);
    if (e != cudaSuccess) return e;
    return pdl_launch(verify_draw_kernel<T>, dim3((unsigned)a.sequences), dim3(THREADS), 0, st, a, pieces, (const Piece *)parts);
}
}  // namespace
}  // namespace ops
}  // namespace ct

extern "C" ct_status ct_verify_drafts_workspace(int64_t sequences, int64_t drafts, int64_t vocab, int64_t max_drafts, size_t *bytes) {
    using namespace ct::ops;
    if (bytes == nullptr) return CT_EINVAL;
    if (sequences < 0 || drafts < 0 || vocab < 0 || sequences > INT32_MAX || drafts > INT32_MAX / 2 || vocab > INT32_MAX ||
        max_drafts < 0 || max_drafts > CT_MAX_DRAFTS || rows_of(sequences, drafts) * pieces_of(vocab) > INT32_MAX)
        return CT_ERANGE;
    *bytes = sizeof(Piece) * (size_t)(rows_of(sequences, drafts) * pieces_of(vocab));
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
