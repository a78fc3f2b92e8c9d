// Low-rank adapters of many requests beside a shared projection, and their
// gradients.
//
//   v[t] = scale[i] A[i] x[t],  y[t] = act(y[t] + B[i] v[t]),  i = ids[t]
//   u[t] = scale[i] B[i]^T dy[t],  dx[t] += A[i]^T u[t],
//   dA[i] = sum_t u[t] x[t]^T,  dB[i] = sum_t dy[t] v[t]^T
//
// v and u carry at least 16 bits: they are short, and rounding them to a result's 8 or 11 would cost it as much
// as its own rounding does.
//
// Many rows are put in the order of their adapters first (one CTA: a counting sort, two where there are more than 254
// adapters), then go through the tensor cores in tiles of 128 rows of one adapter (adapters_shrink.cu,
// adapters_expand.cu, adapters_outer.cu).  Few rows, of about as many adapters, take the two kernels here instead,
// which are bound by the adapters' bytes and the launches: the first row of each adapter speaks for all of its rows.
//
// Measured alone: the order of 8192 rows 8.8 us; 64 rows of 25088 FP16 values with an adapter of rank 16 for each 13.9 us for the first
// product (3.9 TB/s of the adapters), 7.8 us for 4096 columns of the second; 1 row, 4096 to 4096, 5.9 us for both.
#include "adapters.cuh"

namespace ct {
namespace ops {
namespace {

// ---------------------------------------------------------------- the rows' order

constexpr int ORDER_THREADS = 1024, ORDER_WARPS = 32, BINS = 256;

struct OrderArgs {
    const int64_t *ids;
    int64_t t;
    int adapters;
    int32_t *order, *spare;                       // [t]
    int32_t *first, *end;                         // [adapters + 2]
    AdTile *tiles;
    int32_t *n_tiles;
};

__device__ __forceinline__ int key_of(const OrderArgs &a, int64_t i) {
    return i == -1 ? 0 : i >= 0 && i < a.adapters ? (int)i + 1 : a.adapters + 1;
}

// exclusive sum over the block's threads; total: of all
__device__ __forceinline__ int block_sum(int v, int *warps, int &total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int w = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += w;
    }
    __syncthreads();
    if (lane == 31) warps[warp] = s;
    __syncthreads();
    if (warp == 0) {
        int w = warps[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += x;
        }
        warps[lane] = w;
    }
    __syncthreads();
    total = warps[31];
    return s - v + (warp > 0 ? warps[warp - 1] : 0);
}

// f(key, row, have) for a run of rows, 32 at a time in their order; the ids of eight such groups are on their way together
template <typename F> __device__ __forceinline__ void each_row(const OrderArgs &a, const int32_t *from, int64_t r0, int64_t r1, F f) {
    const int lane = threadIdx.x & 31;
    for (int64_t p = r0; p < r1; p += 256) {
        int32_t row[8];
        int64_t id[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t at = min(p + 32 * i + lane, r1 - 1);
            row[i] = from != nullptr ? from[at] : (int32_t)at;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) id[i] = a.ids[row[i]];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (p + 32 * i >= r1) break;
            f(key_of(a, id[i]), row[i], p + 32 * i + lane < r1);
        }
    }
}

__global__ void __launch_bounds__(ORDER_THREADS) order_kernel(const OrderArgs a) {
    __shared__ int count[ORDER_WARPS][BINS];
    __shared__ int sums[32];
    pdl_wait();
    pdl_trigger();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, keys = a.adapters + 2;
    // each warp has a run of the rows; a digit's rows keep their order within and between the runs
    const int64_t run = (a.t + 32 * ORDER_WARPS - 1) / (32 * ORDER_WARPS) * 32;
    const int64_t r0 = min(warp * run, a.t), r1 = min(r0 + run, a.t);
    const int passes = keys <= BINS ? 1 : 2;
    if (passes == 2)
        for (int k = tid; k < keys; k += ORDER_THREADS) a.first[k] = a.end[k] = 0;
    for (int pass = 0; pass < passes; ++pass) {
        const int32_t *from = pass == 0 ? nullptr : a.spare;
        int32_t *to = pass + 1 == passes ? a.order : a.spare;
        for (int b = lane; b < BINS; b += 32) count[warp][b] = 0;
        __syncwarp();
        each_row(a, from, r0, r1, [&](int key, int32_t, bool have) {
            const int d = have ? key >> (8 * pass) & (BINS - 1) : BINS;
            const uint32_t same = __match_any_sync(0xffffffffu, d);
            if (have && lane == __ffs(same) - 1) count[warp][d] += __popc(same);
            __syncwarp();
        });
        __syncthreads();
        // where each warp's rows of each digit go: thread i has digit i / 4, warps 8 (i % 4) to + 7
        int mine[8], s = 0, total;
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            mine[w] = count[tid % 4 * 8 + w][tid / 4];
            s += mine[w];
        }
        s = block_sum(s, sums, total);
        if (passes == 1) {
            // one digit is the whole key: its run of the slots
            if (tid % 4 == 0 && tid / 4 < keys) a.first[tid / 4] = s;
            if (tid % 4 == 0 && tid > 0 && tid / 4 <= keys) a.end[tid / 4 - 1] = s;
            if (keys == BINS && tid == 0) a.end[keys - 1] = total;
        }
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            count[tid % 4 * 8 + w][tid / 4] = s;
            s += mine[w];
        }
        __syncthreads();
        each_row(a, from, r0, r1, [&](int key, int32_t row, bool have) {
            const int d = have ? key >> (8 * pass) & (BINS - 1) : BINS;
            const uint32_t same = __match_any_sync(0xffffffffu, d);
            if (have) to[count[warp][d] + __popc(same & ((1u << lane) - 1u))] = row;
            __syncwarp();
            if (have && lane == __ffs(same) - 1) count[warp][d] += __popc(same);
            __syncwarp();
        });
        __syncthreads();
    }
    if (passes == 2) {
        for (int64_t p = tid; p < a.t; p += ORDER_THREADS) {
            const int k = key_of(a, a.ids[a.order[p]]);
            if (p == 0 || key_of(a, a.ids[a.order[p - 1]]) != k) a.first[k] = (int32_t)p;
            if (p + 1 == a.t || key_of(a, a.ids[a.order[p + 1]]) != k) a.end[k] = (int32_t)p + 1;
        }
        __syncthreads();
    }
    // tiles: each thread has a run of the keys
    const int per = (keys + ORDER_THREADS - 1) / ORDER_THREADS, k0 = min(tid * per, keys), k1 = min(k0 + per, keys);
    int n = 0, total;
    for (int k = k0; k < k1; ++k) n += (a.end[k] - a.first[k] + AD_ROWS - 1) / AD_ROWS;
    int at = block_sum(n, sums, total);
    for (int k = k0; k < k1; ++k)
        for (int s = a.first[k]; s < a.end[k]; s += AD_ROWS) a.tiles[at++] = {s, k};
    if (tid == 0) *a.n_tiles = total;
}

// ---------------------------------------------------------------- few rows

constexpr int FEW = 128;                          // most rows of this kind
constexpr int FEW_THREADS = 256, FEW_WARPS = 8;
constexpr int FEW_J = 4, FEW_R = 4;               // a warp's rows of A, of x

struct FewArgs {
    const void *x;
    int64_t ldx;
    const void *a;
    int64_t a_adapter, a_row;
    const void *b;
    int64_t b_adapter, b_row;
    const int64_t *ids;
    const float *scale;
    int t, adapters, rank;
    int64_t k, n;
    float *v;                                     // [t][rank]
    void *y;
    int32_t y_dtype;
    int64_t ldy;
    int relu;
};

// The rows that row `lead` speaks for: all with its id, if it is the first of them.  Returns their number, 0 if it is not.  At least FEW
// threads.
__device__ __forceinline__ int speak_for(const int64_t *ids, int t, int lead, int16_t *rows, int64_t &id) {
    __shared__ uint32_t masks[FEW / 32];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (ids == nullptr) {
        id = 0;
        if (tid < t) rows[tid] = (int16_t)tid;
        __syncthreads();
        return lead == 0 ? t : 0;
    }
    const int64_t mine = tid < t ? ids[tid] : 0;
    id = ids[lead];
    const bool same = tid < t && mine == id;
    const uint32_t all = __ballot_sync(0xffffffffu, same);
    if (lane == 0 && warp < FEW / 32) masks[warp] = all;
    __syncthreads();
    int n = 0, before = 0;
    bool first = true;
#pragma unroll
    for (int w = 0; w < FEW / 32; ++w) {
        if (w < warp) before += __popc(masks[w]);
        n += __popc(masks[w]);
        const uint32_t early = lead >= 32 * (w + 1) ? 0xffffffffu : lead <= 32 * w ? 0u : (1u << (lead - 32 * w)) - 1u;
        first = first && (masks[w] & early) == 0;
    }
    if (same) rows[before + __popc(all & ((1u << lane) - 1u))] = (int16_t)tid;
    __syncthreads();
    return first ? n : 0;
}

// Eight values on their way; WHOLE: rows start on 16 bytes and are a multiple of 8 values long.
template <typename T, bool WHOLE> struct Way {
    Eight<T> e;
    __device__ __forceinline__ void go(const T *p, int left) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) e.u[i] = ldg_if(reinterpret_cast<const uint4 *>(p) + i, left > 0);
    }
    __device__ __forceinline__ void take(const T *, int, float (&v)[8]) const {
        unpack16<T>(e.u[0], v);
        if constexpr (sizeof(T) == 4) unpack16<T>(e.u[1], v + 4);
    }
};
template <typename T> struct Way<T, false> {
    Units<T> u;
    __device__ __forceinline__ void go(const T *p, int left) { u = load_units(p, left); }
    __device__ __forceinline__ void take(const T *p, int left, float (&v)[8]) const {
        const Eight<T> e = take_eight(u, p, left);
        unpack16<T>(e.u[0], v);
        if constexpr (sizeof(T) == 4) unpack16<T>(e.u[1], v + 4);
    }
};

// Sums of FEW_J rows of A (from j0 on) by R rows of x over every ways-th piece of 256 values, a warp's; into part.
template <typename TX, typename TM, bool WHOLE, int R>
__device__ __forceinline__ void few_dot(const FewArgs &a, const TM *m, const int16_t *rows, int have, int j0, int64_t p0, int64_t p1, int ways,
                                        float (&part)[FEW_J][FEW_R]) {
    constexpr int U = R == 1 ? 4 : 1;             // pieces whose loads are on their way together
    const int lane = threadIdx.x & 31;
    const TX *xr[R];
#pragma unroll
    for (int r = 0; r < R; ++r) xr[r] = static_cast<const TX *>(a.x) + (r < have ? rows[r] * a.ldx : 0);
    float acc[FEW_J][R];
#pragma unroll
    for (int j = 0; j < FEW_J; ++j)
#pragma unroll
        for (int r = 0; r < R; ++r) acc[j][r] = 0.f;
    for (int64_t p = p0; p < p1; p += (int64_t)U * ways) {
        Way<TM, WHOLE> wm[U][FEW_J];
        Way<TX, WHOLE> wx[U][R];
        int left[U];
        int64_t c[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            c[u] = (p + (int64_t)u * ways) * 256 + lane * 8;
            left[u] = p + (int64_t)u * ways < p1 ? left_of(c[u], a.k) : 0;
            if (left[u] == 0) c[u] = 0;
#pragma unroll
            for (int j = 0; j < FEW_J; ++j) wm[u][j].go(m + (j0 + j < a.rank ? (j0 + j) * a.a_row + c[u] : 0), j0 + j < a.rank ? left[u] : 0);
#pragma unroll
            for (int r = 0; r < R; ++r) wx[u][r].go(xr[r] + c[u], r < have ? left[u] : 0);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float fx[R][8];
#pragma unroll
            for (int r = 0; r < R; ++r) wx[u][r].take(xr[r] + c[u], r < have ? left[u] : 0, fx[r]);
#pragma unroll
            for (int j = 0; j < FEW_J; ++j) {
                float fm[8];
                wm[u][j].take(m + (j0 + j < a.rank ? (j0 + j) * a.a_row + c[u] : 0), j0 + j < a.rank ? left[u] : 0, fm);
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[j][r] = fmaf(fm[e], fx[r][e], acc[j][r]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < FEW_J; ++j)
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int s = 16; s > 0; s >>= 1) acc[j][r] += __shfl_xor_sync(0xffffffffu, acc[j][r], s);
            if (lane == 0) part[j][r] = acc[j][r];
        }
}

// v = scale A x.  A cluster for each row that may speak, its CTAs share the long axis; warps share the rows of A, and the axis again
// where those are few.
template <typename TX, typename TM, bool WHOLE> __global__ void __launch_bounds__(FEW_THREADS) few_shrink_kernel(const FewArgs a, int splits) {
    __shared__ int16_t rows[FEW];
    __shared__ float part[FEW_WARPS][FEW_J][FEW_R];
    __shared__ float sums[CT_MAX_RANK][FEW_R];
    pdl_wait();
    pdl_trigger();
    const int rank = splits > 1 ? (int)tc::cluster_ctarank() : 0, tid = threadIdx.x, warp = tid >> 5;
    int64_t id;
    const int n = speak_for(a.ids, a.t, (int)(blockIdx.x / (unsigned)splits), rows, id);
    if (n == 0 || id < 0 || id >= a.adapters) return;                            // the whole cluster alike
    const TM *m = static_cast<const TM *>(a.a) + id * a.a_adapter;
    const float scale = a.scale != nullptr ? a.scale[id] : 1.f;
    // pieces of 256 values (a warp's 32 x 8)
    const int64_t pieces = (a.k + 255) / 256, p0 = pieces * rank / splits, p1 = pieces * (rank + 1) / splits;
    const int groups = (a.rank + FEW_J - 1) / FEW_J, ways = groups >= FEW_WARPS ? 1 : FEW_WARPS / groups;
    for (int r0 = 0; r0 < n; r0 += FEW_R) {
        for (int g0 = 0; g0 < groups; g0 += FEW_WARPS / ways) {
            const int g = g0 + warp / ways, way = warp % ways;
            if (g < groups) {
                if (n - r0 == 1) few_dot<TX, TM, WHOLE, 1>(a, m, rows + r0, 1, g * FEW_J, p0 + way, p1, ways, part[warp]);
                else few_dot<TX, TM, WHOLE, FEW_R>(a, m, rows + r0, n - r0, g * FEW_J, p0 + way, p1, ways, part[warp]);
            }
            __syncthreads();
            // the warps that shared the axis, in their order
            for (int i = tid; i < FEW_WARPS / ways * FEW_J * FEW_R; i += FEW_THREADS) {
                const int w = i / (FEW_J * FEW_R), j = i / FEW_R % FEW_J, r = i % FEW_R, at = (g0 + w) * FEW_J + j;
                if (at >= a.rank || r0 + r >= n) continue;
                float s = 0.f;
                for (int q = 0; q < ways; ++q) s += part[w * ways + q][j][r];
                sums[at][r] = s;
            }
            __syncthreads();
        }
        if (splits > 1) tc::cluster_sync();
        // the CTAs of the cluster share the sums
        for (int i = tid + FEW_THREADS * rank; i < a.rank * FEW_R; i += FEW_THREADS * splits) {
            const int j = i / FEW_R, r = i % FEW_R;
            if (r0 + r >= n) continue;
            float s = sums[j][r];
            if (splits > 1) {
                float p[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) p[q] = q < splits ? ld_peer_f32(tc::smem_u32(&sums[j][r]), q) : 0.f;
                s = p[0];
#pragma unroll
                for (int q = 1; q < 8; ++q) s += p[q];
            }
            a.v[rows[r0 + r] * a.rank + j] = s * scale;
        }
        if (splits > 1) tc::cluster_sync();       // the sums have been read
        else __syncthreads();
    }
}

__device__ __forceinline__ float few_get(const void *p, int dtype, int64_t i) {
    return dtype == CT_DT_F32   ? static_cast<const float *>(p)[i]
           : dtype == CT_DT_F16 ? to_f32(static_cast<const __half *>(p)[i])
                                : to_f32(static_cast<const __nv_bfloat16 *>(p)[i]);
}

// y = act(y + B v): a thread for each column.  The ids and the matrix do not hang on the kernel before, which has itself waited for
// all before it: they are on their way before its end is waited for.
constexpr int FEW_COLS = 128;
template <typename TM> __global__ void __launch_bounds__(FEW_COLS) few_expand_kernel(const FewArgs a) {
    __shared__ int16_t rows[FEW];
    __shared__ float vs[8][CT_MAX_RANK];
    if (a.rank == 0) pdl_wait();                  // no kernel of this call before it
    int64_t id;
    const int n = speak_for(a.ids, a.t, (int)blockIdx.y, rows, id);
    const int64_t c = (int64_t)blockIdx.x * FEW_COLS + threadIdx.x;
    const bool mine = c < a.n, out = id < -1 || id >= a.adapters, product = id >= 0 && !out;
    if (n == 0 || (id == -1 && !a.relu)) {
        pdl_wait();
        return;
    }
    const TM *m = static_cast<const TM *>(a.b) + (product && mine ? id * a.b_adapter + c * a.b_row : 0);
    constexpr int AHEAD = 4;                      // 32 values of a row of B
    Units<TM> um[AHEAD];
    auto fetch = [&](int j0) {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int left = product && mine ? left_of(j0 + j * 8, a.rank) : 0;
            um[j] = load_units(m + (left > 0 ? j0 + j * 8 : 0), left);
        }
    };
    fetch(0);
    pdl_wait();
    for (int r0 = 0; r0 < n; r0 += 8) {
        const int nr = min(8, n - r0);
        float acc[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) acc[r] = mine && r < nr ? few_get(a.y, a.y_dtype, rows[r0 + r] * a.ldy + c) : 0.f;
        float add[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) add[r] = 0.f;
        if (product) {
            for (int i = threadIdx.x; i < nr * a.rank; i += FEW_COLS) vs[i / a.rank][i % a.rank] = a.v[rows[r0 + i / a.rank] * a.rank + i % a.rank];
            __syncthreads();
            if (mine)
                for (int j0 = 0; j0 < a.rank; j0 += 8 * AHEAD) {
                    if (j0 > 0 || (r0 > 0 && a.rank > 8 * AHEAD)) fetch(j0);
#pragma unroll
                    for (int j = 0; j < AHEAD; ++j) {
                        const int at = j0 + j * 8;
                        if (at >= a.rank) break;
                        const Eight<TM> e = take_eight(um[j], m + at, left_of(at, a.rank));
                        float f[8];
                        unpack16<TM>(e.u[0], f);
                        if constexpr (sizeof(TM) == 4) unpack16<TM>(e.u[1], f + 4);
#pragma unroll
                        for (int r = 0; r < 8; ++r) {
                            if (r >= nr) break;
#pragma unroll
                            for (int q = 0; q < 8; ++q)
                                if (at + q < a.rank) add[r] = fmaf(f[q], vs[r][at + q], add[r]);
                        }
                    }
                }
            __syncthreads();
        }
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            if (!mine || r >= nr) break;
            float v = acc[r] + add[r];
            if (a.relu) v = v < 0.f ? 0.f : v;
            put_as(a.y, a.y_dtype, rows[r0 + r] * a.ldy + c, out ? __uint_as_float(0x7FC00000u) : v);
        }
    }
}

template <typename TX, typename TM, bool WHOLE> cudaError_t few_as(const FewArgs &a, cudaStream_t st) {
    if (a.rank > 0) {
        // as many blocks as are resident together (two for each SM), with a piece of the axis at least for each warp that shares it
        const int64_t pieces = (a.k + 255) / 256;
        const int lead = a.ids != nullptr ? a.t : 1, speak = lead < a.adapters ? lead : a.adapters;
        const int groups = (a.rank + FEW_J - 1) / FEW_J, ways = groups >= FEW_WARPS ? 1 : FEW_WARPS / groups;
        int splits = 2 * sm_count() / speak;
        if (splits > 8) splits = 8;
        if (splits > pieces / ways) splits = (int)(pieces / ways);
        if (splits < 1) splits = 1;
        const cudaError_t e = splits > 1 ? pdl_launch_cluster(few_shrink_kernel<TX, TM, WHOLE>, dim3((unsigned)(lead * splits)),
                                                              dim3(FEW_THREADS), 0, st, splits, a, splits)
                                         : pdl_launch(few_shrink_kernel<TX, TM, WHOLE>, dim3((unsigned)lead), dim3(FEW_THREADS), 0, st, a, splits);
        if (e != cudaSuccess) return e;
    }
    // the columns along x: y ends at 65535 blocks
    const dim3 grid((unsigned)((a.n + FEW_COLS - 1) / FEW_COLS), (unsigned)(a.ids != nullptr ? a.t : 1));
    return pdl_launch(few_expand_kernel<TM>, grid, dim3(FEW_COLS), 0, st, a);
}
template <typename TX, typename TM> cudaError_t few(const FewArgs &a, bool whole, cudaStream_t st) {
    return whole ? few_as<TX, TM, true>(a, st) : few_as<TX, TM, false>(a, st);
}

// ---------------------------------------------------------------- host

inline bool adapter_matrix_ok(const void *p, int64_t sa, int64_t sr, int64_t adapters, int64_t rows, int64_t cols, int es) {
    if (adapters == 0 || rows == 0 || cols == 0) return true;
    return p != nullptr && aligned(p, es) && sa >= 0 && sr >= 0 && (rows == 1 || sr >= cols || sr == 0);
}
inline bool matrix_ok(const void *p, int64_t ld, int64_t rows, int64_t cols, int es) {
    if (rows == 0 || cols == 0) return true;
    return p != nullptr && aligned(p, es) && (rows == 1 || ld >= cols);
}
// slots are counted in 32 bits, up to a few tiles and steps past the last
constexpr int64_t ROWS_MOST = ((int64_t)1 << 31) - (1 << 16);
inline bool sizes_ok(int64_t t, int64_t adapters, int64_t rank, int64_t k, int64_t n) {
    return t >= 0 && t <= ROWS_MOST && adapters >= 0 && adapters <= CT_MAX_ADAPTERS && rank >= 0 && rank <= CT_MAX_RANK && k >= 0 &&
           k <= INT32_MAX && n >= 0 && n <= INT32_MAX;
}
inline int64_t tiles_of(int64_t t, int64_t adapters, bool ordered) {
    const int64_t most = (t + AD_ROWS - 1) / AD_ROWS;
    if (!ordered) return most;
    const int64_t partly = t < adapters + 2 ? t : adapters + 2;
    return most + partly;
}

// The workspace: vectors (BF16 parts by slots; few rows: FP32), the order.
struct Space {
    size_t v, u, order, spare, first, end, tiles, n_tiles, total;
};
inline size_t up(size_t n) { return (n + 255) / 256 * 256; }
Space space_of(int64_t t, int64_t adapters, int64_t rank, bool grad) {
    Space s;
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t here = at;
        at += up(bytes);
        return here;
    };
    const size_t vec = (size_t)t * (size_t)ad_padded(rank) * 2 * 3;
    s.v = take(vec);
    s.u = take(grad ? vec : 0);
    s.order = take((size_t)t * 4);
    s.spare = take((size_t)t * 4);
    s.first = take((size_t)(adapters + 2) * 4);
    s.end = take((size_t)(adapters + 2) * 4);
    s.tiles = take((size_t)tiles_of(t, adapters, true) * sizeof(AdTile));
    s.n_tiles = take(4);
    s.total = at;
    return s;
}

cudaError_t make_order(AdOrder &o, const int64_t *ids, int64_t t, int64_t adapters, const Space &s, char *w, cudaStream_t st) {
    o = {nullptr, nullptr, nullptr, nullptr, nullptr, t, (int)adapters};
    if (ids == nullptr) return cudaSuccess;
    OrderArgs a = {ids, t, (int)adapters, reinterpret_cast<int32_t *>(w + s.order), reinterpret_cast<int32_t *>(w + s.spare),
                   reinterpret_cast<int32_t *>(w + s.first), reinterpret_cast<int32_t *>(w + s.end), reinterpret_cast<AdTile *>(w + s.tiles),
                   reinterpret_cast<int32_t *>(w + s.n_tiles)};
    o.order = a.order;
    o.first = a.first;
    o.end = a.end;
    o.tiles = a.tiles;
    o.n_tiles = a.n_tiles;
    return pdl_launch(order_kernel, dim3(1), dim3(ORDER_THREADS), 0, st, a);
}

// whether rows start on 16 bytes and are a multiple of 8 values long (a stride that is not walked does not matter)
inline bool whole(const void *p, int64_t ld, int64_t rows, int64_t cols, int es) {
    return aligned(p, 16) && cols % 8 == 0 && (rows <= 1 || ld * es % 16 == 0);
}
inline bool stack_whole(const void *p, int64_t sa, int64_t sr, int64_t adapters, int64_t rows, int64_t cols, int es) {
    return whole(p, sr, rows, cols, es) && (adapters <= 1 || sa * es % 16 == 0);
}

// whether a matrix lies on one of a stack's
bool on_stack(const Span &m, const void *p, int64_t sa, int64_t sr, int64_t adapters, int64_t rows, int64_t cols, int es) {
    if (adapters == 0 || rows == 0 || cols == 0) return false;
    Span one = span(p, rows, cols, sr, es);
    const Span all = {one.at, 1, (int64_t)(one.end() - one.at) + (adapters - 1) * sa * es, 0};
    if (!share(m, all)) return false;
    for (int64_t i = 0; i < adapters; ++i, one.at += (uintptr_t)(sa * es))
        if (share(m, one)) return true;
    return false;
}
}  // namespace
}  // namespace ops
}  // namespace ct

extern "C" ct_status ct_adapters_workspace(int64_t t, int64_t adapters, int64_t rank, int64_t k, int64_t n, size_t *bytes) {
    using namespace ct::ops;
    if (bytes == nullptr) return CT_EINVAL;
    if (!sizes_ok(t, adapters, rank, k, n)) return CT_ERANGE;
    *bytes = space_of(t, adapters, rank, false).total;
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
    const int es = dtype_size(dtype), xs = dtype_size(x_dtype), ys = dtype_size(y_dtype);
    if (!matrix_ok(y_dev, ldy, t, n, ys) || !matrix_ok(x_dev, ldx, t, k, xs) ||
        !adapter_matrix_ok(a_dev, a_adapter, a_row, adapters, rank, k, es) ||
        !adapter_matrix_ok(b_dev, b_adapter, b_row, adapters, n, rank, es) || !aligned(ids_dev, 8) || !aligned(scale_dev, 4))
        return CT_EINVAL;
    if (ids_dev == nullptr && adapters == 0) return CT_EINVAL;
    const Space s = space_of(t, adapters, rank, false);
    if (workspace_dev == nullptr || !aligned(workspace_dev, 16)) return CT_EINVAL;
    if (workspace_bytes < s.total) return CT_ENOMEM;
    // y is written while b and the ids are read; x and a have been read by then
    const Span y = span(y_dev, t, n, ldy, ys);
    if (on_stack(y, b_dev, b_adapter, b_row, adapters, n, rank, es) || (ids_dev != nullptr && share(y, span(ids_dev, 1, t, t, 8)))) return CT_EINVAL;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    char *w = static_cast<char *>(workspace_dev);
    const bool xw = whole(x_dev, ldx, t, k, xs), aw = stack_whole(a_dev, a_adapter, a_row, adapters, rank, k, es),
               bw = stack_whole(b_dev, b_adapter, b_row, adapters, n, rank, es), yw = whole(y_dev, ldy, t, n, ys);
    cudaError_t e;
    // few rows, and adapters enough that hardly 16 rows have the same one
    if (t <= FEW && t <= 16 * adapters) {
        const FewArgs f = {x_dev, ldx, a_dev, a_adapter, a_row, b_dev, b_adapter, b_row, ids_dev, scale_dev, (int)t, (int)adapters, (int)rank, k,
                           n, reinterpret_cast<float *>(w + s.v), y_dev, y_dtype, ldy, relu != 0};
        if (dtype == CT_DT_F32) e = few<float, float>(f, xw && aw, st);
        else if (dtype == CT_DT_F16) e = x_dtype == CT_DT_F32 ? few<float, __half>(f, xw && aw, st) : few<__half, __half>(f, xw && aw, st);
        else e = x_dtype == CT_DT_F32 ? few<float, __nv_bfloat16>(f, xw && aw, st) : few<__nv_bfloat16, __nv_bfloat16>(f, xw && aw, st);
        return e == cudaSuccess ? CT_OK : CT_ECUDA;
    }
    AdOrder o;
    e = make_order(o, ids_dev, t, adapters, s, w, st);
    const int tiles = (int)tiles_of(t, adapters, ids_dev != nullptr), parts = y_dtype == CT_DT_F32 ? 3 : 2;
    if (e == cudaSuccess && rank > 0 && adapters > 0) {
        const AdShrink x = {x_dev, ldx, k, a_dev, a_adapter, a_row, scale_dev, (int)rank, (int)xw | (int)aw << 1, w + s.v, parts, true};
        e = ad_shrink({x, x}, AD_FORWARD, x_dtype, dtype, o, tiles, st);
    }
    if (e == cudaSuccess)
        e = ad_expand({y_dev, y_dtype, ldy, n, b_dev, b_adapter, b_row, (int)rank, (int)yw | (int)bw << 1, relu != 0, w + s.v, parts, 0}, dtype,
                      false, o, tiles, st);
    return e == cudaSuccess ? CT_OK : CT_ECUDA;
}

extern "C" ct_status ct_adapters_grad_workspace(int64_t t, int64_t adapters, int64_t rank, int64_t k, int64_t n, size_t *bytes) {
    using namespace ct::ops;
    if (bytes == nullptr) return CT_EINVAL;
    if (!sizes_ok(t, adapters, rank, k, n)) return CT_ERANGE;
    *bytes = space_of(t, adapters, rank, true).total;
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
    const int es = dtype_size(dtype), ges = dtype_size(grad_dtype), xs = dtype_size(x_dtype), dys = dtype_size(dy_dtype);
    const int dxs = dx_dev != nullptr ? dtype_size(dx_dtype) : 4;
    if (!matrix_ok(dy_dev, lddy, t, n, dys) || !matrix_ok(x_dev, ldx, t, k, xs) ||
        !adapter_matrix_ok(a_dev, a_adapter, a_row, adapters, rank, k, es) ||
        !adapter_matrix_ok(b_dev, b_adapter, b_row, adapters, n, rank, es) || !aligned(ids_dev, 8) || !aligned(scale_dev, 4) ||
        (dx_dev != nullptr && !matrix_ok(dx_dev, lddx, t, k, dxs)) ||
        (adapters * rank * k > 0 && (da_dev == nullptr || !aligned(da_dev, ges))) ||
        (adapters * rank * n > 0 && (db_dev == nullptr || !aligned(db_dev, ges))))
        return CT_EINVAL;
    if (ids_dev == nullptr && adapters == 0 && t > 0) return CT_EINVAL;
    const Space s = space_of(t, adapters, rank, true);
    if (workspace_dev == nullptr || !aligned(workspace_dev, 16)) return CT_EINVAL;
    if (workspace_bytes < s.total) return CT_ENOMEM;
    // dx is written while a is read and before x and dy are read again, da and db while those are
    const Span x = span(x_dev, t, k, ldx, xs), dy = span(dy_dev, t, n, lddy, dys), dx = span(dx_dev, dx_dev != nullptr ? t : 0, k, lddx, dxs);
    const Span da = span(da_dev, adapters * rank, k, k, ges), db = span(db_dev, adapters * n, rank, rank, ges);
    if (share(dx, x) || share(dx, dy) || on_stack(dx, a_dev, a_adapter, a_row, adapters, rank, k, es) || share(da, x) || share(da, dy) ||
        share(da, dx) || share(db, x) || share(db, dy) || share(db, dx) || share(da, db))
        return CT_EINVAL;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    char *w = static_cast<char *>(workspace_dev);
    const bool xw = whole(x_dev, ldx, t, k, xs), dyw = whole(dy_dev, lddy, t, n, dys), dxw = whole(dx_dev, lddx, t, k, dxs);
    const bool aw = stack_whole(a_dev, a_adapter, a_row, adapters, rank, k, es), bw = stack_whole(b_dev, b_adapter, b_row, adapters, n, rank, es);
    const int r = (int)rank, tiles = (int)tiles_of(t, adapters, ids_dev != nullptr);
    // three parts of the short vectors where a result of 32 bits hangs on them
    if (t == 0) ids_dev = nullptr;                // zeros for all, no rows to order
    const int v_parts = grad_dtype == CT_DT_F32 ? 3 : 2;
    const int u_parts = grad_dtype == CT_DT_F32 || (dx_dev != nullptr && dx_dtype == CT_DT_F32) ? 3 : 2;
    AdOrder o;
    cudaError_t e = make_order(o, ids_dev, t, adapters, s, w, st);
    if (e == cudaSuccess && t > 0 && adapters * rank > 0) {
        const AdShrink v = {x_dev, ldx, k, a_dev, a_adapter, a_row, scale_dev, r, (int)xw | (int)aw << 1, w + s.v, v_parts, true};
        const AdShrink u = {dy_dev, lddy, n, b_dev, b_adapter, b_row, scale_dev, r, (int)dyw | (int)bw << 1, w + s.u, u_parts, false};
        // together where they take the same kernel and are short of CTAs; else one after the other, each with its own share of the axis
        // (8192 rows, 4096 and 8192 columns, rank 64: 49 us, against 55 together; 256 rows, 512 and 1000: 16, against 9)
        if (x_dtype == dy_dtype && v.whole == u.whole && 8 * tiles <= sm_count()) {
            e = ad_shrink({v, u}, AD_BOTH, x_dtype, dtype, o, tiles, st);
        } else {
            e = ad_shrink({v, v}, AD_FORWARD, x_dtype, dtype, o, tiles, st);
            if (e == cudaSuccess) e = ad_shrink({u, u}, AD_BACKWARD, dy_dtype, dtype, o, tiles, st);
        }
    }
    if (e == cudaSuccess && t > 0 && k > 0 && dx_dev != nullptr)
        e = ad_expand({dx_dev, dx_dtype, lddx, k, a_dev, a_adapter, a_row, r, (int)dxw | (int)aw << 1, 0, w + s.u,
                       dx_dtype == CT_DT_F32 ? 3 : 2, 0}, dtype, true, o, tiles, st);
    if (e == cudaSuccess && adapters * rank > 0) {
        const AdOuter da = {x_dev, ldx, k, w + s.u, v_parts, r, (int)xw, da_dev, grad_dtype, 0};
        const AdOuter db = {dy_dev, lddy, n, w + s.v, v_parts, r, (int)dyw, db_dev, grad_dtype, 1};
        if (k > 0 && n > 0 && x_dtype == dy_dtype && xw == dyw) {
            e = ad_outer({da, db}, 2, x_dtype, o, st);
        } else {
            if (k > 0) e = ad_outer({da, da}, 1, x_dtype, o, st);
            if (e == cudaSuccess && n > 0) e = ad_outer({db, db}, 1, dy_dtype, o, st);
        }
    }
    return e == cudaSuccess ? CT_OK : CT_ECUDA;
}
