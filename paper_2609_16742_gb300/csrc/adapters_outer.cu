// The gradients of an adapter's matrices: sums over its rows of outer products.
//
//   g[i](c, j) = sum over the rows t of adapter i of x[t][c] v[t][j]
//
// (x: the activations and v: the gradient's short vectors, or the other way round.)  Bound by x's bytes, with 2 rank operations
// for each value and part of v.  A CTA takes 128 columns of one adapter's rows, 64 rows at a time: both operands lie in
// shared memory with the summed rows along their own rows, as the transposing matrix loads want them.  A cluster's CTAs
// share the rows and add their sums in rank order, so every sum has one order.
// Of each 16 rows, the products of the least parts are added first.
//
// What comes here: FP32 and FP16 values (several parts), rows that start anywhere, and three parts of a rank above 64.  Bound by instructions
// and their latency: three adapters of rank 20 over 1777 rows take 21 us for 5003 FP16 columns, 16 us for 2999 FP32 ones.
#include "adapters.cuh"

namespace ct {
namespace ops {
namespace {

constexpr int COLS = 128;

template <typename TX, int RP> struct Outer {
    static constexpr int PX = Parts<TX>::N;
    static constexpr int LX = ad_pitch(COLS), LV = ad_pitch(RP);
    static constexpr int X_BYTES = AD_STEP * LX, V_BYTES = AD_STEP * LV;
    static constexpr int XV = AD_STEP * (COLS / 8) / AD_THREADS;                  // 4
    static constexpr int V_VECS = AD_STEP * (RP / 8), VV = (V_VECS + AD_THREADS - 1) / AD_THREADS;
    static constexpr int NT = RP / 16, SUM = COLS * sums_pitch(RP) * 4;
    // The tensor cores cut off what they add: sums go from their accumulators into others after 128 rows, or after each 16 where
    // x's values are several parts.
    static constexpr bool EACH = PX > 1;
    static constexpr int FLUSH = 2;
    // Ranks to 32: one buffer and two blocks on an SM, which wait for their rows in turn (8192 rows, 6144 FP32 columns twice, rank 16:
    // 163 us, 316 with two buffers and one block).  Above, the sums' registers leave room for one block.
    static constexpr int BLOCKS = RP <= 32 ? 2 : 1, BUFFERS = BLOCKS == 2 ? 1 : 2;
    static int smem(int parts) {
        const int all = BUFFERS * (PX * X_BYTES + parts * V_BYTES);
        return all > SUM ? all : SUM;
    }
};

template <typename TX, int RP>
__global__ void __launch_bounds__(AD_THREADS, Outer<TX, RP>::BLOCKS) outer_kernel(const __grid_constant__ AdOuters two, const AdOrder o, int splits) {
    using S = Outer<TX, RP>;
    extern __shared__ __align__(128) unsigned char sm[];
    pdl_wait();
    pdl_trigger();
    const int rank = splits > 1 ? (int)tc::cluster_ctarank() : 0, adapter = blockIdx.y;
    const int block = (int)(blockIdx.x / (unsigned)splits);
    const AdOuter &a = two.a[block >= two.first];
    const int64_t cols0 = (int64_t)(block >= two.first ? block - two.first : block) * COLS;
    const int64_t from = o.order != nullptr ? o.first[adapter + 1] : 0, to = o.order != nullptr ? o.end[adapter + 1] : adapter == 0 ? o.t : 0;
    const int64_t steps = (to - from + AD_STEP - 1) / AD_STEP;
    const int64_t s0 = steps * rank / splits, s1 = steps * (rank + 1) / splits;
    const uint32_t base = tc::smem_u32(sm);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, wm = warp & 3, wn = warp >> 2;
    const int buf_bytes = S::PX * S::X_BYTES + a.parts * S::V_BYTES;

    // this thread's vectors: of x, rows tid / 16 + 16 i, 8 values at 8 (tid % 16)
    constexpr int RUN = AD_THREADS / (COLS / 8);
    const int64_t xc = cols0 + (tid % (COLS / 8)) * 8;
    const int x_left = left_of(xc, a.cols), x_to = tid / (COLS / 8) * S::LX + tid % (COLS / 8) * 16;
    const TX *x0 = static_cast<const TX *>(a.x) + (x_left > 0 ? xc : 0);
    auto x_at = [&](int64_t s, int i, int &left) -> const TX * {
        const int64_t t = from + s * AD_STEP + tid / (COLS / 8) + i * RUN;
        left = t < to ? x_left : 0;
        return x0 + (left > 0 ? (o.order != nullptr ? (int64_t)o.order[t] : t) * a.ldx : 0);
    };
    auto v_at = [&](int64_t s, int p, int v, bool &there) -> const uint4 * {
        const int64_t t = from + s * AD_STEP + v / (RP / 8);
        there = v < S::V_VECS && t < to;
        return static_cast<const uint4 *>(a.v) + (there ? (p * o.t + t) * (RP / 8) + v % (RP / 8) : 0);
    };
    auto v_to = [&](int v) { return v / (RP / 8) * S::LV + v % (RP / 8) * 16; };
    Units<TX> ux[S::XV];
    uint4 ev[3][S::VV];
    auto fetch = [&](int64_t s) {
#pragma unroll
        for (int i = 0; i < S::XV; ++i) {
            int left;
            const TX *p = x_at(s, i, left);
            ux[i] = load_units(p, left);
        }
#pragma unroll
        for (int p = 0; p < 3; ++p)
#pragma unroll
            for (int i = 0; i < S::VV; ++i) {
                bool there;
                const uint4 *at = v_at(s, p, tid + i * AD_THREADS, there);
                ev[p][i] = ld_if(at, there && p < a.parts);
            }
    };
    auto store = [&](int64_t s, int buf) {
        const uint32_t bx = base + buf * buf_bytes, bv = bx + S::PX * S::X_BYTES;
#pragma unroll
        for (int i = 0; i < S::XV; ++i) {
            int left;
            const TX *at = x_at(s, i, left);
            uint4 p[S::PX];
            split8<S::PX>(take_eight(ux[i], at, left), p);
#pragma unroll
            for (int q = 0; q < S::PX; ++q) sts16(bx + q * S::X_BYTES + x_to + i * RUN * S::LX, p[q]);
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            if (p >= a.parts) break;
#pragma unroll
            for (int i = 0; i < S::VV; ++i) {
                const int v = tid + i * AD_THREADS;
                if (v < S::V_VECS) sts16(bv + p * S::V_BYTES + v_to(v), ev[p][i]);
            }
        }
    };
    float acc[2][S::NT][4], sum[2][S::NT][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < S::NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] = sum[i][j][e] = 0.f;
    auto flush = [&]() {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < S::NT; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    sum[i][j][e] += acc[i][j][e];
                    acc[i][j][e] = 0.f;
                }
    };
    const int q8 = lane >> 3, r8 = lane & 7;
    // the number of v's parts is fixed in the loop (FP32 rank 128, 8192 rows, 2048 to 2048: a call of 662 us, 680 where it is not)
    auto compute_as = [&](auto parts, int buf) {
        constexpr int PV = decltype(parts)::value, most = PV == 2 ? 1 : 2;
        const uint32_t bx = base + buf * buf_bytes, bv = bx + S::PX * S::X_BYTES;
#pragma unroll
        for (int k = 0; k < AD_STEP; k += 16) {
            uint32_t fa[S::PX][2][4];
#pragma unroll
            for (int p = 0; p < S::PX; ++p)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    ldsm_x4_t(bx + p * S::X_BYTES + (k + (q8 >> 1) * 8 + r8) * S::LX + (wm * 32 + i * 16 + (q8 & 1) * 8) * 2, fa[p][i]);
#pragma unroll
            for (int q = PV - 1; q >= 0; --q) {
                if constexpr (RP == 16) {
                    uint32_t b[4];
                    ldsm_x4_t(bv + q * S::V_BYTES + (k + (q8 & 1) * 8 + r8) * S::LV + wn * 16, b);
#pragma unroll
                    for (int p = S::PX - 1; p >= 0; --p)
                        if (p + q <= most)
#pragma unroll
                            for (int i = 0; i < 2; ++i) mma16<false>(acc[i][0], fa[p][i], b[0], b[1]);
                } else {
#pragma unroll
                    for (int j = 0; j < S::NT; j += 2) {
                        uint32_t b[4];
                        ldsm_x4_t(bv + q * S::V_BYTES + (k + (q8 & 1) * 8 + r8) * S::LV + (wn * (RP / 2) + j * 8 + (q8 >> 1) * 8) * 2, b);
#pragma unroll
                        for (int p = S::PX - 1; p >= 0; --p)
                            if (p + q <= most)
#pragma unroll
                                for (int i = 0; i < 2; ++i) {
                                    mma16<false>(acc[i][j], fa[p][i], b[0], b[1]);
                                    mma16<false>(acc[i][j + 1], fa[p][i], b[2], b[3]);
                                }
                    }
                }
            }
            if constexpr (S::EACH) flush();
        }
    };
    auto compute = [&](int buf) {
        if (a.parts == 2) compute_as(std::integral_constant<int, 2>(), buf);
        else compute_as(std::integral_constant<int, 3>(), buf);
    };
    if (s0 < s1) {
        fetch(s0);
        store(s0, 0);
        __syncthreads();
        for (int64_t s = s0; s < s1; ++s) {
            const int at = (int)(s - s0);
            if (s + 1 < s1) fetch(s + 1);
            compute(S::BUFFERS == 2 ? at & 1 : 0);
            if (!S::EACH && at % S::FLUSH == S::FLUSH - 1) flush();
            if constexpr (S::BUFFERS == 1) __syncthreads();
            if (s + 1 < s1) store(s + 1, S::BUFFERS == 2 ? at & 1 ^ 1 : 0);
            __syncthreads();
        }
    }
    flush();

    float *fs = reinterpret_cast<float *>(sm);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < S::NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                fs[(wm * 32 + i * 16 + (e >> 1) * 8 + (lane >> 2)) * sums_pitch(RP) + wn * (RP / 2) + j * 8 + (lane & 3) * 2 + (e & 1)] = sum[i][j][e];
    if (splits > 1) tc::cluster_sync();
    else __syncthreads();
    write_gradient<RP>(a, adapter, cols0, fs, rank, splits);
    if (splits > 1) tc::cluster_sync();           // no CTA leaves while another reads its sums
}

template <typename TX, int RP> cudaError_t launch(const AdOuters &two, int blocks, const AdOrder &o, int splits, cudaStream_t st) {
    using S = Outer<TX, RP>;
    static std::atomic<bool> sized[MAX_DEVICES];
    auto *kernel = outer_kernel<TX, RP>;
    const cudaError_t e = allow_smem(kernel, sized, (size_t)S::smem(3));
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)(blocks * splits), (unsigned)o.adapters);
    const size_t smem = (size_t)S::smem(two.a[0].parts);
    return ad_launch(kernel, grid, smem, st, splits, true, two, o, splits);
}
template <typename TX> cudaError_t by_rank(const AdOuters &two, int blocks, const AdOrder &o, int splits, cudaStream_t st) {
    switch (ad_padded(two.a[0].rank)) {
        case 16: return launch<TX, 16>(two, blocks, o, splits, st);
        case 32: return launch<TX, 32>(two, blocks, o, splits, st);
        case 64: return launch<TX, 64>(two, blocks, o, splits, st);
        default: return launch<TX, 128>(two, blocks, o, splits, st);
    }
}
// Adapters of a few rows each: a tile's start and end would cost more than its products.  A thread has a column, eight of the rank at a
// time, and adds in FP32 row by row; as all rows may be one adapter's, 64 of them go into a sum, 8 of those into the next, and those into the
// last.  414 rows of 44 adapters, 9924 and 21143 columns, rank 16, BF16: 97 us
// for both gradients, 91 with one sum; the whole call takes 300 us, 346 with tiles here.
constexpr int FEW_COLS = 256, FEW_ROWS = 64, FEW_BLOCKS = 8;
template <typename TX> __global__ void __launch_bounds__(FEW_COLS) few_outer_kernel(const __grid_constant__ AdOuters two, const AdOrder o, int rp) {
    __shared__ float vs[FEW_ROWS][8];
    __shared__ int32_t rows[FEW_ROWS];
    pdl_wait();
    pdl_trigger();
    const int block = blockIdx.x, tid = threadIdx.x, adapter = blockIdx.y;
    const AdOuter &a = two.a[block >= two.first];
    const int64_t c = (int64_t)(block >= two.first ? block - two.first : block) * FEW_COLS + tid;
    const int from = o.first[adapter + 1], to = o.end[adapter + 1];
    const bool mine = c < a.cols;
    const TX *x = static_cast<const TX *>(a.x) + (mine ? c : 0);
    const __nv_bfloat16 *v = static_cast<const __nv_bfloat16 *>(a.v);
    const int64_t g0 = (int64_t)adapter * a.rank * a.cols;
    for (int j0 = 0; j0 < a.rank; j0 += 8) {
        float acc[8], some[8], sum[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = some[j] = sum[j] = 0.f;
        int blocks = 0;
        for (int t0 = from; t0 < to; t0 += FEW_ROWS) {
            const int n = min(FEW_ROWS, to - t0);
            __syncthreads();
            for (int i = tid; i < n * 8; i += FEW_COLS) {
                const int64_t at = (int64_t)(t0 + i / 8) * rp + j0 + i % 8;
                float s = 0.f;
                for (int p = a.parts - 1; p >= 0; --p) s += __bfloat162float(v[p * (o.t * rp) + at]);       // the least part first: exact
                vs[i / 8][i % 8] = s;
            }
            if (tid < n) rows[tid] = o.order[t0 + tid];
            __syncthreads();
#pragma unroll 8
            for (int i = 0; i < n; ++i) {
                const float w = mine ? to_f32(x[(int64_t)rows[i] * a.ldx]) : 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] = fmaf(w, vs[i][j], acc[j]);
            }
            const bool full = ++blocks % FEW_BLOCKS == 0 || t0 + FEW_ROWS >= to;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                some[j] += acc[j];
                acc[j] = 0.f;
                if (full) {
                    sum[j] += some[j];
                    some[j] = 0.f;
                }
            }
        }
        if (mine)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j0 + j < a.rank) put_as(a.g, a.g_dtype, g0 + (a.by_cols ? c * a.rank + j0 + j : (j0 + j) * a.cols + c), sum[j]);
    }
}
template <typename TX> cudaError_t few(const AdOuter (&a)[2], int n, const AdOrder &o, cudaStream_t st) {
    const int first = (int)((a[0].cols + FEW_COLS - 1) / FEW_COLS), blocks = first + (n > 1 ? (int)((a[1].cols + FEW_COLS - 1) / FEW_COLS) : 0);
    const AdOuters two = {{a[0], a[n - 1]}, first};
    return pdl_launch(few_outer_kernel<TX>, dim3((unsigned)blocks, (unsigned)o.adapters), dim3(FEW_COLS), 0, st, two, o, ad_padded(a[0].rank));
}
}  // namespace

cudaError_t ad_outer(const AdOuter (&a)[2], int n, int x_dtype, const AdOrder &o, cudaStream_t st) {
    // 16 rows an adapter at most, on average
    if (o.order != nullptr && o.t <= 16 * (int64_t)o.adapters)
        return x_dtype == CT_DT_F32 ? few<float>(a, n, o, st) : x_dtype == CT_DT_F16 ? few<__half>(a, n, o, st) : few<__nv_bfloat16>(a, n, o, st);
    const int first = (int)((a[0].cols + COLS - 1) / COLS), blocks = first + (n > 1 ? (int)((a[1].cols + COLS - 1) / COLS) : 0);
    // as many CTAs as are resident together (two for each SM), with two steps of an adapter's share of the rows at least for each
    const int64_t steps = (o.t / o.adapters + AD_STEP - 1) / AD_STEP, most = 2 * sm_count() / ((int64_t)blocks * o.adapters);
    int splits = (int)(most < 8 ? most : 8);
    if (splits > steps / 2) splits = (int)(steps / 2);
    if (splits < 1) splits = 1;
    const AdOuters two = {{a[0], a[n - 1]}, first};
    if (x_dtype == CT_DT_BF16 && (a[0].whole & a[n - 1].whole & 1) && ad_outer_tc_takes(a[0].rank, a[0].parts))
        return ad_outer_tc(two, blocks, o, splits, st);
    return x_dtype == CT_DT_F32   ? by_rank<float>(two, blocks, o, splits, st)
           : x_dtype == CT_DT_F16 ? by_rank<__half>(two, blocks, o, splits, st)
                                  : by_rank<__nv_bfloat16>(two, blocks, o, splits, st);
}

}  // namespace ops
}  // namespace ct
