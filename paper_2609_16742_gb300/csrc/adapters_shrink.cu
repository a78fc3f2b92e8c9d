// The first product of an adapter: many rows, their long axis against the few rows of A (or B transposed).
//
//   v[t][j] = scale[i] sum_c x[t][c] m[i](j, c)
//
// Bound by x's bytes: 2 rank operations for each value.  A tile of 128 rows goes along the long axis in steps of 64; a
// cluster's CTAs share the axis, add their sums through distributed shared memory in rank order, and write v in BF16
// parts, as the next products take it.
//
// What comes here has gone through registers: FP32 rows, rows that start anywhere or end within 16 bytes.  Bound by instructions and their
// latency, with few warps an SM: 1777 rows of 5003 FP16 values at rank 20 take 16 us, of 2999 FP32 ones 19 us.
#include "adapters.cuh"

namespace ct {
namespace ops {
namespace {

template <typename TX, typename TM, int RP, bool TRANS> struct Shrink {
    static constexpr bool F16 = sizeof(TX) == 2 && Parts<TX>::N == 2 && Parts<TM>::N == 2;
    static constexpr int PX = F16 ? 1 : Parts<TX>::N, PM = F16 ? 1 : Parts<TM>::N;
    static constexpr int LX = ad_pitch(AD_STEP), LM = ad_pitch(TRANS ? RP : AD_STEP);
    static constexpr int X_BYTES = AD_ROWS * LX, M_ROWS = TRANS ? AD_STEP : RP, M_BYTES = M_ROWS * LM;
    static constexpr int BUF = PX * X_BYTES + PM * M_BYTES;
    static constexpr int SUM = AD_ROWS * sums_pitch(RP) * 4;
    static constexpr int SMEM = 2 * BUF > SUM ? 2 * BUF : SUM;
    static constexpr int XV = AD_ROWS * 8 / AD_THREADS;                          // vectors of 8 values a thread loads
    static constexpr int M_VECS = M_ROWS * (TRANS ? RP / 8 : 8), MV = (M_VECS + AD_THREADS - 1) / AD_THREADS;
    static constexpr int NT = RP / 16;                                           // 8-column tiles of a warp
    // The tensor cores cut off what they add: sums go from their accumulators into others after 256 values, or after each 16
    // where a value is several products.
    static constexpr bool EACH = PX * PM > 1;
    static constexpr int FLUSH = 4;
};

// the i-th part to take of n: FP32's three from the least on
__device__ __forceinline__ constexpr int least(int i, int n) { return n == 3 ? 2 - i : i; }

template <typename TX, typename TM, int RP, bool TRANS>
__device__ __forceinline__ void shrink_tile(const AdShrink &a, const AdOrder &o, const AdRows &tile, int rank, int splits, unsigned char *sm) {
    using S = Shrink<TX, TM, RP, TRANS>;
    const int adapter = tile.key - 1;
    const uint32_t base = tc::smem_u32(sm);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, wm = warp & 3, wn = warp >> 2;
    const int64_t steps = (a.cols + AD_STEP - 1) / AD_STEP;
    const int64_t s0 = steps * rank / splits, s1 = steps * (rank + 1) / splits;

    // this thread's vectors: of x, rows tid / 8 + 32 i, 8 values at 8 (tid % 8)
    const TX *xr[S::XV];
    bool xh[S::XV];
    const int xc = (tid & 7) * 8;
#pragma unroll
    for (int i = 0; i < S::XV; ++i) {
        const int r = tid / 8 + 32 * i;
        const int64_t s = tile.slot0 + r;
        xh[i] = r < tile.rows;
        xr[i] = static_cast<const TX *>(a.x) + (xh[i] ? (o.order != nullptr ? (int64_t)o.order[s] : s) * a.ldx : 0);
    }
    const TM *m = static_cast<const TM *>(a.m) + adapter * a.m_adapter;
    // the matrix's vector v of a step: its address, how many of its values are there, where it goes
    auto m_at = [&](int64_t s, int v, int &left) -> const TM * {
        const int64_t c0 = s * AD_STEP;
        if constexpr (TRANS) {
            const int64_t c = c0 + v / (RP / 8);
            const int j = v % (RP / 8) * 8;
            left = v < S::M_VECS && c < a.cols ? left_of(j, a.rank) : 0;
            return m + (left > 0 ? c * a.m_row + j : 0);
        } else {
            const int j = v / 8;
            const int64_t c = c0 + v % 8 * 8;
            left = v < S::M_VECS && j < a.rank ? left_of(c, a.cols) : 0;
            return m + (left > 0 ? j * a.m_row + c : 0);
        }
    };
    auto m_to = [&](int v) { return v / (TRANS ? RP / 8 : 8) * S::LM + v % (TRANS ? RP / 8 : 8) * 16; };
    const int x_to = tid / 8 * S::LX + xc * 2;
    Units<TX> ux[S::XV];
    Units<TM> um[S::MV];
    auto fetch = [&](int64_t s) {
        const int64_t c = s * AD_STEP + xc;
        const int n = left_of(c, a.cols);
#pragma unroll
        for (int i = 0; i < S::XV; ++i) ux[i] = load_units(xr[i] + (n > 0 ? c : 0), xh[i] ? n : 0);
#pragma unroll
        for (int i = 0; i < S::MV; ++i) {
            int left;
            const TM *p = m_at(s, tid + i * AD_THREADS, left);
            um[i] = load_units(p, left);
        }
    };
    auto store = [&](int64_t s, int buf) {
        const uint32_t bx = base + buf * S::BUF, bm = bx + S::PX * S::X_BYTES;
        const int64_t c = s * AD_STEP + xc;
        const int n = left_of(c, a.cols);
#pragma unroll
        for (int i = 0; i < S::XV; ++i) {
            uint4 p[S::PX];
            split8<S::PX>(take_eight(ux[i], xr[i] + (n > 0 ? c : 0), xh[i] ? n : 0), p);
#pragma unroll
            for (int q = 0; q < S::PX; ++q) sts16(bx + q * S::X_BYTES + x_to + 32 * i * S::LX, p[q]);
        }
#pragma unroll
        for (int i = 0; i < S::MV; ++i) {
            const int v = tid + i * AD_THREADS;
            int left;
            const TM *at = m_at(s, v, left);
            uint4 p[S::PM];
            split8<S::PM>(take_eight(um[i], at, left), p);
            if (v < S::M_VECS)
#pragma unroll
                for (int q = 0; q < S::PM; ++q) sts16(bm + q * S::M_BYTES + m_to(v), p[q]);
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
    const bool busy = wm * 32 < tile.rows;        // else the warp has no rows
    auto compute = [&](int buf) {
        if (!busy) return;
        const uint32_t bx = base + buf * S::BUF, bm = bx + S::PX * S::X_BYTES;
#pragma unroll
        for (int k = 0; k < AD_STEP; k += 16) {
            uint32_t fa[S::PX][2][4];
#pragma unroll
            for (int p = 0; p < S::PX; ++p)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    ldsm_x4(bx + p * S::X_BYTES + (wm * 32 + i * 16 + (q8 & 1) * 8 + r8) * S::LX + (k + (q8 >> 1) * 8) * 2, fa[p][i]);
            if constexpr (RP == 16) {
                // one 8-column tile a warp: both halves of k by lanes 0 to 15's addresses
#pragma unroll
                for (int iq = 0; iq < S::PM; ++iq) {
                    const int q = least(iq, S::PM);
                    uint32_t b[4];
                    if constexpr (TRANS) ldsm_x4_t(bm + q * S::M_BYTES + (k + (q8 & 1) * 8 + r8) * S::LM + wn * 16, b);
                    else ldsm_x4(bm + q * S::M_BYTES + (wn * 8 + r8) * S::LM + (k + (q8 & 1) * 8) * 2, b);
#pragma unroll
                    for (int ip = 0; ip < S::PX; ++ip)
                        if (const int p = least(ip, S::PX); p + q <= 2)
#pragma unroll
                            for (int i = 0; i < 2; ++i) mma16<S::F16>(acc[i][0], fa[p][i], b[0], b[1]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < S::NT; j += 2)
#pragma unroll
                    for (int iq = 0; iq < S::PM; ++iq) {
                        const int q = least(iq, S::PM);
                        uint32_t b[4];
                        const int n = wn * (RP / 2) + j * 8 + (q8 >> 1) * 8;
                        if constexpr (TRANS) ldsm_x4_t(bm + q * S::M_BYTES + (k + (q8 & 1) * 8 + r8) * S::LM + n * 2, b);
                        else ldsm_x4(bm + q * S::M_BYTES + (n + r8) * S::LM + (k + (q8 & 1) * 8) * 2, b);
#pragma unroll
                        for (int ip = 0; ip < S::PX; ++ip)
                            if (const int p = least(ip, S::PX); p + q <= 2)
#pragma unroll
                                for (int i = 0; i < 2; ++i) {
                                    mma16<S::F16>(acc[i][j], fa[p][i], b[0], b[1]);
                                    mma16<S::F16>(acc[i][j + 1], fa[p][i], b[2], b[3]);
                                }
                    }
            }
            if constexpr (S::EACH) flush();
        }
    };

    if (s0 < s1) {
        fetch(s0);
        store(s0, 0);
        __syncthreads();
        for (int64_t s = s0; s < s1; ++s) {
            const int at = (int)(s - s0);
            if (s + 1 < s1) fetch(s + 1);
            compute(at & 1);
            if (!S::EACH && at % S::FLUSH == S::FLUSH - 1) flush();
            if (s + 1 < s1) store(s + 1, at & 1 ^ 1);
            __syncthreads();
        }
    }
    flush();

    // the tile's sums of this CTA, then of all of the cluster
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
    write_vectors<RP>(a, o, tile, adapter, fs, rank, splits);
    if (splits > 1) tc::cluster_sync();           // no CTA leaves while another reads its sums
}

struct AdShrinks {
    AdShrink a[2];
};
// WHICH as AdWhich: both: the tiles of the first, then those of the second
template <typename TX, typename TM, int RP, int WHICH>
__global__ void __launch_bounds__(AD_THREADS) shrink_kernel(const __grid_constant__ AdShrinks two, const AdOrder o, int tiles, int splits) {
    extern __shared__ __align__(128) unsigned char sm[];
    pdl_wait();
    pdl_trigger();
    const int rank = splits > 1 ? (int)tc::cluster_ctarank() : 0;
    int t = (int)(blockIdx.x / (unsigned)splits);
    const bool second = WHICH == AD_BACKWARD || (WHICH == AD_BOTH && t >= tiles);
    if (WHICH == AD_BOTH && second) t -= tiles;
    const AdShrink &a = two.a[WHICH == AD_BOTH && second];
    const AdRows tile = ad_tile(o, t);
    if (tile.rows == 0 || tile.key == 0 || tile.key > o.adapters) return;       // the whole cluster alike
    if (WHICH == AD_FORWARD || (WHICH == AD_BOTH && !second)) shrink_tile<TX, TM, RP, false>(a, o, tile, rank, splits, sm);
    else shrink_tile<TX, TM, RP, true>(a, o, tile, rank, splits, sm);
}

template <typename TX, typename TM, int RP, int WHICH>
cudaError_t launch(const AdShrinks &two, const AdOrder &o, int tiles, int splits, cudaStream_t st) {
    constexpr int F = Shrink<TX, TM, RP, false>::SMEM, B = Shrink<TX, TM, RP, true>::SMEM;
    constexpr int SMEM = WHICH == AD_FORWARD ? F : WHICH == AD_BACKWARD ? B : F > B ? F : B;
    static std::atomic<bool> sized[MAX_DEVICES];
    auto *kernel = shrink_kernel<TX, TM, RP, WHICH>;
    const cudaError_t e = allow_smem(kernel, sized, SMEM);
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)((WHICH == AD_BOTH ? 2 : 1) * tiles * splits));
    return ad_launch(kernel, grid, SMEM, st, splits, true, two, o, tiles, splits);
}
template <typename TX, typename TM, int WHICH> cudaError_t by_rank(const AdShrinks &two, const AdOrder &o, int tiles, int splits, cudaStream_t st) {
    switch (ad_padded(two.a[0].rank)) {
        case 16: return launch<TX, TM, 16, WHICH>(two, o, tiles, splits, st);
        case 32: return launch<TX, TM, 32, WHICH>(two, o, tiles, splits, st);
        case 64: return launch<TX, TM, 64, WHICH>(two, o, tiles, splits, st);
        default: return launch<TX, TM, 128, WHICH>(two, o, tiles, splits, st);
    }
}
template <int WHICH> cudaError_t by_type(const AdShrinks &two, int x_dtype, int dtype, const AdOrder &o, int tiles, int splits, cudaStream_t st) {
    if (dtype == CT_DT_F32) return by_rank<float, float, WHICH>(two, o, tiles, splits, st);
    if (dtype == CT_DT_F16)
        return x_dtype == CT_DT_F32 ? by_rank<float, __half, WHICH>(two, o, tiles, splits, st) : by_rank<__half, __half, WHICH>(two, o, tiles, splits, st);
    return x_dtype == CT_DT_F32 ? by_rank<float, __nv_bfloat16, WHICH>(two, o, tiles, splits, st)
                                : by_rank<__nv_bfloat16, __nv_bfloat16, WHICH>(two, o, tiles, splits, st);
}
}  // namespace

cudaError_t ad_shrink(const AdShrink (&a)[2], AdWhich which, int x_dtype, int dtype, const AdOrder &o, int tiles, cudaStream_t st) {
    const int64_t cols = which == AD_BOTH && a[1].cols > a[0].cols ? a[1].cols : a[0].cols;
    // as many CTAs as are resident together (two for each SM), with two steps at least for each
    const int64_t steps = (cols + AD_STEP - 1) / AD_STEP, most = 2 * sm_count() / ((which == AD_BOTH ? 2 : 1) * (int64_t)tiles);
    int splits = (int)(most < 8 ? most : 8);
    if (splits > steps / 2) splits = (int)(steps / 2);
    if (splits < 1) splits = 1;
    const int whole = a[0].whole & a[which == AD_BOTH].whole;
    if (whole == 3 && dtype != CT_DT_F32 && x_dtype == dtype) return ad_shrink_tc(a, which, dtype == CT_DT_BF16, o, tiles, splits, st);
    const AdShrinks two = {{a[0], a[1]}};
    return which == AD_FORWARD    ? by_type<AD_FORWARD>(two, x_dtype, dtype, o, tiles, splits, st)
           : which == AD_BACKWARD ? by_type<AD_BACKWARD>(two, x_dtype, dtype, o, tiles, splits, st)
                                  : by_type<AD_BOTH>(two, x_dtype, dtype, o, tiles, splits, st);
}

}  // namespace ops
}  // namespace ct
