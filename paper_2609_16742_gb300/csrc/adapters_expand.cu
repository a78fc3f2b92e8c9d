// The second product of an adapter: its short vectors against the many rows of B (or columns of A), added to y in place.
//
//   y[t][c] = act(y[t][c] + sum_j m[i](c, j) v[t][j])
//
// Bound by y's bytes, read once and written once.  A CTA holds the parts of 128 vectors in shared memory and goes along y
// in steps of 64 columns.  The columns of a step are dealt to the tensor cores' so that a thread's sums are eight
// neighbouring columns of a row: y goes from memory to registers and back without shared memory where its rows start on
// 16 bytes.
//
// What comes here: matrices of FP32 or FP16 values (several parts), rows that start anywhere.  Bound by instructions and their latency: 1777 x
// 5003 FP32 values of y that start anywhere, FP16 matrices of rank 20, take 32 us (five products of parts; 42 before y's bits
// came a step ahead without branches or conversions, rows' addresses lay in shared memory and warps without rows idled).
// FP32 of rank 128, 8192 x 2048: 112 us alone; in a call 178 from its early launch on, 278 with a number
// of parts that the loop did not know and the matrix's read again for each of v's.
#include "adapters.cuh"

namespace ct {
namespace ops {
namespace {

template <typename TM, int RP, bool TRANS> struct Expand {
    static constexpr int PM = Parts<TM>::N;
    static constexpr int LV = ad_pitch(RP), LM = ad_pitch(TRANS ? AD_STEP : RP);
    static constexpr int V_BYTES = AD_ROWS * LV, M_ROWS = TRANS ? RP : AD_STEP, M_BYTES = M_ROWS * LM;
    static constexpr int WIDE = 33, OUT = 8 * 8 * WIDE * 4;                      // 8 x 32 sums of each warp, where rows start anywhere
    static constexpr int M_VECS = M_ROWS * (TRANS ? AD_STEP / 8 : RP / 8), MV = (M_VECS + AD_THREADS - 1) / AD_THREADS;
    // blocks that an SM's memory holds
    static constexpr int blocks(bool out) { return 3 * V_BYTES + 2 * PM * M_BYTES + (out ? OUT : 0) <= 112 * 1024 ? 2 : 1; }
    static int smem(int parts, bool out) { return parts * V_BYTES + 2 * PM * M_BYTES + (out ? OUT : 0); }
};

// eight neighbouring values of a row of y, from 16 bytes on
struct YEight {
    uint4 u[2];
};
__device__ __forceinline__ YEight y_load(const char *p, int dtype, bool wanted) {
    YEight e;
    e.u[0] = ld_if(p, wanted);
    e.u[1] = ld_if(p + 16, wanted && dtype == CT_DT_F32);
    return e;
}
__device__ __forceinline__ void y_values(const YEight &e, int dtype, float *v) {
    if (dtype == CT_DT_F32) {
        unpack16<float>(e.u[0], v);
        unpack16<float>(e.u[1], v + 4);
    } else if (dtype == CT_DT_F16) {
        unpack16<__half>(e.u[0], v);
    } else {
        unpack16<__nv_bfloat16>(e.u[0], v);
    }
}
__device__ __forceinline__ void y_store(char *p, int dtype, const float *v) {
    if (dtype == CT_DT_F32) {
        *reinterpret_cast<uint4 *>(p) = pack16<float>(v);
        *reinterpret_cast<uint4 *>(p + 16) = pack16<float>(v + 4);
    } else {
        *reinterpret_cast<uint4 *>(p) = dtype == CT_DT_F16 ? pack16<__half>(v) : pack16<__nv_bfloat16>(v);
    }
}
// The bits of one value of y, or 0: no branch and nothing done with them yet (a value that is converted, or passes the end of a branch, is
// waited for), and no order among other accesses to memory (none is of the same value), so that many are on their way together.
__device__ __forceinline__ uint32_t y_bits_if(const char *p, bool wide, bool wanted) {
    uint32_t v;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %2, 0;\n\tsetp.ne.b32 q, %3, 0;\n\tmov.b32 %0, 0;\n\t"
                 "@p ld.global.b32 %0, [%1];\n\t@q ld.global.u16 %0, [%1];\n\t}"
                 : "=&r"(v) : "l"(p), "r"((int)(wanted && wide)), "r"((int)(wanted && !wide)));
    return v;
}
__device__ __forceinline__ float y_of_bits(uint32_t v, int dtype) {
    return dtype == CT_DT_F32 ? __uint_as_float(v) : dtype == CT_DT_F16 ? __half2float(__ushort_as_half((unsigned short)v)) : __uint_as_float(v << 16);
}

// YW: y's rows are whole
template <typename TM, int RP, bool TRANS, bool YW>
__global__ void __launch_bounds__(AD_THREADS, Expand<TM, RP, TRANS>::blocks(!YW)) expand_kernel(const AdExpand a, const AdOrder o) {
    using S = Expand<TM, RP, TRANS>;
    extern __shared__ __align__(128) unsigned char sm[];
    __shared__ char *rows[AD_ROWS];               // where the rows of y begin; null: no row
    pdl_wait();
    pdl_trigger();
    const AdRows tile = ad_tile(o, (int)blockIdx.x);
    const int64_t c_from = (int64_t)blockIdx.y * a.per, c_to = min(c_from + a.per, a.cols);
    if (tile.rows == 0 || c_from >= c_to || (tile.key == 0 && !a.relu)) return;
    const bool out = tile.key > o.adapters, none = tile.key == 0;               // NaN; act alone
    const uint32_t base = tc::smem_u32(sm), bm0 = base + a.parts * S::V_BYTES;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, wm = warp & 3, wn = warp >> 2;
    const int ys = a.y_dtype == CT_DT_F32 ? 4 : 2;
    if (tid < AD_ROWS)
        rows[tid] = tid < tile.rows ? static_cast<char *>(a.y) + (o.order != nullptr ? (int64_t)o.order[tile.slot0 + tid] : tile.slot0 + tid) * a.ldy * ys
                                    : nullptr;

    const bool product = !out && !none && a.rank > 0;
    const TM *m = static_cast<const TM *>(a.m) + (product ? (int64_t)(tile.key - 1) * a.m_adapter : 0);
    // the matrix's vector v of a step: its address and how many of its values are there
    auto m_at = [&](int64_t c0, int v, int &left) -> const TM * {
        if constexpr (TRANS) {
            const int j = v / 8;
            const int64_t c = c0 + v % 8 * 8;
            left = v < S::M_VECS && j < a.rank ? left_of(c, a.cols) : 0;
            return m + (left > 0 ? j * a.m_row + c : 0);
        } else {
            const int64_t c = c0 + v / (RP / 8);
            const int j = v % (RP / 8) * 8;
            left = v < S::M_VECS && c < a.cols ? left_of(j, a.rank) : 0;
            return m + (left > 0 ? c * a.m_row + j : 0);
        }
    };
    // Where it goes.  With the columns along its rows, chunk t of 32 columns is dealt out: its pair q is what thread t of a quad sums as
    // its pair of tile q.
    auto put = [&](uint32_t at, int v, const uint4 &w) {
        if constexpr (TRANS) {
            const uint32_t row = at + v / 8 * S::LM + (v % 8 / 4) * 64 + (v % 4) * 4;
            sts4(row, w.x);
            sts4(row + 16, w.y);
            sts4(row + 32, w.z);
            sts4(row + 48, w.w);
        } else {
            sts16(at + v / (RP / 8) * S::LM + v % (RP / 8) * 16, w);
        }
    };
    Units<TM> um[S::MV];
    auto fetch = [&](int64_t c0) {
#pragma unroll
        for (int i = 0; i < S::MV; ++i) {
            int left;
            const TM *p = m_at(c0, tid + i * AD_THREADS, left);
            um[i] = load_units(p, left);
        }
    };
    auto store = [&](int64_t c0, int buf) {
        const uint32_t bm = bm0 + buf * (S::PM * S::M_BYTES);
#pragma unroll
        for (int i = 0; i < S::MV; ++i) {
            const int v = tid + i * AD_THREADS;
            int left;
            const TM *at = m_at(c0, v, left);
            uint4 p[S::PM];
            split8<S::PM>(take_eight(um[i], at, left), p);
            if (v < S::M_VECS)
#pragma unroll
                for (int q = 0; q < S::PM; ++q) put(bm + q * S::M_BYTES, v, p[q]);
        }
    };
    if (product) {
        fetch(c_from);
        for (int v = tid; v < a.parts * AD_ROWS * (RP / 8); v += AD_THREADS) {
            const int p = v / (AD_ROWS * (RP / 8)), r = v / (RP / 8) % AD_ROWS, j = v % (RP / 8);
            const bool there = r < tile.rows;
            copy16_if(base + p * S::V_BYTES + r * S::LV + j * 16,
                      static_cast<const uint4 *>(a.v) + (there ? (p * o.t + tile.slot0 + r) * (RP / 8) + j : 0), there);
        }
        copies_end();
        store(c_from, 0);
        copies_wait<0>();
    }
    __syncthreads();
    // this thread's rows: lane / 4 + 8 i of the warp's 32
    char *yr[4];
    bool yh[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        char *p = rows[wm * 32 + i * 8 + (lane >> 2)];
        yh[i] = p != nullptr;
        yr[i] = yh[i] ? p : static_cast<char *>(a.y);
    }
    const int q8 = lane >> 3, r8 = lane & 7;
    auto products = [&](auto parts, uint32_t bm, float (&acc)[2][4][4]) {
        constexpr int PV = decltype(parts)::value, MOST = PV == 2 ? 1 : 2;
        // y of 16 bits has no values so near the end of the range (8192 rows, 4096 to 4096 FP16, rank 64: a call of 147 us, 152 with the least first)
        constexpr bool LEAST_FIRST = PV == 3;
        // two blocks on an SM, 16-bit values and eight values of y ahead: the parts one by one, as registers end
        // (8192 x 4096 FP16, rank 64: 123 us, 135 with all at once; rank 16: 61, 69)
        constexpr int UNROLLED = S::blocks(!YW) == 2 && YW && S::PM < 3 ? 1 : PV;
        auto columns = [&](int k, int q, int j, uint32_t (&b)[4]) {
            const int n = j + (q8 >> 1);
            if constexpr (TRANS) ldsm_x4_t(bm + q * S::M_BYTES + (k + (q8 & 1) * 8 + r8) * S::LM + wn * 64 + n * 16, b);
            else ldsm_x4(bm + q * S::M_BYTES + (wn * 32 + 8 * (r8 >> 1) + 2 * n + (r8 & 1)) * S::LM + (k + (q8 & 1) * 8) * 2, b);
        };
#pragma unroll
        for (int k = 0; k < RP; k += 16) {
            // with the registers of one block on an SM, the matrix's parts are read once for all of the vectors'
            constexpr bool HELD = S::blocks(!YW) == 1;
            uint32_t held[HELD ? S::PM : 1][2][4];
            if constexpr (HELD)
#pragma unroll
                for (int q = 0; q < S::PM; ++q)
#pragma unroll
                    for (int j = 0; j < 2; ++j) columns(k, q, 2 * j, held[q][j]);
#pragma unroll UNROLLED
            for (int ip = 0; ip < PV; ++ip) {
                const int p = LEAST_FIRST ? PV - 1 - ip : ip;
                uint32_t fa[2][4];
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    ldsm_x4(base + p * S::V_BYTES + (wm * 32 + i * 16 + (q8 & 1) * 8 + r8) * S::LV + (k + (q8 >> 1) * 8) * 2, fa[i]);
#pragma unroll
                for (int iq = 0; iq < S::PM; ++iq) {
                    const int q = LEAST_FIRST ? S::PM - 1 - iq : iq;
                    if (p + q > MOST) continue;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        uint32_t(&b)[4] = held[HELD ? q : 0][j];
                        if constexpr (!HELD) columns(k, q, 2 * j, b);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            mma16<false>(acc[i][2 * j], fa[i], b[0], b[1]);
                            mma16<false>(acc[i][2 * j + 1], fa[i], b[2], b[3]);
                        }
                    }
                }
            }
        }
    };
    const float nan = __uint_as_float(0x7FC00000u);
    // y a step ahead: eight neighbouring values of each of the thread's rows, or, of rows that start anywhere, one column's of all of the warp's
    const int64_t mine0 = wn * 32 + (YW ? (lane & 3) * 8 : lane);
    YEight ahead[YW ? 4 : 1];
    uint32_t column[YW ? 1 : 32];
    auto y_fetch = [&](int64_t c0) {
        const int64_t c = c0 + mine0;
        if constexpr (YW) {
#pragma unroll
            for (int i = 0; i < 4; ++i) ahead[i] = y_load(yr[i] + c * ys, a.y_dtype, yh[i] && c < c_to);
        } else {
#pragma unroll
            for (int r = 0; r < 32; ++r) {
                const char *p = rows[wm * 32 + r];
                column[r] = y_bits_if(p + c * ys, ys == 4, p != nullptr && c < c_to);
            }
        }
    };
    const bool busy = wm * 32 < tile.rows;        // else the warp has no rows
    y_fetch(c_from);
    int buf = 0;
    for (int64_t c0 = c_from; c0 < c_to; c0 += AD_STEP, buf ^= 1) {
        const bool more = product && c0 + AD_STEP < c_to;
        if (more) fetch(c0 + AD_STEP);
        const int64_t mine = c0 + mine0;
        YEight y[YW ? 4 : 1];
        if constexpr (YW) {
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = ahead[i];
            y_fetch(c0 + AD_STEP);
        }
        float acc[2][4][4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.f;
        if (product && busy) {
            const uint32_t bm = bm0 + buf * (S::PM * S::M_BYTES);
            // the number of parts is fixed in the loop, so that its loads go ahead of its products
            if (a.parts == 2) products(std::integral_constant<int, 2>(), bm, acc);
            else products(std::integral_constant<int, 3>(), bm, acc);
        }
        if constexpr (YW) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v[8], w[8];
                y_values(y[i], a.y_dtype, w);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[2 * j] = acc[i >> 1][j][(i & 1) * 2] + w[2 * j];
                    v[2 * j + 1] = acc[i >> 1][j][(i & 1) * 2 + 1] + w[2 * j + 1];
                }
                if (a.relu || out)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = out ? nan : v[e] < 0.f ? 0.f : v[e];
                if (yh[i] && mine < c_to) y_store(yr[i] + mine * ys, a.y_dtype, v);
            }
        } else {
            // rows that start anywhere: eight rows of the warp's sums at a time turn in shared memory, so that lanes are neighbouring columns;
            // as a value is done, that of the next step takes its register
            float *w = reinterpret_cast<float *>(sm + a.parts * S::V_BYTES + 2 * S::PM * S::M_BYTES) + warp * 8 * S::WIDE;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (wm * 32 + i * 8 >= tile.rows) break;
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < 2; ++e) w[(lane >> 2) * S::WIDE + (lane & 3) * 8 + 2 * j + e] = acc[i >> 1][j][(i & 1) * 2 + e];
                __syncwarp();
                char *at[8];
                bool there[8];
                float v[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    char *p = rows[wm * 32 + i * 8 + r];
                    there[r] = p != nullptr && mine < c_to;
                    at[r] = p + mine * ys;
                    v[r] = w[r * S::WIDE + lane] + y_of_bits(column[i * 8 + r], a.y_dtype);
                }
                if (a.relu || out)
#pragma unroll
                    for (int r = 0; r < 8; ++r) v[r] = out ? nan : v[r] < 0.f ? 0.f : v[r];
                const bool next = mine + AD_STEP < c_to;
#pragma unroll
                for (int r = 0; r < 8; ++r) column[i * 8 + r] = y_bits_if(at[r] + AD_STEP * ys, ys == 4, there[r] && next);
                if (ys == 4) {
#pragma unroll
                    for (int r = 0; r < 8; ++r)
                        if (there[r]) *reinterpret_cast<float *>(at[r]) = v[r];
                } else {
#pragma unroll
                    for (int r = 0; r < 8; ++r)
                        if (there[r]) *reinterpret_cast<uint16_t *>(at[r]) = (uint16_t)(a.y_dtype == CT_DT_F16 ? pack2<__half>(v[r], 0.f) : pack2<__nv_bfloat16>(v[r], 0.f));
                }
                __syncwarp();
            }
        }
        if (more) store(c0 + AD_STEP, buf ^ 1);
        __syncthreads();
    }
}

template <typename TM, int RP, bool TRANS, bool YW> cudaError_t launch(const AdExpand &q, const AdOrder &o, int tiles, cudaStream_t st) {
    using S = Expand<TM, RP, TRANS>;
    static std::atomic<bool> sized[MAX_DEVICES];
    auto *kernel = expand_kernel<TM, RP, TRANS, YW>;
    const cudaError_t e = allow_smem(kernel, sized, (size_t)S::smem(3, !YW));
    if (e != cudaSuccess) return e;
    // columns of a block: as many as leave each SM three blocks, at most 1024
    AdExpand a = q;
    const int64_t steps = (a.cols + AD_STEP - 1) / AD_STEP;
    int64_t parts = (3 * (int64_t)sm_count() + tiles - 1) / tiles;
    if (parts < (steps + 15) / 16) parts = (steps + 15) / 16;
    if (parts > steps) parts = steps;
    if (parts > 65535) parts = 65535;
    a.per = (steps + parts - 1) / parts * AD_STEP;
    const dim3 grid((unsigned)tiles, (unsigned)((a.cols + a.per - 1) / a.per));
    return ad_launch(kernel, grid, (size_t)S::smem(a.parts, !YW), st, 1, true, a, o);
}
template <typename TM, bool TRANS, bool YW> cudaError_t by_rank(const AdExpand &a, const AdOrder &o, int tiles, cudaStream_t st) {
    switch (ad_padded(a.rank)) {
        case 16: return launch<TM, 16, TRANS, YW>(a, o, tiles, st);
        case 32: return launch<TM, 32, TRANS, YW>(a, o, tiles, st);
        case 64: return launch<TM, 64, TRANS, YW>(a, o, tiles, st);
        default: return launch<TM, 128, TRANS, YW>(a, o, tiles, st);
    }
}
template <bool TRANS, bool YW> cudaError_t by_type(const AdExpand &a, int dtype, const AdOrder &o, int tiles, cudaStream_t st) {
    return dtype == CT_DT_F32   ? by_rank<float, TRANS, YW>(a, o, tiles, st)
           : dtype == CT_DT_F16 ? by_rank<__half, TRANS, YW>(a, o, tiles, st)
                                : by_rank<__nv_bfloat16, TRANS, YW>(a, o, tiles, st);
}
}  // namespace

cudaError_t ad_expand(const AdExpand &a, int dtype, bool trans, const AdOrder &o, int tiles, cudaStream_t st) {
    if (dtype == CT_DT_BF16 && a.whole == 3) return ad_expand_tc(a, trans, o, tiles, st);
    if (a.whole & 1) return trans ? by_type<true, true>(a, dtype, o, tiles, st) : by_type<false, true>(a, dtype, o, tiles, st);
    return trans ? by_type<true, false>(a, dtype, o, tiles, st) : by_type<false, false>(a, dtype, o, tiles, st);
}

}  // namespace ops
}  // namespace ct
