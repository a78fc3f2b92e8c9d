// What the adapters' kernels share: the rows' order by adapter, tiles of 16-bit
// parts in shared memory, and products of those on the tensor cores.
//
// The long products (rows by many) run on the tensor cores with 16-bit operands and FP32
// sums: as tcgen05.mma where rows are 16-bit values that can be copied as they lie
// (adapters_tc.cu), else as mma.sync on what has gone through registers.  BF16 values are taken as they are.  FP16 and FP32 values, and the short FP32
// vectors between two products, are taken apart into BF16 parts of 8 bits each
// (v = hi + mid + lo; two parts hold an FP16 value), and the products of parts
// that matter are added: those of parts p and q with p + q <= 1 where the result has 16
// bits (the rest is below 2^-15 of a term), with p + q <= 2 where it has 32 (2^-22),
// the least first: of the largest FP32 values hi + mid alone can be infinite.
// FP16 by FP16 runs as it is.  (Parts end at 2^-133, BF16's smallest step: FP32 values below 2^-110 keep fewer than 24 bits.)
#pragma once
#include "ops_common.cuh"
#include "tc_common.cuh"

namespace ct {
namespace ops {

constexpr int AD_THREADS = 256;                   // 8 warps: 4 over a tile's rows, 2 over its columns
constexpr int AD_ROWS = 128;                      // rows of a tile
constexpr int AD_STEP = 64;                       // values along the long axis for each step

// Rows of one adapter: order[slot0 .. slot0 + rows).  key 0: rows without an adapter, 1 + i: adapter i, 1 + adapters: ids out of range.
struct AdTile {
    int32_t slot0, key;
};

// The rows in the order of their adapters (each adapter's in their own), on the device; all null where every row has adapter 0.
struct AdOrder {
    const int32_t *order;                         // [t]
    const int32_t *first, *end;                   // [adapters + 2]: the slots of each key
    const AdTile *tiles;
    const int32_t *n_tiles;
    int64_t t;
    int adapters;
};

// One product with a matrix of the adapters.  `whole`: bit 0: x's (y's) rows start on 16 bytes and are a multiple of 8 values long, bit 1:
// the matrix's.
struct AdShrink {
    const void *x;
    int64_t ldx, cols;
    const void *m;
    int64_t m_adapter, m_row;
    const float *scale;
    int rank, whole;
    void *v;                                      // BF16 [parts][t][padded rank], by slots
    int parts;
    bool first;                                   // launched right behind the ordering of the rows
};
struct AdExpand {
    void *y;
    int32_t y_dtype;
    int64_t ldy, cols;
    const void *m;
    int64_t m_adapter, m_row;
    int rank, whole, relu;
    const void *v;
    int parts;
    int64_t per;                                  // columns of a block
};
struct AdOuter {
    const void *x;
    int64_t ldx, cols;
    const void *v;
    int parts;
    int rank, whole;
    void *g;                                      // [adapters][rank][cols], or [adapters][cols][rank] where by_cols
    int32_t g_dtype;
    int by_cols;
};
// One or two of them: blocks of 128 columns, the first one's, then the second one's.
struct AdOuters {
    AdOuter a[2];
    int first;                                    // blocks of the first
};

#ifdef __CUDACC__
struct AdRows {
    int64_t slot0;
    int rows, key;
};
__device__ __forceinline__ AdRows ad_tile(const AdOrder &o, int tile) {
    if (o.order == nullptr) {
        const int64_t s = (int64_t)tile * AD_ROWS;
        return {s, (int)(o.t - s < AD_ROWS ? o.t - s : AD_ROWS), 1};
    }
    if (tile >= *o.n_tiles) return {0, 0, 0};
    const AdTile d = o.tiles[tile];
    const int left = o.end[d.key] - d.slot0;
    return {d.slot0, left < AD_ROWS ? left : AD_ROWS, d.key};
}

// BF16 parts that hold a value
template <typename T> struct Parts { static constexpr int N = 1; };
template <> struct Parts<__half> { static constexpr int N = 2; };
template <> struct Parts<float> { static constexpr int N = 3; };

// Eight values of a row as they lie in memory.
template <typename T> struct Eight {
    uint4 u[sizeof(T) / 2];
};

// 16 bytes, or zeros: one instruction and no branch, so that many are on their way together
__device__ __forceinline__ uint4 ldg_if(const void *p, bool wanted) {
    uint4 v;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
        "@p ld.global.nc.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
        : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w)
        : "l"(p), "r"((int)wanted));
    return v;
}

// the same of what a kernel before wrote, or this one writes
__device__ __forceinline__ uint4 ld_if(const void *p, bool wanted) {
    uint4 v;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
        "@p ld.global.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
        : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w)
        : "l"(p), "r"((int)wanted)
        : "memory");
    return v;
}

// Eight values on their way: the aligned units that hold them.  A unit that holds no wanted byte is not read.
template <typename T> struct Units {
    uint4 u[sizeof(T) / 2 + 1];
};
// left: values of the row from the first on (8 or more, fewer at its end, 0: none)
template <typename T> __device__ __forceinline__ Units<T> load_units(const T *p, int left) {
    constexpr int N = (int)sizeof(T) / 2;
    const uint32_t shift = (uint32_t)(uintptr_t)p & 15u;
    const char *q = reinterpret_cast<const char *>(p) - shift;
    const int bytes = (left > 8 ? 8 : left) * (int)sizeof(T) + (int)shift;       // from q on
    Units<T> r;
#pragma unroll
    for (int i = 0; i <= N; ++i) r.u[i] = ldg_if(q + 16 * i, left > 0 && bytes > 16 * i);
    return r;
}
template <typename T> __device__ __forceinline__ Eight<T> take_eight(const Units<T> &r, const T *p, int left) {
    constexpr int N = (int)sizeof(T) / 2;
    const uint32_t shift = (uint32_t)(uintptr_t)p & 15u;
    Eight<T> e;
#pragma unroll
    for (int i = 0; i < N; ++i) e.u[i] = shifted(r.u[i], r.u[i + 1], shift);
    if (left < 8) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int bytes = left * (int)sizeof(T) - 16 * i;
            e.u[i] = bytes <= 0 ? make_uint4(0u, 0u, 0u, 0u) : bytes >= 16 ? e.u[i] : first_bytes(e.u[i], bytes);
        }
    }
    return e;
}
__device__ __forceinline__ int left_of(int64_t c, int64_t cols) { return c >= cols ? 0 : cols - c > 8 ? 8 : (int)(cols - c); }

// 16 bytes from global to shared memory, or zeros there
__device__ __forceinline__ void copy16_if(uint32_t to, const void *from, bool wanted) {
    const int bytes = wanted ? 16 : 0;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy4_if(uint32_t to, const void *from, bool wanted) {
    const int bytes = wanted ? 4 : 0;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Two values in BF16, and what is left of them (nothing of an infinite or NaN one: CLEAN).  FIRST: of FP32 values as they are.  The largest of
// those are nearer to infinity than to a BF16 value: they get the largest there is, and the next part has the rest.  (An infinity does so
// too, and goes on as the next part; where that is cleaned away it keeps its first.)
template <bool CLEAN, bool FIRST> __device__ __forceinline__ uint32_t split2(float &a, float &b) {
    uint32_t w;
    if constexpr (FIRST && CLEAN) {
        constexpr float MOST = 0x1.FEp127f;
        w = pack2<__nv_bfloat16>(fabsf(a) < __builtin_huge_valf() ? fminf(fmaxf(a, -MOST), MOST) : a,
                                 fabsf(b) < __builtin_huge_valf() ? fminf(fmaxf(b, -MOST), MOST) : b);
    } else if constexpr (FIRST) {
        asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(b), "f"(a));
    } else {
        w = pack2<__nv_bfloat16>(a, b);
    }
    a -= __uint_as_float(w << 16);
    b -= __uint_as_float(w & 0xFFFF0000u);
    if (CLEAN) {
        a = fabsf(a) < __builtin_huge_valf() ? a : 0.f;
        b = fabsf(b) < __builtin_huge_valf() ? b : 0.f;
    }
    return w;
}
template <bool FIRST> __device__ __forceinline__ uint4 split_part(float (&v)[8]) {
    uint4 w;
    w.x = split2<false, FIRST>(v[0], v[1]);
    w.y = split2<false, FIRST>(v[2], v[3]);
    w.z = split2<false, FIRST>(v[4], v[5]);
    w.w = split2<false, FIRST>(v[6], v[7]);
    return w;
}
// eight values as N parts of 16 bytes; the third of an infinite one is NaN, as infinity - infinity
template <int N, typename T> __device__ __forceinline__ void split8(const Eight<T> &e, uint4 (&out)[N]) {
    if constexpr (N == 1) {
        out[0] = e.u[0];
    } else {
        float v[8];
        unpack16<T>(e.u[0], v);
        if constexpr (sizeof(T) == 4) unpack16<T>(e.u[1], v + 4);
        out[0] = split_part<sizeof(T) == 4>(v);
#pragma unroll
        for (int p = 1; p < N; ++p) out[p] = split_part<false>(v);
    }
}

__device__ __forceinline__ void sts16(uint32_t addr, const uint4 &v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void sts4(uint32_t addr, uint32_t v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ void ldsm_x4_t(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr));
}
__device__ __forceinline__ void ldsm_x4(uint32_t addr, uint32_t (&r)[4]) { tc::ldsm_x4(addr, r[0], r[1], r[2], r[3]); }

// D += A (16 x 16) B (16 x 8), 16-bit operands, FP32 sums
template <bool F16> __device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (F16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Row pitch in bytes of a tile of `width` 16-bit values: 16 more than the values, so that eight rows of a matrix lie in different banks.
__host__ __device__ constexpr int ad_pitch(int width) { return 2 * width + 16; }

// four neighbouring sums of all CTAs of a cluster (up to 8), added in rank order; the loads are on their way together
__device__ __forceinline__ void sum_peers(uint32_t addr, int splits, float (&v)[4]) {
    float p[8][4];
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const uint32_t at = tc::mapa_shared(addr, (uint32_t)(c < splits ? c : 0));
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %5, 0;\n\t"
            "mov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
            "@p ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];\n\t}"
            : "=&f"(p[c][0]), "=&f"(p[c][1]), "=&f"(p[c][2]), "=&f"(p[c][3])
            : "r"(at), "r"((int)(c < splits))
            : "memory");
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[e] = p[0][e];
#pragma unroll
        for (int c = 1; c < 8; ++c) v[e] += p[c][e];
    }
}
__device__ __forceinline__ float ld_peer_f32(uint32_t addr, int rank) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(tc::mapa_shared(addr, (uint32_t)rank)) : "memory");
    return v;
}
// A tile's sums in shared memory: rows of `width` and four more, so that eight rows' 16 bytes lie in different banks.
__host__ __device__ constexpr int sums_pitch(int width) { return width + 4; }

// v of a tile: the cluster's sums (fs, at `addr` in each CTA) times scale, 0 behind the rank, in BF16 parts
template <int RP>
__device__ __forceinline__ void write_vectors(const AdShrink &a, const AdOrder &o, const AdRows &tile, int adapter, const float *fs, int rank, int splits) {
    const float scale = a.scale != nullptr ? a.scale[adapter] : 1.f;
    const uint32_t addr = tc::smem_u32(fs);
    const int r0 = AD_ROWS * rank / splits, r1 = AD_ROWS * (rank + 1) / splits;
    for (int i = threadIdx.x; i < (r1 - r0) * (RP / 4); i += AD_THREADS) {
        const int r = r0 + i / (RP / 4), j = i % (RP / 4) * 4;
        if (r >= tile.rows) break;
        float v[4];
        if (splits > 1) {
            sum_peers(addr + (r * sums_pitch(RP) + j) * 4, splits, v);
        } else {
            const float4 w = *reinterpret_cast<const float4 *>(fs + r * sums_pitch(RP) + j);
            v[0] = w.x, v[1] = w.y, v[2] = w.z, v[3] = w.w;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = j + e < a.rank ? v[e] * scale : 0.f;  // 0 and not 0 times what x holds
        uint2 *out = static_cast<uint2 *>(a.v) + ((tile.slot0 + r) * RP + j) / 4;
        for (int p = 0; p < a.parts; ++p) {
            uint2 w;
            w.x = p == 0 ? split2<true, true>(v[0], v[1]) : split2<true, false>(v[0], v[1]);
            w.y = p == 0 ? split2<true, true>(v[2], v[3]) : split2<true, false>(v[2], v[3]);
            out[p * (o.t * RP / 4)] = w;
        }
    }
}

__device__ __forceinline__ void put_as(void *p, int dtype, int64_t i, float v) {
    if (dtype == CT_DT_F32) static_cast<float *>(p)[i] = v;
    else if (dtype == CT_DT_F16) static_cast<__half *>(p)[i] = __float2half_rn(v);
    else static_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(v);
}
// A gradient's 128 columns from cols0 on: the cluster's sums, each CTA its share of the columns.  (Sharing the rank instead, for whole
// runs of columns where those run along the gradient's rows: 30 us for 8192 x 4096 x 64, against 27.)
template <int RP>
__device__ __forceinline__ void write_gradient(const AdOuter &a, int adapter, int64_t cols0, const float *fs, int rank, int splits) {
    constexpr int COLS = 128;
    const uint32_t addr = tc::smem_u32(fs);
    const int c0 = COLS * rank / splits, wide = COLS * (rank + 1) / splits - c0, fours = (a.rank + 3) / 4;
    const int64_t g0 = (int64_t)adapter * a.rank * a.cols;
    for (int i = threadIdx.x; i < wide * fours; i += AD_THREADS) {
        // neighbouring threads: neighbouring values of the gradient
        const int c = c0 + (a.by_cols ? i / fours : i % wide), j = (a.by_cols ? i % fours : i / wide) * 4;
        if (cols0 + c >= a.cols) continue;
        float v[4];
        if (splits > 1) {
            sum_peers(addr + (c * sums_pitch(RP) + j) * 4, splits, v);
        } else {
            const float4 w = *reinterpret_cast<const float4 *>(fs + c * sums_pitch(RP) + j);
            v[0] = w.x, v[1] = w.y, v[2] = w.z, v[3] = w.w;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (j + e < a.rank) put_as(a.g, a.g_dtype, g0 + (a.by_cols ? (cols0 + c) * a.rank + j + e : (j + e) * a.cols + cols0 + c), v[e]);
    }
}
#endif

// A launch that may begin while the kernel before ends, or (early: 0) not.  CTAs that are let in early go to whichever SMs are free first, two to
// one and none to another, where a kernel has not many more than the SMs hold: 8192 rows at rank 64 took 97 us with early launches of all
// kernels, 86 without.  So the tcgen05 kernels wait where they have more CTAs than there are SMs, unless the kernel before is the ordering of the
// rows (one CTA).  The others, which hold fewer registers and less shared memory, lose more by the gap (1777 rows: 144 us, against 135).
template <typename... KArgs, typename... Args>
inline cudaError_t ad_launch(void (*kernel)(KArgs...), dim3 grid, size_t smem, cudaStream_t st, int cluster, bool early, Args &&...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(AD_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = early || (int64_t)grid.x * grid.y <= sm_count();
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}

inline int ad_padded(int64_t rank) { return rank <= 16 ? 16 : rank <= 32 ? 32 : rank <= 64 ? 64 : 128; }

// The products of x with A^T ([rank, cols]; AD_FORWARD), of dy with B ([cols, rank], the rank along its rows; AD_BACKWARD), or of a[0] the one and
// of a[1] the other in one launch (AD_BOTH: of one rank and one type of rows).
enum AdWhich { AD_FORWARD = 0, AD_BACKWARD = 1, AD_BOTH = 2 };
cudaError_t ad_shrink(const AdShrink (&a)[2], AdWhich which, int x_dtype, int dtype, const AdOrder &o, int tiles, cudaStream_t st);
// trans: the matrix has the columns along its rows ([rank, cols])
cudaError_t ad_expand(const AdExpand &a, int dtype, bool trans, const AdOrder &o, int tiles, cudaStream_t st);
// two products of the same rank and number of parts, of x's of one type, in one launch (n = 2), or one (n = 1)
cudaError_t ad_outer(const AdOuter (&a)[2], int n, int x_dtype, const AdOrder &o, cudaStream_t st);

// The same on tcgen05, for 16-bit values in whole rows; splits: CTAs of a cluster that share the summed axis.
cudaError_t ad_shrink_tc(const AdShrink (&a)[2], AdWhich which, bool bf16, const AdOrder &o, int tiles, int splits, cudaStream_t st);
cudaError_t ad_expand_tc(const AdExpand &a, bool trans, const AdOrder &o, int tiles, cudaStream_t st);
bool ad_outer_tc_takes(int64_t rank, int parts);
cudaError_t ad_outer_tc(const AdOuters &two, int blocks, const AdOrder &o, int splits, cudaStream_t st);

}  // namespace ops
}  // namespace ct
