// Block-scaled matrix product in 8-bit floating point on the tcgen05 tensor
// cores:
//
//   y[m, n] = act( sum_b xs[m, b] ws[n / 128, b] P_b[m, n] + bias[n] ),
//   P_b[m, n] = sum over k in block b of xq[m, k] wq[n, k],
//
// x and w in e4m3, one scale for each 128 values of an x row and each
// 128 x 128 block of w.  The scales are any FP32 numbers, so the tensor
// cores cannot apply them: each block's P_b is one group of four MMAs
// (kind::f8f6f4, K = 32 each) into a TMEM accumulator of its own, and
// epilogue warps add factor * P_b to FP32 registers while the next block's
// MMAs run into another accumulator.
//
// Warp roles: 8 epilogue warps (warp w reads TMEM lanes 32 (w % 4) ..), one TMA
// warp, one MMA warp (a second one that took K blocks in turn changed
// nothing).  A stage of shared memory holds one K block of both operands:
// 128-byte rows, 128-byte swizzle; rows and columns past the ends are the
// zeros TMA fills in.
//
// Two kernels:
//   wide (many rows): rows of x on the TMEM lanes, tiles of 256 rows x BN
//     columns on CTA pairs (cta_group::2: each CTA stages half of both
//     operands), persistent; the factor of a thread's values is one product
//     per block.  A K block of 256 columns takes ~790 cycles, of which the MMAs
//     need 512: the epilogue's loads from TMEM and additions set the pace (16
//     epilogue warps instead of 8 make it slower, 262 us and more against 201).
//     8192 x 8192 x 4096 to BF16 in 200 us, 2.75 PFLOP/s, at 2070 MHz, in 222 us
//     after 0.1 s at the power limit (1.84 GHz);
//   narrow (few rows): rows of w on the lanes, 128 x BN tiles with BN as
//     narrow as the rows allow, so that a few rows cost no 128-wide tile; the
//     K range is split over a cluster of up to 8 CTAs so that the whole GPU
//     streams the weights, and the cluster adds its partial sums through
//     distributed shared memory, in rank order: no workspace, no atomics, one
//     launch, the same bits each time.  For few rows that are not yet in 8 bits
//     8 more warps quantise them on the way into shared memory (X: their type;
//     uint8_t: they are in 8 bits).  Bound by HBM with a start of ~3 us and a
//     join of ~2: 64 x 4096 x 25088 in 21.7 us, 4.7 TB/s of weights.
#include <atomic>
#include <cudaTypedefs.h>
#include <math.h>

#include "fp8_quantize.cuh"
#include "tc_common.cuh"

namespace ct {
namespace ops {
namespace {

using namespace ct::tc;

constexpr int BL = 128;                 // lane side of a tile
constexpr int BK = 128;                 // K block: one scale, one 128-byte row
constexpr int L_BYTES = BL * BK;
constexpr int N_EPI = 8;
constexpr int TMA_WARP = 8, MMA_WARP = 9;
constexpr int THREADS = 320;

// narrow: scales are fetched this many of a warp's K blocks at a time, that
// many ahead
constexpr int AHEAD = 4;

// error codes of the bounded waits
constexpr uint32_t E_TMA = 0x100, E_MMA = 0x200, E_ACC = 0x400, E_EPI = 0x800, E_DRAIN = 0x1000;

struct MmArgs {
    const float *xs;
    int64_t xs_row, xs_blk;
    const float *ws;
    int64_t ws_row, ws_blk;
    const float *bias;
    void *y;
    int64_t ldy;
    int M, N, KB;
    int out, relu;
    int tiles_l, tiles_c;               // tiles along the lane side and along the columns
    int splits;                         // CTAs of a cluster that share a tile's K blocks
    int group;                          // wide: row tiles walked together
    int vec;                            // wide: TMA can address y's rows, and they are whole 16-byte units
    int vec4;                           // 4 values of a row of y, from a multiple of 4 on, are one aligned store
    int early;                          // narrow: the kernel before does not write w
    const void *x;                      // narrow: rows to quantise, their pitch and length
    int64_t ldx;
    int K;
    uint32_t *err;
};

constexpr int QUANT_WARP = 10, N_QUANT = 8;   // narrow: warps that quantise x
// blocks whose scales are kept, each with a barrier: more than stages and accumulators together
constexpr int X_SLOTS = 16;

template <int BN, typename X = uint8_t> struct Narrow {
    static constexpr bool QUANT = sizeof(X) > 1;
    static constexpr int THREADS = ct::ops::THREADS + (QUANT ? 32 * N_QUANT : 0);
    // teams of the quantising warps, which take K blocks in turn, as what a block costs them is latency: 1 x 4096 x
    // 25088 FP16 in 24.9 us with one team, 20.9 with two, 19.8 with four; as many as leave a lane 4 rows
    static constexpr int TEAMS = (BN == 16 ? 4 : 2) / (sizeof(X) == 4 ? 2 : 1);
    static constexpr int C_BYTES = BN * BK;
    static constexpr int STAGE = L_BYTES + C_BYTES;
    static constexpr int STAGES = BN == 16 ? 10 : BN == 128 ? 6 : 8;
    static constexpr int NBUF = BN <= 64 ? 4 : 2;
    static constexpr int TMEM_COLS = NBUF * BN;
    // up to 64 columns: the two halves of the epilogue warps take K blocks in
    // turn, all columns each (what a block costs them is latency); 128
    // columns: every block, half the columns each
    static constexpr int GROUPS = BN <= 64 ? 2 : 1;
    static constexpr int CPW = BN / (2 / GROUPS);          // columns of an epilogue warp
    static constexpr int LDN = CPW < 32 ? CPW : 32;        // columns of one TMEM load
    static constexpr int FAC = N_EPI * 2 * CPW * 4;
    static constexpr size_t SMEM = 1024 + (size_t)STAGES * STAGE + FAC + 8 * (2 * STAGES + 2 * NBUF) + 16 +
                                   (QUANT ? X_SLOTS * (BN * 4 + 8) : 0);
    static_assert(STAGES + NBUF < X_SLOTS, "a slot is read, and its barrier's phase seen, before it is written again");
};

template <int N> __device__ __forceinline__ void tmem_ld_nw(uint32_t taddr, uint32_t (&r)[N]) {
    if constexpr (N == 16) {
        tmem_ld16_nw(taddr, r);
    } else if constexpr (N == 48) {
        tmem_ld_nw<32>(taddr, reinterpret_cast<uint32_t (&)[32]>(r[0]));
        tmem_ld_nw<16>(taddr + 32u, reinterpret_cast<uint32_t (&)[16]>(r[32]));
    } else {
        static_assert(N == 32, "16, 32 or 48 columns");
        asm volatile(
            "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
            "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
            : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
              "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
              "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
              "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
            : "r"(taddr));
    }
}

// kind::f8f6f4, A = B = E4M3 (format 0), D = FP32, both K-major
__host__ __device__ constexpr uint32_t idesc_e4m3(int M, int N) {
    return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

__device__ __forceinline__ void umma_e4m3(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a), "l"(b), "r"(idesc), "r"(acc));
}

__device__ __forceinline__ float4 ld_cluster_f32x4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(addr)
                 : "memory");
    return v;
}

__device__ __forceinline__ void store_out(const MmArgs &a, int64_t at, float v) {
    if (a.out == CT_DT_F32) static_cast<float *>(a.y)[at] = v;
    else if (a.out == CT_DT_F16) static_cast<__half *>(a.y)[at] = __float2half_rn(v);
    else static_cast<__nv_bfloat16 *>(a.y)[at] = __float2bfloat16_rn(v);
}

// 4 sums with their bias, `have` of them in the row: act, rounding, one store where y is aligned for it
__device__ __forceinline__ void store4(const MmArgs &a, int64_t at, const float (&f)[4], int have) {
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a.relu ? relu_keep_nan(f[i]) : f[i];
    if (a.vec4 && have >= 4) {
        if (a.out == CT_DT_F32) *reinterpret_cast<float4 *>(static_cast<float *>(a.y) + at) = make_float4(v[0], v[1], v[2], v[3]);
        else if (a.out == CT_DT_F16)
            *reinterpret_cast<uint2 *>(static_cast<__half *>(a.y) + at) =
                make_uint2(pack2<__half>(v[0], v[1]), pack2<__half>(v[2], v[3]));
        else
            *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(a.y) + at) =
                make_uint2(pack2<__nv_bfloat16>(v[0], v[1]), pack2<__nv_bfloat16>(v[2], v[3]));
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < have) store_out(a, at + i, v[i]);
}

// acc += f * p on two values at once.  Volatile, like the TMEM load and the
// wait before it: volatile asm keeps its order, so no value is read before
// its load is complete.
__device__ __forceinline__ void fma2(uint64_t &acc, uint64_t f, uint32_t p0, uint32_t p1) {
    asm volatile("{\n\t.reg .b64 p;\n\tmov.b64 p, {%2, %3};\n\tfma.rn.f32x2 %0, %1, p, %0;\n\t}"
                 : "+l"(acc)
                 : "l"(f), "r"(p0), "r"(p1));
}
__device__ __forceinline__ uint64_t dup2(float f) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %1};" : "=l"(r) : "f"(f));
    return r;
}
__device__ __forceinline__ uint64_t join2(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void split2(uint64_t v, float &a, float &b) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
}

// ---------------------------------------------------------------------------
// narrow: few rows
// ---------------------------------------------------------------------------
// Blocks `first`, first + 1, ... of x's BN rows from m0 on, quantised into the
// stages as TMA would put them there; a row's 16 bytes a lane, a team's next
// block on its way meanwhile.
template <int BN, typename X>
__device__ __forceinline__ void quantize_stages(const MmArgs &a, uint8_t *Cs, float *xsc, uint64_t *xs_full, uint64_t *full,
                                                uint64_t *empty, int m0, int first, int nkb) {
    using S = Narrow<BN, X>;
    constexpr int TEAMS = S::TEAMS, V = Vec16<X>::N, G = BK / V;            // lanes a row
    constexpr int SIDE = 32 * N_QUANT / TEAMS / G, N = BN / SIDE;           // rows at once, rows of a lane
    static_assert(BN % SIDE == 0 && N == 4, "whole passes; the rows that the teams' number is made for");
    const int t = ((int)threadIdx.x - 32 * QUANT_WARP) % (32 * N_QUANT / TEAMS), g = t / G, l = t % G;
    const int team = ((int)threadIdx.x / 32 - QUANT_WARP) / (N_QUANT / TEAMS);
    const X *rows = static_cast<const X *>(a.x) + (int64_t)(m0 + g) * a.ldx;
    uint4 u[N], n[N];
    const auto load = [&](int it) {
        const int c = (first + it) * BK + l * V, bytes = it < nkb ? max(0, min(V, a.K - c)) * (int)sizeof(X) : 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uintptr_t p = reinterpret_cast<uintptr_t>(rows + (int64_t)(i * SIDE) * a.ldx + c);
            const uint4 *at = reinterpret_cast<const uint4 *>(p & ~(uintptr_t)15);
            const bool any = bytes > 0 && m0 + g + i * SIDE < a.M;
            u[i] = n[i] = make_uint4(0, 0, 0, 0);
            if (any) u[i] = __ldg(at);
            if (any && (int)(p & 15u) + bytes > 16) n[i] = __ldg(at + 1);
        }
    };
    load(team);
    for (int it = team; it < nkb; it += TEAMS) {
        const int s = it % S::STAGES, c = (first + it) * BK + l * V;
        uint4 w[N];
        uint32_t mx[N];
        bool odd = false;                                  // something that is not finite
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uintptr_t p = reinterpret_cast<uintptr_t>(rows + (int64_t)(i * SIDE) * a.ldx + c);
            w[i] = first_bytes(shifted(u[i], n[i], (uint32_t)p & 15u), max(0, min(V, a.K - c)) * (int)sizeof(X));
            mx[i] = largest_any<X>(w[i]);
            odd |= mx[i] >= 0x7F800000u;
        }
        load(it + TEAMS);
        if (__any_sync(~0u, odd)) {
#pragma unroll
            for (int i = 0; i < N; ++i) mx[i] = largest<X, V>(w[i]);
        }
#pragma unroll
        for (int e = G / 2; e > 0; e /= 2)
#pragma unroll
            for (int i = 0; i < N; ++i) mx[i] = max(mx[i], __shfl_xor_sync(~0u, mx[i], e));
        if (!warp_wait(smem_u32(&empty[s]), ((uint32_t)(it / S::STAGES) & 1u) ^ 1u, a.err, E_TMA)) break;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = g + i * SIDE;
            float scale, inv;
            block_scale(mx[i], scale, inv);
            uint32_t q[V / 4];
            convert<X, V>(w[i], inv, q);
            uint8_t *to = Cs + s * S::C_BYTES + r * BK + ((l * V / 16) ^ (r & 7)) * 16 + l * V % 16;
            if constexpr (V == 8) *reinterpret_cast<uint2 *>(to) = make_uint2(q[0], q[1]);
            else *reinterpret_cast<uint32_t *>(to) = q[0];
            if (l == 0) xsc[it % X_SLOTS * BN + r] = scale;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (threadIdx.x % 32 == 0) {
            // the values for the MMAs, the scales for the epilogue: what reaches it by way of the MMAs' completion
            // orders only what they did
            mbar_arrive(smem_u32(&xs_full[it % X_SLOTS]));
            mbar_arrive(smem_u32(&full[s]));
        }
    }
}

template <int BN, typename X>
__global__ void __launch_bounds__((Narrow<BN, X>::THREADS), 1)
fp8_narrow_kernel(const __grid_constant__ CUtensorMap lmap, const __grid_constant__ CUtensorMap cmap, const MmArgs a) {
    using S = Narrow<BN, X>;
    constexpr bool QUANT = S::QUANT;
    constexpr int CPW = S::CPW, LDN = S::LDN, STAGES = S::STAGES, NBUF = S::NBUF, GROUPS = S::GROUPS;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t *Ls = smem;
    uint8_t *Cs = Ls + STAGES * L_BYTES;
    float *fac = (float *)(Cs + STAGES * S::C_BYTES);
    uint64_t *full = (uint64_t *)((uint8_t *)fac + S::FAC);
    uint64_t *empty = full + STAGES;
    uint64_t *acc_full = empty + STAGES;
    uint64_t *acc_empty = acc_full + NBUF;
    uint32_t *tmem_holder = (uint32_t *)(acc_empty + NBUF);
    // QUANT: a barrier for each slot's scales, [slot][row], of x's blocks
    uint64_t *xs_full = (uint64_t *)(tmem_holder + 4);
    float *xsc = (float *)(xs_full + X_SLOTS);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)(blockIdx.x % (unsigned)a.splits);
    const int tile = (int)(blockIdx.x / (unsigned)a.splits);
    const int tl = tile % a.tiles_l, tc = tile / a.tiles_l;
    const int kb0 = (int)((int64_t)a.KB * rank / a.splits), kb1 = (int)((int64_t)a.KB * (rank + 1) / a.splits);
    const int nkb = kb1 - kb0;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(smem_u32(&full[s]), 1 + (QUANT ? N_QUANT / S::TEAMS : 0));
            mbar_init(smem_u32(&empty[s]), 1);
        }
        for (int b = 0; b < NBUF; ++b) {
            mbar_init(smem_u32(&acc_full[b]), 1);
            mbar_init(smem_u32(&acc_empty[b]), N_EPI / GROUPS);
        }
        if (QUANT)
            for (int i = 0; i < X_SLOTS; ++i) mbar_init(smem_u32(&xs_full[i]), N_QUANT / S::TEAMS);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == MMA_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)),
                     "r"((uint32_t)S::TMEM_COLS));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *tmem_holder;
    pdl_trigger();

    if (warp == TMA_WARP) {
        const auto load_l = [&](int i) {
            const int s = i % STAGES;
            mbar_arrive_expect_tx(smem_u32(&full[s]), (uint32_t)(QUANT ? L_BYTES : S::STAGE));
            tma_load_2d(smem_u32(Ls + s * L_BYTES), &lmap, smem_u32(&full[s]), (kb0 + i) * BK, tl * BL);
        };
        const auto load_c = [&](int i) {
            const int s = i % STAGES;
            if (!QUANT) tma_load_2d(smem_u32(Cs + s * S::C_BYTES), &cmap, smem_u32(&full[s]), (kb0 + i) * BK, tc * BN);
        };
        // the weights of the first stages may be on their way while the kernel before still quantises x
        const int ahead = a.early ? min(STAGES, nkb) : 0;
        if (elect_one()) {
            for (int i = 0; i < ahead; ++i) load_l(i);
            pdl_wait();
            for (int i = 0; i < ahead; ++i) load_c(i);
            int it = ahead;
            for (; it < nkb; ++it) {
                if (!mbar_wait(smem_u32(&empty[it % STAGES]), ((uint32_t)(it / STAGES) & 1u) ^ 1u, a.err, E_TMA)) break;
                load_l(it);
                load_c(it);
            }
            // No copy and no commit is under way when the CTA ends: the last
            // use of each stage has been released (or, after a wait that ran
            // out, its copies have landed).
            for (int j = max(0, it - STAGES); j < it; ++j)
                mbar_wait(smem_u32(it < nkb ? &full[j % STAGES] : &empty[j % STAGES]), (uint32_t)(j / STAGES) & 1u, a.err,
                          E_DRAIN);
        }
        __syncwarp();
    } else if (warp == MMA_WARP) {
        pdl_wait();                                        // its waits' limits do not run while the kernel before works
        constexpr uint32_t idesc = idesc_e4m3(BL, BN);
        if (elect_one()) {
            for (int it = 0; it < nkb; ++it) {
                const int s = it % STAGES, b = it % NBUF;
                if (!mbar_wait(smem_u32(&acc_empty[b]), ((uint32_t)(it / NBUF) & 1u) ^ 1u, a.err, E_ACC) ||
                    !mbar_wait(smem_u32(&full[s]), (uint32_t)(it / STAGES) & 1u, a.err, E_MMA))
                    break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint64_t ld = smem_desc_sw128(smem_u32(Ls + s * L_BYTES));
                const uint64_t cd = smem_desc_sw128(smem_u32(Cs + s * S::C_BYTES));
#pragma unroll
                for (int k = 0; k < BK / 32; ++k)
                    umma_e4m3(tmem + (uint32_t)(b * BN), ld + 2 * k, cd + 2 * k, idesc, k > 0 ? 1u : 0u);
                umma_commit(smem_u32(&acc_full[b]));
                umma_commit(smem_u32(&empty[s]));
            }
        }
        __syncwarp();
    } else if (QUANT && warp >= QUANT_WARP) {
        pdl_wait();
        if constexpr (QUANT) quantize_stages<BN, X>(a, Cs, xsc, xs_full, full, empty, tc * BN, kb0, nkb);
    } else {
        pdl_wait();
        const int quad = warp & 3, half = warp >> 2;
        const int row = quad * 32 + lane;                  // lane row of this thread within the tile
        const int cw = GROUPS == 1 ? half * CPW : 0;       // first of this warp's columns in the tile
        const int c0 = tc * BN + cw;                       // ... its row of x
        const uint32_t tbase = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)cw;
        uint64_t acc[CPW / 2];
#pragma unroll
        for (int i = 0; i < CPW / 2; ++i) acc[i] = 0;

        // scales of this warp's next blocks: lane j holds column j's, and the
        // warp shares the products through shared memory
        constexpr int NF = (CPW + 31) / 32;
        const int first = GROUPS == 1 ? 0 : half;
        float nx[AHEAD][NF], nw[AHEAD];
        const float *xp[NF];
        bool xin[NF];
#pragma unroll
        for (int j = 0; j < NF; ++j) {
            const int m = c0 + j * 32 + lane;
            xin[j] = j * 32 + lane < CPW && m < a.M;
            xp[j] = a.xs + (int64_t)(xin[j] ? m : 0) * a.xs_row;
        }
        const float *wp = a.ws + (int64_t)tl * a.ws_row;
        const auto fetch = [&](int i) {
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const bool in = i + u * GROUPS < nkb;
                const int64_t kb = kb0 + i + u * GROUPS;
#pragma unroll
                for (int j = 0; j < NF; ++j) nx[u][j] = QUANT ? 1.f : in && xin[j] ? __ldg(xp[j] + kb * a.xs_blk) : 0.f;
                nw[u] = in ? __ldg(wp + kb * a.ws_blk) : 0.f;
            }
        };
        fetch(first);

        bool ok = true;
        for (int its = first; its < nkb && ok; its += AHEAD * GROUPS) {
            float f[AHEAD][NF];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
#pragma unroll
                for (int j = 0; j < NF; ++j) f[u][j] = nx[u][j] * nw[u];
            if (its + AHEAD * GROUPS < nkb) fetch(its + AHEAD * GROUPS);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int it = its + u * GROUPS, b = it % NBUF;
                if (it >= nkb) break;
                float *fs = fac + (warp * 2 + (u & 1)) * CPW;
                if (QUANT) {                               // x's scales, which come before the block's products
                    ok = warp_wait(smem_u32(&xs_full[it % X_SLOTS]), (uint32_t)(it / X_SLOTS) & 1u, a.err, E_EPI);
                    if (!ok) break;
                }
#pragma unroll
                for (int j = 0; j < NF; ++j)
                    if (j * 32 + lane < CPW)
                        fs[j * 32 + lane] = QUANT ? f[u][j] * xsc[it % X_SLOTS * BN + cw + j * 32 + lane] : f[u][j];
                __syncwarp();
                ok = warp_wait(smem_u32(&acc_full[b]), (uint32_t)(it / NBUF) & 1u, a.err, E_EPI);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                for (int c = 0; c < CPW; c += LDN) {
                    uint32_t r[LDN];
                    tmem_ld_nw<LDN>(tbase + (uint32_t)(b * BN + c), r);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < LDN; i += 4) {
                        const ulonglong2 q = *reinterpret_cast<const ulonglong2 *>(fs + c + i);
                        fma2(acc[(c + i) / 2], q.x, r[i], r[i + 1]);
                        fma2(acc[(c + i) / 2 + 1], q.y, r[i + 2], r[i + 3]);
                    }
                }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&acc_empty[b]));
            }
        }
        // Partial sums [column][lane row], over the stages: once both halves
        // are here every copy has landed and every MMA has read it.  (After a
        // wait that ran out, which is reported, the output is invalid.)
        float *part = (float *)smem;
        const auto put = [&](bool add) {
#pragma unroll
            for (int i = 0; i < CPW / 2; ++i) {
                float u, v;
                split2(acc[i], u, v);
                float *p = part + (cw + 2 * i) * BL + row;
                p[0] = add ? p[0] + u : u;
                p[BL] = add ? p[BL] + v : v;
            }
        };
        asm volatile("bar.sync 1, %0;" ::"n"(N_EPI * 32) : "memory");
        if (GROUPS == 1 || half == 1) put(false);
        if (GROUPS == 2) {
            asm volatile("bar.sync 1, %0;" ::"n"(N_EPI * 32) : "memory");
            if (half == 0) put(true);
        }
    }
    __syncwarp();
    cluster_sync();
    if (warp < N_EPI) {
        // this CTA finishes its share of the tile's columns: a warp a column, 4 lane rows a thread
        const int l = tl * BL + 4 * lane;
        const int cols = min(BN, a.M - tc * BN);
        float bias[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) bias[i] = a.bias != nullptr && l + i < a.N ? __ldg(a.bias + l + i) : 0.f;
#pragma unroll 2
        for (int c = rank * N_EPI + warp; c < cols; c += a.splits * N_EPI) {
            const uint32_t at = smem_u32((const float *)smem + c * BL + 4 * lane);
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
            for (int s = 0; s < a.splits; ++s) {
                const float4 p = ld_cluster_f32x4(mapa_shared(at, (uint32_t)s));
                v.x += p.x; v.y += p.y; v.z += p.z; v.w += p.w;
            }
            const float f[4] = {v.x + bias[0], v.y + bias[1], v.z + bias[2], v.w + bias[3]};
            store4(a, (int64_t)(tc * BN + c) * a.ldy + l, f, a.N - l);
        }
    }
    cluster_sync();                                        // no CTA leaves while its sums may still be read
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == MMA_WARP) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)S::TMEM_COLS));
    }
}

// ---------------------------------------------------------------------------
// wide: CTA pairs
// ---------------------------------------------------------------------------
constexpr int W_THREADS = 384;       // warps 0-7 epilogue, 8 TMA, 9 MMA, 10-11 scales
constexpr int SCALE_WARP = 10, N_SCALE = 2;

// registers a thread after the split: 2 x 224 + 56 for three warpgroups that
// were launched with 168 each (3 x 168 = 504)
constexpr int W_REGS_EPI = 224, W_REGS_REST = 56;
constexpr int W_BOX_BYTES = 32 * 128;
constexpr int W_LINES_BYTES = 32 * 33 * 8;   // or a warp's rows where TMA does not address y

template <int BN> struct Wide {
    static constexpr int C_BYTES = BN / 2 * BK;            // this CTA's half of the column operand
    static constexpr int STAGES = BN == 256 ? 4 : BN == 192 ? 5 : 6;
    static constexpr int BOXES = 2;                        // epilogue: 32 rows of 128 bytes on their way to y, for each warp
    static constexpr int NBUF = BN >= 192 ? 2 : 4;         // accumulators
    static constexpr int TMEM = BN == 192 ? 512 : NBUF * BN;  // columns: a power of two
    static constexpr int FAC_SLOTS = 2 * NBUF;
    static constexpr int CPW = BN / 2;                     // columns of an epilogue warp
    static constexpr int LDN = BN == 64 ? 16 : BN == 192 ? 48 : 32;   // columns on their way together: an even number of times
    static constexpr int PITCH = BN + 4;                   // row of partial sums, in floats: 8 rows hit all banks
    static_assert(BL * PITCH * 4 <= STAGES * (L_BYTES + C_BYTES) + N_EPI * BOXES * W_BOX_BYTES,
                  "partial sums over the stages and boxes");
    static_assert(BOXES * W_BOX_BYTES <= W_LINES_BYTES, "one or the other");
    static constexpr size_t SMEM = 1024 + (size_t)STAGES * (L_BYTES + C_BYTES) + N_EPI * W_LINES_BYTES +
                                   FAC_SLOTS * 2 * BL * 4 + 8 * (2 * STAGES + 2 * NBUF + 1) + 16;
};

__device__ __forceinline__ void umma_e4m3_pair(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a), "l"(b), "r"(idesc), "r"(acc));
}

// Arrive on the even CTA's barrier.  Relaxed: what it orders is the TMEM reads
// before it (complete at their wait, then tcgen05.fence), not memory; a
// release would wait for the scale loads and output stores in flight.
__device__ __forceinline__ void mbar_arrive_relaxed(uint32_t bar_cluster) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar_cluster) : "memory");
}

__device__ __forceinline__ void tma_store_2d(const CUtensorMap *map, uint32_t src, int x, int y) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"((uint64_t)map),
                 "r"(src), "r"(x), "r"(y)
                 : "memory");
}

// tile -> (row tile, column tile): `group` row tiles are walked together, so
// that the pairs at work share operand tiles in L2
__device__ __forceinline__ void tile_at(const MmArgs &a, int t, int &l, int &c) {
    const int per = a.group * a.tiles_c;
    const int g = t / per, r = t % per;
    const int rows = min(a.group, a.tiles_l - g * a.group);
    l = g * a.group + r % rows;
    c = r / rows;
}

// bias and activation on a thread's row, as passes of their own: the code of
// a tile's end runs once in thousands of cycles, so what it does not need
// should not be fetched with it
template <int CPW> __device__ __forceinline__ void finish_row(const MmArgs &a, uint64_t *acc, int c0) {
    if (a.bias != nullptr) {
#pragma unroll
        for (int i = 0; i < CPW / 2; ++i) {
            float u, v;
            split2(acc[i], u, v);
            u += __ldg(a.bias + min(c0 + 2 * i, a.N - 1));
            v += __ldg(a.bias + min(c0 + 2 * i + 1, a.N - 1));
            acc[i] = join2(u, v);
        }
    }
    if (a.relu) {
#pragma unroll
        for (int i = 0; i < CPW / 2; ++i) {
            float u, v;
            split2(acc[i], u, v);
            acc[i] = join2(relu_keep_nan(u), relu_keep_nan(v));
        }
    }
}

// Rows of y that TMA can address, of whole 16-byte units: through shared memory in boxes of 32 rows
// by COLS columns, 128 bytes (64 where the warp's columns are fewer), swizzled
// so that the 16-byte pieces of 8 rows hit 8 bank groups, stored by TMA,
// which clips what lies past the ends, while the next tile's products are added.
template <typename O, int CPW, int BOXES>
__device__ __forceinline__ void store_boxes(const MmArgs &a, const CUtensorMap *ymap, const uint64_t *acc, uint8_t *boxes,
                                            uint32_t &stored, int m_warp, int c0, int lane) {
    constexpr int COLS = CPW % (128 / (int)sizeof(O)) == 0 ? 128 / (int)sizeof(O) : 32;
    constexpr int PER16 = 16 / (int)sizeof(O);             // values of 16 bytes
    constexpr int PIECES = COLS / PER16;                   // 16-byte pieces of a box row
    static_assert((PIECES == 8 || PIECES == 4) && CPW % COLS == 0, "box rows of 128 or 64 bytes");
    const int swz = PIECES == 8 ? lane & 7 : (lane >> 1) & 3;
#pragma unroll
    for (int c = 0; c < CPW; c += COLS) {
        if (c0 + c >= a.N) break;
        uint8_t *box = boxes + stored++ % BOXES * W_BOX_BYTES;
        // the store before from this box has been read
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(BOXES - 1) : "memory");
        __syncwarp();
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            float v[PER16];
#pragma unroll
            for (int i = 0; i < PER16 / 2; ++i) split2(acc[(c + j * PER16) / 2 + i], v[2 * i], v[2 * i + 1]);
            *reinterpret_cast<uint4 *>(box + lane * (PIECES * 16) + ((j ^ swz) * 16)) = pack16<O>(v);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
            if (m_warp < a.M) tma_store_2d(ymap, smem_u32(box), c0 + c, m_warp);
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
    }
}

// Rows that start or end anywhere: segments of 256 bytes of a row (fewer where the
// warp's columns are fewer) through shared memory.  A lane moves its row up to
// its place in the aligned 8-byte units of y, then the warp stores rows of
// units, and what is left at a segment's ends value by value.  Few instructions
// decide: two warps a scheduler are all that run here, and the products of the
// next tile wait.  (4170 x 7300 x 1018 to 16 bits: 56.7 us with single values
// from 32 x 32 squares, 48.9 us with the shift at the second step, 41.4 us this
// way, 34.5 us where TMA can address the rows, with 7296 columns.)
template <typename O, int CPW>
__device__ __forceinline__ void store_lines(const MmArgs &a, const uint64_t *acc, uint64_t *sq, int m_warp, int c0, int lane) {
    constexpr int PER8 = 8 / (int)sizeof(O);               // values of a unit
    constexpr int MOST = 256 / (int)sizeof(O) < CPW ? 256 / (int)sizeof(O) : CPW;
    constexpr int COLS = CPW % MOST == 0 ? MOST : CPW / 2;
    constexpr int UNITS = COLS / PER8, STEP = 32 / UNITS;  // rows of one store
    constexpr int PITCH = UNITS + 1;                       // odd: neither side hits a bank twice
    static_assert(CPW % COLS == 0 && UNITS <= 32 && UNITS % 8 == 0, "segments of whole units");
    static_assert(32 * PITCH * 8 <= W_LINES_BYTES, "a segment of 32 rows");
    const int rows = min(32, a.M - m_warp);
    const int64_t pitch = a.ldy * (int)sizeof(O);
#pragma unroll
    for (int c = 0; c < CPW; c += COLS) {
        if (c0 + c >= a.N) break;
        const uintptr_t y = reinterpret_cast<uintptr_t>(static_cast<O *>(a.y) + (int64_t)m_warp * a.ldy + c0 + c);
        {
            const uint32_t off = (uint32_t)(y + lane * pitch) & 7u, bits = (off & 3u) * 8u;
            uint32_t last = 0, moved = 0;                  // the word before, as it was and as it became
#pragma unroll
            for (int u = 0; u <= UNITS; ++u) {
                float v[PER8];
                uint64_t piece = 0;
                if (u < UNITS) {
#pragma unroll
                    for (int i = 0; i < PER8 / 2; ++i) split2(acc[(c + u * PER8) / 2 + i], v[2 * i], v[2 * i + 1]);
                    piece = pack8<O>(v);
                }
                const uint32_t w0 = (uint32_t)piece, w1 = (uint32_t)(piece >> 32);
                const uint32_t m0 = __funnelshift_l(last, w0, bits), m1 = __funnelshift_l(w0, w1, bits);
                sq[lane * PITCH + u] = off & 4u ? (uint64_t)m0 << 32 | moved : (uint64_t)m1 << 32 | m0;
                last = w1;
                moved = m1;
            }
        }
        __syncwarp();
        const int have = min(COLS, a.N - c0 - c);
        {
            const int u = lane % UNITS;
            uintptr_t row = y + lane / UNITS * pitch;
            const uint64_t *src = sq + lane / UNITS * PITCH + u;
#pragma unroll 4
            for (int r = lane / UNITS; r < rows; r += STEP, row += STEP * pitch, src += STEP * PITCH) {
                const int off = (int)(row & 7u);
                if (lane < STEP * UNITS && u * 8 >= off && u * 8 + 8 <= off + have * (int)sizeof(O))
                    *reinterpret_cast<uint64_t *>((row & ~(uintptr_t)7) + u * 8) = *src;
            }
        }
        if ((((uint32_t)y | (uint32_t)pitch | (uint32_t)(have * (int)sizeof(O))) & 7u) != 0) {
            // values of the first and the last unit, where not whole
            constexpr int ENDS = 2 * PER8;
            const int e = lane % ENDS;
            for (int r = lane / ENDS; r < rows; r += 32 / ENDS) {
                const uintptr_t row = y + r * pitch;
                const int off = (int)(row & 7u) / (int)sizeof(O), end = off + have;
                const int i = e < PER8 ? (off > 0 ? e : -1) : end / PER8 * PER8 + e - PER8;
                if (i >= off && i < end)
                    reinterpret_cast<O *>(row & ~(uintptr_t)7)[i] = reinterpret_cast<const O *>(sq + r * PITCH)[i];
            }
        }
        __syncwarp();
    }
}

// A CTA's share of the columns of its rows, added over the cluster's pairs in
// their order.  A function of its own: inlined, it costs the kernel's main loop
// registers.
template <int BN>
__device__ __noinline__ void finish_split(const MmArgs &a, uint32_t part, int tile, uint32_t crank, uint32_t pair) {
    const int width = BN / a.splits, lanes = width / 4;    // a row's, 4 columns a thread
    int tl, tc;
    tile_at(a, tile, tl, tc);
    const int c = (int)pair * width + (int)threadIdx.x % lanes * 4, n = tc * BN + c;
    if (n >= a.N) return;
    const int m0 = (2 * tl + (int)crank) * BL;
    float bias[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) bias[i] = a.bias != nullptr && n + i < a.N ? __ldg(a.bias + n + i) : 0.f;
    const int step = N_EPI * 32 / lanes;
#pragma unroll 2
    for (int row = (int)threadIdx.x / lanes; row < min(BL, a.M - m0); row += step) {
        const uint32_t at = part + (uint32_t)(row * Wide<BN>::PITCH + c) * 4u;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
        for (int s = 0; s < a.splits; ++s) {
            const float4 p = ld_cluster_f32x4(mapa_shared(at, (uint32_t)(2 * s) + crank));
            v.x += p.x; v.y += p.y; v.z += p.z; v.w += p.w;
        }
        const float f[4] = {v.x + bias[0], v.y + bias[1], v.z + bias[2], v.w + bias[3]};
        store4(a, (int64_t)(m0 + row) * a.ldy + n, f, a.N - n);
    }
}

template <int BN, bool SPLIT>
__global__ void __launch_bounds__(W_THREADS, 1)
fp8_wide_kernel(const __grid_constant__ CUtensorMap lmap, const __grid_constant__ CUtensorMap cmap,
                const __grid_constant__ CUtensorMap ymap, const MmArgs a) {
    using S = Wide<BN>;
    constexpr int CPW = S::CPW, LDN = S::LDN, NBUF = S::NBUF, FAC_SLOTS = S::FAC_SLOTS;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t *Ls = smem;
    uint8_t *Cs = Ls + S::STAGES * L_BYTES;
    uint8_t *boxes = Cs + S::STAGES * S::C_BYTES;
    float *fac = (float *)(boxes + N_EPI * W_LINES_BYTES);   // [slot][column half][row]: scale of a block's sums
    uint64_t *full = (uint64_t *)(fac + FAC_SLOTS * 2 * BL);   // even CTA's: both CTAs' copies of a stage
    uint64_t *empty = full + S::STAGES;                    // each CTA: the pair's MMAs have read the stage
    uint64_t *acc_full = empty + S::STAGES;                // each CTA: a block's products are in TMEM, its scales in fac
    uint64_t *acc_empty = acc_full + NBUF;                   // even CTA's: both CTAs' epilogues have read them
    uint64_t *mma_done = acc_empty + NBUF;
    uint32_t *tmem_holder = (uint32_t *)(mma_done + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // SPLIT: a cluster is `splits` pairs, which share one tile's K blocks
    const uint32_t crank = cluster_ctarank() & 1u, pair = SPLIT ? cluster_ctarank() >> 1 : 0u, even = 2u * pair;
    const bool leader = crank == 0;
    const uint16_t both = (uint16_t)(3u << even);
    const unsigned ctas = SPLIT ? 2u * (unsigned)a.splits : 2u;
    const int cid = (int)(blockIdx.x / ctas), ncl = (int)(gridDim.x / ctas);
    const int tiles = a.tiles_l * a.tiles_c;
    const int kb0 = SPLIT ? (int)((int64_t)a.KB * pair / a.splits) : 0;     // this pair's
    const int KB = SPLIT ? (int)((int64_t)a.KB * (pair + 1) / a.splits) - kb0 : a.KB;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; ++s) {
            mbar_init(smem_u32(&full[s]), 1);
            mbar_init(smem_u32(&empty[s]), 1);
        }
        for (int b = 0; b < NBUF; ++b) {
            mbar_init(smem_u32(&acc_full[b]), 1 + N_SCALE);
            mbar_init(smem_u32(&acc_empty[b]), 2 * N_EPI);
        }
        mbar_init(smem_u32(mma_done), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == MMA_WARP) {
        // one warp of each CTA of the pair allocates the same columns in both
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)),
                     "r"((uint32_t)S::TMEM));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync();                                        // the peer's barriers exist before anything targets them
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *tmem_holder;
    pdl_wait();
    pdl_trigger();

    if (warp >= N_EPI) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(W_REGS_REST));
        if (warp == TMA_WARP) {
            const uint32_t full_even = mapa_shared(smem_u32(full), even);
            if (elect_one()) {
                int it = 0;
                bool ok = true;
                for (int t = cid; t < tiles && ok; t += ncl) {
                    int tl, tc;
                    tile_at(a, t, tl, tc);
                    const int m0 = (2 * tl + (int)crank) * BL, n0 = tc * BN + (int)crank * (BN / 2);
                    for (int kb = 0; kb < KB; ++kb, ++it) {
                        const int s = it % S::STAGES;
                        ok = mbar_wait(smem_u32(&empty[s]), ((uint32_t)(it / S::STAGES) & 1u) ^ 1u, a.err, E_TMA);
                        if (!ok) break;
                        const uint32_t fb = full_even + (uint32_t)(s * 8);
                        if (leader) mbar_arrive_expect_tx(smem_u32(&full[s]), 2u * (L_BYTES + S::C_BYTES));
                        tma_load_2d_pair(smem_u32(Ls + s * L_BYTES), &lmap, fb, (kb0 + kb) * BK, m0);
                        tma_load_2d_pair(smem_u32(Cs + s * S::C_BYTES), &cmap, fb, (kb0 + kb) * BK, n0);
                    }
                }
                // no copy and no commit is under way when the CTA ends, see the narrow kernel (the even CTA's
                // barriers count both CTAs' copies)
                if (ok || leader)
                    for (int j = max(0, it - S::STAGES); j < it; ++j)
                        mbar_wait(smem_u32(ok ? &empty[j % S::STAGES] : &full[j % S::STAGES]),
                                  (uint32_t)(j / S::STAGES) & 1u, a.err, E_DRAIN);
            }
        } else if (warp >= SCALE_WARP) {
            // Scale loads take up to 1000 cycles while the tiles stream, so
            // these warps make them DEPTH blocks ahead: 2 rows a lane, both
            // column halves.  Block `it` goes to slot it % (2 NBUF) once block
            // it - NBUF is complete: the epilogue has then read block
            // it - 2 NBUF's TMEM, and before it the slot.
            constexpr int DEPTH = 4;
            const int r0 = (warp - SCALE_WARP) * (BL / N_SCALE) + lane;
            int it = 0;
            bool ok = true;
            for (int t = cid; t < tiles && ok; t += ncl) {
                int tl, tc;
                tile_at(a, t, tl, tc);
                const int m0 = (2 * tl + (int)crank) * BL + r0, last = (a.N - 1) / 128;
                const float *xp[2], *wp[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    xp[i] = a.xs + (int64_t)min(m0 + 32 * i, a.M - 1) * a.xs_row + kb0 * a.xs_blk;
                    wp[i] = a.ws + (int64_t)min(BN == 192 ? tc * BN / 128 + i : (tc * BN + i * CPW) / 128, last) * a.ws_row +
                            kb0 * a.ws_blk;
                }
                float x[DEPTH][2], w[DEPTH][2];
                const auto load = [&](int kb, int u) {
                    if (kb < KB) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            x[u][i] = __ldg(xp[i] + kb * a.xs_blk);
                            w[u][i] = __ldg(wp[i] + kb * a.ws_blk);
                        }
                    }
                };
#pragma unroll
                for (int u = 0; u < DEPTH; ++u) load(u, u);
                for (int kb = 0; kb < KB && ok; kb += DEPTH) {
#pragma unroll
                    for (int u = 0; u < DEPTH; ++u, ++it) {
                        if (kb + u >= KB) break;
                        ok = it < NBUF || warp_wait(smem_u32(&acc_full[it % NBUF]), (uint32_t)(it / NBUF - 1) & 1u, a.err, E_EPI);
                        if (!ok) break;
                        float *slot = fac + it % FAC_SLOTS * (2 * BL) + r0;
#pragma unroll
                        for (int q = 0; q < 2; ++q)
#pragma unroll
                            for (int i = 0; i < 2; ++i) slot[q * BL + 32 * i] = x[u][i] * w[u][q];
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&acc_full[it % NBUF]));
                        load(kb + u + DEPTH, u);
                    }
                }
            }
        } else if (warp == MMA_WARP && leader) {
            constexpr uint32_t idesc = idesc_e4m3(2 * BL, BN);
            if (elect_one()) {
                // this pair's blocks, all tiles in a row
                const int64_t all = (int64_t)((tiles - cid + ncl - 1) / ncl) * KB;
                int s = 0, round = 0;                      // stage, times it was used before
                for (int64_t it = 0; it < all; ++it) {
                    const int b = (int)(it % NBUF);
                    if (!mbar_wait(smem_u32(&full[s]), (uint32_t)round & 1u, a.err, E_MMA) ||
                        !mbar_wait(smem_u32(&acc_empty[b]), ((uint32_t)(it / NBUF) & 1u) ^ 1u, a.err, E_ACC))
                        break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t ld = smem_desc_sw128(smem_u32(Ls + s * L_BYTES));
                    const uint64_t cd = smem_desc_sw128(smem_u32(Cs + s * S::C_BYTES));
#pragma unroll
                    for (int k = 0; k < BK / 32; ++k)
                        umma_e4m3_pair(tmem + (uint32_t)(b * BN), ld + 2 * k, cd + 2 * k, idesc, k > 0 ? 1u : 0u);
                    umma_commit_pair_mc(smem_u32(&acc_full[b]), both);
                    umma_commit_pair_mc(smem_u32(&empty[s]), both);
                    if (++s == S::STAGES) { s = 0; ++round; }
                }
                umma_commit_pair_mc(smem_u32(mma_done), both);
            }
        }
        __syncwarp();
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(W_REGS_EPI));
        const int quad = warp & 3, half = warp >> 2;
        const uint32_t tbase = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(half * CPW);
        const uint32_t acc_empty_even = mapa_shared(smem_u32(acc_empty), even);
        uint8_t *mine = boxes + warp * S::BOXES * W_BOX_BYTES;
        const float *my_fac = fac + (BN == 192 ? 0 : half * BL) + quad * 32 + lane;
        uint32_t stored = 0;                               // boxes this warp has stored
        uint32_t it = 0;
        bool ok = true;
        for (int t = cid; t < tiles && ok; t += ncl) {
            int tl, tc;
            tile_at(a, t, tl, tc);
            const int m_warp = (2 * tl + (int)crank) * BL + quad * 32;
            // the warp's columns lie inside one 128-row block of w, or, 192 wide, in the tile's first up to
            // its 32-column group `turn` and from there on in the second
            const int c0 = tc * BN + half * CPW;
            const int turn = (128 - tc * BN % 128 - half * CPW) / 32;
            uint64_t acc[CPW / 2];
#pragma unroll
            for (int i = 0; i < CPW / 2; ++i) acc[i] = 0;

            uint32_t r[2][LDN];
            ok = warp_wait(smem_u32(&acc_full[(it & (NBUF - 1))]), (uint32_t)(it / NBUF) & 1u, a.err, E_EPI);
            if (!SPLIT && !ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            if (!SPLIT || ok) tmem_ld_nw<LDN>(tbase + (uint32_t)((it & (NBUF - 1)) * BN), r[0]);
            for (int kb = 0; kb < KB && ok; ++kb, ++it) {
                const uint32_t src = tbase + (uint32_t)((it & (NBUF - 1)) * BN);
                constexpr int GROUPS = BN == 192 ? 3 : 1;
                uint64_t f[GROUPS];
                const float first = my_fac[(it & (FAC_SLOTS - 1)) * (2 * BL)];
                f[0] = dup2(first);
                if constexpr (BN == 192) {
                    const float second = my_fac[(it & (FAC_SLOTS - 1)) * (2 * BL) + BL];
#pragma unroll
                    for (int g = 0; g < GROUPS; ++g) f[g] = dup2(g < turn ? first : second);
                }
                // LDN columns are on their way while the LDN before are added,
                // across blocks too
#pragma unroll
                for (int c = 0; c < CPW; c += LDN) {
                    const int h = c / LDN & 1;
                    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                    if (c + LDN < CPW) {
                        tmem_ld_nw<LDN>(src + (uint32_t)(c + LDN), r[h ^ 1]);
                    } else {
                        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) mbar_arrive_relaxed(acc_empty_even + (uint32_t)((it & (NBUF - 1)) * 8));
                        if (kb + 1 < KB) {
                            ok = warp_wait(smem_u32(&acc_full[((it + 1) & (NBUF - 1))]), (uint32_t)((it + 1) / NBUF) & 1u,
                                           a.err, E_EPI);
                            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                            if (ok) tmem_ld_nw<LDN>(tbase + (uint32_t)(((it + 1) & (NBUF - 1)) * BN), r[h ^ 1]);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < LDN / 2; ++i)
                        fma2(acc[c / 2 + i], f[GROUPS == 1 ? 0 : (c + 2 * i) / 32], r[h][2 * i], r[h][2 * i + 1]);
                }
            }
            // After a wait that ran out, which is reported, the output is invalid;
            // a split tile's warps still meet at their barriers.
            if (!SPLIT && !ok) break;

            if constexpr (SPLIT) {
                // partial sums [row][column], over the stages and boxes (see the narrow kernel); one tile
                float *part = (float *)smem + (quad * 32 + lane) * S::PITCH + half * CPW;
                asm volatile("bar.sync 1, %0;" ::"n"(N_EPI * 32) : "memory");
#pragma unroll
                for (int i = 0; i < CPW / 2; i += 2)
                    *reinterpret_cast<ulonglong2 *>(part + 2 * i) = make_ulonglong2(acc[i], acc[i + 1]);
            } else {
                finish_row<CPW>(a, acc, c0);
                if (a.vec) {
                    if (a.out == CT_DT_F32) store_boxes<float, CPW, S::BOXES>(a, &ymap, acc, mine, stored, m_warp, c0, lane);
                    else if (a.out == CT_DT_F16)
                        store_boxes<__half, CPW, S::BOXES>(a, &ymap, acc, mine, stored, m_warp, c0, lane);
                    else
                        store_boxes<__nv_bfloat16, CPW, S::BOXES>(a, &ymap, acc, mine, stored, m_warp, c0, lane);
                } else {
                    uint64_t *lines = (uint64_t *)(boxes + warp * W_LINES_BYTES);
                    if (a.out == CT_DT_F32) store_lines<float, CPW>(a, acc, lines, m_warp, c0, lane);
                    else if (a.out == CT_DT_F16) store_lines<__half, CPW>(a, acc, lines, m_warp, c0, lane);
                    else store_lines<__nv_bfloat16, CPW>(a, acc, lines, m_warp, c0, lane);
                }
            }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    __syncwarp();
    if constexpr (SPLIT) {
        cluster_sync();
        if (warp < N_EPI) finish_split<BN>(a, smem_u32(smem), cid, crank, pair);
    }
    __syncthreads();
    // every MMA of the pair has completed before TMEM is freed in either CTA,
    // and no CTA leaves while its peer may still arrive on its barriers
    if (warp == MMA_WARP) warp_wait(smem_u32(mma_done), 0u, a.err, E_DRAIN);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    cluster_sync();
    if (warp == MMA_WARP) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)S::TMEM));
    }
}

// y = act(bias) where K is 0
__global__ void bias_only_kernel(const MmArgs a) {
    pdl_wait();
    pdl_trigger();
    const int64_t n_all = (int64_t)a.M * a.N;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n_all; i += (int64_t)gridDim.x * blockDim.x) {
        const float v = a.bias != nullptr ? __ldg(a.bias + i % a.N) : 0.f;
        store_out(a, i / a.N * a.ldy + i % a.N, a.relu ? relu_keep_nan(v) : v);
    }
}

PFN_cuTensorMapEncodeTiled_v12000 encoder() {
    static std::atomic<PFN_cuTensorMapEncodeTiled_v12000> found{nullptr};
    PFN_cuTensorMapEncodeTiled_v12000 f = found.load(std::memory_order_relaxed);
    if (f == nullptr) {
        cudaDriverEntryPointQueryResult q;
        void *p = nullptr;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            return nullptr;
        f = (PFN_cuTensorMapEncodeTiled_v12000)p;
        found.store(f, std::memory_order_relaxed);
    }
    return f;
}

int64_t q_pitch(int64_t k) { return (k + 15) / 16 * 16; }

// [rows, cols] values of `size` bytes, row pitch ld bytes, in boxes of box_bytes (128 or 64) x box_rows, swizzled
// within box_bytes
bool encode(CUtensorMap *map, const void *p, CUtensorMapDataType type, int size, int64_t rows, int64_t cols, int64_t ld,
            int box_bytes, int box_rows) {
    PFN_cuTensorMapEncodeTiled_v12000 f = encoder();
    if (f == nullptr) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)ld};
    const cuuint32_t box[2] = {(cuuint32_t)(box_bytes / size), (cuuint32_t)box_rows};
    const cuuint32_t es[2] = {1, 1};
    return f(map, type, 2, const_cast<void *>(p), dims, strides, box, es,
             CU_TENSOR_MAP_INTERLEAVE_NONE, box_bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// (the pitch of a single row does not matter)
bool encode8(CUtensorMap *map, const uint8_t *p, int64_t rows, int64_t k, int64_t ld, int box_rows) {
    if (rows == 1) ld = q_pitch(k);
    return encode(map, p, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, rows, k, ld, BK, box_rows);
}

// (the kernels' shared memory was allowed when choose() asked for their residency)
template <int BN, typename X = uint8_t>
cudaError_t launch_narrow(const CUtensorMap &lmap, const CUtensorMap &cmap, const MmArgs &a, int grid, cudaStream_t st) {
    using S = Narrow<BN, X>;
    if (a.splits == 1)
        return pdl_launch(fp8_narrow_kernel<BN, X>, dim3((unsigned)grid), dim3(S::THREADS), S::SMEM, st, lmap, cmap, a);
    return pdl_launch_cluster(fp8_narrow_kernel<BN, X>, dim3((unsigned)grid), dim3(S::THREADS), S::SMEM, st, a.splits,
                              lmap, cmap, a);
}

template <int BN>
cudaError_t launch_wide(const CUtensorMap &lmap, const CUtensorMap &cmap, const CUtensorMap &ymap, const MmArgs &a,
                        int clusters, cudaStream_t st) {
    const dim3 grid((unsigned)(2 * a.splits * clusters)), block(W_THREADS);
    if (a.splits == 1)
        return pdl_launch_cluster(fp8_wide_kernel<BN, false>, grid, block, Wide<BN>::SMEM, st, 2, lmap, cmap, ymap, a);
    return pdl_launch_cluster(fp8_wide_kernel<BN, true>, grid, block, Wide<BN>::SMEM, st, 2 * a.splits, lmap, cmap, ymap, a);
}

struct Operands {
    const uint8_t *xq;
    int64_t ldx;
    const uint8_t *wq;
    int64_t ldw;
    int64_t k;
};

// CTAs of a kernel that device `dev`, the current one, holds at once in clusters of `cluster`, asked once:
// clusters must fit into a GPC, so it is not always the SMs' number.  0: it does not run.
template <typename K>
int resident(K *kernel, int threads, size_t smem, int cluster, std::atomic<int> &known) {
    int n = known.load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return 0;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)cluster);
        cfg.blockDim = dim3((unsigned)threads);
        cfg.dynamicSmemBytes = smem;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)cluster;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        int clusters = 0;
        if (cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg) != cudaSuccess || clusters < 1) {
            cudaGetLastError();
            return 0;
        }
        n = clusters * cluster;
        known.store(n, std::memory_order_relaxed);
    }
    return n;
}

constexpr int N_SPLITS = 6;
constexpr int NARROW_SPLITS[N_SPLITS] = {1, 2, 3, 4, 6, 8};

constexpr int W_COLS[4] = {64, 128, 192, 256};

// [dev][log2 of the columns / 16][index of the split], [dev][index of the columns][splits - 1]
std::atomic<int> g_narrow[MAX_DEVICES][4][N_SPLITS], g_wide[MAX_DEVICES][4][2];

template <int BN, typename X = uint8_t> int narrow_resident(int splits, std::atomic<int> &known) {
    return resident(fp8_narrow_kernel<BN, X>, Narrow<BN, X>::THREADS, Narrow<BN, X>::SMEM, splits, known);
}
template <int BN> int wide_resident(int splits, std::atomic<int> &known) {
    return splits == 1 ? resident(fp8_wide_kernel<BN, false>, W_THREADS, Wide<BN>::SMEM, 2, known)
                       : resident(fp8_wide_kernel<BN, true>, W_THREADS, Wide<BN>::SMEM, 2 * splits, known);
}

struct Choice {
    bool wide;
    int bn, splits;
    int ctas;               // that run at once
    double us;              // estimate
};

// figures of the estimate, see choose()
constexpr double N_BLOCK[4] = {0.2, 0.25, 0.33, 0.5}, N_TILE[4] = {1.0, 1.3, 2.7, 3.3};
constexpr double N_SPLIT[N_SPLITS] = {0, 1.4, 1.7, 2.0, 2.2, 2.2};

// of the narrow kernel with tiles of 16 << i columns and split q; `block`: a K block's us
double narrow_us(int M, int N, int KB, int sms, int i, int q, int ctas, double block) {
    const int bn = 16 << i, s = NARROW_SPLITS[q];
    const int64_t tiles = (int64_t)((N + 127) / 128) * ((M + bn - 1) / bn);
    const double nkb = (KB + s - 1) / s, all = (double)tiles * s, busy = all < sms ? all : sms;
    const double rounds = (double)((tiles * s + ctas - 1) / ctas);
    const double l2 = all * nkb * (BL + bn) * BK / 9e6;
    const double hbm = (double)N * KB * BK / (busy < 110 ? 58e3 * busy : 6.4e6);
    return rounds * N_TILE[i] + (rounds - 1) + N_SPLIT[q] + fmax(rounds * nkb * block, fmax(l2, hbm));
}

// Which kernel, how wide its tiles, over how many CTAs (pairs) K is split: the
// least of an estimate in us, whose figures were fitted to every candidate's
// times at 67 shapes.  At 72 shapes (1 to 8000 rows, 16 to 15618 columns, K from
// 64 to 25088) the choice is 4.3% slower than the best candidate on average,
// 48% at worst (8000 x 100 x 1000: 9.6 us in narrow tiles, 6.5 in wide ones).
//   A K block costs a CTA 0.2 to 0.5 us (16 to 128 columns), a pair 0.2 to
//   0.41 us (64 to 256; 192 a little less than 256, which counts where neither
//   fills its last round: 1777 x 2999 x 5003, two rounds of either, takes 40.8
//   and 44.8 us, 42.3 in 128 columns); launch, start and end of a tile 1 to 3.3
//   us, 3.9 to 4.8 us; adding the shares of a split 1.4 to 2.2 us, 3.5 us.
//   No kernel is faster than its operands: 9 to 11 bytes a ns from L2, 6.4 of
//   weights from HBM, 58 bytes a ns to one SM.
Choice choose(int M, int N, int KB, int sms, int dev) {
    static const double w_block[4] = {0.2, 0.28, 0.385, 0.41};
    Choice best = {false, 16, 1, 0, 1e30};
    const double weights = (double)N * KB * BK;
    const int64_t rows_n = (N + 127) / 128, rows_m = (M + 2 * BL - 1) / (2 * BL);
    for (int i = 0; i < 4; ++i) {
        const int bn = 16 << i;
        if (bn > 16 && bn / 2 >= M) break;
        const int64_t tiles = rows_n * ((M + bn - 1) / bn);
        for (int q = 0; q < N_SPLITS; ++q) {
            const int s = NARROW_SPLITS[q];
            if (s > KB || (s > 1 && tiles * s > sms)) break;
            std::atomic<int> &known = g_narrow[dev][i][q];
            const int ctas = bn == 16   ? narrow_resident<16>(s, known)
                             : bn == 32 ? narrow_resident<32>(s, known)
                             : bn == 64 ? narrow_resident<64>(s, known)
                                        : narrow_resident<128>(s, known);
            if (ctas == 0) continue;
            const double t = narrow_us(M, N, KB, sms, i, q, ctas, N_BLOCK[i]);
            if (t < best.us) best = Choice{false, bn, s, ctas, t};
        }
    }
    for (int i = 0; i < 4 && M > 64; ++i) {
        const int bn = W_COLS[i];
        const int64_t tiles = rows_m * ((N + bn - 1) / bn);
        for (int s = 1; s <= (bn == 192 ? 1 : 2) && s <= KB; ++s) {
            std::atomic<int> &known = g_wide[dev][i][s - 1];
            const int ctas = bn == 64    ? wide_resident<64>(s, known)
                             : bn == 128 ? wide_resident<128>(s, known)
                             : bn == 192 ? resident(fp8_wide_kernel<192, false>, W_THREADS, Wide<192>::SMEM, 2, known)
                                         : wide_resident<256>(s, known);
            const int64_t pairs = ctas / 2;
            if (ctas == 0 || (s > 1 && tiles * s > pairs)) continue;
            const double nkb = (KB + s - 1) / s, rounds = (double)((tiles * s + pairs - 1) / pairs);
            const double l2 = (double)tiles * s * nkb * (2 * BL + bn) * BK / 11e6;
            const double t = 3.6 + 0.0047 * bn + (s > 1 ? 3.5 : 0) +
                             fmax(rounds * nkb * w_block[i] + (rounds - 1) * 0.8, fmax(l2, weights / 6.4e6));
            if (t < best.us) best = Choice{true, bn, s, ctas, t};
        }
    }
    return best;
}

// The same for the kernels that quantise rows of X: one launch less (LAUNCH us),
// no 8-bit copy, but each CTA quantises the rows it multiplies, which sets the
// pace of long K: only tiles of 16 and 32 columns do.  In one launch and in two:
// 256 x 1000 x 512 FP16 5.1 and 6.0 us, 500 x 500 x 500 5.1 and 8.1, 1 x 4096 x
// 25088 20.0 and 21.3, 256 x 1000 x 4096 13.6 and 10.9.
constexpr double LAUNCH = 2.0;
constexpr double Q_BLOCK[2][2] = {{0.35, 0.65}, {0.5, 0.95}};   // 16-bit, FP32 rows
std::atomic<int> g_quant[MAX_DEVICES][3][2][N_SPLITS];     // [dev][type][log2 of the columns / 16][index of the split]

// It adds in the order that `two`, the choice for 8-bit rows, does: the same
// bits, so the same split of K over CTAs and, within one, over epilogue halves.
template <typename X> Choice choose_quantising(const Choice &two, int M, int N, int KB, int sms, int dev, int type) {
    Choice best = {false, 16, two.splits, 0, 1e30};
    if (two.ctas == 0 || two.wide || Narrow<16, X>::GROUPS != (two.bn <= 64 ? 2 : 1)) return best;
    int q = 0;
    while (NARROW_SPLITS[q] != two.splits) ++q;
    for (int i = 0; i < 2; ++i) {
        const int bn = 16 << i;
        if (bn > 16 && bn / 2 >= M) break;
        std::atomic<int> &known = g_quant[dev][type][i][q];
        const int ctas = bn == 16 ? narrow_resident<16, X>(two.splits, known) : narrow_resident<32, X>(two.splits, known);
        if (ctas == 0) continue;
        const double t = narrow_us(M, N, KB, sms, i, q, ctas, Q_BLOCK[sizeof(X) == 4][i]);
        if (t < best.us) best = Choice{false, bn, two.splits, ctas, t};
    }
    return best;
}

// The kernel that quantises and multiplies rows of `type` in one launch, where that is estimated to take less than a
// launch for each (`two`: the product's); ctas = 0: it is not.
Choice choose_one_launch(const Choice &two, int M, int N, int64_t k, int dev, int type) {
    const int KB = (int)((k + BK - 1) / BK), sms = sm_count();
    Choice ch = type == CT_DT_F32   ? choose_quantising<float>(two, M, N, KB, sms, dev, 0)
                : type == CT_DT_F16 ? choose_quantising<__half>(two, M, N, KB, sms, dev, 1)
                                    : choose_quantising<__nv_bfloat16>(two, M, N, KB, sms, dev, 2);
    const double apart = two.us + LAUNCH + (double)M * k * (dtype_size(type) + 1) / 6e6;
    const int64_t tiles = (int64_t)((N + 127) / 128) * ((M + ch.bn - 1) / ch.bn);
    if (ch.us >= apart || tiles > INT32_MAX / 16) ch.ctas = 0;
    return ch;
}

template <typename X> ct_status quantise_and_multiply(MmArgs a, const Operands &o, const Choice &ch, cudaStream_t st) {
    a.tiles_l = (a.N + 127) / 128;
    a.tiles_c = (a.M + ch.bn - 1) / ch.bn;
    a.splits = ch.splits;
    a.err = device_error_word();
    CUtensorMap lmap;
    if (a.err == nullptr || !encode8(&lmap, o.wq, a.N, o.k, o.ldw, BL)) return CT_ECUDA;
    const int grid = a.tiles_l * a.tiles_c * a.splits;
    const cudaError_t e = ch.bn == 16 ? launch_narrow<16, X>(lmap, lmap, a, grid, st) : launch_narrow<32, X>(lmap, lmap, a, grid, st);
    return e == cudaSuccess ? CT_OK : CT_ECUDA;
}

ct_status matmul(MmArgs a, const Operands &o, cudaStream_t st, const Choice *chosen = nullptr) {
    if (a.KB == 0) {
        const int64_t grid = ((int64_t)a.M * a.N + 255) / 256;
        return pdl_launch(bias_only_kernel, dim3((unsigned)(grid < 65536 ? grid : 65536)), dim3(256), 0, st, a) == cudaSuccess
                   ? CT_OK
                   : CT_ECUDA;
    }
    a.err = device_error_word();
    if (a.err == nullptr) return CT_ECUDA;
    CUtensorMap lmap, cmap;
    cudaError_t e;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev >= MAX_DEVICES) return CT_ECUDA;
    const Choice ch = chosen != nullptr ? *chosen : choose(a.M, a.N, a.KB, sm_count(), dev);
    if (ch.ctas == 0) return CT_ECUDA;
    const int bn = ch.bn;
    a.splits = ch.splits;
    if (ch.wide) {
        a.tiles_l = (a.M + 2 * BL - 1) / (2 * BL);
        a.tiles_c = (a.N + bn - 1) / bn;
        a.group = 8;
        const int pairs = ch.ctas / 2;
        const int64_t tiles = (int64_t)a.tiles_l * a.tiles_c;
        if (tiles > INT32_MAX / 16) return CT_ERANGE;
        CUtensorMap ymap = {};
        const int es = dtype_size(a.out);
        // TMA clips a store at the 16-byte unit in which a row ends, not at the row's end: what lies beside y in a
        // wider matrix would be written
        a.vec = aligned(a.y, 16) && a.ldy * es % 16 == 0 && (int64_t)a.N * es % 16 == 0;
        if (!encode8(&lmap, o.xq, a.M, o.k, o.ldx, BL) || !encode8(&cmap, o.wq, a.N, o.k, o.ldw, bn / 2) ||
            (a.vec && !encode(&ymap, a.y, a.out == CT_DT_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16,
                              es, a.M, a.N, a.ldy * es, bn % 128 == 64 && es == 2 ? 64 : 128, 32)))
            return CT_ECUDA;
        const int n = (int)(a.splits > 1 || tiles < pairs ? tiles : pairs);
        e = bn == 64    ? launch_wide<64>(lmap, cmap, ymap, a, n, st)
            : bn == 128 ? launch_wide<128>(lmap, cmap, ymap, a, n, st)
            : bn == 192 ? pdl_launch_cluster(fp8_wide_kernel<192, false>, dim3((unsigned)(2 * n)), dim3(W_THREADS),
                                             Wide<192>::SMEM, st, 2, lmap, cmap, ymap, a)
                        : launch_wide<256>(lmap, cmap, ymap, a, n, st);
    } else {
        a.tiles_l = (a.N + 127) / 128;
        a.tiles_c = (a.M + bn - 1) / bn;
        const int64_t tiles = (int64_t)a.tiles_l * a.tiles_c;
        if (tiles > INT32_MAX / 16) return CT_ERANGE;
        if (!encode8(&lmap, o.wq, a.N, o.k, o.ldw, BL) || !encode8(&cmap, o.xq, a.M, o.k, o.ldx, bn)) return CT_ECUDA;
        const int grid = (int)tiles * a.splits;
        e = bn == 16   ? launch_narrow<16>(lmap, cmap, a, grid, st)
            : bn == 32 ? launch_narrow<32>(lmap, cmap, a, grid, st)
            : bn == 64 ? launch_narrow<64>(lmap, cmap, a, grid, st)
                       : launch_narrow<128>(lmap, cmap, a, grid, st);
    }
    return e == cudaSuccess ? CT_OK : CT_ECUDA;
}

// checks shared by the two entry points (everything but x)
ct_status check(int64_t m, int64_t n, int64_t k, const uint8_t *w, int64_t ldw, const float *ws, const float *bias,
                const void *y, int out, int64_t ldy) {
    if (!dtype_ok(out)) return CT_EINVAL;
    if (m < 0 || n < 0 || k < 0 || m > INT32_MAX - 256 || n > INT32_MAX - 256 || k > INT32_MAX - 256) return CT_ERANGE;
    if (m == 0 || n == 0) return CT_OK;
    if (y == nullptr || ldy < n || !aligned(y, dtype_size(out)) || !aligned(bias, 4)) return CT_EINVAL;
    if (k > 0 && (w == nullptr || ws == nullptr || (n > 1 && (ldw < k || ldw % 16 != 0)) || !aligned(w, 16) || !aligned(ws, 4)))
        return CT_EINVAL;
    return CT_OK;
}

MmArgs make_args(int64_t m, int64_t n, int64_t k, const float *ws, int64_t ws_row, int64_t ws_blk, const float *bias,
                 int relu, void *y, int out, int64_t ldy) {
    MmArgs a = {};
    a.ws = ws; a.ws_row = ws_row; a.ws_blk = ws_blk;
    a.bias = bias; a.y = y; a.ldy = ldy;
    a.M = (int)m; a.N = (int)n; a.KB = (int)((k + BK - 1) / BK);
    a.out = out; a.relu = relu != 0;
    a.vec4 = aligned(y, 4 * dtype_size(out)) && (m == 1 || ldy % 4 == 0);
    return a;
}

// workspace of ct_fp8_linear: the 8-bit rows (pitch a multiple of 16 bytes), then their scales [block][row]
size_t scales_at(int64_t m, int64_t k) { return ((size_t)m * (size_t)q_pitch(k) + 255) / 256 * 256; }

}  // namespace
}  // namespace ops
}  // namespace ct

extern "C" ct_status ct_fp8_matmul(const uint8_t *x_dev, int64_t ldx, const float *x_scale_dev, int64_t x_scale_row,
                                   int64_t x_scale_blk, const uint8_t *w_dev, int64_t ldw, const float *w_scale_dev,
                                   int64_t w_scale_row, int64_t w_scale_blk, const float *bias_dev, int32_t relu,
                                   void *y_dev, int32_t y_dtype, int64_t ldy, int64_t m, int64_t n, int64_t k,
                                   void *stream) {
    using namespace ct::ops;
    const ct_status s = check(m, n, k, w_dev, ldw, w_scale_dev, bias_dev, y_dev, y_dtype, ldy);
    if (s != CT_OK || m == 0 || n == 0) return s;
    if (k > 0 && (x_dev == nullptr || x_scale_dev == nullptr || (m > 1 && (ldx < k || ldx % 16 != 0)) || !aligned(x_dev, 16) ||
                  !aligned(x_scale_dev, 4)))
        return CT_EINVAL;
    MmArgs a = make_args(m, n, k, w_scale_dev, w_scale_row, w_scale_blk, bias_dev, relu, y_dev, y_dtype, ldy);
    a.xs = x_scale_dev; a.xs_row = x_scale_row; a.xs_blk = x_scale_blk;
    return matmul(a, Operands{x_dev, ldx, w_dev, ldw, k}, static_cast<cudaStream_t>(stream));
}

extern "C" ct_status ct_fp8_linear_workspace(int64_t m, int64_t k, size_t *bytes) {
    using namespace ct::ops;
    if (bytes == nullptr) return CT_EINVAL;
    if (m < 0 || k < 0 || m > INT32_MAX - 256 || k > INT32_MAX - 256) return CT_ERANGE;
    *bytes = scales_at(m, k) + (size_t)m * (size_t)((k + BK - 1) / BK) * 4;
    return CT_OK;
}

extern "C" ct_status ct_fp8_linear(const void *x_dev, int32_t x_dtype, int64_t ldx, const uint8_t *w_dev, int64_t ldw,
                                   const float *w_scale_dev, int64_t w_scale_row, int64_t w_scale_blk,
                                   const float *bias_dev, int32_t relu, void *y_dev, int32_t y_dtype, int64_t ldy,
                                   int64_t m, int64_t n, int64_t k, void *workspace_dev, size_t workspace_bytes,
                                   void *stream) {
    using namespace ct::ops;
    const ct_status s = check(m, n, k, w_dev, ldw, w_scale_dev, bias_dev, y_dev, y_dtype, ldy);
    if (s != CT_OK) return s;
    if (!dtype_ok(x_dtype)) return CT_EINVAL;
    if (m == 0 || n == 0) return CT_OK;
    MmArgs a = make_args(m, n, k, w_scale_dev, w_scale_row, w_scale_blk, bias_dev, relu, y_dev, y_dtype, ldy);
    if (k == 0) return matmul(a, Operands{}, static_cast<cudaStream_t>(stream));
    size_t need = 0;
    ct_fp8_linear_workspace(m, k, &need);
    if (x_dev == nullptr || ldx < k || !aligned(x_dev, dtype_size(x_dtype))) return CT_EINVAL;
    if (workspace_dev == nullptr || !aligned(workspace_dev, 16)) return CT_EINVAL;
    if (workspace_bytes < need) return CT_ENOMEM;
    a.x = x_dev; a.ldx = ldx; a.K = (int)k;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev >= MAX_DEVICES) return CT_ECUDA;
    const Choice two = choose(a.M, a.N, a.KB, sm_count(), dev);
    const Operands w = {nullptr, 0, w_dev, ldw, k};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const Choice one = choose_one_launch(two, a.M, a.N, k, dev, x_dtype);
    if (one.ctas > 0)
        return x_dtype == CT_DT_F32   ? quantise_and_multiply<float>(a, w, one, st)
               : x_dtype == CT_DT_F16 ? quantise_and_multiply<__half>(a, w, one, st)
                                      : quantise_and_multiply<__nv_bfloat16>(a, w, one, st);
    uint8_t *q = static_cast<uint8_t *>(workspace_dev);
    float *xs = reinterpret_cast<float *>(q + scales_at(m, k));
    const ct_status r = quantize(x_dev, x_dtype, m, k, ldx, 1, q, q_pitch(k), xs, 1, m, st);
    if (r != CT_OK) return r;
    a.xs = xs; a.xs_row = 1; a.xs_blk = m;
    // the quantisation lets this kernel start only after all work before itself
    // is complete, and does not write w
    a.early = 1;
    return matmul(a, Operands{q, q_pitch(k), w_dev, ldw, k}, st, &two);
}

// Which kernel a product of these sizes takes (x_dtype -1), or a linear layer on
// rows of x_dtype: {quantises in the launch, wide, columns of a tile, splits of
// K}.  Not part of the interface: the tests ask it whether they reach every kernel.
extern "C" ct_status ct_internal_fp8_kernel(int64_t m, int64_t n, int64_t k, int32_t x_dtype, int32_t *kernel) {
    using namespace ct::ops;
    if (kernel == nullptr || (x_dtype != -1 && !dtype_ok(x_dtype))) return CT_EINVAL;
    if (m < 1 || n < 1 || k < 1 || m > INT32_MAX - 256 || n > INT32_MAX - 256 || k > INT32_MAX - 256) return CT_ERANGE;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev >= MAX_DEVICES) return CT_ECUDA;
    Choice ch = choose((int)m, (int)n, (int)((k + BK - 1) / BK), sm_count(), dev);
    const Choice one = x_dtype < 0 ? Choice{} : choose_one_launch(ch, (int)m, (int)n, k, dev, x_dtype);
    if (one.ctas > 0) ch = one;
    if (ch.ctas == 0) return CT_ECUDA;
    kernel[0] = one.ctas > 0;
    kernel[1] = ch.wide;
    kernel[2] = ch.bn;
    kernel[3] = ch.splits;
    return CT_OK;
}
