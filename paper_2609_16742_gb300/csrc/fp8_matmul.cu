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
// Warp roles: 8 epilogue warps (warp w reads TMEM lanes 32 (w % 4) .. and the
// column half w / 4), one TMA warp, one MMA warp.  A stage of shared memory
// holds one K block of both operands: 128-byte rows, 128-byte swizzle; rows
// and columns past the ends are the zeros TMA fills in.
//
// Two orientations:
//   rows of x on the TMEM lanes (many rows): 128 x 256 tiles, persistent
//     CTAs; the factor of a thread's values is one product per block;
//   rows of w on the lanes (few rows): 128 x BN tiles with BN as narrow as
//     the rows allow, so that a few rows cost no 128-wide tile; the K range
//     is split over a cluster of up to 8 CTAs so that the whole GPU streams
//     the weights, and the cluster adds its partial sums through distributed
//     shared memory, in rank order: no workspace, no atomics, one launch, the
//     same bits each time.
#include <atomic>
#include <cudaTypedefs.h>
#include <string.h>

#include "ops_common.cuh"
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
    int group;                          // lane tiles walked together (persistent grids)
    int vec;                            // y rows may be written 32 bytes at a time
    uint32_t *err;
};

template <int BN, bool SWAP> struct Shape {
    static constexpr int C_BYTES = BN * BK;
    static constexpr int STAGE = L_BYTES + C_BYTES;
    // two CTAs share an SM where the tiles are narrow
    static constexpr int STAGES = BN <= 32 ? 5 : BN == 64 ? 4 : BN == 128 ? 6 : 4;
    static constexpr int NBUF = BN <= 64 ? 4 : 2;
    static constexpr int TMEM_COLS = NBUF * BN < 32 ? 32 : NBUF * BN;
    static constexpr int CPW = BN / 2;                     // columns of an epilogue warp
    static constexpr int FAC = SWAP ? N_EPI * 2 * CPW * 4 : 0;
    static constexpr size_t SMEM = 1024 + (size_t)STAGES * STAGE + FAC + 8 * (2 * STAGES + 2 * NBUF) + 16;
};

template <int N> __device__ __forceinline__ void tmem_ld_nw(uint32_t taddr, uint32_t (&r)[N]) {
    if constexpr (N == 8) {
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                     : "r"(taddr));
    } else if constexpr (N == 16) {
        tmem_ld16_nw(taddr, r);
    } else {
        static_assert(N == 32, "8, 16 or 32 columns");
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

__device__ __forceinline__ float ld_cluster_f32(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}

__device__ __forceinline__ void store_out(const MmArgs &a, int64_t at, float v) {
    if (a.out == CT_DT_F32) static_cast<float *>(a.y)[at] = v;
    else if (a.out == CT_DT_F16) static_cast<__half *>(a.y)[at] = __float2half_rn(v);
    else static_cast<__nv_bfloat16 *>(a.y)[at] = __float2bfloat16_rn(v);
}

__device__ __forceinline__ float finish(const MmArgs &a, float v, int n) {
    if (a.bias != nullptr) v += __ldg(a.bias + n);
    return a.relu ? relu_keep_nan(v) : v;
}

// tile -> (lane tile, column tile): `group` lane tiles are walked together,
// so that the CTAs at work share operand tiles in L2
__device__ __forceinline__ void tile_at(const MmArgs &a, int t, int &l, int &c) {
    const int per = a.group * a.tiles_c;
    const int g = t / per, r = t % per;
    const int rows = min(a.group, a.tiles_l - g * a.group);
    l = g * a.group + r % rows;
    c = r / rows;
}

template <int BN, bool SWAP>
__global__ void __launch_bounds__(THREADS, 1)
fp8_matmul_kernel(const __grid_constant__ CUtensorMap lmap, const __grid_constant__ CUtensorMap cmap, const MmArgs a) {
    using S = Shape<BN, SWAP>;
    constexpr int CPW = S::CPW;
    constexpr int LDN = CPW < 32 ? CPW : 32;               // columns of one TMEM load
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t *Ls = smem;
    uint8_t *Cs = Ls + S::STAGES * L_BYTES;
    float *fac = (float *)(Cs + S::STAGES * S::C_BYTES);
    uint64_t *full = (uint64_t *)((uint8_t *)fac + S::FAC);
    uint64_t *empty = full + S::STAGES;
    uint64_t *acc_full = empty + S::STAGES;
    uint64_t *acc_empty = acc_full + S::NBUF;
    uint32_t *tmem_holder = (uint32_t *)(acc_empty + S::NBUF);
    volatile uint32_t *abort_flag = tmem_holder + 1;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)(blockIdx.x % (unsigned)a.splits);
    const int cid = (int)(blockIdx.x / (unsigned)a.splits), ncl = (int)(gridDim.x / (unsigned)a.splits);
    const int tiles = a.tiles_l * a.tiles_c;
    const int kb0 = (int)((int64_t)a.KB * rank / a.splits), kb1 = (int)((int64_t)a.KB * (rank + 1) / a.splits);

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; ++s) {
            mbar_init(smem_u32(&full[s]), 1);
            mbar_init(smem_u32(&empty[s]), 1);
        }
        for (int b = 0; b < S::NBUF; ++b) {
            mbar_init(smem_u32(&acc_full[b]), 1);
            mbar_init(smem_u32(&acc_empty[b]), N_EPI);
        }
        *abort_flag = 0;
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
    pdl_wait();
    pdl_trigger();

    if (warp == TMA_WARP) {
        int it = 0;
        bool ok = true;
        for (int t = cid; t < tiles && ok; t += ncl) {
            int tl, tc;
            tile_at(a, t, tl, tc);
            for (int kb = kb0; kb < kb1; ++kb, ++it) {
                const int s = it % S::STAGES;
                if (!warp_wait(smem_u32(&empty[s]), ((uint32_t)(it / S::STAGES) & 1u) ^ 1u, a.err, E_TMA) ||
                    __any_sync(0xffffffffu, *abort_flag)) {
                    ok = false;
                    break;
                }
                if (elect_one()) {
                    const uint32_t fb = smem_u32(&full[s]);
                    mbar_arrive_expect_tx(fb, (uint32_t)S::STAGE);
                    tma_load_2d(smem_u32(Ls + s * L_BYTES), &lmap, fb, kb * BK, tl * BL);
                    tma_load_2d(smem_u32(Cs + s * S::C_BYTES), &cmap, fb, kb * BK, tc * BN);
                }
                __syncwarp();
            }
        }
        if (!ok) {
            if (lane == 0) *abort_flag = 1;
            // copies still in flight land before the CTA ends
            for (int j = max(0, it - S::STAGES); j < it; ++j)
                warp_wait(smem_u32(&full[j % S::STAGES]), (uint32_t)(j / S::STAGES) & 1u, a.err, E_DRAIN);
        }
    } else if (warp == MMA_WARP) {
        constexpr uint32_t idesc = idesc_e4m3(BL, BN);
        int it = 0;
        bool ok = true;
        for (int t = cid; t < tiles && ok; t += ncl) {
            for (int kb = kb0; kb < kb1; ++kb, ++it) {
                const int s = it % S::STAGES, b = it % S::NBUF;
                if (!warp_wait(smem_u32(&acc_empty[b]), ((uint32_t)(it / S::NBUF) & 1u) ^ 1u, a.err, E_ACC) ||
                    !warp_wait(smem_u32(&full[s]), (uint32_t)(it / S::STAGES) & 1u, a.err, E_MMA) ||
                    __any_sync(0xffffffffu, *abort_flag)) {
                    ok = false;
                    break;
                }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (elect_one()) {
                    const uint64_t ld = smem_desc_sw128(smem_u32(Ls + s * L_BYTES));
                    const uint64_t cd = smem_desc_sw128(smem_u32(Cs + s * S::C_BYTES));
#pragma unroll
                    for (int k = 0; k < BK / 32; ++k)
                        umma_e4m3(tmem + (uint32_t)(b * BN), ld + 2 * k, cd + 2 * k, idesc, k > 0 ? 1u : 0u);
                    umma_commit(smem_u32(&empty[s]));
                    umma_commit(smem_u32(&acc_full[b]));
                }
                __syncwarp();
            }
        }
        if (!ok && lane == 0) *abort_flag = 1;
    } else {
        const int quad = warp & 3, half = warp >> 2;
        const int row = quad * 32 + lane;                  // lane row of this thread within the tile
        const uint32_t tbase = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(half * CPW);
        int it = 0;
        bool ok = true;
        for (int t = cid; t < tiles && ok; t += ncl) {
            int tl, tc;
            tile_at(a, t, tl, tc);
            const int l = tl * BL + row;                   // global index on the lane side
            const int c0 = tc * BN + half * CPW;           // first global column of this warp
            float acc[CPW];
#pragma unroll
            for (int i = 0; i < CPW; ++i) acc[i] = 0.f;

            // scales of the next block, fetched one block ahead
            constexpr int NF = (CPW + 31) / 32;
            float nx[NF], nw;
            const float *xp[NF];
            bool xin[NF];
            const float *wp;
            if constexpr (SWAP) {
#pragma unroll
                for (int j = 0; j < NF; ++j) {
                    const int m = c0 + j * 32 + lane;
                    xin[j] = j * 32 + lane < CPW && m < a.M;
                    xp[j] = a.xs + (int64_t)(xin[j] ? m : 0) * a.xs_row;
                }
                wp = a.ws + (int64_t)tl * a.ws_row;
            } else {
                xin[0] = l < a.M;
                xp[0] = a.xs + (int64_t)(xin[0] ? l : 0) * a.xs_row;
                wp = a.ws + (int64_t)min(c0 / 128, (a.N - 1) / 128) * a.ws_row;
            }
            const auto fetch = [&](int kb) {
#pragma unroll
                for (int j = 0; j < NF; ++j)
                    if (SWAP || j == 0) nx[j] = xin[j] ? __ldg(xp[j] + kb * a.xs_blk) : 0.f;
                nw = __ldg(wp + kb * a.ws_blk);
            };
            if (kb0 < kb1) fetch(kb0);

            for (int kb = kb0; kb < kb1; ++kb, ++it) {
                const int b = it % S::NBUF;
                float f = nx[0] * nw;
                const float *fs = fac + (warp * 2 + (it & 1)) * CPW;
                if constexpr (SWAP) {
#pragma unroll
                    for (int j = 0; j < NF; ++j)
                        if (j * 32 + lane < CPW) const_cast<float *>(fs)[j * 32 + lane] = nx[j] * nw;
                    __syncwarp();
                }
                if (kb + 1 < kb1) fetch(kb + 1);
                ok = warp_wait(smem_u32(&acc_full[b]), (uint32_t)(it / S::NBUF) & 1u, a.err, E_EPI) &&
                     !__any_sync(0xffffffffu, *abort_flag);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                for (int c = 0; c < CPW; c += LDN) {
                    uint32_t r[LDN];
                    tmem_ld_nw<LDN>(tbase + (uint32_t)(b * BN + c), r);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < LDN; ++i) {
                        const float p = tmem_done(r[i]);
                        acc[c + i] = fmaf(SWAP ? fs[c + i] : f, p, acc[c + i]);
                    }
                }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&acc_empty[b]));
            }
            if (!ok) break;

            if constexpr (SWAP) {
                if (a.splits > 1) {
                    // partial sums [column][lane row], over the stages: every copy has
                    // landed and every MMA has read it (the last block is complete)
                    float *part = (float *)smem;
#pragma unroll
                    for (int i = 0; i < CPW; ++i) part[(half * CPW + i) * BL + row] = acc[i];
                } else if (l < a.N) {
#pragma unroll
                    for (int i = 0; i < CPW; ++i)
                        if (c0 + i < a.M) store_out(a, (int64_t)(c0 + i) * a.ldy + l, finish(a, acc[i], l));
                }
            } else if (l < a.M) {
#pragma unroll
                for (int i = 0; i < CPW; ++i) {
                    const int n = c0 + i;
                    if (n < a.N) store_out(a, (int64_t)l * a.ldy + n, finish(a, acc[i], n));
                }
            }
        }
        if (!ok && lane == 0) *abort_flag = 1;
    }
    __syncwarp();
    if constexpr (SWAP) {
        if (a.splits > 1) {
            cluster_sync();
            if (warp < N_EPI) {
                // this CTA finishes every splits-th column of the cluster's tile
                int tl, tc;
                tile_at(a, cid, tl, tc);
                const int row = (int)threadIdx.x & (BL - 1), l = tl * BL + row;
                const int cols = min(BN, a.M - tc * BN);
                for (int c = rank * 2 + ((int)threadIdx.x >> 7); c < cols; c += 2 * a.splits) {
                    float v = 0.f;
                    const uint32_t at = smem_u32((float *)smem + c * BL + row);
#pragma unroll 4
                    for (int s = 0; s < a.splits; ++s) v += ld_cluster_f32(mapa_shared(at, (uint32_t)s));
                    if (l < a.N) store_out(a, (int64_t)(tc * BN + c) * a.ldy + l, finish(a, v, l));
                }
            }
            cluster_sync();
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == MMA_WARP) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)S::TMEM_COLS));
    }
}

// y = act(bias) where K is 0
__global__ void bias_only_kernel(const MmArgs a) {
    pdl_wait();
    pdl_trigger();
    const int64_t n_all = (int64_t)a.M * a.N;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n_all; i += (int64_t)gridDim.x * blockDim.x)
        store_out(a, i / a.N * a.ldy + i % a.N, finish(a, 0.f, (int)(i % a.N)));
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

// [rows, k] bytes, row pitch ld, in boxes of 128 bytes x box_rows, 128-byte swizzle
bool encode(CUtensorMap *map, const uint8_t *p, int64_t rows, int64_t k, int64_t ld, int box_rows) {
    PFN_cuTensorMapEncodeTiled_v12000 f = encoder();
    if (f == nullptr) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)ld};
    const cuuint32_t box[2] = {(cuuint32_t)BK, (cuuint32_t)box_rows};
    const cuuint32_t es[2] = {1, 1};
    return f(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t *>(p), dims, strides, box, es,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int BN, bool SWAP>
cudaError_t launch(const CUtensorMap &lmap, const CUtensorMap &cmap, const MmArgs &a, int grid, cudaStream_t st) {
    using S = Shape<BN, SWAP>;
    static std::atomic<bool> sized[MAX_DEVICES];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= MAX_DEVICES || !sized[dev].load(std::memory_order_relaxed)) {
        e = cudaFuncSetAttribute(fp8_matmul_kernel<BN, SWAP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::SMEM);
        if (e != cudaSuccess) return e;
        if (dev < MAX_DEVICES) sized[dev].store(true, std::memory_order_relaxed);
    }
    return pdl_launch_cluster(fp8_matmul_kernel<BN, SWAP>, dim3((unsigned)grid), dim3(THREADS), S::SMEM, st, a.splits,
                              lmap, cmap, a);
}

struct Operands {
    const uint8_t *xq;
    int64_t ldx;
    const uint8_t *wq;
    int64_t ldw;
    int64_t k;
};

ct_status matmul(MmArgs a, const Operands &o, cudaStream_t st) {
    if (a.KB == 0) {
        const int64_t grid = ((int64_t)a.M * a.N + 255) / 256;
        return pdl_launch(bias_only_kernel, dim3((unsigned)(grid < 65536 ? grid : 65536)), dim3(256), 0, st, a) == cudaSuccess
                   ? CT_OK
                   : CT_ECUDA;
    }
    a.err = device_error_word();
    if (a.err == nullptr) return CT_ECUDA;
    const int sms = sm_count();
    const int nt = (a.N + 127) / 128;
    CUtensorMap lmap, cmap;
    cudaError_t e;
    if (a.M > 256) {
        a.tiles_l = (a.M + 127) / 128;
        a.tiles_c = (a.N + 255) / 256;
        a.splits = 1;
        a.group = 8;
        if (!encode(&lmap, o.xq, a.M, o.k, o.ldx, BL) || !encode(&cmap, o.wq, a.N, o.k, o.ldw, 256)) return CT_ECUDA;
        const int64_t tiles = (int64_t)a.tiles_l * a.tiles_c;
        if (tiles > INT32_MAX / 2) return CT_ERANGE;
        e = launch<256, false>(lmap, cmap, a, (int)(tiles < sms ? tiles : sms), st);
    } else {
        const int bn = a.M <= 16 ? 16 : a.M <= 32 ? 32 : a.M <= 64 ? 64 : 128;
        a.tiles_l = nt;
        a.tiles_c = (a.M + bn - 1) / bn;
        a.group = nt;
        const int64_t tiles = (int64_t)a.tiles_l * a.tiles_c;
        a.splits = 1;
        while (a.splits < 8 && tiles * a.splits * 2 <= sms && a.splits * 2 <= a.KB) a.splits *= 2;
        if (tiles > INT32_MAX / 16) return CT_ERANGE;
        if (!encode(&lmap, o.wq, a.N, o.k, o.ldw, BL) || !encode(&cmap, o.xq, a.M, o.k, o.ldx, bn)) return CT_ECUDA;
        const int grid = (int)tiles * a.splits;
        e = bn == 16   ? launch<16, true>(lmap, cmap, a, grid, st)
            : bn == 32 ? launch<32, true>(lmap, cmap, a, grid, st)
            : bn == 64 ? launch<64, true>(lmap, cmap, a, grid, st)
                       : launch<128, true>(lmap, cmap, a, grid, st);
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
    if (k > 0 && (w == nullptr || ws == nullptr || ldw < k || ldw % 16 != 0 || !aligned(w, 16) || !aligned(ws, 4)))
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
    a.vec = aligned(y, 32) && ldy * dtype_size(out) % 32 == 0;
    return a;
}

// workspace of ct_fp8_linear: the 8-bit rows (pitch a multiple of 16 bytes), then their scales [block][row]
int64_t q_pitch(int64_t k) { return (k + 15) / 16 * 16; }
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
    if (k > 0 && (x_dev == nullptr || x_scale_dev == nullptr || ldx < k || ldx % 16 != 0 || !aligned(x_dev, 16) ||
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
    uint8_t *q = static_cast<uint8_t *>(workspace_dev);
    float *xs = reinterpret_cast<float *>(q + scales_at(m, k));
    const ct_status r = quantize(x_dev, x_dtype, m, k, ldx, 1, q, q_pitch(k), xs, 1, m, static_cast<cudaStream_t>(stream));
    if (r != CT_OK) return r;
    a.xs = xs; a.xs_row = 1; a.xs_blk = m;
    return matmul(a, Operands{q, q_pitch(k), w_dev, ldw, k}, static_cast<cudaStream_t>(stream));
}
