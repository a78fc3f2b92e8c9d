// The adapters' products of many rows on the tcgen05 tensor cores, for 16-bit values in whole rows (16-byte starts, a multiple
// of 8 values): what shrink_kernel, expand_kernel and outer_kernel compute, in the same order of tiles and splits.
//
// At rank 64 a value of x takes part in 128 operations, so that HBM's rate asks for some 420 TFLOP/s: more than mma.sync
// reaches here (175 measured), a quarter of what tcgen05.mma does.  All threads copy (rows come in any order: cp.async, 16
// bytes a thread, into the swizzled layouts that the tensor cores read), one issues the products; sums lie in tensor
// memory and are moved to registers after every 256 values (the tensor cores cut off what they add) while the next go on into
// other columns.  Operands whose summed axis runs along their rows in memory are read as they lie (MN-major).
//
// Measured alone (BF16, rank 64): 8192 rows of 4096 against A 18.5 us (3.6 TB/s), of 8192 against B 30 us (4.5 TB/s); added to 8192 x 8192
// of y 49 us (5.5 TB/s read and written), to 8192 x 4096 29 us; both gradients, 4096 and 8192 columns, 55 us (3.7 TB/s).
//
// Every wait is bounded: one that runs out sets the operators' error word, ends the work after the copies and products under way,
// and frees the tensor memory.
#include "adapters.cuh"

namespace ct {
namespace ops {
namespace {

constexpr uint32_t E_ADAPTERS = 0x8000;

// shared-memory operand: byte distances between atoms along MN (lbo) and along K or, K-major, along MN (sbo)
enum { SW128 = 2, SW64 = 4, SW32 = 6 };
__device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t lbo, uint32_t sbo, int swizzle) {
    return (uint64_t)((addr >> 4) & 0x3FFF) | (uint64_t)((lbo >> 4) & 0x3FFF) << 16 | (uint64_t)((sbo >> 4) & 0x3FFF) << 32 | (uint64_t)1 << 46 |
           (uint64_t)swizzle << 61;
}
// instruction descriptor: FP32 sums of two FP16 or two BF16 operands; a_mn, b_mn: the summed axis runs along the operand's rows
__host__ __device__ constexpr uint32_t product(bool bf16, bool a_mn, bool b_mn, int m, int n) {
    return 1u << 4 | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 |
           (uint32_t)(m >> 4) << 24;
}

// A matrix of `width` 16-bit values a row, MN-major or K-major alike: blocks of 64 values a row (128 bytes), or narrower ones.
template <int WIDTH> struct Tile {
    static constexpr int ROW = WIDTH >= 64 ? 128 : 2 * WIDTH;                    // bytes of a row in a block
    static constexpr int SWIZZLE = ROW == 128 ? SW128 : ROW == 64 ? SW64 : SW32;
    static constexpr int CHUNKS = WIDTH / 8;                                     // 16-byte chunks of a row, of all blocks
    // chunk c of row r of a block of `rows` rows
    static __device__ __forceinline__ uint32_t at(int r, int c, int rows) {
        if (ROW == 128) return (uint32_t)((c >> 3) * rows * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4));
        if (ROW == 64) return (uint32_t)(r * 64 + ((c ^ (r >> 1 & 3)) << 4));
        return (uint32_t)(r * 32 + ((c ^ (r >> 2 & 1)) << 4));
    }
};

__device__ __forceinline__ void tmem_ld8(uint32_t addr, float (&v)[8]) {
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = tc::tmem_done(r[i]);
}
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
// what this thread wrote to shared memory is seen by the tensor cores
__device__ __forceinline__ void fence_operands() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// The barriers that a CTA's products arrive on, and its tensor memory.  It is taken after the kernel before has ended and before the next may
// begin: no CTA holds some while it waits for a kernel that may want it.
template <int BARS, int COLUMNS> __device__ __forceinline__ uint32_t tensor_begin(uint64_t (&bars)[BARS], uint32_t &holder) {
    if (threadIdx.x == 0) {
        for (int i = 0; i < BARS; ++i) tc::mbar_init(tc::smem_u32(&bars[i]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x < 32) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(&holder)), "r"((uint32_t)COLUMNS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    fence_before();
    __syncthreads();
    fence_after();
    return holder;
}
template <int COLUMNS> __device__ __forceinline__ void tensor_end(uint32_t addr) {
    fence_before();
    __syncthreads();
    fence_after();
    if (threadIdx.x < 32) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"((uint32_t)COLUMNS));
}
constexpr int columns_of(int n) { return n <= 32 ? 32 : n <= 64 ? 64 : n <= 128 ? 128 : n <= 256 ? 256 : 512; }

constexpr int FLUSH = 4;                          // steps whose sums stay in the tensor cores' accumulators: 256 values

// ---------------------------------------------------------------- shrink

template <int RP> struct Shrink {
    static constexpr int X_BYTES = AD_ROWS * 128, M_BYTES = RP * 128, STAGE = X_BYTES + M_BYTES, STAGES = RP == 128 ? 3 : 4;
    static constexpr int SMEM = STAGES * STAGE + 1024, COLUMNS = columns_of(2 * RP);
    static constexpr int MV = (RP * 8 + AD_THREADS - 1) / AD_THREADS;
};

template <typename T, int RP, bool TRANS>
__device__ __forceinline__ void shrink_tile(const AdShrink &a, const AdOrder &o, const AdRows &tile, int rank, int splits, unsigned char *raw,
                                            uint32_t bar, uint32_t tmem, uint32_t *err) {
    using S = Shrink<RP>;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t base = (tc::smem_u32(raw) + 1023u) & ~1023u;
    const int adapter = tile.key - 1, steps = (int)((a.cols + AD_STEP - 1) / AD_STEP);
    const int s0 = (int)((int64_t)steps * rank / splits), n = (int)((int64_t)steps * (rank + 1) / splits) - s0;

    // Each thread's copies, a step's worth further on with each step: of x, rows tid / 8 + 32 i, 16 bytes at 16 (tid % 8)
    const char *xp[4], *mp[S::MV];
    bool xh[4], mh[S::MV];
    const int64_t c0 = (int64_t)s0 * AD_STEP;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = tid / 8 + 32 * i;
        const int64_t s = tile.slot0 + r;
        xh[i] = r < tile.rows;
        xp[i] = reinterpret_cast<const char *>(static_cast<const T *>(a.x) +
                                               (xh[i] ? (o.order != nullptr ? (int64_t)o.order[s] : s) * a.ldx : 0) + c0 + (tid & 7) * 8);
    }
    using MT = Tile<TRANS ? RP : AD_STEP>;
    uint32_t m_to[S::MV];
    int m_left[S::MV];                            // steps whose values are there
#pragma unroll
    for (int i = 0; i < S::MV; ++i) {
        const int v = tid + i * AD_THREADS, r = v / MT::CHUNKS, q = v % MT::CHUNKS, j = TRANS ? q * 8 : r;
        const int64_t c = c0 + (TRANS ? r : q * 8);
        mh[i] = v < RP * 8;
        m_to[i] = MT::at(r, q, TRANS ? AD_STEP : RP);
        m_left[i] = j < a.rank && c < a.cols ? (int)((a.cols - c + AD_STEP - 1) / AD_STEP) : 0;
        mp[i] = reinterpret_cast<const char *>(static_cast<const T *>(a.m) + adapter * a.m_adapter +
                                               (m_left[i] > 0 ? (TRANS ? c * a.m_row + j : j * a.m_row + c) : 0));
    }
    const int64_t m_step = 2 * (TRANS ? AD_STEP * a.m_row : AD_STEP);
    const int x_left = c0 + (tid & 7) * 8 < a.cols ? (int)((a.cols - c0 - (tid & 7) * 8 + AD_STEP - 1) / AD_STEP) : 0;
    const uint32_t x_to = Tile<AD_STEP>::at(tid / 8, tid & 7, AD_ROWS);
    int to_copy = 0, copy_stage = 0;              // the next step to copy, its stage
    auto copy = [&]() {
        const uint32_t bx = base + copy_stage * S::STAGE, bm = bx + S::X_BYTES;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool there = xh[i] && to_copy < x_left;
            copy16_if(bx + x_to + 32 * i * 128, there ? xp[i] : static_cast<const char *>(a.x), there);
            xp[i] += 2 * AD_STEP;
        }
#pragma unroll
        for (int i = 0; i < S::MV; ++i) {
            const bool there = to_copy < m_left[i];
            if (mh[i]) copy16_if(bm + m_to[i], there ? mp[i] : static_cast<const char *>(a.m), there);
            mp[i] += m_step;
        }
        ++to_copy;
        copy_stage = copy_stage + 1 == S::STAGES ? 0 : copy_stage + 1;
    };
    float sum[RP / 2];
#pragma unroll
    for (int j = 0; j < RP / 2; ++j) sum[j] = 0.f;
    bool ok = true;
    int groups = 0;                               // whose sums are in registers
    const uint32_t mine = tmem + ((uint32_t)(warp & 3) << 21) + (uint32_t)(warp >> 2) * (RP / 2);
    auto collect = [&]() {
        ok = ok && tc::mbar_wait(bar + 8 * (S::STAGES + (groups & 1)), (groups >> 1) & 1, err, E_ADAPTERS);
        __syncwarp();
        fence_after();
#pragma unroll
        for (int j = 0; j < RP / 2; j += 8) {
            float v[8];
            tmem_ld8(mine + (groups & 1) * RP + j, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[j + e] += v[e];
        }
        fence_before();
        ++groups;
    };
#pragma unroll
    for (int i = 0; i < S::STAGES; ++i) {
        if (i < n) copy();
        copies_end();
    }
    constexpr uint32_t how = product(Parts<T>::N == 1, false, TRANS, AD_ROWS, RP);
    int at = 0, stage = 0;                        // the step, its stage
    uint32_t done = 0;                            // bit s: parity of stage s's next end of products
    for (; at < n; ++at) {
        copies_wait<S::STAGES - 1>();
        fence_operands();
        if (!__syncthreads_and(ok)) break;
        if (warp == 0 && tc::elect_one()) {
            fence_after();
            const uint32_t bx = base + stage * S::STAGE, bm = bx + S::X_BYTES;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint64_t da = operand(bx + 32 * k, 16, 1024, SW128);
                const uint64_t db = TRANS ? operand(bm + 16 * k * MT::ROW, AD_STEP * 128, 8 * MT::ROW, MT::SWIZZLE)
                                          : operand(bm + 32 * k, 16, 1024, SW128);
                tc::umma_f16(tmem + (at / FLUSH & 1) * RP, da, db, how, at % FLUSH > 0 || k > 0);
            }
            tc::umma_commit(bar + 8 * stage);
            if (at % FLUSH == FLUSH - 1 || at == n - 1) tc::umma_commit(bar + 8 * (S::STAGES + (at / FLUSH & 1)));
        }
        __syncwarp();
        if (at + S::STAGES < n) {
            // the stage again, once its products are done: they take a fraction of the time that the next stages' copies do
            ok = ok && tc::mbar_wait(bar + 8 * stage, done >> stage & 1, err, E_ADAPTERS);
            done ^= 1u << stage;
            if (ok) copy();
        }
        copies_end();
        if (at % FLUSH == 1 && at > FLUSH) collect();
        stage = stage + 1 == S::STAGES ? 0 : stage + 1;
    }
    copies_wait<0>();
    if (at == n) {
        while (groups < (n + FLUSH - 1) / FLUSH) collect();
    } else if (warp == 0 && tc::elect_one()) {
        tc::umma_commit(bar + 8 * (S::STAGES + 2));                              // gave up: what was issued, before its memory goes
    }
    if (at < n) tc::mbar_wait(bar + 8 * (S::STAGES + 2), 0, err, E_ADAPTERS);
    tensor_end<S::COLUMNS>(tmem);

    // the tile's sums of this CTA, then of all of the cluster
    float *fs = reinterpret_cast<float *>(raw) + ((warp & 3) * 32 + lane) * sums_pitch(RP) + (warp >> 2) * (RP / 2);
#pragma unroll
    for (int j = 0; j < RP / 2; j += 4) *reinterpret_cast<float4 *>(fs + j) = make_float4(sum[j], sum[j + 1], sum[j + 2], sum[j + 3]);
    if (splits > 1) tc::cluster_sync();
    else __syncthreads();
    write_vectors<RP>(a, o, tile, adapter, reinterpret_cast<const float *>(raw), rank, splits);
    if (splits > 1) tc::cluster_sync();           // no CTA leaves while another reads its sums
}

// The rows of x that a CTA would have if they were in order already, on their way to L2 while the order is made (which touches
// nothing of x, and has itself waited for all before it).
__device__ __forceinline__ void shrink_ahead(const AdShrink &a, int size, int64_t t, int tile, int rank, int splits) {
    const int steps = (int)((a.cols + AD_STEP - 1) / AD_STEP), s0 = steps * rank / splits, s1 = steps * (rank + 1) / splits;
    const int64_t row = (int64_t)tile * AD_ROWS + threadIdx.x / 2;
    if (row >= t) return;
    const char *p = static_cast<const char *>(a.x) + row * a.ldx * size;
    for (int s = s0 + (threadIdx.x & 1); s < s1; s += 2) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + (int64_t)s * AD_STEP * size));
}

// x A^T, or (WHICH 1) dy B, or both: the tiles of the first, then those of the second
struct AdShrinks {
    AdShrink a[2];
};
constexpr int FORWARD = AD_FORWARD, BACKWARD = AD_BACKWARD, BOTH = AD_BOTH;
template <typename T, int RP, int WHICH>
__global__ void __launch_bounds__(AD_THREADS, 2)
shrink_tc_kernel(const __grid_constant__ AdShrinks two, const AdOrder o, int tiles, int splits, uint32_t *err) {
    using S = Shrink<RP>;
    extern __shared__ __align__(128) unsigned char raw[];
    __shared__ uint64_t bars[S::STAGES + 3];      // a stage's products are done; a group's sums are there (two, in turn); all
    __shared__ uint32_t holder;
    const int rank = splits > 1 ? (int)tc::cluster_ctarank() : 0;
    int t = (int)(blockIdx.x / (unsigned)splits);
    const bool second = WHICH == BACKWARD || (WHICH == BOTH && t >= tiles);
    if (WHICH == BOTH && second) t -= tiles;
    const AdShrink &a = two.a[WHICH == BOTH && second];
    if (a.first && o.order != nullptr) shrink_ahead(a, 2, o.t, t, rank, splits);
    pdl_wait();
    const uint32_t tmem = tensor_begin<S::STAGES + 3, S::COLUMNS>(bars, holder);
    pdl_trigger();
    const AdRows tile = ad_tile(o, t);
    if (tile.rows == 0 || tile.key == 0 || tile.key > o.adapters) {             // the whole cluster alike
        tensor_end<S::COLUMNS>(tmem);
        return;
    }
    if (WHICH == FORWARD || (WHICH == BOTH && !second)) shrink_tile<T, RP, false>(a, o, tile, rank, splits, raw, tc::smem_u32(bars), tmem, err);
    else shrink_tile<T, RP, true>(a, o, tile, rank, splits, raw, tc::smem_u32(bars), tmem, err);
}

// ---------------------------------------------------------------- expand

// Columns of a block: 256 bytes of y a row.  Its columns are dealt to the products' so that what the four lanes of a quad
// read from tensor memory for a row are 16 neighbouring bytes of y each: column c = 4 W g + W t + 2 q + e (W = 16 bytes of values, t < 4,
// e < 2) is the product's column 4 W g + 8 q + 2 t + e.
template <int RP, int YS> struct Expand {
    static constexpr int COLS = 256 / YS, HALF = COLS / 2, W = 16 / YS, V_BYTES = AD_ROWS * 2 * RP, M_BYTES = COLS * 2 * RP, STAGES = 3;
    static constexpr int COLUMNS = columns_of(2 * COLS);
    static int smem(int parts) { return parts * V_BYTES + STAGES * M_BYTES + 1024; }
    static constexpr int MV = COLS * (RP / 8) / AD_THREADS > 0 ? COLS * (RP / 8) / AD_THREADS : 1;
    static __device__ __forceinline__ int dealt(int c) { return c / (4 * W) * (4 * W) + c % W / 2 * 8 + c % (4 * W) / W * 2 + c % 2; }
};

// W columns' sums of rows lane / 4 and lane / 4 + 8 of 16 rows: columns W (lane % 4) on of 4 W
template <int W> __device__ __forceinline__ void tmem_quads(uint32_t addr, float (&lo)[W], float (&hi)[W]) {
    uint32_t r[2 * W];
    if constexpr (W == 8)
        asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                       "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                     : "r"(addr));
    else
        asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                     : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int q = 0; q < W / 2; ++q)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            lo[2 * q + e] = tc::tmem_done(r[4 * q + e]);
            hi[2 * q + e] = tc::tmem_done(r[4 * q + 2 + e]);
        }
}

template <int RP, bool TRANS, int YS>
__global__ void __launch_bounds__(AD_THREADS) expand_tc_kernel(const AdExpand a, const AdOrder o, uint32_t *err) {
    using S = Expand<RP, YS>;
    extern __shared__ __align__(128) unsigned char raw[];
    __shared__ uint64_t bars[3];                  // a block's products are done (two, in turn); all
    __shared__ uint32_t holder;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_wait();
    const uint32_t tmem = tensor_begin<3, S::COLUMNS>(bars, holder), bar = tc::smem_u32(bars);
    pdl_trigger();
    const AdRows tile = ad_tile(o, (int)blockIdx.x);
    const int64_t c_from = (int64_t)blockIdx.y * a.per, c_to = min(c_from + a.per, a.cols);
    if (tile.rows == 0 || c_from >= c_to || (tile.key == 0 && !a.relu)) {
        tensor_end<S::COLUMNS>(tmem);
        return;
    }
    const bool out = tile.key > o.adapters, none = tile.key == 0;               // NaN; act alone
    const bool product_wanted = !out && !none && a.rank > 0;                     // rank 0: no vectors have been written
    const uint32_t vb = (tc::smem_u32(raw) + 1023u) & ~1023u, mb = vb + a.parts * S::V_BYTES;
    const __nv_bfloat16 *m = static_cast<const __nv_bfloat16 *>(a.m) + (product_wanted ? (int64_t)(tile.key - 1) * a.m_adapter : 0);
    const int n = (int)((c_to - c_from + S::COLS - 1) / S::COLS);
    using VT = Tile<RP>;
    using MT = Tile<TRANS ? S::COLS : RP>;
    // each thread's copies of the matrix, a block further on with each block
    const char *mp[S::MV];
    uint32_t m_to[S::MV];
    int m_left[S::MV];                            // blocks whose values are there
#pragma unroll
    for (int i = 0; i < S::MV; ++i) {
        const int v = tid + i * AD_THREADS, r = v / MT::CHUNKS, q = v % MT::CHUNKS, j = TRANS ? r : q * 8;
        const int64_t c = c_from + (TRANS ? q * 8 : r);
        m_left[i] = v < S::COLS * (RP / 8) ? j < a.rank && c < a.cols ? (int)((a.cols - c + S::COLS - 1) / S::COLS) : 0 : -1;
        m_to[i] = MT::at(TRANS ? r : S::dealt(r), q, TRANS ? RP : S::COLS);
        mp[i] = reinterpret_cast<const char *>(m + (m_left[i] > 0 ? (TRANS ? j * a.m_row + c : c * a.m_row + j) : 0));
    }
    const int64_t m_step = 2 * (TRANS ? S::COLS : S::COLS * a.m_row);
    auto copy = [&](int b) {
        const uint32_t bm = mb + (b % S::STAGES) * S::M_BYTES;
#pragma unroll
        for (int i = 0; i < S::MV; ++i) {
            if (m_left[i] < 0) break;
            const bool there = b < m_left[i];
            const char *p = there ? mp[i] : reinterpret_cast<const char *>(m);
            if constexpr (TRANS) {
                // four pairs of columns, each to its place
                const int v = tid + i * AD_THREADS, r = v / MT::CHUNKS, q = v % MT::CHUNKS;
#pragma unroll
                for (int i2 = 0; i2 < 4; ++i2) {
                    const int to = S::dealt(q * 8 + 2 * i2);
                    copy4_if(bm + MT::at(r, to / 8, RP) + to % 8 * 2, p + 4 * i2, there);
                }
            } else {
                copy16_if(bm + m_to[i], p, there);
            }
            mp[i] += m_step;
        }
    };
    if (product_wanted) {
        for (int v = tid; v < a.parts * AD_ROWS * (RP / 8); v += AD_THREADS) {
            const int p = v / (AD_ROWS * (RP / 8)), r = v / (RP / 8) % AD_ROWS, q = v % (RP / 8);
            const bool there = r < tile.rows;
            copy16_if(vb + p * S::V_BYTES + VT::at(r, q, AD_ROWS),
                      static_cast<const uint4 *>(a.v) + (there ? (p * o.t + tile.slot0 + r) * (RP / 8) + q : 0), there);
        }
#pragma unroll
        for (int i = 0; i < S::STAGES - 1; ++i) {
            if (i < n) copy(i);
            copies_end();
        }
    }
    // This thread's rows: lane / 4 + 8 i of the warp's 32; its columns: W from W (lane % 4) on of each 4 W of the warp's half.
    constexpr int W = S::W, G = S::HALF / (4 * W);
    const int half = (warp >> 2) * S::HALF, lane_c = half + (lane & 3) * W;
    char *yr[4];
    bool have[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = (warp & 3) * 32 + i * 8 + (lane >> 2);
        have[i] = row < tile.rows;
        yr[i] = static_cast<char *>(a.y) + (have[i] ? (o.order != nullptr ? (int64_t)o.order[tile.slot0 + row] : tile.slot0 + row) * a.ldy * YS : 0);
    }
    const float nan = __uint_as_float(0x7FC00000u);
    using Y = uint4[G][4];
    Y even, odd;                                  // y of the blocks of even and of odd number, two ahead
    auto y_fetch = [&](int b, Y &y) {
        const int64_t c = c_from + (int64_t)b * S::COLS + lane_c;
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) y[g][i] = ld_if(yr[i] + (c + g * 4 * W) * YS, have[i] && c + g * 4 * W < c_to);
    };
    y_fetch(0, even);
    y_fetch(1, odd);
    const uint32_t mine = tmem + ((uint32_t)(warp & 3) << 21) + (uint32_t)half;
    // adds a block's sums (none where there is no product) to y
    auto finish = [&](int b, const Y &y) {
        const int64_t c = c_from + (int64_t)b * S::COLS + lane_c;
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float v[2][W];
                if (product_wanted) {
                    tmem_quads<W>(mine + ((uint32_t)h << 20) + (b & 1) * S::COLS + g * 4 * W, v[0], v[1]);
                } else {
#pragma unroll
                    for (int e = 0; e < W; ++e) v[0][e] = v[1][e] = 0.f;
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float w[W];
                    if constexpr (YS == 4) unpack16<float>(y[g][2 * h + i], w);
                    else if (a.y_dtype == CT_DT_F16) unpack16<__half>(y[g][2 * h + i], w);
                    else unpack16<__nv_bfloat16>(y[g][2 * h + i], w);
#pragma unroll
                    for (int e = 0; e < W; ++e) w[e] += v[i][e];
                    if (a.relu || out)
#pragma unroll
                        for (int e = 0; e < W; ++e) w[e] = out ? nan : w[e] < 0.f ? 0.f : w[e];
                    if (have[2 * h + i] && c + g * 4 * W < c_to) {
                        uint4 *p = reinterpret_cast<uint4 *>(yr[2 * h + i] + (c + g * 4 * W) * YS);
                        if constexpr (YS == 4) *p = pack16<float>(w);
                        else *p = a.y_dtype == CT_DT_F16 ? pack16<__half>(w) : pack16<__nv_bfloat16>(w);
                    }
                }
            }
    };
    bool ok = true;
    constexpr uint32_t how = product(true, false, TRANS, AD_ROWS, S::COLS);
    // one block's products on their way, those of the block before (whose y is given) into y, the y of the block after next
    auto advance = [&](int b, Y &y) -> bool {
        copies_wait<S::STAGES - 2>();
        fence_operands();
        fence_before();
        if (!__syncthreads_and(ok)) return false;
        if (warp == 0 && tc::elect_one()) {
            fence_after();
            const uint32_t bm = mb + (b % S::STAGES) * S::M_BYTES;
            for (int p = a.parts - 1; p >= 0; --p)
#pragma unroll
                for (int k = 0; k < RP / 16; ++k) {
                    // 16 values along the rank: 32 bytes of a row, in the next block of 64 after four
                    const uint32_t av = vb + p * S::V_BYTES + (k >> 2) * AD_ROWS * 128 + (k & 3) * 32;
                    const uint64_t da = operand(av, 16, 8 * VT::ROW, VT::SWIZZLE);
                    const uint64_t db = TRANS ? operand(bm + 16 * k * 128, RP * 128, 1024, SW128)
                                              : operand(bm + (k >> 2) * S::COLS * 128 + (k & 3) * 32, 16, 8 * MT::ROW, MT::SWIZZLE);
                    tc::umma_f16(tmem + (b & 1) * S::COLS, da, db, how, p < a.parts - 1 || k > 0);
                }
            tc::umma_commit(bar + 8 * (b & 1));
        }
        __syncwarp();
        if (b > 0) {
            ok = ok && tc::mbar_wait(bar + 8 * (b - 1 & 1), (b - 1) >> 1 & 1, err, E_ADAPTERS);
            __syncwarp();
        }
        if (ok && b + S::STAGES - 1 < n) copy(b + S::STAGES - 1);               // into the stage whose products are done
        copies_end();
        if (b > 0 && ok) {
            fence_after();
            finish(b - 1, y);
            y_fetch(b + 1, y);
        }
        return true;
    };
    int b = 0;
    if (product_wanted) {
        for (; b < n; b += 2) {
            if (!advance(b, odd)) break;
            if (b + 1 < n && !advance(b + 1, even)) break;
        }
        copies_wait<0>();
        if (b >= n) {
            ok = ok && tc::mbar_wait(bar + 8 * (n - 1 & 1), (n - 1) >> 1 & 1, err, E_ADAPTERS);
            __syncwarp();
            fence_after();
            if (ok && (n & 1)) finish(n - 1, even);
            else if (ok) finish(n - 1, odd);
        } else {
            if (warp == 0 && tc::elect_one()) tc::umma_commit(bar + 16);        // gave up: what was issued, before its memory goes
            tc::mbar_wait(bar + 16, 0, err, E_ADAPTERS);
        }
    } else {
        for (; b < n; b += 2) {
            finish(b, even);
            y_fetch(b + 2, even);
            if (b + 1 < n) {
                finish(b + 1, odd);
                y_fetch(b + 3, odd);
            }
        }
    }
    tensor_end<S::COLUMNS>(tmem);
}

// ---------------------------------------------------------------- outer

constexpr int OUTER_COLS = 128;

// The parts of v lie side by side as columns of one product; their sums are added when they are moved to registers.
template <int RP, int PARTS> struct Outer {
    static constexpr int N = RP * PARTS, X_BYTES = AD_STEP * OUTER_COLS * 2, V_BYTES = AD_STEP * 2 * RP, STAGE = X_BYTES + PARTS * V_BYTES;
    static constexpr int STAGES = STAGE <= 24576 ? 4 : STAGE <= 32768 ? 3 : 4, SMEM = STAGES * STAGE + 1024, COLUMNS = columns_of(2 * N);
    static constexpr int SUM = OUTER_COLS * sums_pitch(RP) * 4;
    static constexpr int VV = (AD_STEP * (RP / 8) * PARTS + AD_THREADS - 1) / AD_THREADS;
    static_assert(N <= 256 && SUM <= SMEM, "one product's columns, and the sums in the stages' memory");
};

template <int RP, int PARTS>
__global__ void __launch_bounds__(AD_THREADS) outer_tc_kernel(const __grid_constant__ AdOuters two, const AdOrder o, int splits, uint32_t *err) {
    using S = Outer<RP, PARTS>;
    extern __shared__ __align__(128) unsigned char raw[];
    __shared__ uint64_t bars[S::STAGES + 3];      // a stage's products are done; a group's sums are there (two, in turn); all
    __shared__ uint32_t holder;
    const int rank = splits > 1 ? (int)tc::cluster_ctarank() : 0, adapter = blockIdx.y, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int block = (int)(blockIdx.x / (unsigned)splits);
    const AdOuter &a = two.a[block >= two.first];
    const int64_t cols0 = (int64_t)(block >= two.first ? block - two.first : block) * OUTER_COLS;
    pdl_wait();
    const uint32_t tmem = tensor_begin<S::STAGES + 3, S::COLUMNS>(bars, holder), bar = tc::smem_u32(bars);
    const uint32_t base = (tc::smem_u32(raw) + 1023u) & ~1023u;
    pdl_trigger();
    const int64_t from = o.order != nullptr ? o.first[adapter + 1] : 0, to = o.order != nullptr ? o.end[adapter + 1] : adapter == 0 ? o.t : 0;
    const int64_t steps = (to - from + AD_STEP - 1) / AD_STEP;
    const int64_t s0 = steps * rank / splits, t0 = from + s0 * AD_STEP;
    const int n = (int)(steps * (rank + 1) / splits - s0), left = (int)min((int64_t)n * AD_STEP, to - t0);      // steps, rows
    using XT = Tile<OUTER_COLS>;
    using VT = Tile<RP>;
    // Each thread's copies, 64 rows further on with each step: of x, rows tid / 16 + 16 i, 16 bytes at 16 (tid % 16)
    const int64_t xc = cols0 + (tid & 15) * 8;
    const bool x_there = xc < a.cols;
    const char *x0 = reinterpret_cast<const char *>(static_cast<const __nv_bfloat16 *>(a.x) + (x_there ? xc : 0));
    const uint32_t x_to = XT::at(tid / 16, tid & 15, AD_STEP);
    int32_t next[4];                              // the rows of the next step to copy
    auto rows_of = [&](int step) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = step * AD_STEP + tid / 16 + 16 * i;
            next[i] = o.order == nullptr ? (int32_t)(t0 + r) : r < left ? o.order[t0 + r] : 0;
        }
    };
    rows_of(0);
    const uint4 *vp[S::VV];
    uint32_t v_to[S::VV];
    int v_row[S::VV];
#pragma unroll
    for (int i = 0; i < S::VV; ++i) {
        const int v = tid + i * AD_THREADS, p = v / (AD_STEP * (RP / 8)), r = v / (RP / 8) % AD_STEP, q = v % (RP / 8);
        v_row[i] = v < AD_STEP * (RP / 8) * PARTS ? r : INT32_MAX / 2;
        v_to[i] = p * S::V_BYTES + VT::at(r, q, AD_STEP);
        vp[i] = static_cast<const uint4 *>(a.v) + ((p < PARTS ? p : 0) * o.t + t0 + r) * (RP / 8) + q;
    }
    int to_copy = 0, copy_stage = 0;              // the next step to copy, its stage
    auto copy = [&]() {
        const uint32_t bx = base + copy_stage * S::STAGE, bv = bx + S::X_BYTES;
        const int rest = left - to_copy * AD_STEP;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool there = x_there && tid / 16 + 16 * i < rest;
            copy16_if(bx + x_to + 16 * i * 128, x0 + (there ? (int64_t)next[i] * a.ldx * 2 : 0), there);
        }
#pragma unroll
        for (int i = 0; i < S::VV; ++i) {
            const bool there = v_row[i] < rest;
            if (v_row[i] < AD_STEP) copy16_if(bv + v_to[i], there ? vp[i] : static_cast<const uint4 *>(a.v), there);
            vp[i] += AD_STEP * (RP / 8);
        }
        ++to_copy;
        copy_stage = copy_stage + 1 == S::STAGES ? 0 : copy_stage + 1;
        rows_of(to_copy);
    };
    float sum[RP / 2];
#pragma unroll
    for (int j = 0; j < RP / 2; ++j) sum[j] = 0.f;
    bool ok = true;
    int groups = 0;                               // whose sums are in registers
    const uint32_t mine = tmem + ((uint32_t)(warp & 3) << 21) + (uint32_t)(warp >> 2) * (RP / 2);
    auto collect = [&]() {
        ok = ok && tc::mbar_wait(bar + 8 * (S::STAGES + (groups & 1)), (groups >> 1) & 1, err, E_ADAPTERS);
        __syncwarp();
        fence_after();
#pragma unroll
        for (int j = 0; j < RP / 2; j += 8) {
            float all[8], v[8];
            tmem_ld8(mine + (groups & 1) * S::N + (PARTS - 1) * RP + j, all);
#pragma unroll
            for (int p = PARTS - 2; p >= 0; --p) {                               // the least parts first
                tmem_ld8(mine + (groups & 1) * S::N + p * RP + j, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) all[e] += v[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[j + e] += all[e];
        }
        fence_before();
        ++groups;
    };
#pragma unroll
    for (int i = 0; i < S::STAGES; ++i) {
        if (i < n) copy();
        copies_end();
    }
    constexpr uint32_t how = product(true, true, true, OUTER_COLS, S::N);
    int at = 0, stage = 0;                        // the step, its stage
    uint32_t done = 0;                            // bit s: parity of stage s's next end of products
    for (; at < n; ++at) {
        copies_wait<S::STAGES - 1>();
        fence_operands();
        if (!__syncthreads_and(ok)) break;
        if (warp == 0 && tc::elect_one()) {
            fence_after();
            const uint32_t bx = base + stage * S::STAGE, bv = bx + S::X_BYTES;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                tc::umma_f16(tmem + (at / FLUSH & 1) * S::N, operand(bx + 16 * k * 128, AD_STEP * 128, 1024, SW128),
                             operand(bv + 16 * k * VT::ROW, AD_STEP * VT::ROW, 8 * VT::ROW, VT::SWIZZLE), how, at % FLUSH > 0 || k > 0);
            tc::umma_commit(bar + 8 * stage);
            if (at % FLUSH == FLUSH - 1 || at == n - 1) tc::umma_commit(bar + 8 * (S::STAGES + (at / FLUSH & 1)));
        }
        __syncwarp();
        if (at + S::STAGES < n) {
            // the stage again, once its products are done: they take a fraction of the time that the next stages' copies do
            ok = ok && tc::mbar_wait(bar + 8 * stage, done >> stage & 1, err, E_ADAPTERS);
            done ^= 1u << stage;
            if (ok) copy();
        }
        copies_end();
        if (at % FLUSH == 1 && at > FLUSH) collect();
        stage = stage + 1 == S::STAGES ? 0 : stage + 1;
    }
    copies_wait<0>();
    if (at == n) {
        while (groups < (n + FLUSH - 1) / FLUSH) collect();
    } else if (warp == 0 && tc::elect_one()) {
        tc::umma_commit(bar + 8 * (S::STAGES + 2));                              // gave up: what was issued, before its memory goes
    }
    if (at < n) tc::mbar_wait(bar + 8 * (S::STAGES + 2), 0, err, E_ADAPTERS);
    tensor_end<S::COLUMNS>(tmem);

    float *fs = reinterpret_cast<float *>(raw) + ((warp & 3) * 32 + lane) * sums_pitch(RP) + (warp >> 2) * (RP / 2);
#pragma unroll
    for (int j = 0; j < RP / 2; j += 4) *reinterpret_cast<float4 *>(fs + j) = make_float4(sum[j], sum[j + 1], sum[j + 2], sum[j + 3]);
    if (splits > 1) tc::cluster_sync();
    else __syncthreads();
    write_gradient<RP>(a, adapter, cols0, reinterpret_cast<const float *>(raw), rank, splits);
    if (splits > 1) tc::cluster_sync();           // no CTA leaves while another reads its sums
}

// ---------------------------------------------------------------- host

template <typename T, int RP, int WHICH> cudaError_t shrink(const AdShrinks &two, const AdOrder &o, int tiles, int splits, uint32_t *err, cudaStream_t st) {
    using S = Shrink<RP>;
    static std::atomic<bool> sized[MAX_DEVICES];
    auto *kernel = shrink_tc_kernel<T, RP, WHICH>;
    const cudaError_t e = allow_smem(kernel, sized, S::SMEM);
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)((WHICH == BOTH ? 2 : 1) * tiles * splits));
    return ad_launch(kernel, grid, S::SMEM, st, splits, two.a[0].first && o.order != nullptr, two, o, tiles, splits, err);
}
template <typename T, int WHICH> cudaError_t shrink_rank(const AdShrinks &two, const AdOrder &o, int tiles, int splits, uint32_t *err, cudaStream_t st) {
    switch (ad_padded(two.a[0].rank)) {
        case 16: return shrink<T, 16, WHICH>(two, o, tiles, splits, err, st);
        case 32: return shrink<T, 32, WHICH>(two, o, tiles, splits, err, st);
        case 64: return shrink<T, 64, WHICH>(two, o, tiles, splits, err, st);
        default: return shrink<T, 128, WHICH>(two, o, tiles, splits, err, st);
    }
}

template <int RP, bool TRANS, int YS> cudaError_t expand(const AdExpand &q, const AdOrder &o, int tiles, uint32_t *err, cudaStream_t st) {
    using S = Expand<RP, YS>;
    static std::atomic<bool> sized[MAX_DEVICES];
    auto *kernel = expand_tc_kernel<RP, TRANS, YS>;
    const cudaError_t e = allow_smem(kernel, sized, (size_t)S::smem(3));
    if (e != cudaSuccess) return e;
    // columns of a CTA: as many as leave each SM two CTAs, which are resident together, at most 32 blocks
    AdExpand a = q;
    const int64_t blocks = (a.cols + S::COLS - 1) / S::COLS;
    int64_t parts = 2 * (int64_t)sm_count() / tiles;
    if (parts < (blocks + 31) / 32) parts = (blocks + 31) / 32;
    if (parts > blocks) parts = blocks;
    if (parts > 65535) parts = 65535;
    a.per = (blocks + parts - 1) / parts * S::COLS;
    const dim3 grid((unsigned)tiles, (unsigned)((a.cols + a.per - 1) / a.per));
    return ad_launch(kernel, grid, (size_t)S::smem(a.parts), st, 1, false, a, o, err);
}
template <bool TRANS, int YS> cudaError_t expand_rank(const AdExpand &a, const AdOrder &o, int tiles, uint32_t *err, cudaStream_t st) {
    switch (ad_padded(a.rank)) {
        case 16: return expand<16, TRANS, YS>(a, o, tiles, err, st);
        case 32: return expand<32, TRANS, YS>(a, o, tiles, err, st);
        case 64: return expand<64, TRANS, YS>(a, o, tiles, err, st);
        default: return expand<128, TRANS, YS>(a, o, tiles, err, st);
    }
}

template <int RP, int PARTS> cudaError_t outer(const AdOuters &two, int blocks, const AdOrder &o, int splits, uint32_t *err, cudaStream_t st) {
    using S = Outer<RP, PARTS>;
    static std::atomic<bool> sized[MAX_DEVICES];
    auto *kernel = outer_tc_kernel<RP, PARTS>;
    const cudaError_t e = allow_smem(kernel, sized, S::SMEM);
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)(blocks * splits), (unsigned)o.adapters);
    return ad_launch(kernel, grid, S::SMEM, st, splits, false, two, o, splits, err);
}
}  // namespace

cudaError_t ad_shrink_tc(const AdShrink (&a)[2], AdWhich which, bool bf16, const AdOrder &o, int tiles, int splits, cudaStream_t st) {
    uint32_t *err = device_error_word();
    if (err == nullptr) return cudaErrorUnknown;
    const AdShrinks two = {{a[0], a[1]}};
    if (bf16)
        return which == AD_FORWARD    ? shrink_rank<__nv_bfloat16, FORWARD>(two, o, tiles, splits, err, st)
               : which == AD_BACKWARD ? shrink_rank<__nv_bfloat16, BACKWARD>(two, o, tiles, splits, err, st)
                                      : shrink_rank<__nv_bfloat16, BOTH>(two, o, tiles, splits, err, st);
    return which == AD_FORWARD    ? shrink_rank<__half, FORWARD>(two, o, tiles, splits, err, st)
           : which == AD_BACKWARD ? shrink_rank<__half, BACKWARD>(two, o, tiles, splits, err, st)
                                  : shrink_rank<__half, BOTH>(two, o, tiles, splits, err, st);
}
cudaError_t ad_expand_tc(const AdExpand &a, bool trans, const AdOrder &o, int tiles, cudaStream_t st) {
    uint32_t *err = device_error_word();
    if (err == nullptr) return cudaErrorUnknown;
    if (a.y_dtype == CT_DT_F32) return trans ? expand_rank<true, 4>(a, o, tiles, err, st) : expand_rank<false, 4>(a, o, tiles, err, st);
    return trans ? expand_rank<true, 2>(a, o, tiles, err, st) : expand_rank<false, 2>(a, o, tiles, err, st);
}
bool ad_outer_tc_takes(int64_t rank, int parts) { return ad_padded(rank) * parts <= 256; }
cudaError_t ad_outer_tc(const AdOuters &two, int blocks, const AdOrder &o, int splits, cudaStream_t st) {
    uint32_t *err = device_error_word();
    if (err == nullptr) return cudaErrorUnknown;
    const bool p2 = two.a[0].parts == 2;
    switch (ad_padded(two.a[0].rank)) {
        case 16: return p2 ? outer<16, 2>(two, blocks, o, splits, err, st) : outer<16, 3>(two, blocks, o, splits, err, st);
        case 32: return p2 ? outer<32, 2>(two, blocks, o, splits, err, st) : outer<32, 3>(two, blocks, o, splits, err, st);
        case 64: return p2 ? outer<64, 2>(two, blocks, o, splits, err, st) : outer<64, 3>(two, blocks, o, splits, err, st);
        default: return outer<128, 2>(two, blocks, o, splits, err, st);
    }
}

}  // namespace ops
}  // namespace ct
