// Helpers shared by the operators of the 8-bit answer head (quantisation,
// block-scaled products, log probabilities): element types, tensor checks on
// the host, the device-side error word.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "ct_internal.h"

namespace ct {
namespace ops {

inline int dtype_size(int dtype) { return dtype == CT_DT_F32 ? 4 : 2; }
inline bool dtype_ok(int dtype) { return dtype == CT_DT_F32 || dtype == CT_DT_F16 || dtype == CT_DT_BF16; }
inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// Memory that a call reads or writes: rows of `width` bytes, `pitch` bytes apart (0: all the same; else at least `width`).
struct Span {
    uintptr_t at;
    int64_t rows, width, pitch;
    uintptr_t end() const { return at + (uintptr_t)(rows - 1) * (uintptr_t)pitch + (uintptr_t)width; }
};
inline Span span(const void *p, int64_t rows, int64_t cols, int64_t ld, int size) {
    return {(uintptr_t)p, cols > 0 ? rows : 0, cols * size, rows > 1 ? ld * size : 0};
}
// Whether two have a byte in common.  Rows of one pitch (columns of one matrix) are compared at once, others row by row of the one that has
// fewer, where their ranges cross.
inline bool share(Span a, Span b) {
    if (a.pitch == 0 && a.rows > 1) a.rows = 1;
    if (b.pitch == 0 && b.rows > 1) b.rows = 1;
    if (a.rows <= 0 || b.rows <= 0 || a.width <= 0 || b.width <= 0 || a.at >= b.end() || b.at >= a.end()) return false;
    if (a.rows > b.rows) {
        const Span c = a;
        a = b;
        b = c;
    }
    if (b.rows == 1) return true;
    // b's first row that ends behind byte s of its store, were there rows before its own and behind them
    const auto first = [&](int64_t s) {
        const int64_t d = s - b.width, q = d / b.pitch;
        return (d % b.pitch < 0 ? q - 1 : q) + 1;
    };
    const int64_t d = (int64_t)(a.at - b.at);     // of a's first row, from b's
    if (a.rows > 1 && a.pitch == b.pitch) {
        // row i of a meets b's rows j + i and j + 1 + i, or one of them, or none
        for (int64_t j = first(d), k = j + 1; j <= k; ++j)
            if (j * b.pitch < d + a.width && j < b.rows && j + a.rows > 0) return true;
        return false;
    }
    const int64_t last = (int64_t)(b.end() - b.at);
    for (int64_t i = d + a.width > 0 ? 0 : -(d + a.width) / a.pitch + 1; i < a.rows; ++i) {
        const int64_t s = d + i * a.pitch;
        if (s >= last) return false;
        const int64_t j = s < b.width ? 0 : first(s);
        if (j < b.rows && j * b.pitch < s + a.width) return true;
    }
    return false;
}

constexpr int MAX_DEVICES = 64;

// Error word of the current device, OR-ed into by kernels whose bounded wait
// expired (ops.cu).
uint32_t *device_error_word();

// SM count of the current device, looked up once per device.
int sm_count();

// ct_fp8_quantize after its checks (fp8_quantize.cu).
ct_status quantize(const void *x, int dtype, int64_t m, int64_t k, int64_t ldx, int block_rows, uint8_t *q, int64_t ldq,
                   float *scale, int64_t srow, int64_t sblk, cudaStream_t st);

// once per kernel and device: the shared memory it may ask for
template <typename K> inline cudaError_t allow_smem(K *kernel, std::atomic<bool> (&sized)[MAX_DEVICES], size_t bytes) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < MAX_DEVICES && sized[dev].load(std::memory_order_relaxed)) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == cudaSuccess && dev < MAX_DEVICES) sized[dev].store(true, std::memory_order_relaxed);
    return e;
}

#ifdef __CUDACC__
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// 16 bytes of T as floats (4 or 8 of them)
template <typename T> struct Vec16 { static constexpr int N = 16 / (int)sizeof(T); };

template <typename T> __device__ __forceinline__ void unpack16(const uint4 &u, float *v);
template <> __device__ __forceinline__ void unpack16<float>(const uint4 &u, float *v) {
    v[0] = __uint_as_float(u.x); v[1] = __uint_as_float(u.y); v[2] = __uint_as_float(u.z); v[3] = __uint_as_float(u.w);
}
template <> __device__ __forceinline__ void unpack16<__half>(const uint4 &u, float *v) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
        v[2 * i] = f.x; v[2 * i + 1] = f.y;
    }
}
template <> __device__ __forceinline__ void unpack16<__nv_bfloat16>(const uint4 &u, float *v) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}

// 16 bytes from `shift` bytes on of the 32 in p, n; no branch, so that the loads of several units stay in flight
// together
__device__ __forceinline__ uint4 shifted(const uint4 &p, const uint4 &n, uint32_t shift) {
    const uint32_t bits = (shift & 3u) * 8u;
    const bool two = shift & 8u, one = shift & 4u;
    uint32_t w[6] = {two ? p.z : p.x, two ? p.w : p.y, two ? n.x : p.z, two ? n.y : p.w, two ? n.z : n.x, two ? n.w : n.y};
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = one ? w[i + 1] : w[i];
    return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits),
                      __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits));
}

// the first `bytes` (0 to 16) of 16, then zeros
__device__ __forceinline__ uint4 first_bytes(uint4 u, int bytes) {
    uint32_t *w = &u.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int keep = bytes - 4 * i;
        if (keep < 4) w[i] = keep <= 0 ? 0u : w[i] & ((1u << (8 * keep)) - 1u);
    }
    return u;
}

// two floats rounded to T, packed in 32 bits (16-bit types)
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <typename T> __device__ __forceinline__ uint4 pack16(const float *v) {
    return make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
}
template <> __device__ __forceinline__ uint4 pack16<float>(const float *v) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
// 8 bytes of packed values (4 or 2)
template <typename T> __device__ __forceinline__ uint64_t pack8(const float *v) {
    return (uint64_t)pack2<T>(v[2], v[3]) << 32 | pack2<T>(v[0], v[1]);
}
template <> __device__ __forceinline__ uint64_t pack8<float>(const float *v) {
    return (uint64_t)__float_as_uint(v[1]) << 32 | __float_as_uint(v[0]);
}
#endif

}  // namespace ops
}  // namespace ct
