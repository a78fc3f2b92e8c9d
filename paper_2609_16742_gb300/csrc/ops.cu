// Device facts shared by the operators of the 8-bit answer head.
#include <atomic>

#include "ops_common.cuh"

namespace ct {
namespace ops {

namespace {

__device__ uint32_t g_error_word;

std::atomic<uint32_t *> g_error_addr[MAX_DEVICES];
std::atomic<int> g_sms[MAX_DEVICES];

}  // namespace

uint32_t *device_error_word() {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return nullptr;
    uint32_t *p = g_error_addr[dev].load(std::memory_order_relaxed);
    if (p == nullptr) {
        void *q = nullptr;
        if (cudaGetSymbolAddress(&q, g_error_word) != cudaSuccess) return nullptr;
        p = static_cast<uint32_t *>(q);
        g_error_addr[dev].store(p, std::memory_order_relaxed);
    }
    return p;
}

int sm_count() {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return device_sm_count();
    int n = g_sms[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        n = device_sm_count();
        g_sms[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

}  // namespace ops
}  // namespace ct

extern "C" ct_status ct_ops_device_error(uint32_t *code) {
    if (code == nullptr) return CT_EINVAL;
    *code = 0;
    uint32_t *w = ct::ops::device_error_word();
    if (w == nullptr || cudaDeviceSynchronize() != cudaSuccess) return CT_ECUDA;
    if (cudaMemcpy(code, w, sizeof(*code), cudaMemcpyDeviceToHost) != cudaSuccess) return CT_ECUDA;
    if (*code != 0 && cudaMemset(w, 0, sizeof(*code)) != cudaSuccess) return CT_ECUDA;
    return CT_OK;
}
