// Shared by the operators at the ends of a training step (embedding.cu, losses.cu, adamw.cu): whole-number operands, 32-byte
// stores, the device's size.
#pragma once

#include <atomic>

#include "blocks.cuh"

namespace srq {

// SMs of the current device (0 on an error); looked up once per device.
inline int sm_count() {
    static std::atomic<int> known[64];
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    if (dev >= 0 && dev < 64 && (n = known[dev].load(std::memory_order_relaxed)) != 0) return n;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    if (dev >= 0 && dev < 64) known[dev].store(n, std::memory_order_relaxed);
    return n;
}

// Element i of a vector of ids, targets or offsets.
__device__ __forceinline__ int64_t whole_at(const void* p, int wide, int64_t i) {
    return wide ? reinterpret_cast<const int64_t*>(p)[i] : (int64_t)reinterpret_cast<const int32_t*>(p)[i];
}

// Ordinary 32-byte stores (one instruction on this architecture).  Volatile, so that none moves ahead of the wait a kernel starts with.
struct alignas(32) Word8 { uint32_t w[8]; };
__device__ __forceinline__ void store32(void* p, const Word8& r) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]), "r"(r.w[4]), "r"(r.w[5]), "r"(r.w[6]), "r"(r.w[7]) : "memory");
}

}  // namespace srq
