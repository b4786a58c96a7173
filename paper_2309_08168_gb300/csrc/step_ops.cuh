// step_ops.cuh - what the operators of ssd_step.h share.
#pragma once

#include <initializer_list>
#include <mutex>

#include "ssd_step.h"
#include "tree_ops.cuh"

namespace ssd {
namespace step {
using namespace tree;

// whether two ranges of bytes meet; NULL meets nothing
struct Range {
    const void* p;
    size_t n;
};
inline bool meet(const void* a, size_t na, const void* b, size_t nb) {
    return a && b && (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}
// whether some range of one list meets one of the other
template <size_t N, size_t M>
inline bool meet(const Range (&a)[N], const Range (&b)[M]) {
    for (const Range& x : a)
        for (const Range& y : b)
            if (meet(x.p, x.n, y.p, y.n)) return true;
    return false;
}
// bytes from the first row's start to the last row's end
inline size_t span(int n_rows, int64_t stride, int64_t width, int dtype) {
    return ((size_t)(n_rows - 1) * (size_t)stride + (size_t)width) * (dtype == SSD_F32 ? 4 : 2);
}

// whether all of these addresses are multiples of `to` bytes
inline bool aligned(size_t to, std::initializer_list<const void*> all) {
    uintptr_t bits = 0;
    for (const void* p : all) bits |= (uintptr_t)p;
    return bits % to == 0;
}

// the current device
constexpr int kMaxDevices = 64;
inline int device_of(const char* call, int* dev) {
    if (cudaGetDevice(dev) != cudaSuccess || *dev < 0 || *dev >= kMaxDevices) {
        (void)cudaGetLastError();
        return refuse(SSD_ERR_CUDA, call, "no usable current device");
    }
    return SSD_OK;
}

// Loads kernels that need no other set-up.  (Left to a first launch, it may come inside a stream capture.)
inline cudaError_t loaded(std::initializer_list<const void*> kernels) {
    cudaFuncAttributes at;
    cudaError_t e = cudaSuccess;
    for (const void* k : kernels)
        if (e == cudaSuccess) e = cudaFuncGetAttributes(&at, k);
    return e;
}
// ... once a device
template <auto... kKernels>
inline int set_up_once(const char* call) {
    static std::mutex mu;
    static bool ready[kMaxDevices] = {};
    int dev = 0;
    if (int rc = device_of(call, &dev)) return rc;
    std::lock_guard<std::mutex> lock(mu);
    if (ready[dev]) return SSD_OK;
    if (const cudaError_t e = loaded({(const void*)kKernels...})) return refuse(SSD_ERR_CUDA, call, "set-up: %s", cudaGetErrorString(e));
    ready[dev] = true;
    return SSD_OK;
}

// ---------------------------------------------------------------------------
// two fp32 operations in one instruction
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint64_t pair_of(float x, float y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};\n" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ float2 of_pair(uint64_t p) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;\n" : "=f"(r.x), "=f"(r.y) : "l"(p));
    return r;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t x, uint64_t y) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;\n" : "=l"(r) : "l"(x), "l"(y));
    return r;
}
__device__ __forceinline__ uint64_t mul_pair(uint64_t x, uint64_t y) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;\n" : "=l"(r) : "l"(x), "l"(y));
    return r;
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t x, uint64_t y, uint64_t z) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;\n" : "=l"(r) : "l"(x), "l"(y), "l"(z));
    return r;
}

// ---------------------------------------------------------------------------
// clusters
// ---------------------------------------------------------------------------
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;\n" ::: "memory");
}
__device__ __forceinline__ uint32_t peer_address(const void* p, uint32_t cta) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(at) : "r"(smem_u32(p)), "r"(cta));
    return at;
}
__device__ __forceinline__ uint64_t peer_load(const void* p, uint32_t cta) {
    uint64_t v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];\n" : "=l"(v) : "r"(peer_address(p, cta)) : "memory");
    return v;
}
__device__ __forceinline__ void peer_store(void* p, uint32_t cta, uint64_t v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;\n" ::"r"(peer_address(p, cta)), "l"(v) : "memory");
}

}  // namespace step
}  // namespace ssd
