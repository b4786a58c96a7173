// tree_ops.cuh - what the operators of ssd_ops.h share: checks of their
// arguments, launches, and the places of cache rows.
#pragma once

#include <cstdarg>
#include <cstdio>

#include "ssd.h"
#include "ssd_internal.cuh"
#include "ssd_ops.h"

namespace ssd {
namespace tree {

constexpr int kMaxNodes = 256;     // nodes of a tree with masks, and of one that is committed
constexpr int kMaxRequests = 4096;

// sets the message "call: ..." and returns the code
inline int refuse(int code, const char* call, const char* fmt, ...) {
    char text[320];
    const int n = snprintf(text, sizeof text, "%s: ", call);
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(text + n, sizeof text - (size_t)n, fmt, ap);
    va_end(ap);
    return set_last_error(code, text);
}
inline int refuse_arg(const char* call, const char* what) { return refuse(SSD_ERR_INVALID_ARG, call, "%s", what); }

inline int check_batch(const char* call, const ssd_batch* b) {
    if (!b || !b->row_start || !b->lens || !b->block_table) return refuse_arg(call, "NULL pointer in the batch");
    if (b->n_requests < 1 || b->n_requests > kMaxRequests || b->n_rows < 0 || b->max_rows < 1 || b->max_blocks < 1)
        return refuse_arg(call, "need 1 <= n_requests <= 4096, n_rows >= 0, max_rows >= 1, max_blocks >= 1");
    return SSD_OK;
}
inline int check_page_size(const char* call, int page_size, int n_pages) {
    if (page_size < 16 || page_size > 65536 || page_size % 16 || n_pages < 1 || (long long)page_size * n_pages >= (1ll << 31))
        return refuse_arg(call, "need page_size a multiple of 16, 16 .. 65536, n_pages >= 1, n_pages * page_size < 2^31");
    return SSD_OK;
}
inline int check_pages(const char* call, const ssd_pages* c) {
    if (!c || !c->k || !c->v) return refuse_arg(call, "NULL pointer in the cache");
    if (((uintptr_t)c->k | (uintptr_t)c->v) & 15u) return refuse_arg(call, "the cache must be 16-byte aligned");
    if (c->dtype != SSD_F16 && c->dtype != SSD_BF16) return refuse_arg(call, "the cache must be fp16 or bf16");
    if (c->head_dim != 64 && c->head_dim != 128) return refuse_arg(call, "head_dim must be 64 or 128");
    if (c->n_layers < 1 || c->n_kv_heads < 1) return refuse_arg(call, "need n_layers >= 1 and n_kv_heads >= 1");
    if (int rc = check_page_size(call, c->page_size, c->n_pages)) return rc;
    // (2^37 elements are the 2^38 bytes that one GPU's memory does not exceed)
    const int64_t most = int64_t(1) << 37;
    const int64_t s[4] = {c->layer_stride, c->page_stride, c->head_stride, c->pos_stride};
    for (int i = 0; i < 4; ++i)
        if (s[i] < 0 || s[i] > most || s[i] % 8)
            return refuse_arg(call, "cache strides must be multiples of 8 elements, 0 .. 2^37");
    if (c->pos_stride < c->head_dim) return refuse_arg(call, "pos_stride is shorter than a head");
    if ((c->n_kv_heads > 1 && c->head_stride < c->head_dim) || (c->n_pages > 1 && c->page_stride < c->head_dim) ||
        (c->n_layers > 1 && c->layer_stride < c->head_dim))
        return refuse_arg(call, "a cache stride is shorter than a head");
    return SSD_OK;
}
// rows of fp32 and fp16 go with an fp16 cache, of bf16 with a bf16 cache
inline int check_rows_type(const char* call, int dtype, const ssd_pages* c) {
    const bool ok = c->dtype == SSD_F16 ? dtype == SSD_F32 || dtype == SSD_F16 : dtype == SSD_BF16;
    return ok ? SSD_OK : refuse_arg(call, "rows are fp32 or fp16 over an fp16 cache, bf16 over a bf16 cache");
}
inline int check_rows(const char* call, const char* what, const void* p, int64_t stride, int dtype, int64_t width) {
    const int64_t per16 = dtype == SSD_F32 ? 4 : 8;
    if (((uintptr_t)p & 15u) || stride % per16 || stride < width || stride > (int64_t(1) << 37))
        return refuse(SSD_ERR_INVALID_ARG, call, "%s: rows must be 16-byte aligned, a multiple of 16 bytes apart and not overlap", what);
    return SSD_OK;
}

// whether p is memory of the current device (of a call's tensors one is looked at)
inline int check_device(const char* call, const void* p) {
    int dev = 0;
    cudaPointerAttributes at = {};
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaPointerGetAttributes(&at, p);
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        return refuse(SSD_ERR_CUDA, call, "%s", cudaGetErrorString(e));
    }
    if ((at.type != cudaMemoryTypeDevice && at.type != cudaMemoryTypeManaged) || at.device != dev)
        return refuse(SSD_ERR_INVALID_ARG, call, "the tensors are not in memory of the current device (%d)", dev);
    return SSD_OK;
}

// Launch that may start while the previous kernel of the stream ends (every
// kernel waits for that one's results before it touches memory that either writes).
template <typename... P, typename... A>
inline int launch(const char* call, void (*k)(P...), dim3 grid, int threads, size_t smem, void* stream, const A&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, k, args...);
    return e == cudaSuccess ? SSD_OK : refuse(SSD_ERR_CUDA, call, "%s", cudaGetErrorString(e));
}

// ---------------------------------------------------------------------------
// device side
// ---------------------------------------------------------------------------
// the rows of a request, kept inside [0, n_rows) whatever row_start holds
struct Rows {
    int r0, n;
};
__device__ __forceinline__ Rows rows_of(const int32_t* row_start, int b, int n_rows) {
    const int s = min(max(__ldcg(row_start + b), 0), n_rows), e = min(max(__ldcg(row_start + b + 1), s), n_rows);
    return {s, e - s};
}

__device__ __forceinline__ void say(int32_t* status, int bit) {
    if (status) atomicOr(status, bit);
}

// element types: 16 bytes of rows to and from fp32
template <typename T>
struct Vec;
template <>
struct Vec<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void get(const uint4& u, float (&f)[4]) {
        f[0] = __uint_as_float(u.x), f[1] = __uint_as_float(u.y), f[2] = __uint_as_float(u.z), f[3] = __uint_as_float(u.w);
    }
    static __device__ __forceinline__ uint4 put(const float (&f)[4]) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};
__device__ __forceinline__ uint32_t pack2(float a, float b, f16) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack2(float a, float b, bf16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float2 unpack2(uint32_t u, f16) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }
__device__ __forceinline__ float2 unpack2(uint32_t u, bf16) { return make_float2(bf16_lo(u), bf16_hi(u)); }
template <typename T>
struct Vec16 {
    static constexpr int N = 8;
    static __device__ __forceinline__ void get(const uint4& u, float (&f)[8]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 p = unpack2(w[i], T());
            f[2 * i] = p.x;
            f[2 * i + 1] = p.y;
        }
    }
    static __device__ __forceinline__ uint4 put(const float (&f)[8]) {
        return make_uint4(pack2(f[0], f[1], T()), pack2(f[2], f[3], T()), pack2(f[4], f[5], T()), pack2(f[6], f[7], T()));
    }
};
template <>
struct Vec<f16> : Vec16<f16> {};
template <>
struct Vec<bf16> : Vec16<bf16> {};

}  // namespace tree
}  // namespace ssd
