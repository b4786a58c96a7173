// tree_attn.cuh - what the kernels of ssd_tree_attention share: their arguments, the
// workspace, a CTA's range, arithmetic.
#pragma once

#include "tree_ops.cuh"
#include "tree_sched.cuh"

namespace ssd {
namespace tree {

constexpr int kTile = 128;   // most rows of a tile
constexpr int kFewRows = 2;  // most rows of a tile of few_kernel

// what a CTA whose range ends inside an item leaves for join_kernel
struct alignas(16) Cut {
    int first, last;  // CTAs that hold parts of the item; last < 0: the range does not end inside one
    int first_slot;   // the first one's part is its slot 0 or 1 (the others': 0)
    int row0, rows;   // of the request: first row of its tile, rows of the tile that exist
    int r0, kvh, pad;
};

struct AttnOpArgs {
    Shape shape;
    int grid;
    const int32_t* block_table;
    const void* q;
    void* out;
    int64_t q_stride, out_stride;
    const uint64_t* masks;
    int words;
    const void *kc, *vc;  // the layer's K and V
    int64_t page_stride, head_stride, pos_stride;
    int n_heads, n_pages;
    int box_shift;  // positions per copy, log2: 16 .. 64 of them, which divide page_size
    int at_pos, at_head, at_page;  // which coordinate (1 .. 3) of the tensor maps is which
    float scale2;  // log2(e) * scale
    int tile;      // rows: up to kFewRows, or kTile
    uint64_t group_inv;  // ceil(2^32 / group)
    Cut* cuts;     // [grid]
    float* stats;  // [grid][2][2][kTile]: maximum, sum
    float4* part;  // [grid][2][HD / 4][kTile]
    int32_t* status;
    long long wait_clocks;  // after which a wait gives up
    int stall;              // a CTA that asks for no keys, so that waits of it give up; -1: none
};

// of the rows' type: the cache's, and how many of those hold a value of q on the tensor cores
template <typename T>
struct Types {
    typedef T C;
    static constexpr int PARTS = 1;
};
template <>
struct Types<float> {
    typedef f16 C;
    static constexpr int PARTS = 2;
};

// few_kernel for the rows' type and head_dim (tree_few.cu)
int launch_few(const char* call, const AttnOpArgs& a, int dtype, int hd, void* stream);

#ifdef __CUDACC__
// 2^x; below 2^-126: 0
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// two fp32 values in one register pair: fma, add and mul of both in one instruction
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 two(float a, float b) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void of_two(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// This CTA's range, from the units of all requests, a run of requests per thread of THREADS.
// Returns the units of all; every thread has passed two barriers.
template <int THREADS>
struct RangeOf {
    long long sum[THREADS / 32], off, head;  // head: units of a KV head of it
    int b;
    Req req;  // the request that the range starts in
};
template <int THREADS>
__device__ __forceinline__ long long range_of(const AttnOpArgs& a, int tile, RangeOf<THREADS>& s, Walk& walk, int& ctas) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Shape& sh = a.shape;
    const int per = (sh.n_requests + THREADS - 1) / THREADS;
    const int b0 = min(tid * per, sh.n_requests), b1 = min(b0 + per, sh.n_requests);
    long long mine = 0, head = 0;  // (a prompt's is a sum over its tiles: formed once, if the thread has one request)
    Req last{};
#pragma unroll 1
    for (int b = b0; b < b1; ++b) {
        last = req_of(sh, b);
        if (last.clipped && last.n && blockIdx.x == 0) say(a.status, SSD_STATUS_TABLE);
        if (!sh.chain && last.n > 64 * a.words && blockIdx.x == 0) say(a.status, SSD_STATUS_PARENT);
        head = head_units(sh, last, tile);
        mine += head * sh.n_kv_heads;
    }
    long long before = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += x;
    }
    if (lane == 31) s.sum[warp] = before;
    __syncthreads();
    before -= mine;
    long long units = 0;
#pragma unroll 4
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) before += s.sum[w];
        units += s.sum[w];
    }
    const int cta = blockIdx.x;
    ctas = ctas_of(units, a.grid);
    const long long lo = cta < ctas ? range_start(units, ctas, cta) : 0, hi = cta < ctas ? range_start(units, ctas, cta + 1) : 0;
    if (before <= lo && lo < before + mine) {
        long long off = lo - before;
#pragma unroll 1
        for (int b = b0; b < b1; ++b) {
            const Req q = per == 1 ? last : req_of(sh, b);
            if (per != 1) head = head_units(sh, q, tile);
            const long long n = head * sh.n_kv_heads;
            if (off < n) {
                s.head = head;
                s.b = b;
                s.req = q;
                s.off = off;
                break;
            }
            off -= n;
        }
    }
    __syncthreads();
    walk_init(walk, sh, tile, s.b, s.req, s.off, lo, hi - lo, s.head);
    return units;
}
#endif

}  // namespace tree
}  // namespace ssd
