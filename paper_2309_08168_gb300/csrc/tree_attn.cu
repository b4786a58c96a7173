// tree_attn.cu - ssd_tree_attention (ssd_ops.h): attention of a batch's rows
// over a paged cache, with the masks of their trees.
//
//   o = sum_x w_x v_x / sum_x w_x,  w_x = 2^(s_x - m),  s_x = log2(e) scale q . k_x
//
// over the positions x that a row sees, m a running maximum.  All query heads
// that share a KV head, and all nodes of the request's tree, are rows of one
// tile, so K and V are read once for all of them: with R rows a position costs
// 4 hd bytes and 4 hd R flops.  Up to some 250 rows the bound is HBM, beyond it the
// tensor cores and the exponentials.
//
// A CTA walks its range of units (tree_sched.cuh), 64 positions at a time:
//   warp TILE / 32     : TMA producer: K and V of a unit, 16 to 64 rows of a page per
//                        copy, into a ring;
//   warp TILE / 32 + 1 : MMA issuer: S = q K^T (tcgen05.mma, 128 x 64 x 16, TMEM
//                        accumulators) a unit ahead of O += P V (P in TMEM over the
//                        columns of S, V as it lies in the cache, MN-major);
//   warps 0 ..         : softmax, a row per thread: S from TMEM, P back to it, running
//                        maximum and sum; at an item's end O / sum, or O, maximum
//                        and sum to the workspace if other CTAs hold parts of the item.
// The tile has 128 rows or, for requests of up to 32 rows, 32 (the other lanes
// of the MMA are not read).  join_kernel adds the parts of cut items.
//
// O is rescaled only when a row's maximum has grown by more than kSlack (log2)
// over the one its weights are relative to (the running softmax of Milakov and
// Gimelshein, 2018).  Weights are relative to the maximum less kShift, so that
// fp16 keeps 22 bits of pairs, and 11 of single weights, down to 2^-20 of the
// largest one.
//
// fp32 rows: q and the weights enter the products as fp16 pairs hi + lo (22 bits).  A
// row of q is scaled by a power of two first, which the scores take back, so that
// no fp32 value is too large or too small for the pair; hi is rounded towards
// zero and lo is not 0, so that an infinite key gives the product the sign of q.
// 16-bit rows: q as it is; the weights rounded to the type once, like the output.
//
// Units with positions that some row does not see: scores by the row's 64 mask
// bits, and V rows behind the last position, which may hold anything, are set
// to zero in shared memory, as 0 x NaN would reach every row.  Values of the round's own nodes that
// are not finite are set to zero there too and added at the end to the rows that see them.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <cmath>
#include <mutex>

#include "tc_gemm.cuh"
#include "tree_ops.cuh"
#include "tree_sched.cuh"

namespace ssd {
namespace tree {
namespace {

constexpr float kSlack = 8.f, kShift = 6.f;  // weights up to 2^14: finite in fp16
constexpr unsigned long long kWaitNs = 2000000000ull;
constexpr int kTmem = 256;  // columns: O 0 .. hd, S / P of even units at 128, of odd ones at 192
constexpr int kJoinThreads = 128;

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
    const void* vc;  // the layer's V
    int64_t page_stride, head_stride, pos_stride;
    int n_heads, n_pages;
    int box_shift;  // positions per copy, log2: 16 .. 64 of them, which divide page_size
    int at_pos, at_head, at_page;  // which coordinate (1 .. 3) of the tensor maps is which
    float scale2;  // log2(e) * scale
    Cut* cuts;     // [grid]
    float* stats;  // [grid][2][2][TILE]: maximum, sum
    float4* part;  // [grid][2][HD / 4][TILE]
    int32_t* status;
};

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

template <typename T, int HD, int TILE>
struct Lay {
    static constexpr int PARTS = Types<T>::PARTS, BOXES = HD / 64;
    static constexpr int QB = TILE * 128;             // bytes of 64 dims of the tile's q, one part
    static constexpr int Q = PARTS * BOXES * QB;
    static constexpr int KB = kUnit * 128;            // bytes of 64 dims of a unit of K or V
    static constexpr int STAGE = 2 * BOXES * KB;      // K boxes, then V boxes
    // two CTAs an SM, except for fp32 rows in tiles of 128 at hd 128, whose q takes 64 KB
    static constexpr int CTAS = Q > 32 * 1024 ? 1 : 2;
    static constexpr int FIT = ((CTAS == 1 ? 220 : 110) * 1024 - Q) / STAGE;
    static constexpr int STAGES = FIT > 6 ? 6 : FIT;
    // (the MMA reads 128 rows of q whatever TILE is: what lies behind has to be shared memory of the CTA)
    static constexpr size_t BYTES = 1024 + (size_t)Q + (size_t)STAGES * STAGE;
    static constexpr int THREADS = TILE + 64;
    static_assert(STAGES >= 2 && Q + STAGES * STAGE >= Q - QB + 128 * 128, "");
};

__device__ __forceinline__ void tma4d(void* dst, const CUtensorMap* map, int x, int c1, int c2, int c3, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
        ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(c1), "r"(c2), "r"(c3), "r"(smem_u32(bar))
        : "memory");
}
// kind::f16, A = B = fp16 or bf16, D = fp32, M = 128, N = 64; B K-major or (V) MN-major
template <typename C>
__device__ __forceinline__ constexpr uint32_t idesc(bool b_mn) {
    return (1u << 4) | (sizeof(C) == 2 && std::is_same<C, bf16>::value ? (1u << 7) | (1u << 10) : 0u) | (b_mn ? 1u << 16 : 0u) |
           ((64u >> 3) << 17) | ((128u >> 4) << 24);
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t ad, uint64_t bd, uint32_t id, uint32_t acc) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n"
        ::"r"(d), "l"(ad), "l"(bd), "r"(id), "r"(acc)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t bd, uint32_t id, uint32_t acc) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n"
        ::"r"(d), "r"(a), "l"(bd), "r"(id), "r"(acc)
        : "memory");
}
__device__ __forceinline__ void commit(uint64_t* b) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void arrive(uint64_t* b) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(b)) : "memory");
}
#define SSD_R8(r, o) "=r"(r[o]), "=r"(r[o + 1]), "=r"(r[o + 2]), "=r"(r[o + 3]), "=r"(r[o + 4]), "=r"(r[o + 5]), "=r"(r[o + 6]), "=r"(r[o + 7])
#define SSD_I8(r, o) "r"(r[o]), "r"(r[o + 1]), "r"(r[o + 2]), "r"(r[o + 3]), "r"(r[o + 4]), "r"(r[o + 5]), "r"(r[o + 6]), "r"(r[o + 7])
// 32 columns of this thread's TMEM lane
__device__ __forceinline__ void ld32(uint32_t t, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : SSD_R8(r, 0), SSD_R8(r, 8), SSD_R8(r, 16), SSD_R8(r, 24)
        : "r"(t));
}
__device__ __forceinline__ void st32(uint32_t t, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
        ::SSD_I8(r, 0), SSD_I8(r, 8), SSD_I8(r, 16), SSD_I8(r, 24), "r"(t)
        : "memory");
}
#undef SSD_R8
#undef SSD_I8
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// bounded wait; false after kWaitNs, or once another thread of the CTA has given up
__device__ __forceinline__ bool mb_wait(uint64_t* b, unsigned parity, volatile int* fail) {
    if (tc::mb_try(b, parity)) return true;
    const unsigned long long t0 = tc::gtime();
    while (!tc::mb_try(b, parity)) {
        if (*fail) return false;
        if (tc::gtime() - t0 > kWaitNs) {
            *fail = 1;
            return false;
        }
    }
    return true;
}

// fp16 pair of x: hi towards zero, lo the rest, of the same sign and not 0 unless x is
__device__ __forceinline__ void split_away(float a, float b, uint32_t& hi, uint32_t& lo) {
    const __half2 h = __halves2half2(__float2half_rz(a), __float2half_rz(b));
    const float2 f = __half22float2(h);
    const float la = a - f.x, lb = b - f.y;
    __half2 l = __floats2half2_rn(la, lb);
    hi = *reinterpret_cast<const uint32_t*>(&h);
    lo = *reinterpret_cast<const uint32_t*>(&l);
    if ((lo & 0x7fffu) == 0 && a != 0.f) lo = (lo & 0xffff0000u) | (hi & 0x8000u) | 1u;
    if ((lo & 0x7fff0000u) == 0 && b != 0.f) lo = (lo & 0xffffu) | (hi & 0x80000000u) | 0x10000u;
}
// hi = rn(a, b), lo = rn((a, b) - hi), packed
__device__ __forceinline__ void split_rn(float a, float b, uint32_t& hi, uint32_t& lo) {
    const __half2 h = __floats2half2_rn(a, b);
    const float2 f = __half22float2(h);
    hi = *reinterpret_cast<const uint32_t*>(&h);
    lo = pack2(a - f.x, b - f.y, f16());
}

// which of the positions p0 .. p0 + 63 node `node` (mask words m) sees, as bits
__device__ __forceinline__ uint64_t visible(const Req& q, int chain, int words, const uint64_t (&m)[4], int node, int p0) {
    const int end = q.total - p0;  // the unit's positions below it exist
    uint64_t v;
    if (chain) {
        const long long last = (long long)q.len + node - p0;
        v = last >= 63 ? ~0ull : last < 0 ? 0ull : (2ull << last) - 1ull;
    } else {
        const int j0 = p0 - q.len;  // node of the unit's first position
        if (j0 <= -64) {
            v = ~0ull;
        } else if (j0 <= 0) {
            v = j0 == 0 ? m[0] : (m[0] << -j0) | ((1ull << -j0) - 1ull);
        } else {
            const int w = j0 >> 6, s = j0 & 63;
            const uint64_t a = w == 0 ? m[0] : w == 1 ? m[1] : w == 2 ? m[2] : w == 3 ? m[3] : 0ull;
            const uint64_t b = w == 0 ? m[1] : w == 1 ? m[2] : w == 2 ? m[3] : 0ull;
            v = s ? (a >> s) | (b << (64 - s)) : a;
        }
    }
    return end >= 64 ? v : end <= 0 ? 0ull : v & ((1ull << end) - 1ull);
}

__device__ __forceinline__ uint32_t exps_all_ones(uint32_t u, f16) { return ((u & 0x7c00u) == 0x7c00u) | ((u & 0x7c000000u) == 0x7c000000u) << 1; }
__device__ __forceinline__ uint32_t exps_all_ones(uint32_t u, bf16) { return ((u & 0x7f80u) == 0x7f80u) | ((u & 0x7f800000u) == 0x7f800000u) << 1; }

template <typename T, int HD, int TILE>
__global__ void __launch_bounds__(Lay<T, HD, TILE>::THREADS, Lay<T, HD, TILE>::CTAS)
    attn_kernel(const __grid_constant__ AttnOpArgs a, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v) {
    using L = Lay<T, HD, TILE>;
    using C = typename Types<T>::C;
    constexpr int BOXES = L::BOXES, PARTS = L::PARTS, NW = TILE / 32, S = L::STAGES;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    unsigned char* kv = smem + L::Q;
    __shared__ __align__(8) uint64_t k_full[S], v_full[S], kv_empty[S], q_ready, s_full[2], p_ready[2], pv_done[2];
    __shared__ uint32_t s_tmem;
    __shared__ int s_fail, s_odd;  // a wait gave up; a node's value is not finite
    __shared__ long long s_sum[L::THREADS / 32], s_off;
    __shared__ int s_b;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        s_fail = s_odd = 0;
        s_b = -1;
        for (int s = 0; s < S; ++s) {
            tc::mb_init(k_full + s, 1);
            tc::mb_init(v_full + s, 1);
            tc::mb_init(kv_empty + s, 1);
        }
        tc::mb_init(&q_ready, NW);
        for (int i = 0; i < 2; ++i) {
            tc::mb_init(s_full + i, 1);
            tc::mb_init(p_ready + i, NW);
            tc::mb_init(pv_done + i, 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == NW) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(kTmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_launch_dependents();
    pdl_wait();  // everything below may come from the previous kernel
    if (tid == 0) a.cuts[blockIdx.x].last = -1;

    // this CTA's range: units of all requests, a run of requests per thread
    const Shape& sh = a.shape;
    const int per = (sh.n_requests + L::THREADS - 1) / L::THREADS;
    const int b0 = min(tid * per, sh.n_requests), b1 = min(b0 + per, sh.n_requests);
    long long mine = 0;
    for (int b = b0; b < b1; ++b) {
        const Req q = req_of(sh, b);
        if (q.clipped && q.n && blockIdx.x == 0) say(a.status, SSD_STATUS_TABLE);
        mine += head_units(sh, q, TILE) * sh.n_kv_heads;
    }
    long long before = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += x;
    }
    if (lane == 31) s_sum[warp] = before;
    __syncthreads();
    before -= mine;
    long long units = 0;
    for (int w = 0; w < L::THREADS / 32; ++w) {
        if (w < warp) before += s_sum[w];
        units += s_sum[w];
    }
    const int ctas = ctas_of(units, a.grid), cta = blockIdx.x;
    const long long lo = cta < ctas ? range_start(units, ctas, cta) : 0, hi = cta < ctas ? range_start(units, ctas, cta + 1) : 0;
    if (before <= lo && lo < before + mine) {
        long long off = lo - before;
        for (int b = b0; b < b1; ++b) {
            const long long n = head_units(sh, req_of(sh, b), TILE) * sh.n_kv_heads;
            if (off < n) {
                s_b = b;
                s_off = off;
                break;
            }
            off -= n;
        }
    }
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = s_tmem;
    Walk walk;
    walk_init(walk, sh, TILE, s_b, s_off, hi - lo);
    Seg g;
    bool ok = true;

    if (warp == NW) {
        // page ids are asked for 32 copies ahead, one per lane
        asm volatile("fence.proxy.async.global;" ::: "memory");  // K / V rows that the previous kernel wrote
        const int n_box = kUnit >> a.box_shift, batch = 32 << a.box_shift;  // copies per unit, positions per 32 copies
        unsigned j = 0;
        while (ok && walk_next(walk, sh, TILE, g)) {
            const int32_t* table = a.block_table + (size_t)g.b * sh.max_blocks;
            auto fetch = [&](long long x) {  // page of this lane's copy of the 32 from x on; -1: outside, reads as zeros
                x += lane << a.box_shift;
                int page = -1;
                if (x < g.q.total) page = __ldcg(table + (int)x / sh.page_size);
                return page >= 0 && page < a.n_pages ? page : -1;
            };
            int x0 = g.u0 * kUnit, got = fetch(x0), ahead = fetch((long long)x0 + batch);
            for (int u = g.u0; u < g.u1 && ok; ++u, ++j) {
                if (u * kUnit - x0 >= batch) {
                    x0 += batch;
                    got = ahead;
                    ahead = fetch((long long)x0 + batch);
                }
                const int s = j % S;
                ok = __all_sync(0xffffffffu, mb_wait(kv_empty + s, (j / S + 1) & 1u, &s_fail));
                if (!ok) break;
                unsigned char* st = kv + s * L::STAGE;
                const bool one = elect_one();
                if (one) {
                    tc::mb_arrive_tx(k_full + s, (unsigned)(BOXES * L::KB));
                    tc::mb_arrive_tx(v_full + s, (unsigned)(BOXES * L::KB));
                }
#pragma unroll
                for (int kvp = 0; kvp < 2; ++kvp)
                    for (int i = 0; i < n_box; ++i) {
                        const int page = __shfl_sync(0xffffffffu, got, ((u * kUnit - x0) >> a.box_shift) + i);
                        if (one) {
                            const int in_page = (u * kUnit + (i << a.box_shift)) % sh.page_size;
                            const int c1 = a.at_pos == 1 ? in_page : a.at_head == 1 ? g.kvh : page;
                            const int c2 = a.at_pos == 2 ? in_page : a.at_head == 2 ? g.kvh : page;
                            const int c3 = a.at_pos == 3 ? in_page : a.at_head == 3 ? g.kvh : page;
#pragma unroll
                            for (int b = 0; b < BOXES; ++b)
                                tma4d(st + (kvp * BOXES + b) * L::KB + (i << a.box_shift) * 128, kvp ? &tm_v : &tm_k, b * 64, c1, c2, c3, (kvp ? v_full : k_full) + s);
                        }
                    }
                __syncwarp();
            }
        }
    } else if (warp == NW + 1) {
        const uint64_t q0 = tc::sdesc(smem_u32(smem)), kv0 = tc::sdesc(smem_u32(kv));
        auto wait = [&](uint64_t* b, unsigned phase) {
            ok = ok && __all_sync(0xffffffffu, mb_wait(b, phase & 1u, &s_fail));
            return ok;
        };
        // S of unit j; its K has landed and P of unit j - 2, which held these columns, is used up
        auto scores = [&](unsigned j) {
            if (!wait(k_full + j % S, j / S)) return;
            if (j >= 2 && !wait(pv_done + (j & 1), (j - 2) >> 1)) return;
            tc::fence_after();
            if (elect_one()) {
                const uint64_t k0 = kv0 + (uint64_t)((j % S) * (L::STAGE >> 4));
                const uint32_t d = tmem + 128u + 64u * (j & 1);
#pragma unroll
                for (int h = 0; h < PARTS; ++h)
#pragma unroll
                    for (int b = 0; b < BOXES; ++b)
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks)
                            mma_ss(d, q0 + (uint64_t)(((h * BOXES + b) * L::QB + ks * 32) >> 4), k0 + (uint64_t)((b * L::KB + ks * 32) >> 4),
                                   idesc<C>(false), (h | b | ks) ? 1u : 0u);
                commit(s_full + (j & 1));
            }
            __syncwarp();
        };
        unsigned j = 0, n_seg = 0;
        while (ok && walk_next(walk, sh, TILE, g)) {
            if (!wait(&q_ready, n_seg++)) break;
            scores(j);
            for (int u = g.u0; u < g.u1 && ok; ++u, ++j) {
                if (u + 1 < g.u1) scores(j + 1);
                if (!ok || !wait(p_ready + (j & 1), j >> 1) || !wait(v_full + j % S, j / S)) break;
                tc::fence_after();
                if (elect_one()) {
                    // V: 64 dims (MN) x 16 positions (K) per MMA; 8 positions are 1024 bytes apart
                    const uint64_t v0 = kv0 + (uint64_t)(((j % S) * L::STAGE + BOXES * L::KB) >> 4);
                    const uint64_t mn = (uint64_t)((1024 >> 4) - 1) << 16;  // leading byte offset 1024 too
                    const uint32_t p = tmem + 128u + 64u * (j & 1);
#pragma unroll
                    for (int b = 0; b < BOXES; ++b)
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                            for (int h = 0; h < PARTS; ++h)
                                mma_ts(tmem + 64u * b, p + 32u * h + 8u * ks, v0 + mn + (uint64_t)((b * L::KB + ks * 2048) >> 4), idesc<C>(true),
                                       (u > g.u0 || ks || h) ? 1u : 0u);
                    commit(kv_empty + j % S);
                    commit(pv_done + (j & 1));
                }
                __syncwarp();
            }
        }
    } else {
        const uint32_t tl = tmem + ((uint32_t)(warp * 32) << 16);
        // q of the segment's rows (K-major, 128-byte swizzle: row r of 64 dims at r * 128, 16-byte
        // chunk c at (c ^ (r & 7)) * 16), a few rows of this warp's 32 at a time; returns the power
        // of two that this thread's row was divided by
        float q_scale = 1.f;
        auto load_q = [&](const Seg& s) {
            constexpr int V = Vec<T>::N, LPR = HD / V, RPI = 32 / LPR, N = 8;  // lanes per row, rows per step, steps at once
            const int rows = s.q.n * sh.group;
            float mult = 1.f;
            for (int i0 = 0; i0 < 32; i0 += N * RPI) {
                uint4 x[N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int r = s.mt * TILE + warp * 32 + i0 + i * RPI + lane / LPR, e = (lane % LPR) * V;
                    x[i] = make_uint4(0, 0, 0, 0);
                    if (r < rows) {
                        const int node = r / sh.group, head = s.kvh * sh.group + r - node * sh.group;
                        x[i] = __ldcg(reinterpret_cast<const uint4*>((const T*)a.q + (int64_t)(s.q.r0 + node) * a.q_stride + head * HD + e));
                    }
                }
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int r = warp * 32 + i0 + i * RPI + lane / LPR, e = (lane % LPR) * V;
                    unsigned char* at = smem + (e >> 6) * L::QB + r * 128 + ((((e & 63) >> 3) ^ (r & 7)) << 4) + (e & 7) * 2;
                    if constexpr (PARTS == 1) {
                        *reinterpret_cast<uint4*>(at) = x[i];
                    } else {
                        float f[4];
                        Vec<float>::get(x[i], f);
                        float m = fmaxf(fmaxf(fabsf(f[0]), fabsf(f[1])), fmaxf(fabsf(f[2]), fabsf(f[3])));
#pragma unroll
                        for (int o = LPR / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
                        // 2^e with the row's largest value at 2^9 .. 2^10 (rows of zeros, infinities and subnormals: as if 2^-126 or 2^127)
                        const int e2 = min(max((int)(__float_as_uint(m) >> 23), 10), 254) - 127 - 9;
                        const float down = __uint_as_float((uint32_t)(127 - e2) << 23);
                        uint2 h, l;
                        split_away(f[0] * down, f[1] * down, h.x, l.x);
                        split_away(f[2] * down, f[3] * down, h.y, l.y);
                        *reinterpret_cast<uint2*>(at) = h;
                        *reinterpret_cast<uint2*>(at + BOXES * L::QB) = l;
                        const float up = __uint_as_float((uint32_t)(127 + e2) << 23);
                        // lane i0 + i RPI + (row in step) holds that row
#pragma unroll
                        for (int k = 0; k < RPI; ++k) {
                            const float v = __shfl_sync(0xffffffffu, up, k * LPR);
                            if (lane == i0 + i * RPI + k) mult = v;
                        }
                    }
                }
            }
            q_scale = mult;
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) arrive(&q_ready);
        };

        unsigned j = 0;
        bool more = walk_next(walk, sh, TILE, g);
        if (more) load_q(g);
        long long at = lo;  // global unit of the segment's start
        bool first_seg = true;
        while (more && ok) {
            const int rows = g.q.n * sh.group - g.mt * TILE;     // of the tile that exist
            const bool active = warp * 32 < rows;                // some row of the warp
            const int r = g.mt * TILE + warp * 32 + lane, node = min(r / sh.group, g.q.n - 1), head = g.kvh * sh.group + r % sh.group;
            const bool valid = warp * 32 + lane < rows;
            const float sc = a.scale2 * q_scale;
            uint64_t m[4] = {0, 0, 0, 0};
            if (!sh.chain && valid)
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    if (w < a.words) m[w] = __ldcg(a.masks + (size_t)(g.q.r0 + node) * a.words + w);
            const int all_seen = sh.chain ? g.q.len + min(g.mt * TILE / sh.group, g.q.n - 1) + 1 : g.q.len;  // positions below it are seen by every row
            float mx = 0.f, l = 0.f;  // maximum that the weights are relative to, their sum
            for (int u = g.u0; u < g.u1; ++u, ++j) {
                const int p0 = u * kUnit;
                const uint32_t ts = tl + 128u + 64u * (j & 1);
                ok = __all_sync(0xffffffffu, mb_wait(s_full + (j & 1), (j >> 1) & 1u, &s_fail));
                if (!ok) break;
                tc::fence_after();
                const bool tail = p0 + kUnit > min(all_seen, g.q.total);
                if (tail) {  // V of positions that not every row sees
                    ok = __all_sync(0xffffffffu, mb_wait(v_full + j % S, (j / S) & 1u, &s_fail));
                    if (!ok) break;
                    unsigned char* vs = kv + (j % S) * L::STAGE + BOXES * L::KB;
                    for (int i = tid; i < BOXES * kUnit * 8; i += TILE) {
                        const int x = p0 + ((i >> 3) & 63);
                        if (x < g.q.len && x < g.q.total) continue;
                        uint4* v = reinterpret_cast<uint4*>(vs + i * 16);
                        if (x >= g.q.total) {
                            *v = make_uint4(0, 0, 0, 0);
                            continue;
                        }
                        uint32_t w[4] = {v->x, v->y, v->z, v->w}, odd = 0;
#pragma unroll
                        for (int k = 0; k < 4; ++k) odd |= exps_all_ones(w[k], C()) << (2 * k);
                        if (odd) {
#pragma unroll
                            for (int k = 0; k < 4; ++k) w[k] &= (odd >> (2 * k) & 1 ? 0u : 0xffffu) | (odd >> (2 * k) & 2 ? 0u : 0xffff0000u);
                            *v = make_uint4(w[0], w[1], w[2], w[3]);
                            *(volatile int*)&s_odd = 1;
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                if (active) {
                    uint32_t u0[32], u1[32];
                    ld32(ts, u0);
                    ld32(ts + 32, u1);
                    wait_ld();
                    if (tail) {
                        const uint64_t v = visible(g.q, sh.chain, a.words, m, node, p0);
                        const uint32_t v0 = (uint32_t)v, v1 = (uint32_t)(v >> 32);
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            if (!(v0 >> i & 1u)) u0[i] = 0xff800000u;
                            if (!(v1 >> i & 1u)) u1[i] = 0xff800000u;
                        }
                    }
                    float bm4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int i = 0; i < 32; ++i) bm4[i & 3] = fmaxf(bm4[i & 3], fmaxf(__uint_as_float(u0[i]), __uint_as_float(u1[i])));
                    const float bm = fmaxf(fmaxf(bm4[0], bm4[1]), fmaxf(bm4[2], bm4[3])) * sc;
                    if (u == g.u0) {
                        mx = bm;
                    } else if (__any_sync(0xffffffffu, bm > mx + kSlack)) {
                        // O and the sum move to the new maximum (all rows of the warp)
                        ok = __all_sync(0xffffffffu, mb_wait(pv_done + ((j - 1) & 1), ((j - 1) >> 1) & 1u, &s_fail));
                        if (!ok) break;
                        tc::fence_after();
                        const float nm = fmaxf(mx, bm), f = nm == -INFINITY ? 1.f : exp2f(mx - nm);
                        for (int c = 0; c < HD; c += 32) {
                            uint32_t o[32];
                            ld32(tl + c, o);
                            wait_ld();
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                            st32(tl + c, o);
                        }
                        l *= f;
                        mx = nm;
                    }
                    // (a row that has seen nothing yet, or only scores of -inf: weights 0)
                    const float ref = (mx == -INFINITY ? 0.f : mx) - kShift;
                    float l4[4] = {0.f, 0.f, 0.f, 0.f};
                    uint32_t ph[32], pl[32];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float p0f = exp2f(fmaf(__uint_as_float(u0[2 * i]), sc, -ref)), p1f = exp2f(fmaf(__uint_as_float(u0[2 * i + 1]), sc, -ref));
                        const float p2f = exp2f(fmaf(__uint_as_float(u1[2 * i]), sc, -ref)), p3f = exp2f(fmaf(__uint_as_float(u1[2 * i + 1]), sc, -ref));
                        l4[i & 3] += (p0f + p1f) + (p2f + p3f);
                        if constexpr (PARTS == 2) {
                            split_rn(p0f, p1f, ph[i], pl[i]);
                            split_rn(p2f, p3f, ph[i + 16], pl[i + 16]);
                        } else {
                            ph[i] = pack2(p0f, p1f, C());
                            ph[i + 16] = pack2(p2f, p3f, C());
                        }
                    }
                    l += (l4[0] + l4[1]) + (l4[2] + l4[3]);
                    st32(ts, ph);
                    if constexpr (PARTS == 2) st32(ts + 32, pl);
                    wait_st();
                }
                tc::fence_before();
                __syncwarp();
                if (lane == 0) arrive(p_ready + (j & 1));
            }
            if (!ok) break;
            const Seg done = g;
            const bool whole = done.u0 == 0 && done.u1 == done.n;
            const long long item = at - done.u0;  // global unit of the item's start
            const int slot = first_seg ? 0 : 1;
            at += done.u1 - done.u0;
            first_seg = false;
            // the next rows' q while the last products run (all scores of this segment are done)
            more = walk_next(walk, sh, TILE, g);
            if (more) load_q(g);
            if (tid == 0 && done.u1 < done.n) {
                Cut c;
                c.first = cta_of(units, ctas, item);
                c.last = cta_of(units, ctas, item + done.n - 1);
                c.first_slot = range_start(units, ctas, c.first) == item ? 0 : 1;
                c.row0 = done.mt * TILE;
                c.rows = min(rows, TILE);
                c.r0 = done.q.r0;
                c.kvh = done.kvh;
                c.pad = 0;
                a.cuts[cta] = c;
            }
            ok = __all_sync(0xffffffffu, mb_wait(pv_done + ((j - 1) & 1), ((j - 1) >> 1) & 1u, &s_fail));
            if (!ok) break;
            tc::fence_after();
            if (active) {
                const bool odd = *(volatile int*)&s_odd;
                const float inv = l == 0.f ? 0.f : 1.f / l;
                if (!whole && valid) {
                    float* st = a.stats + (size_t)(cta * 2 + slot) * 2 * TILE + warp * 32 + lane;
                    st[0] = mx == -INFINITY ? mx : mx - kShift;
                    st[TILE] = l;
                }
                for (int c = 0; c < HD; c += 32) {
                    uint32_t o[32];
                    ld32(tl + c, o);
                    wait_ld();
                    if (!valid) continue;
                    if (odd) {  // values that are not finite, of nodes that this row sees
                        for (int u = done.u0; u < done.u1; ++u) {
                            const int p0 = u * kUnit;
                            if (p0 + kUnit <= done.q.len) continue;
                            const uint64_t v = visible(done.q, sh.chain, a.words, m, node, p0);
                            for (int k = 0; k < kUnit; ++k) {
                                const int x = p0 + k;
                                if (x < done.q.len || !(v >> k & 1)) continue;
                                const int page = __ldcg(a.block_table + (size_t)done.b * sh.max_blocks + x / sh.page_size);
                                if (page < 0 || page >= a.n_pages) continue;
                                const C* vr = (const C*)a.vc + page * a.page_stride + done.kvh * a.head_stride + (x % sh.page_size) * a.pos_stride + c;
#pragma unroll
                                for (int i = 0; i < 32; ++i) {
                                    const float f = (float)vr[i];
                                    if (!isfinite(f)) o[i] = __float_as_uint(__uint_as_float(o[i]) + f);
                                }
                            }
                        }
                    }
                    if (whole) {
                        T* to = (T*)a.out + (int64_t)(done.q.r0 + node) * a.out_stride + head * HD + c;
                        constexpr int V = Vec<T>::N;
#pragma unroll
                        for (int i = 0; i < 32; i += V) {
                            float f[V];
#pragma unroll
                            for (int k = 0; k < V; ++k) f[k] = __uint_as_float(o[i + k]) * inv;
                            *reinterpret_cast<uint4*>(to + i) = Vec<T>::put(f);
                        }
                    } else {
                        float4* to = a.part + ((size_t)(cta * 2 + slot) * (HD / 4) + c / 4) * TILE + warp * 32 + lane;
#pragma unroll
                        for (int i = 0; i < 32; i += 4)
                            to[(i / 4) * TILE] = make_float4(__uint_as_float(o[i]), __uint_as_float(o[i + 1]), __uint_as_float(o[i + 2]), __uint_as_float(o[i + 3]));
                    }
                }
            }
        }
    }
    if (!ok) s_fail = 1;
    tc::fence_before();
    __syncwarp();
    __syncthreads();
    if (s_fail && tid == 0) {  // let copies and MMAs in flight finish
        say(a.status, SSD_STATUS_TIMEOUT);
        const unsigned long long t0 = tc::gtime();
        while (tc::gtime() - t0 < 2000000ull) __nanosleep(1000);
    }
    __syncthreads();
    if (warp == NW) {
        tc::fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmem) : "memory");
    }
}


// Joins the parts of the items that range ends cut.  CTA c of the attention left a
// Cut if its range ends inside an item; with n such ends in an item, n CTAs share
// it here: a warp takes 32 rows (a lane each) and 4 dims at a time, first the
// largest maximum of the parts, then the weighted sums, in the order of the parts.
template <typename T, int HD, int TILE>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const AttnOpArgs a) {
    pdl_launch_dependents();
    pdl_wait();
    const int cta = blockIdx.x, lane = threadIdx.x & 31;
    const int4 c0 = __ldcg(reinterpret_cast<const int4*>(a.cuts + cta)), c1 = __ldcg(reinterpret_cast<const int4*>(a.cuts + cta) + 1);
    const int first = c0.x, last = c0.y, slot = c0.z, row0 = c0.w, rows = c1.x, r0 = c1.y, kvh = c1.z;
    if (last < 0) return;
    const int warps = (last - first) * (kJoinThreads / 32), items = (rows + 31) / 32 * (HD / 4);
    for (int w = (cta - first) * (kJoinThreads / 32) + (threadIdx.x >> 5); w < items; w += warps) {
        const int chunk = w % (HD / 4), row = w / (HD / 4) * 32 + lane;
        if (row >= rows) continue;
        auto part_of = [&](int p) { return (size_t)(p * 2 + (p == first ? slot : 0)); };
        float top = -INFINITY;
#pragma unroll 8
        for (int p = first; p <= last; ++p) top = fmaxf(top, __ldcg(a.stats + part_of(p) * 2 * TILE + row));
        float l = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int p = first; p <= last; ++p) {
            const float* st = a.stats + part_of(p) * 2 * TILE + row;
            const float m = __ldcg(st), lp = __ldcg(st + TILE);
            const float4 x = __ldcg(a.part + (part_of(p) * (HD / 4) + chunk) * TILE + row);
            const float f = m == -INFINITY ? 0.f : exp2f(m - top);  // (0 x NaN stays NaN)
            l = fmaf(lp, f, l);
            o.x = fmaf(x.x, f, o.x);
            o.y = fmaf(x.y, f, o.y);
            o.z = fmaf(x.z, f, o.z);
            o.w = fmaf(x.w, f, o.w);
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const int r = row0 + row, node = r / a.shape.group, head = kvh * a.shape.group + r - node * a.shape.group;
        T* to = (T*)a.out + (int64_t)(r0 + node) * a.out_stride + head * HD + chunk * 4;
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4*>(to) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
        } else {
            *reinterpret_cast<uint2*>(to) = make_uint2(pack2(o.x * inv, o.y * inv, T()), pack2(o.z * inv, o.w * inv, T()));
        }
    }
}

// -- host ----------------------------------------------------------------------

// the workspace: cuts, statistics and parts of the largest grid (two CTAs an SM) and tile
constexpr int kMaxTile = 128, kMaxCtas = 2;
size_t workspace_need(int n_sms, int hd) {
    const size_t grid = (size_t)kMaxCtas * n_sms;
    return grid * (sizeof(Cut) + 2 * 2 * kMaxTile * sizeof(float) + 2 * (size_t)kMaxTile * hd * sizeof(float));
}

// Per device, once: kernel attributes and the SM count.
struct AttnDevice {
    bool ready = false;
    int n_sms = 0;
};
constexpr int kMaxDevices = 64;
AttnDevice g_attn_dev[kMaxDevices];
PFN_cuTensorMapEncodeTiled_v12000 g_encode = nullptr;
std::mutex g_attn_mu;

template <typename T, int HD, int TILE>
cudaError_t set_up_one() {
    return cudaFuncSetAttribute(attn_kernel<T, HD, TILE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Lay<T, HD, TILE>::BYTES);
}
template <typename T>
cudaError_t set_up_type() {
    cudaError_t e = set_up_one<T, 64, 32>();
    if (e == cudaSuccess) e = set_up_one<T, 64, 128>();
    if (e == cudaSuccess) e = set_up_one<T, 128, 32>();
    if (e == cudaSuccess) e = set_up_one<T, 128, 128>();
    return e;
}
int set_up(const char* call, int* n_sms) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || dev < 0 || dev >= kMaxDevices) {
        (void)cudaGetLastError();
        return refuse(SSD_ERR_CUDA, call, "no usable current device");
    }
    std::lock_guard<std::mutex> lock(g_attn_mu);
    AttnDevice& d = g_attn_dev[dev];
    if (!d.ready) {
        e = set_up_type<float>();
        if (e == cudaSuccess) e = set_up_type<f16>();
        if (e == cudaSuccess) e = set_up_type<bf16>();
        if (e == cudaSuccess) e = cudaDeviceGetAttribute(&d.n_sms, cudaDevAttrMultiProcessorCount, dev);
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
        if (e == cudaSuccess) e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found);
        if (e != cudaSuccess) return refuse(SSD_ERR_CUDA, call, "set-up: %s", cudaGetErrorString(e));
        if (!fn || found != cudaDriverEntryPointSuccess) return refuse(SSD_ERR_CUDA, call, "cuTensorMapEncodeTiled unavailable");
        g_encode = (PFN_cuTensorMapEncodeTiled_v12000)fn;
        d.ready = true;
    }
    *n_sms = d.n_sms;
    return SSD_OK;
}

// K or V of a layer as {hd, then positions of a page, heads and pages by their strides}, box 64 dims x box_rows positions
int encode(const char* call, CUtensorMap* m, const void* base, const ssd_pages* c, AttnOpArgs& a) {
    struct Dim {
        cuuint64_t n, stride;
        cuuint32_t box;
        int* at;
    } d[3] = {{(cuuint64_t)c->page_size, (cuuint64_t)c->pos_stride * 2, 1u << a.box_shift, &a.at_pos},
              {(cuuint64_t)c->n_kv_heads, (cuuint64_t)c->head_stride * 2, 1, &a.at_head},
              {(cuuint64_t)c->n_pages, (cuuint64_t)c->page_stride * 2, 1, &a.at_page}};
    for (Dim& x : d)  // (the stride of a dimension of one is not used)
        if (x.n == 1) x.stride = cuuint64_t(1) << 39;
    std::stable_sort(d, d + 3, [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
    for (int i = 0; i < 3; ++i) *d[i].at = i + 1;
    const cuuint64_t dims[4] = {(cuuint64_t)c->head_dim, d[0].n, d[1].n, d[2].n}, strides[3] = {d[0].stride, d[1].stride, d[2].stride};
    const cuuint32_t box[4] = {64, d[0].box, d[1].box, d[2].box}, step[4] = {1, 1, 1, 1};
    const CUresult r = g_encode(m, c->dtype == SSD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(base), dims,
                                strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? SSD_OK : refuse(SSD_ERR_CUDA, call, "cuTensorMapEncodeTiled failed (%d)", (int)r);
}

template <typename T, int HD, int TILE>
int run_tile(const char* call, AttnOpArgs& a, const CUtensorMap& k, const CUtensorMap& v, int n_sms, void* workspace, void* stream) {
    using L = Lay<T, HD, TILE>;
    a.grid = L::CTAS * n_sms;
    a.cuts = (Cut*)workspace;
    a.part = (float4*)(a.cuts + a.grid);
    a.stats = (float*)(a.part + (size_t)a.grid * 2 * (HD / 4) * TILE);
    if (int rc = launch(call, attn_kernel<T, HD, TILE>, dim3((unsigned)a.grid), L::THREADS, L::BYTES, stream, a, k, v)) return rc;
    // an item of one unit is never cut
    if ((long long)a.shape.max_blocks * a.shape.page_size <= kUnit) return SSD_OK;
    return launch(call, join_kernel<T, HD, TILE>, dim3((unsigned)(a.grid - 1)), kJoinThreads, 0, stream, a);
}
// Tiles of 32 rows where every request has at most that many per KV head.
template <typename T>
int run(const char* call, AttnOpArgs& a, int hd, int max_rows, const CUtensorMap& k, const CUtensorMap& v, int n_sms, void* ws, void* stream) {
    const bool small = (long long)max_rows * a.shape.group <= 32;
    if (hd == 64) return small ? run_tile<T, 64, 32>(call, a, k, v, n_sms, ws, stream) : run_tile<T, 64, 128>(call, a, k, v, n_sms, ws, stream);
    return small ? run_tile<T, 128, 32>(call, a, k, v, n_sms, ws, stream) : run_tile<T, 128, 128>(call, a, k, v, n_sms, ws, stream);
}

}  // namespace
}  // namespace tree
}  // namespace ssd

using namespace ssd;
using namespace ssd::tree;

extern "C" int ssd_tree_attention_workspace(int head_dim, size_t* bytes) {
    static const char call[] = "ssd_tree_attention_workspace";
    if (!bytes) return refuse_arg(call, "NULL pointer");
    if (head_dim != 64 && head_dim != 128) return refuse_arg(call, "head_dim must be 64 or 128");
    int n_sms = 0;
    if (int rc = set_up(call, &n_sms)) return rc;
    *bytes = workspace_need(n_sms, head_dim);
    return SSD_OK;
}

extern "C" int ssd_tree_attention(const ssd_batch* batch, const ssd_pages* cache, int layer, int dtype, int n_heads,
                                  const void* q, int64_t q_stride, const uint64_t* masks, int mask_words, float scale, void* out,
                                  int64_t out_stride, void* workspace, size_t workspace_bytes, int32_t* status,
                                  void* cuda_stream) {
    static const char call[] = "ssd_tree_attention";
    if (int rc = check_batch(call, batch)) return rc;
    if (int rc = check_pages(call, cache)) return rc;
    if (layer < 0 || layer >= cache->n_layers) return refuse_arg(call, "no such layer");
    if (int rc = check_rows_type(call, dtype, cache)) return rc;
    if (n_heads < 1 || n_heads > 65536 || n_heads % cache->n_kv_heads)
        return refuse_arg(call, "n_heads must be a multiple of n_kv_heads, at most 65536");
    const int group = n_heads / cache->n_kv_heads;
    if ((long long)batch->n_rows * group >= (1ll << 30)) return refuse_arg(call, "need n_rows * n_heads / n_kv_heads < 2^30");
    if (!(scale > 0.f) || !std::isfinite(scale)) return refuse_arg(call, "scale must be positive and finite");
    if (masks ? mask_words < 1 || mask_words > 4 : mask_words != 0)
        return refuse_arg(call, "masks need 1 <= mask_words <= 4, chains (masks = NULL) 0");
    if (batch->n_rows == 0) return SSD_OK;
    if (!q || !out || !workspace) return refuse_arg(call, "NULL pointer");
    if (int rc = check_rows(call, "q", q, q_stride, dtype, (int64_t)n_heads * cache->head_dim)) return rc;
    if (int rc = check_rows(call, "out", out, out_stride, dtype, (int64_t)n_heads * cache->head_dim)) return rc;
    if (q == out) return refuse_arg(call, "out must be memory of its own");
    if ((uintptr_t)workspace & 15u) return refuse_arg(call, "the workspace must be 16-byte aligned");
    if (workspace_bytes < workspace_need(1, cache->head_dim)) return refuse(SSD_ERR_CAPACITY, call, "the workspace is too small");
    if (int rc = check_device(call, cache->k)) return rc;
    int n_sms = 0;
    if (int rc = set_up(call, &n_sms)) return rc;
    const size_t need = workspace_need(n_sms, cache->head_dim);
    if (workspace_bytes < need) return refuse(SSD_ERR_CAPACITY, call, "the workspace needs %zu bytes", need);
    AttnOpArgs a{};
    a.shape.n_requests = batch->n_requests;
    a.shape.n_rows = batch->n_rows;
    a.shape.max_blocks = batch->max_blocks;
    a.shape.page_size = cache->page_size;
    a.shape.n_kv_heads = cache->n_kv_heads;
    a.shape.group = group;
    a.shape.chain = masks == nullptr;
    a.shape.row_start = batch->row_start;
    a.shape.lens = batch->lens;
    a.block_table = batch->block_table;
    a.q = q;
    a.out = out;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.masks = masks;
    a.words = mask_words;
    a.vc = (const char*)cache->v + 2 * layer * cache->layer_stride;
    a.page_stride = cache->page_stride;
    a.head_stride = cache->head_stride;
    a.pos_stride = cache->pos_stride;
    a.n_heads = n_heads;
    a.n_pages = cache->n_pages;
    a.box_shift = cache->page_size % 64 == 0 ? 6 : cache->page_size % 32 == 0 ? 5 : 4;
    a.scale2 = (float)(1.4426950408889634 * scale);
    a.status = status;
    CUtensorMap k, v;
    if (int rc = encode(call, &k, (const char*)cache->k + 2 * layer * cache->layer_stride, cache, a)) return rc;
    if (int rc = encode(call, &v, a.vc, cache, a)) return rc;
    const int hd = cache->head_dim, rows = batch->max_rows;
    if (dtype == SSD_F32) return run<float>(call, a, hd, rows, k, v, n_sms, workspace, cuda_stream);
    if (dtype == SSD_F16) return run<f16>(call, a, hd, rows, k, v, n_sms, workspace, cuda_stream);
    return run<bf16>(call, a, hd, rows, k, v, n_sms, workspace, cuda_stream);
}
