// tree_attn.cu - ssd_tree_attention (ssd_ops.h): attention of a batch's rows
// over a paged cache, with the masks of their trees.
//
//   o = sum_x w_x v_x / sum_x w_x,  w_x = 2^(s_x - m),  s_x = log2(e) scale q . k_x
//
// over the positions x that a row sees, m a running maximum.  All query heads
// that share a KV head, and all nodes of the request's tree, are rows of tiles
// of 128, each of which reads K and V once: with R rows of a tile a position costs
// 4 hd bytes and 4 hd R flops.  Up to one tile a request the bound is HBM; further tiles
// find K and V in L2.
//
// A CTA (one per SM) walks its range of units (tree_sched.cuh), 128 positions at a time:
//   warps 8, 9 : TMA producers of K and of V, a lane per copy of 16 to 64 rows of a page,
//                into a ring each (K in slots of 64 dims, free once multiplied; V in
//                slots of 64 positions);
//   warp 10    : issues S = q K^T (tcgen05.mma, 128 x 128 x 16, TMEM accumulators);
//   warp 11    : issues O += P V (P in TMEM over the columns of S, V as it lies in the
//                cache, MN-major, N = hd);
//   warps 0-3, 4-7 : softmax of the even and of the odd units, a row per thread: S from
//                TMEM, P back to it.  Three units' S and P have a place (two for fp32 rows of
//                128 dims), so that the tensor cores multiply for one while both groups work;
//                there is one accumulator, and the maximum that weights are relative to goes
//                from unit to unit, from a group's warp to the other's (before its weights
//                are computed, so that the groups overlap).
//   warps 12-15 : q of the next item to shared memory; adds each run's product (fp32 rows: a
//                unit's) to the sums; at an item's end O / sum, or O, maximum and sum to the
//                workspace if other CTAs hold parts of the item, while the others are at
//                the next item.  join_kernel adds those.
// The tile has 128 rows (with fewer, the others' lanes hold what no one reads; tiles of 32, with q of two
// items in shared memory, were no faster); two rows or less are few_kernel's (tree_few.cu).
//
// Measured, with join_kernel (copy rate 6.79 TB/s, tensor cores 1.92 PFLOP/s):
//   9 nodes, 8 heads a KV head, 100001 positions, fp16: 78 us, 5.2 TB/s - HBM, and the gap where a run of
//     units ends (below);
//   6 trees of 33 nodes, 8 heads a KV head, 4096 positions, bf16: 36 us, 1.9 TB/s - 8 us until the
//     first unit's scores, then 1.4 us a unit (S, softmax, P V of a buffer one after the other), join 5;
//   2048 rows over 4000 positions, 8 heads a KV head, bf16: 382 us, 0.88 PFLOP/s counted once, 1.3 done (P V in two
//     passes) - 1.4 us a unit: no part is busy all of the time (tensor pipe 59 % of the cycles, L2 31 % of its rate,
//     issue slots 50 %).  By clock stamps a softmax group waits for scores for 54 % of its unit, computes
//     weights for 31 %, the maximum for 9 % and waits for the reference for 6 %; the warp of P V waits for weights for a tenth
//     of the time and for V for a third, with three units of V in the ring as with two;
//   2 x 1023 rows over 700 positions, 40 heads, fp32: 135 us, 0.35 PFLOP/s counted once, 0.7 done
//     (two passes each) - 1.9 us a unit, as its product and the sum of the one before take turns at the
//     accumulator, and 7 us an item until its q, which has one buffer, is there as pairs;
//   32 trees of 9 nodes, 32 heads, 90 to 270 positions: fp16 56 us, fp32 68, for 13 us of bytes - the hand-offs at the
//     ends of 1024 items of two or three units.
//
// O is rescaled only when a row's maximum has grown by more than kSlack (log2)
// over the one its weights are relative to (the running softmax of Milakov and
// Gimelshein, 2018).  Weights are relative to the maximum less kShift, and enter the product as pairs hi + lo of the
// cache's type: in fp16 22 bits down to 2^-20 of the largest one, in bf16 16 bits.  (Rounded to the type
// once, as their sum is not, they made the error of 16-bit rows 1.4 times that of rounding the result: 2.3e-3 against
// 1.7e-3 in bf16.  The second pass costs 2 % of the time where HBM bounds, 9 % on trees, 18 % on prompts.)
//
// fp32 rows: q enters its product as fp16 pairs too.  A
// row of q is scaled by a power of two first, which the scores take back, so that
// no fp32 value is too large or too small for the pair; hi is rounded towards
// zero and lo is not 0, so that an infinite key gives the product the sign of q.
// The tensor cores cut off what their sums cannot hold, always downwards in size: 1.5e-8 of the sum a
// position, 6e-4 after 100000 in one accumulator.  So a run of units (Lay::RUN) starts from zero
// (lo first), and runs are added in fp32.  fp32 rows: a run is a unit, 1e-6 at any length.  16-bit rows: 24 units, 4e-5 at any length
// (of fp16's half step, 2.4e-4 to 4.9e-4, a sixth; 32 units 5e-5).  A run's end is a gap of 3 to 4 us in the products: 100001 positions
// 73.6 -> 78.7 us, 160 items of 60000 472 -> 508, bf16 prompt of 2048 rows 366 -> 382, items of two or three units
// (code that they do not reach) 54 -> 56.
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
#include "tree_attn.cuh"

namespace ssd {
namespace tree {
namespace {

constexpr float kSlack = 8.f, kShift = 6.f;  // weights up to 2^14: finite in fp16
constexpr double kWaitSeconds = 2.0, kClocksPerSecond = 2e9;
constexpr int kThreads = 512;
constexpr int kTmem = 512;  // columns (Lay)
constexpr int kMaxSlots = 12, kSegs = 32;
constexpr int kJoinThreads = 128, kJoinLines = 16;

template <typename T, int HD>
struct Lay {
    static constexpr int PARTS = Types<T>::PARTS, BOXES = HD / 64;
    static constexpr int KSLOT = kUnit * 128;         // 64 dims of a unit's K
    static constexpr int VBOX = 64 * 128;             // 64 dims of 64 positions of V
    static constexpr int VSLOT = BOXES * VBOX;
    static constexpr int RING = 210 * 1024;           // shared memory for q and the rings
    // TMEM columns: O; sums of earlier runs, if SUMS_IN_TMEM; S / P of unit j at S0 + 128 (j mod NB)
    static constexpr int M0 = HD, S0 = PARTS == 2 && HD == 128 ? 256 : 128, NB = (kTmem - S0) / kUnit;
    // Units whose products are added in the accumulator, from zero on; then they are added to the sums in fp32, in TMEM if
    // it has room for those, else in the workspace (above).  (Sums in TMEM with two S / P buffers instead of three: bf16 prompt
    // 438 us against 382; copies of the accumulator added up behind the next run's products: no faster.)
    static constexpr int RUN = PARTS == 2 ? 1 : 24;
    static constexpr bool SUMS_IN_TMEM = M0 + HD <= S0;
    static constexpr int QBOX = kTile * 128;          // 64 dims of the tile's q
    static constexpr int Q_ALL = PARTS * BOXES * QBOX;
    // Slots.  The scores wait for K more often than the products for V, which is asked for at the same time and
    // needed later: K takes 13 / 20 of the rings (10 and 11 / 20: the same within 1 %; 9 / 20: 2 % slower), but leaves two
    // units of V (softmax: half_done).
    static constexpr int ROOM = RING - Q_ALL, MOST_K = (ROOM - 4 * VSLOT) / KSLOT, SHARE = ROOM * 13 / 20 / KSLOT;
    static constexpr int least(int a, int b) { return a < b ? a : b; }
    static constexpr unsigned NK = least(least(SHARE, MOST_K), kMaxSlots), NV = least((ROOM - (int)NK * KSLOT) / VSLOT, kMaxSlots);
    static_assert(NK >= 2 * BOXES && NV >= 4, "a unit of K and two of V");
    static constexpr size_t BYTES = 1024 + (size_t)RING;
};

__device__ __forceinline__ void tma4d(void* dst, const CUtensorMap* map, int x, int c1, int c2, int c3, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
        ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(c1), "r"(c2), "r"(c3), "r"(smem_u32(bar))
        : "memory");
}
// kind::f16, A = B = fp16 or bf16, D = fp32, M = 128, N = n; B K-major or (V) MN-major
template <typename C>
__device__ __forceinline__ constexpr uint32_t idesc(int n, bool b_mn) {
    return (1u << 4) | (sizeof(C) == 2 && std::is_same<C, bf16>::value ? (1u << 7) | (1u << 10) : 0u) | (b_mn ? 1u << 16 : 0u) |
           ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24);
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
// 16 columns
__device__ __forceinline__ void st16(uint32_t t, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::SSD_I8(r, 0), SSD_I8(r, 8), "r"(t)
                 : "memory");
}
#undef SSD_R8
#undef SSD_I8
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// bounded wait; false after `limit` clocks, or once another thread of the CTA has given up
__device__ __noinline__ bool mb_wait_on(uint64_t* b, unsigned parity, volatile int* fail, long long limit) {
    const long long t0 = clock64();
#pragma unroll 1
    while (!tc::mb_try(b, parity)) {
        if (*fail) return false;
        if (clock64() - t0 > limit) {
            *fail = 1;
            return false;
        }
    }
    return true;
}
__device__ __forceinline__ bool mb_wait(uint64_t* b, unsigned parity, volatile int* fail, long long limit) {
    return tc::mb_try(b, parity) || mb_wait_on(b, parity, fail, limit);
}

__device__ __noinline__ bool known_wait(volatile int* known, int i, volatile int* fail, long long limit) {
    const long long t0 = clock64();
#pragma unroll 1
    while (*known <= i) {
        if (*fail) return false;
        if (clock64() - t0 > limit) {
            *fail = 1;
            return false;
        }
    }
    return true;
}

// the upper 11 bits of two values, and the rest
__device__ __forceinline__ f32x2 upper(f32x2 v) { return v & 0xffffe000ffffe000ull; }
__device__ __forceinline__ f32x2 rest(f32x2 v, f32x2 hi) { return fma2(hi, two(-1.f, -1.f), v); }
__device__ __forceinline__ uint32_t half2_of(f32x2 v) {
    float a, b;
    of_two(v, a, b);
    return pack2(a, b, f16());
}
// fp16 pairs of two values of q: hi towards zero, lo the rest and 2^-24 of the value, so that it has
// the value's sign and (down to 2^-16 of the row's largest value) is not 0
__device__ __forceinline__ void split_away(f32x2 v, uint32_t& hi, uint32_t& lo) {
    const f32x2 h = upper(v);
    hi = half2_of(h);
    lo = half2_of(fma2(v, two(0x1p-24f, 0x1p-24f), rest(v, h)));
}
// two weights as pairs of the cache's type: hi the upper bits (fp16 11, bf16 8), lo the rest
__device__ __forceinline__ void split_bits(f32x2 v, uint32_t& hi, uint32_t& lo, f16) {
    const f32x2 h = upper(v);
    hi = half2_of(h);
    lo = half2_of(rest(v, h));
}
__device__ __forceinline__ void split_bits(f32x2 v, uint32_t& hi, uint32_t& lo, bf16) {
    const f32x2 h = v & 0xffff0000ffff0000ull;
    float a, b;
    of_two(h, a, b);
    hi = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
    of_two(rest(v, h), a, b);
    lo = pack2(a, b, bf16());
}

// Which of the positions p0 .. p0 + 63 node `node` of a request sees, as bits; masks: its row's words, nullptr: a
// chain.  (Arguments of functions that are not inlined are values: a reference would put what it refers to into
// local memory.  The words are read here, for the few units that need them, rather than kept in registers.)
__device__ __noinline__ uint64_t visible(int len, int total, const uint64_t* masks, int words, int node, int p0) {
    const int end = total - p0;  // the unit's positions below it exist
    uint64_t v;
    if (!masks) {
        const long long last = (long long)len + node - p0;
        v = last >= 63 ? ~0ull : last < 0 ? 0ull : (2ull << last) - 1ull;
    } else {
        const int j0 = p0 - len;  // node of the unit's first position
        if (j0 <= -64) {
            v = ~0ull;
        } else if (j0 <= 0) {
            const uint64_t m = __ldcg(masks);
            v = j0 == 0 ? m : (m << -j0) | ((1ull << -j0) - 1ull);
        } else {
            const int w = j0 >> 6, s = j0 & 63;
            v = w < words ? __ldcg(masks + w) >> s : 0ull;
            if (s && w + 1 < words) v |= __ldcg(masks + w + 1) << (64 - s);
        }
    }
    return end >= 64 ? v : end <= 0 ? 0ull : v & ((1ull << end) - 1ull);
}

__device__ __forceinline__ uint32_t exps_all_ones(uint32_t u, f16) { return ((u & 0x7c00u) == 0x7c00u) | ((u & 0x7c000000u) == 0x7c000000u) << 1; }
__device__ __forceinline__ uint32_t exps_all_ones(uint32_t u, bf16) { return ((u & 0x7f80u) == 0x7f80u) | ((u & 0x7f800000u) == 0x7f800000u) << 1; }

// 0 if both values are finite, else a NaN in some half
__device__ __forceinline__ uint32_t finite2(uint32_t u, uint32_t acc, f16) {
    const __half2 r = __hfma2(*reinterpret_cast<const __half2*>(&u), __float2half2_rn(0.f), *reinterpret_cast<const __half2*>(&acc));
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t finite2(uint32_t u, uint32_t acc, bf16) {
    const __nv_bfloat162 r = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&u), __float2bfloat162_rn(0.f), *reinterpret_cast<const __nv_bfloat162*>(&acc));
    return *reinterpret_cast<const uint32_t*>(&r);
}
// Rows lo .. hi - 1 of 64 positions of V in shared memory, of which those from end on
// do not exist: zeros there, and in the place of values that are not finite.  By 128 threads.
template <typename C, int HD>
__device__ __noinline__ void clean_v(unsigned char* v8, int lo, int end, int hi, int t, int* odd_seen) {
    constexpr int PER_ROW = HD / 8;  // 16-byte pieces
    auto piece = [&](int c) {
        const int r = lo + c / PER_ROW, k = c % PER_ROW;
        return reinterpret_cast<uint4*>(v8 + (k >> 3) * (64 * 128) + r * 128 + (k & 7) * 16);
    };
    const int n = (max(end - lo, 0)) * PER_ROW, all = (hi - lo) * PER_ROW;
#pragma unroll 1
    for (int c = t; c < all; c += kTile) {
        uint4* v = piece(c);
        if (c >= n) {
            *v = make_uint4(0, 0, 0, 0);
            continue;
        }
        uint32_t w[4] = {v->x, v->y, v->z, v->w};
        if (!exps_all_ones(finite2(w[0], finite2(w[1], finite2(w[2], finite2(w[3], 0, C()), C()), C()), C()), C())) continue;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t odd = exps_all_ones(w[k], C());
            w[k] &= (odd & 1 ? 0u : 0xffffu) | (odd & 2 ? 0u : 0xffff0000u);
        }
        *v = make_uint4(w[0], w[1], w[2], w[3]);
        *(volatile int*)odd_seen = 1;
    }
}

// Adds to 32 dims of a row's result, in memory, the values that are not finite of positions
// from .. to - 1 that the row sees (clean_v left them out of the products).  Dim i lies at
// out[(i / 4) * stride + i % 4].
struct OddArgs {
    const uint64_t* masks;   // of the row (nullptr: chain)
    const int32_t* table;    // of the request
    const void* v;           // of the layer and head, at the first dim
    int64_t page_stride, pos_stride;
    int words, page_size, n_pages;
};
template <typename C, typename E>
__device__ __noinline__ void add_odd(OddArgs a, int len, int total, int node, int from, int to, E* out, int stride) {
#pragma unroll 1
    for (int x = max(from, len); x < min(to, total); ++x) {
        if (!(visible(len, total, a.masks, a.words, node, x) & 1)) continue;
        const int page = __ldcg(a.table + x / a.page_size);
        if (page < 0 || page >= a.n_pages) continue;
        const uint4* v = reinterpret_cast<const uint4*>((const C*)a.v + page * a.page_stride + (x % a.page_size) * a.pos_stride);
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {
            float f[8];
            Vec<C>::get(__ldcg(v + i), f);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (!isfinite(f[k])) {
                    E* p = out + (2 * i + k / 4) * stride + k % 4;
                    *p = (E)((float)*p + f[k]);
                }
        }
    }
}

// 32 dims of a row, 16 bytes of them kTile apart
__device__ __forceinline__ void to_memory(float4* to, const uint32_t (&o)[32]) {
#pragma unroll
    for (int i = 0; i < 32; i += 4)
        to[(i / 4) * kTile] = make_float4(__uint_as_float(o[i]), __uint_as_float(o[i + 1]), __uint_as_float(o[i + 2]), __uint_as_float(o[i + 3]));
}
// and back
__device__ __forceinline__ void from_memory(const float4* from, uint32_t (&o)[32]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float4 x = __ldcg(from + k * kTile);
        o[4 * k] = __float_as_uint(x.x), o[4 * k + 1] = __float_as_uint(x.y), o[4 * k + 2] = __float_as_uint(x.z), o[4 * k + 3] = __float_as_uint(x.w);
    }
}
// o += f times those
__device__ __forceinline__ void add_memory(const float4* from, float f, uint32_t (&o)[32]) {
    float4 m[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) m[k] = __ldcg(from + k * kTile);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        o[4 * k] = __float_as_uint(fmaf(f, m[k].x, __uint_as_float(o[4 * k])));
        o[4 * k + 1] = __float_as_uint(fmaf(f, m[k].y, __uint_as_float(o[4 * k + 1])));
        o[4 * k + 2] = __float_as_uint(fmaf(f, m[k].z, __uint_as_float(o[4 * k + 2])));
        o[4 * k + 3] = __float_as_uint(fmaf(f, m[k].w, __uint_as_float(o[4 * k + 3])));
    }
}

template <typename T, int HD>
__global__ void __launch_bounds__(kThreads, 1)
    attn_kernel(const __grid_constant__ AttnOpArgs a, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v) {
    using L = Lay<T, HD>;
    using C = typename Types<T>::C;
    constexpr int BOXES = L::BOXES, PARTS = L::PARTS, NB = L::NB;
    constexpr unsigned NK = L::NK, NV = L::NV;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    unsigned char *ks = smem + L::Q_ALL, *vs = ks + NK * L::KSLOT;
    __shared__ __align__(8) uint64_t k_full[kMaxSlots], k_empty[kMaxSlots], v_full[kMaxSlots], v_empty[kMaxSlots];
    __shared__ __align__(8) uint64_t q_ready, q_free, o_free, run_done, s_full[3], p_ready[3][2], pv_done[3], ends_ready[4], ref_ready[2][4];
    __shared__ uint32_t s_tmem;
    __shared__ int s_fail, s_odd;  // a wait gave up; a node's value is not finite
    __shared__ RangeOf<kThreads> s_range;
    // The CTA's segments, written by the K producer one ahead of itself, the one behind the last with n = 0; s_known: how
    // many so far.  (K is at most kMaxSlots units ahead of the scores, those three ahead of what is multiplied, and
    // results at most a segment behind that: a place is not written again before everyone has left it.)
    __shared__ Seg s_seg[kSegs];
    __shared__ int s_known;
    // (four segments: scores are at most three units ahead of the accumulator)
    __shared__ float s_scale[4][kTile];    // [segment & 3]: power of two that a row of q was divided by
    __shared__ float2 s_end[4][2][kTile];  // [segment & 3][group]: what a row's weights are relative to, and their sum
    __shared__ float s_ref[4][kTile];      // [unit & 3]: what a unit's weights are relative to
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        s_fail = s_odd = s_known = 0;
#pragma unroll 1
        for (int i = 0; i < kMaxSlots; ++i) {
            tc::mb_init(k_full + i, 1);
            tc::mb_init(k_empty + i, 1);
            tc::mb_init(v_full + i, 1);
            tc::mb_init(v_empty + i, 1);
        }
        tc::mb_init(&q_ready, 4);
        tc::mb_init(&q_free, 1);
        tc::mb_init(&o_free, 4);
        tc::mb_init(&run_done, 1);
        for (int i = 0; i < 3; ++i) {
            tc::mb_init(s_full + i, 1);
            tc::mb_init(&p_ready[i][0], 4);
            tc::mb_init(&p_ready[i][1], 4);
            tc::mb_init(pv_done + i, 1);
        }
        for (int i = 0; i < 4; ++i) {
            tc::mb_init(ends_ready + i, 8);
            tc::mb_init(&ref_ready[0][i], 1);
            tc::mb_init(&ref_ready[1][i], 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 8) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(kTmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_launch_dependents();
    pdl_wait();  // everything below may come from the previous kernel
    if (tid == 0) a.cuts[blockIdx.x].last = -1;

    const Shape& sh = a.shape;
    const int cta = blockIdx.x;
    tc::fence_before();
    Walk walk;
    int ctas;
    const long long units = range_of<kThreads>(a, kTile, s_range, walk, ctas);
    tc::fence_after();
    const uint32_t tmem = s_tmem;
    Seg g;
    bool ok = true;
    auto wait = [&](uint64_t* b, unsigned phase) {
        ok = ok && __all_sync(0xffffffffu, mb_wait(b, phase & 1u, &s_fail, a.wait_clocks));
        return ok;
    };

    // segment i to g, if there is one
    auto segment = [&](unsigned i) {
        ok = ok && __all_sync(0xffffffffu, *(volatile int*)&s_known > (int)i || known_wait(&s_known, (int)i, &s_fail, a.wait_clocks));
        __threadfence_block();
        g = s_seg[i % kSegs];
        return ok && g.n > 0;
    };

    // node of row `row` of a tile whose first row is `rem` heads into its first node, from that node on
    auto node_of = [&](int rem, int row) { return (int)(((uint64_t)(unsigned)(rem + row) * a.group_inv) >> 32); };

    if (warp == 8 || warp == 9) {
        // page ids are asked for 32 copies (of one 64-dim half) ahead, one per lane
        asm volatile("fence.proxy.async.global;" ::: "memory");  // K / V rows that the previous kernel wrote
        const bool is_v = warp == 9;
        const unsigned n_slots = is_v ? NV : NK;
        unsigned char* ring = is_v ? vs : ks;
        uint64_t *full = is_v ? v_full : k_full, *empty = is_v ? v_empty : k_empty;
        const CUtensorMap* map = is_v ? &tm_v : &tm_k;
        const int batch = 32 << a.box_shift;  // positions of 32 copies
        // a slot: V 64 positions x BOXES halves, K 128 positions x one half
        const int slot_rows = is_v ? 64 : kUnit, copies = slot_rows >> a.box_shift;
        const int my_box = is_v ? lane % copies : lane, my_half = is_v ? lane / copies : 0;
        const bool mine_too = lane < (is_v ? copies * BOXES : copies);
        const unsigned bytes = is_v ? L::VSLOT : L::KSLOT;
        unsigned slot = 0, phase = 1;
        unsigned published = 0;
        bool more = true;
        for (unsigned n_seg = 0; ok; ++n_seg) {
            if (!is_v)
#pragma unroll 1
                for (; published < n_seg + 2 && more; ++published) {
                    more = walk_next(walk, sh, kTile, g);
                    if (!more) g.n = 0;
                    if (lane == 0) {
                        s_seg[published % kSegs] = g;
                        __threadfence_block();
                        *(volatile int*)&s_known = (int)published + 1;
                    }
                    __syncwarp();
                }
            if (!segment(n_seg)) break;
            if (!is_v && cta == a.stall) break;  // (ssd_debug_tree_stall)
            const int32_t* table = a.block_table + (size_t)g.b * sh.max_blocks;
            auto fetch = [&](long long x) {  // page of this lane's copy of the 32 from x on; -1: outside, reads as zeros
                x += lane << a.box_shift;
                int page = -1;
                if (x < g.q.total) page = __ldcg(table + (int)x / sh.page_size);
                return page >= 0 && page < a.n_pages ? page : -1;
            };
            const int n = (g.u1 - g.u0) * (is_v ? 2 : BOXES);  // slots of the segment
            long long x0 = (long long)g.u0 * kUnit;
            int got = fetch(x0), ahead = fetch(x0 + batch);
#pragma unroll 1
            for (int i = 0; i < n; ++i) {
                const long long x = (long long)g.u0 * kUnit + (is_v ? i * 64 : i / BOXES * kUnit);  // the slot's first position
                if (x - x0 >= batch) {
                    x0 += batch;
                    got = ahead;
                    ahead = fetch(x0 + batch);
                }
                const int page = __shfl_sync(0xffffffffu, got, ((int)(x - x0) >> a.box_shift) + my_box);
                const int in_page = (int)((unsigned)(x + (my_box << a.box_shift)) % (unsigned)sh.page_size);
                if (!wait(empty + slot, phase)) break;
                if (elect_one()) tc::mb_arrive_tx(full + slot, bytes);
                __syncwarp();
                if (mine_too) {
                    const int c1 = a.at_pos == 1 ? in_page : a.at_head == 1 ? g.kvh : page;
                    const int c2 = a.at_pos == 2 ? in_page : a.at_head == 2 ? g.kvh : page;
                    const int c3 = a.at_pos == 3 ? in_page : a.at_head == 3 ? g.kvh : page;
                    const int half = is_v ? my_half : i % BOXES;
                    tma4d(ring + slot * bytes + my_half * L::VBOX + (my_box << a.box_shift) * 128, map, half * 64, c1, c2, c3, full + slot);
                }
                __syncwarp();
                if (++slot == n_slots) slot = 0, phase ^= 1u;
                if (!is_v && n_seg && i == BOXES) {  // the rows of q that will be asked for at the end of the segment before, into L2
                    const int start = g.mt * kTile, rows = min(g.q.n * sh.group - start, kTile), node0 = start / sh.group, rem = start - node0 * sh.group;
#pragma unroll 1
                    for (int r = lane; r < rows; r += 32) {
                        const int node = node_of(rem, r), head = g.kvh * sh.group + rem + r - node * sh.group;
                        const T* row = (const T*)a.q + (int64_t)(g.q.r0 + node0 + node) * a.q_stride + head * HD;
                        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(row), "n"(HD * sizeof(T)) : "memory");
                    }
                }
            }
        }
    } else if (warp == 10) {
        const uint64_t q0 = tc::sdesc(smem_u32(smem)), k0 = tc::sdesc(smem_u32(ks));
        unsigned slot = 0, phase = 0, buf = 0, turn = 0;  // unit 3 turn + buf
        for (unsigned n_seg = 0; ok && segment(n_seg); ++n_seg) {
            if (!wait(&q_ready, n_seg)) break;
#pragma unroll 1
            for (int u = g.u0; u < g.u1 && ok; ++u) {
                // P of unit j - NB, which held these columns, is used up
                if (turn && !wait(pv_done + buf, turn - 1)) break;
                const uint32_t d = tmem + (uint32_t)L::S0 + 128u * buf;
                auto multiply = [&](int h, int b, unsigned slot, bool more) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        mma_ss(d, q0 + (uint64_t)(((h * BOXES + b) * L::QBOX + k * 32) >> 4), k0 + (uint64_t)((slot * L::KSLOT + k * 32) >> 4),
                               idesc<C>(kUnit, false), (more || k) ? 1u : 0u);
                };
                unsigned slots[BOXES];
#pragma unroll
                for (int b = 0; b < BOXES; ++b) {
                    if (!wait(k_full + slot, phase)) break;
                    slots[b] = slot;
                    if (++slot == NK) slot = 0, phase ^= 1u;
                    if (PARTS == 1) {
                        tc::fence_after();
                        if (elect_one()) {
                            multiply(0, b, slots[b], b > 0);
                            commit(k_empty + slots[b]);
                        }
                        __syncwarp();
                    }
                }
                if (!ok) break;
                tc::fence_after();
                if (elect_one()) {
                    if (PARTS == 2)  // lo first: the accumulator truncates at every step, relative to what it holds
#pragma unroll
                        for (int h = 1; h >= 0; --h)
#pragma unroll
                            for (int b = 0; b < BOXES; ++b) {
                                multiply(h, b, slots[b], h == 0 || b > 0);
                                if (h == 0) commit(k_empty + slots[b]);
                            }
                    commit(s_full + buf);
                    if (u == g.u1 - 1) commit(&q_free);
                }
                __syncwarp();
                if (++buf == NB) buf = 0, ++turn;
            }
        }
    } else if (warp == 11) {
        // V: hd dims (MN) x 16 positions (K) per MMA; 8 positions are 1024 bytes apart, 64 dims a box
        const uint64_t v0 = tc::sdesc(smem_u32(vs)) + ((uint64_t)((L::VBOX >> 4) - 1) << 16);
        unsigned slot = 0, phase = 0, buf = 0, turn = 0;
        // every run's products start from 0, once the last one's have been added to the sums or written
        unsigned taken = 0;
        for (unsigned n_seg = 0; ok && segment(n_seg); ++n_seg) {
#pragma unroll 1
            for (int u = g.u0; u < g.u1 && ok; ++u) {
                const bool fresh = (u - g.u0) % L::RUN == 0;
                if (fresh && taken++ && !wait(&o_free, taken - 2)) break;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    if (!wait(&p_ready[buf][half], turn) || !wait(v_full + slot, phase)) break;
                    tc::fence_after();
                    if (elect_one()) {
                        const uint32_t p = tmem + (uint32_t)L::S0 + 128u * buf + 64u * half;
#pragma unroll
                        for (int h = 1; h >= 0; --h)  // (lo first, as above)
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                mma_ts(tmem, p + 32u * (k >> 1) + 16u * h + 8u * (k & 1), v0 + (uint64_t)((slot * L::VSLOT + k * 2048) >> 4), idesc<C>(HD, true),
                                       (!fresh || half || k || h == 0) ? 1u : 0u);
                        commit(v_empty + slot);
                        if (half) {
                            commit(pv_done + buf);
                            if ((u - g.u0) % L::RUN == L::RUN - 1 || u == g.u1 - 1) commit(&run_done);
                        }
                    }
                    __syncwarp();
                    if (++slot == NV) slot = 0, phase ^= 1u;
                }
                if (++buf == NB) buf = 0, ++turn;
            }
        }
    } else if (warp >= 12) {
        const int quarter = warp & 3, mine32 = quarter * 32 + lane;  // this thread's row of the tile
        const uint32_t tl = tmem + ((uint32_t)(quarter * 32) << 16);
        // q of the segment's rows (K-major, 128-byte swizzle: row r of 64 dims at r * 128, 16-byte
        // chunk c at (c ^ (r & 7)) * 16), a few rows a step, steps over the four warps.  Rows that do not
        // exist keep what lies there: no one reads their lanes.
        // fp32 rows come as they are into the place of their pairs - a row has 16 bytes of each for 16 bytes of dims -
        // and are converted there.
        auto load_q = [&](const Seg& s, unsigned n_seg) {
            constexpr int V = Vec<T>::N, LPR = HD / V, RPI = 32 / LPR;  // lanes per row, rows per step
            const int start = s.mt * kTile, rows = min(s.q.n * sh.group - start, kTile), node0 = start / sh.group, rem = start - node0 * sh.group;
            const int piece = lane % LPR;
            unsigned char* to = smem + (piece >> 3) * L::QBOX;
#pragma unroll 4
            for (int r = quarter * RPI + lane / LPR; r < rows; r += 4 * RPI) {
                const int node = node_of(rem, r), head = s.kvh * sh.group + rem + r - node * sh.group;
                const T* from = (const T*)a.q + (int64_t)(s.q.r0 + node0 + node) * a.q_stride + head * HD + piece * V;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to + r * 128 + (((piece & 7) ^ (r & 7)) << 4))), "l"(from) : "memory");
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            __syncwarp();
            if constexpr (PARTS == 2) {
                constexpr int N = 4;  // steps at once
                const int e = piece * V;
                unsigned char* hi = smem + (e >> 6) * L::QBOX + (e & 7) * 2;
#pragma unroll 1
                for (int i0 = quarter * RPI + lane / LPR; i0 - lane / LPR < rows; i0 += N * 4 * RPI) {
                    uint4 x[N];
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const int r = min(i0 + i * 4 * RPI, kTile - 1);
                        x[i] = *reinterpret_cast<const uint4*>(to + r * 128 + (((piece & 7) ^ (r & 7)) << 4));
                    }
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const int r = i0 + i * 4 * RPI;
                        float f[4];
                        Vec<float>::get(x[i], f);
                        // the row's largest absolute value (as bits: their order is the same, NaN above all)
                        const float m = fmaxf(max3(fabsf(f[0]), fabsf(f[1]), fabsf(f[2])), fabsf(f[3]));
                        const uint32_t top = __reduce_max_sync(LPR == 32 ? 0xffffffffu : lane < 16 ? 0xffffu : 0xffff0000u, __float_as_uint(m));
                        // 2^e2 with that at 2^14 .. 2^15 of it (zeros and the smallest values: as if it were 2^-111)
                        const int e2 = min(max((int)(top >> 23), 16), 254) - 127 - 14;
                        const float down = __uint_as_float((uint32_t)(127 - e2) << 23);
                        uint2 h, l;
                        split_away(mul2(two(f[0], f[1]), two(down, down)), h.x, l.x);
                        split_away(mul2(two(f[2], f[3]), two(down, down)), h.y, l.y);
                        if (r < rows) {
                            unsigned char* at = hi + r * 128 + ((((e & 63) >> 3) ^ (r & 7)) << 4);
                            *reinterpret_cast<uint2*>(at) = h;
                            *reinterpret_cast<uint2*>(at + BOXES * L::QBOX) = l;
                            if (piece == 0) s_scale[n_seg & 3][r] = __uint_as_float((uint32_t)(127 + e2) << 23);
                        }
                    }
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) arrive(&q_ready);
        };
        bool more = segment(0);
        if (more) load_q(g, 0);
        unsigned j = 0;       // of the segment's first unit
        unsigned n_runs = 0;  // (the accumulator is one run's until o_free, so this warp is never a phase behind)
        for (unsigned n_seg = 0; more && ok; ++n_seg) {
            const Seg cur = g;
            const int n = cur.u1 - cur.u0, start = cur.mt * kTile, rows = min(cur.q.n * sh.group - start, kTile);
            const bool active = quarter * 32 < rows, valid = mine32 < rows, whole = cur.u0 == 0 && cur.u1 == cur.n;
            const unsigned j_last = j + (unsigned)n - 1;
            float ref = -INFINITY;  // what the sums of earlier runs are relative to
            float top = 0.f, sum = 0.f;  // what the result is relative to, and the weights' sum
            auto ends = [&] {
                if (!wait(ends_ready + (n_seg & 3), n_seg >> 2)) return false;
                // (the last unit's group has what the accumulator is relative to now)
                const float2 e = s_end[n_seg & 3][j_last & 1u][mine32], f = s_end[n_seg & 3][~j_last & 1u][mine32];
                top = e.x;
                sum = e.y + f.y * (f.x == -INFINITY ? 0.f : ex2(f.x - e.x));
                return true;
            };
            // the next rows' q, once all scores of this segment are there
            auto next_q = [&] {
                more = segment(n_seg + 1);
                if (more && wait(&q_free, n_seg)) load_q(g, n_seg + 1);
            };
            // the segment's place in the workspace (written again by the next segment only if this one is the whole item)
            const int slot = n_seg ? 1 : 0;
            float4* const part = a.part + (size_t)(cta * 2 + slot) * (HD / 4) * kTile + mine32;
            // (q before the products that are still to be added, as scores are up to NB units ahead of them: with fp32 rows' q
            // asked for after all others were added, multiplying stopped for 10 us an item, and for 5 so; 16-bit rows:
            // before the last run's, as nothing of an earlier one waits for it)
            const int runs = (n + L::RUN - 1) / L::RUN, q_at = L::RUN == 1 ? max(n - NB, 0) : runs - 1;
#pragma unroll 1
            for (int i = 0; i < runs; ++i) {
                if (i == q_at) next_q();
                const unsigned ju = min(j + (unsigned)((i + 1) * L::RUN) - 1, j_last);
                if (i == runs - 1 && !ends()) break;
                if (!wait(&run_done, L::RUN == 1 ? ju : n_runs++)) break;
                tc::fence_after();
                if (L::RUN > 1 && runs == 1) break;  // (written from the accumulator)
                const float r = *(volatile float*)&s_ref[ju & 3][mine32], f = ref == -INFINITY ? 0.f : ex2(ref - r);
                if (active) {
#pragma unroll 1
                    for (int c = 0; c < HD; c += 32) {
                        uint32_t o[32];
                        ld32(tl + c, o);
                        if constexpr (L::SUMS_IN_TMEM) {
                            uint32_t m[32];
                            if (i) ld32(tl + L::M0 + c, m);
                            wait_ld();
                            if (i)
#pragma unroll
                                for (int k = 0; k < 32; k += 2) {
                                    float a0, a1;
                                    of_two(fma2(two(__uint_as_float(m[k]), __uint_as_float(m[k + 1])), two(f, f), two(__uint_as_float(o[k]), __uint_as_float(o[k + 1]))), a0, a1);
                                    o[k] = __float_as_uint(a0);
                                    o[k + 1] = __float_as_uint(a1);
                                }
                            st32(tl + L::M0 + c, o);
                        } else {
                            wait_ld();
                            if (i) add_memory(part + c / 4 * kTile, f, o);
                            if (valid) to_memory(part + c / 4 * kTile, o);
                        }
                    }
                    if constexpr (L::SUMS_IN_TMEM) wait_st();
                }
                tc::fence_before();
                __syncwarp();
                if (lane == 0) arrive(&o_free);
                ref = r;
            }
            if (!ok) break;
            if (tid == 12 * 32 && cur.u1 < cur.n) {
                Cut c;
                holders(cur, units, ctas, c.first, c.last, c.first_slot);
                c.row0 = start;
                c.rows = rows;
                c.r0 = cur.q.r0;
                c.kvh = cur.kvh;
                c.pad = 0;
                a.cuts[cta] = c;
            }
            const int node0 = start / sh.group, rem = start - node0 * sh.group, row = min(mine32, rows - 1);
            const int node = node0 + node_of(rem, row), head = cur.kvh * sh.group + rem + row - (node - node0) * sh.group;
            if (active) {
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
                const bool odd = *(volatile int*)&s_odd;
                // positions below it are seen by every row, and their values multiplied as they are
                const int all_seen = min(sh.chain ? cur.q.len + node0 + 1 : cur.q.len, cur.q.total);
                auto odd_to = [&](int c, auto* to, int stride) {
                    const OddArgs oa = {sh.chain ? nullptr : a.masks + (size_t)(cur.q.r0 + node) * a.words, a.block_table + (size_t)cur.b * sh.max_blocks,
                                        (const C*)a.vc + cur.kvh * a.head_stride + c, a.page_stride, a.pos_stride, a.words, sh.page_size, a.n_pages};
                    add_odd<C>(oa, cur.q.len, cur.q.total, node, max(cur.u0, all_seen / kUnit) * kUnit, cur.u1 * kUnit, to, stride);
                };
                if (!whole && valid) {
                    float* st = a.stats + (size_t)(cta * 2 + slot) * 2 * kTile + mine32;
                    st[0] = top;
                    st[kTile] = sum;
                }
#pragma unroll 1
                for (int c = 0; c < HD; c += 32) {
                    uint32_t o[32];
                    if (L::SUMS_IN_TMEM || runs == 1) {
                        ld32(tl + (L::RUN == 1 || runs > 1 ? L::M0 : 0) + c, o);
                        wait_ld();
                    } else {
                        from_memory(part + c / 4 * kTile, o);
                    }
                    if (!valid) continue;
                    if (whole) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * inv);
                        T* to = (T*)a.out + (int64_t)(cur.q.r0 + node) * a.out_stride + head * HD + c;
                        constexpr int V = Vec<T>::N;
#pragma unroll
                        for (int i = 0; i < 32; i += V) {
                            float f[V];
#pragma unroll
                            for (int k = 0; k < V; ++k) f[k] = __uint_as_float(o[i + k]);
                            *reinterpret_cast<uint4*>(to + i) = Vec<T>::put(f);
                        }
                        if (odd) odd_to(c, to, 4);
                    } else {
                        float4* to = part + c / 4 * kTile;
                        to_memory(to, o);
                        if (odd) odd_to(c, reinterpret_cast<float*>(to), 4 * kTile);
                    }
                }
            }
            if (L::RUN > 1 && runs == 1) {
                tc::fence_before();
                __syncwarp();
                if (lane == 0) arrive(&o_free);
            }
            j += (unsigned)n;
        }
    } else {
        const int grp = warp >> 2, quarter = warp & 3, mine32 = quarter * 32 + lane;  // this thread's row of the tile
        const uint32_t tl = tmem + ((uint32_t)(quarter * 32) << 16);
        unsigned j = 0;  // of the segment's first unit
        for (unsigned n_seg = 0; ok && segment(n_seg); ++n_seg) {
            const int n = g.u1 - g.u0, start = g.mt * kTile, rows = min(g.q.n * sh.group - start, kTile);  // units; rows that exist
            const bool active = quarter * 32 < rows;
            const int node0 = start / sh.group, node = node0 + node_of(start - node0 * sh.group, min(mine32, rows - 1));
            // positions below it are seen by every row of the tile
            const int all_seen = min(sh.chain ? g.q.len + node0 + 1 : g.q.len, g.q.total);
            const int first = (int)((j ^ (unsigned)grp) & 1u);  // this group's first unit of the segment
            float ref = -INFINITY, l = 0.f, sc = a.scale2;  // what the weights are relative to (and kShift), their sum
#pragma unroll 1
            for (int i = first; i < n; i += 2) {
                const unsigned ju = j + (unsigned)i, turn = ju / NB, buf = ju - NB * turn;
                const int p0 = (g.u0 + i) * kUnit;
                const uint32_t ts = tl + (uint32_t)L::S0 + 128u * buf;
                if (!wait(s_full + buf, turn)) break;
                tc::fence_after();
                if constexpr (PARTS == 2)
                    if (i == first) sc = a.scale2 * s_scale[n_seg & 3][mine32];
                const bool tail = p0 + kUnit > all_seen;
                // The weights of half of the unit are there: V, if some row does not see all of it, and the word to
                // the multiplying warp.  (Unit ju - 2 is used up: then the slots' fills before these
                // ones are complete, and the parity of the wait means these.)
                auto half_done = [&](int half) {
                    if (tail && ok) {
                        const unsigned s = 2 * ju + half;
                        const int x0 = p0 + 64 * half, lo_row = max(min(g.q.len, g.q.total) - x0, 0);
                        // (copies that begin behind the last position have brought zeros)
                        const int hi_row = min((max(g.q.total - x0, 0) + (1 << a.box_shift) - 1) >> a.box_shift << a.box_shift, 64);
                        if (lo_row < hi_row && (ju < 2 || wait(pv_done + (ju - 2) % NB, (ju - 2) / NB)) && wait(v_full + s % NV, s / NV)) {
                            clean_v<C, HD>(vs + s % NV * L::VSLOT, lo_row, min(g.q.total - x0, 64), hi_row, tid & (kTile - 1), &s_odd);
                            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        }
                    }
                    tc::fence_before();
                    __syncwarp();
                    if (lane == 0) arrive(&p_ready[buf][half]);
                };
                if (active) {
                    // 32 scores of the unit.  (Twice, once for the maximum and once for the weights, in loops that are not
                    // unrolled: the code of a unit is an eighth of what it was unrolled, and takes fewer registers.)
                    uint32_t x[32];
                    auto load = [&](int c) {
                        ld32(ts + 32 * c, x);
                        wait_ld();
                    };
                    if (tail) {  // scores of positions that the row does not see: -inf
                        uint64_t v = 0;
#pragma unroll 1
                        for (int c = 0; c < kUnit / 32; ++c) {
                            v = c & 1 ? v >> 32 : visible(g.q.len, g.q.total, sh.chain ? nullptr : a.masks + (size_t)(g.q.r0 + node) * a.words, a.words, node, p0 + 32 * c);
                            load(c);
#pragma unroll
                            for (int k = 0; k < 32; ++k)
                                if (!((uint32_t)v >> k & 1u)) x[k] = 0xff800000u;
                            st32(ts + 32 * c, x);
                        }
                        wait_st();
                    }
                    float bm = -INFINITY;
#pragma unroll 1
                    for (int c = 0; c < kUnit / 32; ++c) {
                        load(c);
                        float m4[4] = {bm, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                        for (int k = 0; k < 32; k += 2) m4[k >> 1 & 3] = max3(m4[k >> 1 & 3], __uint_as_float(x[k]), __uint_as_float(x[k + 1]));
                        bm = max3(fmaxf(m4[0], m4[1]), m4[2], m4[3]);
                    }
                    bm = mine32 < rows ? bm * sc : -INFINITY;  // (lanes of no row hold anything)
                    // from the unit before, and on to the next one (in every unit, so that the groups stay in step)
                    float r = bm - kShift;
                    if (ju && !wait(&ref_ready[grp ^ 1][quarter], (ju - 1) >> 1)) break;
                    if (i > 0) {
                        r = *(volatile float*)&s_ref[(ju - 1) & 3][mine32];
                        if (__any_sync(0xffffffffu, bm - kShift > r + kSlack)) {
                            const float nr = bm - kShift > r + kSlack ? bm - kShift : r;  // (each row by what it sees alone)
                            if (L::RUN > 1 && i % L::RUN) {  // (a run's first unit finds it empty) the accumulator moves to the new maximum (the other rows of the warp: by a factor of 1)
                                const unsigned tb = (ju - 1) / NB, bb = ju - 1 - NB * tb;
                                if (!wait(pv_done + bb, tb)) break;
                                tc::fence_after();
                                const float f = nr == r ? 1.f : ex2(r - nr);
#pragma unroll 1
                                for (int c = 0; c < HD; c += 32) {
                                    ld32(tl + c, x);
                                    wait_ld();
#pragma unroll
                                    for (int k = 0; k < 32; ++k) x[k] = __float_as_uint(__uint_as_float(x[k]) * f);
                                    st32(tl + c, x);
                                }
                            }
                            r = nr;
                        }
                    }
                    *(volatile float*)&s_ref[ju & 3][mine32] = r;
                    __syncwarp();
                    if (lane == 0) arrive(&ref_ready[grp][quarter]);
                    if (ref != -INFINITY) l *= ex2(ref - r);
                    ref = r;
                    // (a row that has seen nothing yet, or only scores of -inf: weights 0)
                    const float sub = r == -INFINITY ? 0.f : r;
#pragma unroll 1
                    for (int c = 0; c < kUnit / 32; ++c) {
                        load(c);
                        f32x2 l4[4] = {0, 0, 0, 0};
                        // 32 weights in the place of their scores: 16 columns of pairs (hi), 16 of lo
                        uint32_t ph[16], pl[16];
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            float e0, e1;
                            of_two(fma2(two(__uint_as_float(x[2 * k]), __uint_as_float(x[2 * k + 1])), two(sc, sc), two(-sub, -sub)), e0, e1);
                            e0 = ex2(e0);
                            e1 = ex2(e1);
                            const f32x2 e = two(e0, e1);
                            l4[k & 3] = add2(l4[k & 3], e);
                            split_bits(e, ph[k], pl[k], C());
                        }
                        st16(ts + 32 * c, ph);
                        st16(ts + 32 * c + 16, pl);
                        float la, lb;
                        of_two(add2(add2(l4[0], l4[1]), add2(l4[2], l4[3])), la, lb);
                        l += la + lb;
                        if (c & 1) {
                            wait_st();
                            half_done(c >> 1);
                        }
                    }
                } else {
                    if (ju && !wait(&ref_ready[grp ^ 1][quarter], (ju - 1) >> 1)) break;
                    if (lane == 0) arrive(&ref_ready[grp][quarter]);
#pragma unroll 1
                    for (int h = 0; h < 2; ++h) half_done(h);
                }
            }
            if (!ok) break;
            s_end[n_seg & 3][grp][mine32] = make_float2(ref, l);
            __syncwarp();
            if (lane == 0) arrive(ends_ready + (n_seg & 3));
            j += (unsigned)n;
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
    if (warp == 8) {
        tc::fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmem) : "memory");
    }
}

// Joins the parts of the items that range ends cut.  CTA c of the attention left a
// Cut if its range ends inside an item; with n such ends in an item, n lines of CTAs
// (gridDim.y each) share it here.  A piece of work is 32 rows (a lane each) and 16 bytes of
// dims; 1, 2, 4 or 8 warps take up to four parts of it each at once, in the order of
// the parts, and the first one adds their sums, in order.  Bound by L2 latency: with more
// parts a warp one after the other (19 parts of 8 items) the long request took 4 us more.
template <typename T, int HD>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const AttnOpArgs a) {
    constexpr int W = kJoinThreads / 32, D = Vec<T>::N, AHEAD = 4;
    __shared__ float s_o[W][D + 2][32];
    pdl_launch_dependents();
    pdl_wait();
    const int cta = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int4 c0 = __ldcg(reinterpret_cast<const int4*>(a.cuts + cta)), c1 = __ldcg(reinterpret_cast<const int4*>(a.cuts + cta) + 1);
    const int first = c0.x, last = c0.y, slot = c0.z, row0 = c0.w, rows = c1.x, r0 = c1.y, kvh = c1.z;
    if (last < 0) return;
    const int parts = last - first + 1;
    int team = 1;  // warps of a piece
    while (team < W && parts > AHEAD * team) team *= 2;
    const int per = (parts + team - 1) / team, mate = warp & (team - 1), teams = W / team;
    const int lines = (last - first) * (int)gridDim.y, items = (rows + 31) / 32 * (HD / D);
    for (int w0 = ((cta - first) * (int)gridDim.y + blockIdx.y) * teams; w0 < items; w0 += lines * teams) {  // (the same for the CTA's warps)
        const int w = w0 + warp / team, chunk = w % (HD / D), row = w / (HD / D) * 32 + lane;
        const bool mine = w < items && row < rows;
        float top = -INFINITY, l = 0.f, o[D];
#pragma unroll
        for (int i = 0; i < D; ++i) o[i] = 0.f;
        auto add = [&](float m, float lp, const float (&x)[D]) {
            const float t = fmaxf(top, m), f = top == -INFINITY ? 0.f : ex2(top - t), g = m == -INFINITY ? 0.f : ex2(m - t);  // (0 x NaN stays NaN)
            l = l * f + lp * g;
#pragma unroll
            for (int i = 0; i < D; ++i) o[i] = o[i] * f + x[i] * g;
            top = t;
        };
        const int p1 = min(first + (mate + 1) * per, last + 1);
        if (mine)
            for (int p = first + mate * per; p < p1; p += AHEAD) {
                float m[AHEAD], lp[AHEAD];
                float4 x[AHEAD][D / 4];
#pragma unroll
                for (int i = 0; i < AHEAD; ++i)
                    if (p + i < p1) {
                        const size_t part = (size_t)((p + i) * 2 + (p + i == first ? slot : 0));
                        const float* st = a.stats + part * 2 * kTile + row;
                        m[i] = __ldcg(st);
                        lp[i] = __ldcg(st + kTile);
#pragma unroll
                        for (int k = 0; k < D / 4; ++k) x[i][k] = __ldcg(a.part + (part * (HD / 4) + chunk * (D / 4) + k) * kTile + row);
                    }
#pragma unroll
                for (int i = 0; i < AHEAD; ++i)
                    if (p + i < p1) {
                        float f[D];
#pragma unroll
                        for (int k = 0; k < D / 4; ++k) f[4 * k] = x[i][k].x, f[4 * k + 1] = x[i][k].y, f[4 * k + 2] = x[i][k].z, f[4 * k + 3] = x[i][k].w;
                        add(m[i], lp[i], f);
                    }
            }
        if (team > 1) {
            if (mate) {
                s_o[warp][0][lane] = top;
                s_o[warp][1][lane] = l;
#pragma unroll
                for (int i = 0; i < D; ++i) s_o[warp][2 + i][lane] = o[i];
            }
            __syncthreads();
            if (!mate)
                for (int k = 1; k < team; ++k) {
                    float f[D];
#pragma unroll
                    for (int i = 0; i < D; ++i) f[i] = s_o[warp + k][2 + i][lane];
                    add(s_o[warp + k][0][lane], s_o[warp + k][1][lane], f);
                }
            __syncthreads();
        }
        if (!mine || mate) continue;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const int r = row0 + row, node = r / a.shape.group, head = kvh * a.shape.group + r - node * a.shape.group;
        T* to = (T*)a.out + (int64_t)(r0 + node) * a.out_stride + head * HD + chunk * D;
#pragma unroll
        for (int i = 0; i < D; ++i) o[i] *= inv;
        *reinterpret_cast<uint4*>(to) = Vec<T>::put(o);
    }
}

// -- host ----------------------------------------------------------------------

// the workspace: cuts, parts and statistics of a grid of one CTA an SM
size_t workspace_need(int n_sms, int hd) {
    return (size_t)n_sms * (sizeof(Cut) + 2 * 2 * kTile * sizeof(float) + 2 * (size_t)kTile * hd * sizeof(float));
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
// ssd_debug_tree_stall, for one call (guarded by g_attn_mu)
int g_stall = -1;
double g_stall_wait_s = 0.0;

template <typename T>
cudaError_t set_up_type() {
    cudaError_t e = cudaFuncSetAttribute(attn_kernel<T, 64>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Lay<T, 64>::BYTES);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(attn_kernel<T, 128>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Lay<T, 128>::BYTES);
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

template <typename T, int HD>
int run_hd(const char* call, AttnOpArgs& a, int dtype, const CUtensorMap& k, const CUtensorMap& v, void* stream) {
    using L = Lay<T, HD>;
    int rc;
    if (a.tile <= kFewRows) {
        rc = launch_few(call, a, dtype, HD, stream);
    } else {
        rc = launch(call, attn_kernel<T, HD>, dim3((unsigned)a.grid), kThreads, L::BYTES, stream, a, k, v);
    }
    // an item of one unit is never cut
    if (rc || (long long)a.shape.max_blocks * a.shape.page_size <= kUnit || a.grid == 1) return rc;
    return launch(call, join_kernel<T, HD>, dim3((unsigned)(a.grid - 1), kJoinLines), kJoinThreads, 0, stream, a);
}
template <typename T>
int run(const char* call, AttnOpArgs& a, int dtype, int hd, const CUtensorMap& k, const CUtensorMap& v, void* stream) {
    return hd == 64 ? run_hd<T, 64>(call, a, dtype, k, v, stream) : run_hd<T, 128>(call, a, dtype, k, v, stream);
}

}  // namespace
}  // namespace tree
}  // namespace ssd

using namespace ssd;
using namespace ssd::tree;

extern "C" void ssd_debug_tree_stall(int cta, double wait_limit_s) {
    std::lock_guard<std::mutex> lock(g_attn_mu);
    g_stall = cta >= 0 && wait_limit_s > 0.0 && wait_limit_s <= 10.0 ? cta : -1;
    g_stall_wait_s = wait_limit_s;
}

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
    a.kc = (const char*)cache->k + 2 * layer * cache->layer_stride;
    a.vc = (const char*)cache->v + 2 * layer * cache->layer_stride;
    a.page_stride = cache->page_stride;
    a.head_stride = cache->head_stride;
    a.pos_stride = cache->pos_stride;
    a.n_heads = n_heads;
    a.n_pages = cache->n_pages;
    a.stall = -1;
    a.wait_clocks = (long long)(kWaitSeconds * kClocksPerSecond);
    a.box_shift = cache->page_size % 64 == 0 ? 6 : cache->page_size % 32 == 0 ? 5 : 4;
    a.scale2 = (float)(1.4426950408889634 * scale);
    a.status = status;
    const long long rows = (long long)batch->max_rows * group;
    a.tile = rows <= kFewRows ? (int)rows : kTile;  // (both sides measured: tree_few.cu)
    a.group_inv = ((1ull << 32) + group - 1) / group;
    a.grid = n_sms;
    a.cuts = (Cut*)workspace;
    a.part = (float4*)(a.cuts + a.grid);
    a.stats = (float*)(a.part + (size_t)a.grid * 2 * (cache->head_dim / 4) * kTile);
    CUtensorMap k, v;
    if (a.tile > kFewRows) {
        if (int rc = encode(call, &k, a.kc, cache, a)) return rc;
        if (int rc = encode(call, &v, a.vc, cache, a)) return rc;
        std::lock_guard<std::mutex> lock(g_attn_mu);
        if (g_stall >= 0) {
            a.stall = g_stall;
            a.wait_clocks = (long long)(g_stall_wait_s * kClocksPerSecond);
            g_stall = -1;
        }
    }
    const int hd = cache->head_dim;
    if (dtype == SSD_F32) return run<float>(call, a, dtype, hd, k, v, cuda_stream);
    if (dtype == SSD_F16) return run<f16>(call, a, dtype, hd, k, v, cuda_stream);
    return run<bf16>(call, a, dtype, hd, k, v, cuda_stream);
}
