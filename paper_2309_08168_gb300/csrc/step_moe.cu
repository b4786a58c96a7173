// step_moe.cu - a mixture-of-experts layer for the rows of a decoding step:
// the router (ssd_moe_route) and the experts' products (ssd_moe_mlp) of ssd_step.h.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <cmath>
#include <mutex>

#include "step_ops.cuh"
#include "tc_gemm.cuh"

namespace ssd {
namespace step {

constexpr int kMaxExperts = 1024, kMaxSlots = 16, kMaxMoeRows = 1024;

// ---------------------------------------------------------------------------
// ssd_moe_route
// ---------------------------------------------------------------------------
constexpr int kRouteThreads = 512, kRouteWarps = kRouteThreads / 32, kRouteSplit = 8;  // CTAs of a row at most, 2 at least
constexpr int kRouteShare = kMaxExperts / 2;  // experts of a CTA at most

struct RouteArgs {
    const void *x, *w;
    const float* favour;
    int32_t* ids;
    float* weights;
    int64_t x_stride;
    int d, n_experts, k, score, renorm;
    float scale;
};

// what a double sorts by; NaN is below all
__device__ __forceinline__ uint64_t order_of(double v) {
    if (v != v) return 0ull;
    const uint64_t u = (uint64_t)__double_as_longlong(v + 0.0);
    return u >> 63 ? ~u : u | 1ull << 63;
}

// s + c += q without loss but in c
__device__ __forceinline__ void add_exactly(float& s, float& c, float q) {
    const float t = __fadd_rn(s, q), b = __fsub_rn(t, s);
    c = __fadd_rn(c, __fadd_rn(__fsub_rn(s, __fsub_rn(t, b)), __fsub_rn(q, b)));
    s = t;
}

// A cluster of CTAs (8 to 2) takes a row, each a share of the experts.  Which of two experts comes first must not hang on the order of a sum,
// so the products (exact in fp32: two values of 8 or 11 bits) are added without loss to a pair of floats, 6 additions each
// (Knuth's two-sum), over lanes too; fp64 sums would be slower by an order, with two fp64 units an SM.
// Scores decide by z itself where that is the same order, in fp64 where something is added to them.  The rank of an
// expert is the number of better ones, counted by a warp of the CTA that has it; the winners go to the first CTA.
template <typename T>
__global__ void __launch_bounds__(kRouteThreads, 2) route_kernel(const __grid_constant__ RouteArgs a) {
    __shared__ float2 s_part[kRouteShare];  // [warp of an expert][expert], with more than one warp for up to 8 experts
    __shared__ double s_z[kRouteShare];
    __shared__ uint64_t s_key[kRouteShare], s_all[kMaxExperts];
    __shared__ double s_top[kMaxSlots];  // the winners' z and expert, in the first CTA
    __shared__ uint64_t s_who[kMaxSlots], s_stat[kRouteSplit];
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, rank = blockIdx.x, row = blockIdx.y, split = gridDim.x;
    const int share = (a.n_experts + split - 1) / split, e0 = min(rank * share, a.n_experts), mine = min(share, a.n_experts - e0);
    // warps of an expert, each a part of d
    const int per = share <= 2 ? 8 : share <= 4 ? 4 : share <= 8 ? 2 : 1, part = warp % per;
    const int pieces = a.d / 8, p0 = (int)((int64_t)pieces * part / per), p1 = (int)((int64_t)pieces * (part + 1) / per);
    const uint4* x = reinterpret_cast<const uint4*>((const T*)a.x + (int64_t)row * a.x_stride);
    for (int e = warp / per; e < mine; e += kRouteWarps / per) {
        const uint4* w = reinterpret_cast<const uint4*>((const T*)a.w + (int64_t)(e0 + e) * a.d);
        float s = 0.f, c = 0.f;
        for (int p = p0 + lane; p < p1; p += 128) {
            uint4 u[4], v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool in = p + 32 * i < p1;
                u[i] = in ? w[p + 32 * i] : make_uint4(0u, 0u, 0u, 0u);
                v[i] = in ? x[p + 32 * i] : make_uint4(0u, 0u, 0u, 0u);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float f[8], g[8];
                Vec<T>::get(u[i], f);
                Vec<T>::get(v[i], g);
#pragma unroll
                for (int j = 0; j < 8; ++j) add_exactly(s, c, __fmul_rn(f[j], g[j]));
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const float q = __shfl_xor_sync(0xffffffffu, s, o), r = __shfl_xor_sync(0xffffffffu, c, o);
            add_exactly(s, c, q);
            c = __fadd_rn(c, r);
        }
        if (lane == 0) s_part[part * share + e] = make_float2(s, c);
    }
    __syncthreads();
    for (int e = tid; e < mine; e += kRouteThreads) {
        float2 v = s_part[e];
        for (int i = 1; i < per; ++i) {
            const float2 o = s_part[i * share + e];
            add_exactly(v.x, v.y, o.x);
            v.y = __fadd_rn(v.y, o.y);
        }
        s_z[e] = isfinite(v.x) ? (double)v.x + (double)v.y : (double)v.x;
    }
    __syncthreads();
    // softmax over all experts where the scores or the weights need it: the row's maximum and sum (without NaN; of +inf each has the same share)
    const bool whole = a.score == SSD_MOE_SOFTMAX && (a.favour || !a.renorm);
    if (whole) {
        cluster_sync();  // (every CTA has started)
        double m = -INFINITY;
        if (warp == 0) {
            for (int e = lane; e < mine; e += 32) m = fmax(m, s_z[e]);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) m = fmax(m, __shfl_xor_sync(0xffffffffu, m, o));
            if (lane < split) peer_store(&s_stat[rank], lane, (uint64_t)__double_as_longlong(m));
        }
        cluster_sync();
        m = -INFINITY;
        for (int i = 0; i < split; ++i) m = fmax(m, __longlong_as_double((long long)s_stat[i]));
        auto above = [&](double z) { return z == m ? 1.0 : exp(z - m); };
        double sum = 0.0;
        if (warp == 0) {
            for (int e = lane; e < mine; e += 32) sum += s_z[e] == s_z[e] ? above(s_z[e]) : 0.0;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        }
        cluster_sync();  // (the maxima are read)
        if (warp == 0 && lane < split) peer_store(&s_stat[rank], lane, (uint64_t)__double_as_longlong(sum));
        cluster_sync();
        sum = 0.0;
        for (int i = 0; i < split; ++i) sum += __longlong_as_double((long long)s_stat[i]);
        for (int e = tid; e < mine; e += kRouteThreads) {
            const double p = above(s_z[e]) / sum;
            s_key[e] = order_of(a.favour ? p + (double)__ldcg(a.favour + e0 + e) : s_z[e]);
            s_z[e] = p;  // (from here on the score)
        }
    } else {
        for (int e = tid; e < mine; e += kRouteThreads) {
            if (a.favour) s_key[e] = order_of(1.0 / (1.0 + exp(-s_z[e])) + (double)__ldcg(a.favour + e0 + e));
            else s_key[e] = order_of(s_z[e]);
        }
    }
    cluster_sync();
    for (int e = tid; e < a.n_experts; e += kRouteThreads) s_all[e] = peer_load(&s_key[e % share], e / share);
    __syncthreads();
    for (int e = warp; e < mine; e += kRouteWarps) {
        const uint64_t key = s_key[e];
        int better = 0;
        for (int i = lane; i < a.n_experts; i += 32) better += s_all[i] > key || (s_all[i] == key && i < e0 + e);
        better = __reduce_add_sync(0xffffffffu, better);
        if (better < a.k && lane == 0) {
            peer_store(&s_top[better], 0, (uint64_t)__double_as_longlong(s_z[e]));
            peer_store(&s_who[better], 0, (uint64_t)(e0 + e));
        }
    }
    cluster_sync();
    if (rank || warp) return;
    // Weights of the winners, a lane each.  Renormalised ones are formed relative to the largest, so that scores below fp32 (sigmoids far below
    // 0, or experts that favour alone puts first) keep their ratios.
    auto exp_of = [](double z) {  // (what rounding the exponent to fp32 leaves is a factor)
        const float near = (float)z, rest = (float)(z - (double)near);
        return expf(near) * (1.f + (isfinite(near) ? rest : 0.f));
    };
    double v = lane < a.k ? s_top[lane] : -INFINITY;
    const float lead = warp_max((float)v);
    float p = 0.f;
    if (whole) {
        if (a.renorm && lead < 0x1p-100f) {
            double m = v;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) m = fmax(m, __shfl_xor_sync(0xffffffffu, m, o));
            v /= m;
        }
        p = (float)v;
    } else if (a.score == SSD_MOE_SIGMOID) {
        const float shift = a.renorm ? fminf(lead, 0.f) : 0.f;
        p = (v > 0.0 ? 1.f : exp_of(v - (double)shift)) / (1.f + exp_of(-fabs(v)));
    } else {
        p = v == s_top[0] ? 1.f : exp_of(v - s_top[0]);
    }
    if (lane >= a.k) p = 0.f;
    if (a.renorm) p /= warp_sum(p == p ? p : 0.f);
    if (lane < a.k) {
        a.ids[(int64_t)row * a.k + lane] = (int)s_who[lane];
        a.weights[(int64_t)row * a.k + lane] = p * a.scale;
    }
}

// ---------------------------------------------------------------------------
// ssd_moe_mlp
// ---------------------------------------------------------------------------
constexpr int kMoeWarps = 8;                         // that multiply; one more asks for weights
constexpr int kMoeSums = 32 * kMoeWarps;
constexpr int kChunk = 32;                           // k of a warp in a stage: 4 lanes have 16 bytes each of a row
constexpr int kStageK = kChunk * kMoeWarps;
constexpr double kWaitSeconds = 2.0, kClocksPerSecond = 2e9;

struct MoeArgs {
    const void *x, *residual;
    void* out;
    const int32_t* ids;
    const float* weights;
    int64_t x_stride, residual_stride, out_stride;
    void* h;   // [kPlanes][pair][f]: silu(gate x) * (up x) in values of the type
    float* y;  // [pair][part][d]: weights * down h over a part of f
    int n_rows, k, n_experts, d, f;
    int parts;  // of f, each summed by a unit of its own
    int up_depth, down_depth;  // stages of the rings
    int32_t* status;
    long long wait_clocks;
    int stall;  // test hook: the CTA of the first kernel that asks for nothing (-1: none)
};

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, bf16) {
    mma_bf16_16816(d, a0, a1, a2, a3, b0, b1);
}
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, f16) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 "
        "{%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// silu(..) * (..) goes to the second product as a sum of values of the type, each what the ones before leave of it: three of bf16, the 24 bits of
// fp32, or two of fp16, the second times 2^11, which are off by 2^-22 of it or by 2^-36 (without the factor by 2^-25: nothing is left of small ones).
template <typename T>
constexpr int kPlanes = 2;
template <>
constexpr int kPlanes<bf16> = 3;
template <typename T>
constexpr float kRestScale = 1.f;
template <>
constexpr float kRestScale<f16> = 0x1p11f;

__device__ __forceinline__ uint4 load_shared(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void tma3d(uint32_t to, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n" ::"r"(to), "l"(map), "r"(x), "r"(y),
                 "r"(z), "r"(smem_u32(bar))
                 : "memory");
}
// 16 bytes of a row; zeros and no access if not there
__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}
// arrives once this thread's copies so far have
__device__ __forceinline__ void arrive_copies(uint64_t* b) { asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];\n" ::"r"(smem_u32(b)) : "memory"); }
__device__ __forceinline__ void arrive(uint64_t* b) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(smem_u32(b)) : "memory"); }
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
__device__ __forceinline__ void sums_sync() { asm volatile("bar.sync 1, %0;\n" ::"n"(kMoeSums) : "memory"); }

// The rows' experts, as every CTA of both kernels works them out for itself from ids: the (row, slot) pairs sorted by
// expert, and groups of up to `size` pairs of one expert.
__host__ __device__ inline int max_groups(int n_pairs, int n_experts, int size) { return (n_experts < n_pairs ? n_experts : n_pairs) + n_pairs / size; }
struct Group {
    int expert, first, n;  // pairs pairs[first ..]
};
struct Plan {
    int n_groups;
    uint32_t* groups;  // expert << 21 | pairs << 15 | first
    uint16_t* pairs;
    __device__ __forceinline__ Group operator[](int i) const {
        const uint32_t g = groups[i];
        return {(int)(g >> 21), (int)(g & 0x7fffu), (int)(g >> 15 & 63u)};
    }
};
static_assert(kMaxExperts <= 1 << 11 && kMaxMoeRows * kMaxSlots < 1 << 15, "a group in 32 bits");

template <int kThreads>
__device__ __forceinline__ Plan make_plan(const MoeArgs& a, int size, unsigned char* smem, int* s_count, int* s_scan) {
    const int tid = threadIdx.x, lane = tid % 32, n = a.n_rows * a.k;
    constexpr int kEach = kMaxExperts / kMoeSums;
    Plan p;
    p.groups = reinterpret_cast<uint32_t*>(smem);
    p.pairs = reinterpret_cast<uint16_t*>(p.groups + max_groups(n, a.n_experts, size));
    uint16_t* of_pair = p.pairs + n;  // experts, kMaxExperts: none
    for (int e = tid; e < kMaxExperts; e += kThreads) s_count[e] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) {
        const int e = __ldcg(a.ids + i);
        const bool ok = e >= 0 && e < a.n_experts;
        of_pair[i] = (uint16_t)(ok ? e : kMaxExperts);
        if (ok) atomicAdd(s_count + e, 1);
    }
    __syncthreads();
    // groups and pairs of the experts before (groups in the upper half): 4 experts a thread, summed over the warps
    int mine[kEach], sum = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        mine[i] = tid < kMoeSums ? s_count[tid * kEach + i] : 0;
        sum += (mine[i] + size - 1) / size << 16 | mine[i];
    }
    int upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
    }
    if (lane == 31 && tid < kMoeSums) s_scan[tid / 32] = upto;
    __syncthreads();
    int at = upto - sum;
    p.n_groups = 0;
    for (int w = 0; w < kMoeWarps; ++w) {
        if (w < tid / 32) at += s_scan[w];
        p.n_groups += s_scan[w] >> 16;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int e = tid * kEach + i;
        if (tid < kMoeSums) s_count[e] = at & 0xffff;  // (where its next pair goes)
        for (int done = 0; done < mine[i]; done += size, at += 1 << 16)
            p.groups[at >> 16] = (uint32_t)e << 21 | (uint32_t)min(size, mine[i] - done) << 15 | (uint32_t)((at & 0xffff) + done);
        at += mine[i];
    }
    __syncthreads();
    // one warp sorts, so that every CTA has the same order
    if (tid < 32) {
        for (int i = 0; i < n; i += 32) {
            const int e = i + lane < n ? of_pair[i + lane] : kMaxExperts;
            const bool ok = e < kMaxExperts;
            const unsigned same = __match_any_sync(0xffffffffu, e);
            const int before = __popc(same & ((1u << lane) - 1u));
            const int to = ok ? s_count[e] + before : 0;
            __syncwarp();
            if (ok) p.pairs[to] = (uint16_t)(i + lane);
            if (ok && before == 0) s_count[e] = to + __popc(same);
            __syncwarp();
        }
    }
    __syncthreads();
    return p;
}

// Both products: units (group, tile of output rows, part of k), a CTA each, in turns over the grid.  A stage is 256 k of a unit's
// 32 or 64 weight rows (TMA boxes of 64 k, 128-byte swizzle, zeros past the ends of rows and matrices), in a ring that goes on over
// the units: while the 8 warps of a CTA join their sums, the next unit's weights are on their way.  A warp multiplies its 32 k of
// a stage.  Columns (PL planes each): up to 8 come from L2 straight to a warp's registers, a stage ahead, over the units' ends
// too; more of them (64 weight rows then, so that they are read half as often) are copied into the ring by three warps, since a
// stage ahead is too late (64 rows, 8 an expert, h in two planes: 1215 us, copied 990).  The k that
// a lane holds go to the matrix instruction in an order of their own, the same for both operands, so that every operand is 16 bytes
// in a row; lane group g has row (g / 2) + 4 (g mod 2) of 8, so that the 8 lanes that shared memory serves at once meet
// different banks.  The matrix instructions cut off what is below their sum, so a stage's products are summed from 0, the smallest plane first, and added to the
// sums before them with a rounding.  (With two planes of bf16 and one sum for all stages 26 of 24576 results of a layer of 4096 x 11008, two experts of 8, were
// neighbours of the nearest value, now 4 are, and 4 of fp32 products; its one row took 102.9 us instead of 106.5, 64 rows of 5120 x 13824 1010
// instead of 1065, with rings of their own for weights and columns, four and three stages, 1074; the third plane loaded and not
// multiplied 103.4 and 1037.)  Bound by HBM: two CTAs have 160 KB of weights under way on an SM.
//
// kUp: h = silu(gate x) * (up x); a tile of 16 weight rows is 8 of gate and the same 8 of up, so that both sums of an output are in
// one lane.  Else y = weights * (down h), h in kPlanes planes.
template <typename T, int NT, bool kUp>
struct Products {
    static constexpr int kTiles = NT == 1 ? 2 : 4, kWeightRows = 16 * kTiles;
    static constexpr int kBox = kWeightRows * 128, kStage = kStageK / 64 * kBox;  // 64 k of them; 16 or 32 KB
    static constexpr int PL = kUp ? 1 : kPlanes<T>, kRows = kWeightRows / (kUp ? 2 : 1);   // output rows of a unit
    static constexpr int kColumns = 8 * NT, kCtas = NT == 1 ? 2 : 1;              // of an SM
    static constexpr bool kCopied = NT > 1;                                       // columns
    static constexpr int kLoaders = kCopied ? 3 : 0, kThreads = kMoeSums + 32 + 32 * kLoaders;
    static constexpr int kSums = kMoeWarps * kTiles * 32, kSumBuffers = NT == 1 ? 2 : 1;  // of the warps' sums
    static constexpr int kColumnBox = kColumns * 128, kSlot = kStage + (kCopied ? PL * kStageK / 64 * kColumnBox : 0);
    static constexpr int kDepth = kCopied ? 200 * 1024 / kSlot : 5;               // at most

    static __device__ __forceinline__ void run(const MoeArgs& a, const CUtensorMap* map0, const CUtensorMap* map1, const Plan& p, uint32_t ring, float4* s_red, uint64_t* full,
                                               uint64_t* empty, volatile int* s_fail) {
        const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, parts = kUp ? 1 : a.parts;
        const int K = kUp ? a.d : a.f, rows = kUp ? a.f : a.d, tiles = (rows + kRows - 1) / kRows;
        const int units = p.n_groups * tiles * parts, stages = (K + kStageK - 1) / kStageK;
        const int64_t plane = (int64_t)a.n_rows * a.k * a.f;
        const int depth = kUp ? a.up_depth : a.down_depth;
        bool ok = true;
        auto begin_of = [&](int u) { return u % parts * stages / parts; };
        auto end_of = [&](int u) { return (u % parts + 1) * stages / parts; };
        if (warp == kMoeWarps) {
            int n = 0;  // stages asked for
            for (int u = kUp && a.stall == (int)blockIdx.x ? units : (int)blockIdx.x; u < units && ok; u += gridDim.x) {
                const int rest = u / parts, row = rest % tiles * kRows, expert = p[rest / tiles].expert;
                const int end = end_of(u);
                for (int stage = begin_of(u); stage < end; ++stage, ++n) {
                    const int slot = n % depth;
                    if (n >= depth) ok = __all_sync(0xffffffffu, mb_wait(empty + slot, (unsigned)(n / depth - 1) & 1u, s_fail, a.wait_clocks));
                    if (!ok) break;
                    if (elect_one()) {
                        tc::mb_arrive_tx(full + slot, kStage);
                        const uint32_t to = ring + slot * kSlot;
#pragma unroll
                        for (int i = 0; i < kStageK / 64; ++i) {
                            tma3d(to + i * kBox, map0, stage * kStageK + 64 * i, row, expert, full + slot);
                            if (kUp) tma3d(to + i * kBox + kBox / 2, map1, stage * kStageK + 64 * i, row, expert, full + slot);
                        }
                    }
                    __syncwarp();
                }
            }
            if (!ok || *s_fail) {  // copies in flight end before the CTA does
                const long long t0 = clock64();
                for (int i = max(0, n - depth); i < n; ++i)
                    while (!tc::mb_try(full + i % depth, (unsigned)(i / depth) & 1u) && clock64() - t0 < 4000000ll) {
                    }
            }
            return;
        }
        if (kCopied && warp > kMoeWarps) {
            // copies columns, a row (512 bytes) at a time: lane l its 16 bytes number l, swizzled as the weights' boxes are
            if (!kUp) pdl_wait();
            const int loader = warp - kMoeWarps - 1;
            const uint32_t to = ring + kStage + lane / 8 * kColumnBox;
            int n = 0, group = -1, rows_here = 0;
            unsigned long long row = 0;  // where the group's row number `lane` is
            for (int u = blockIdx.x; u < units && ok; u += gridDim.x) {
                const int end = end_of(u);
                if (u / parts / tiles != group) {
                    group = u / parts / tiles;
                    const Group q = p[group];
                    rows_here = q.n;
                    if (lane < q.n) {
                        const int pair = p.pairs[q.first + lane];
                        row = (unsigned long long)(kUp ? (const T*)a.x + (int64_t)(pair / a.k) * a.x_stride : (const T*)a.h + (int64_t)pair * a.f);
                    }
                }
                for (int stage = begin_of(u); stage < end; ++stage, ++n) {
                    const int slot = n % depth, k = stage * kStageK + lane * 8;
                    if (n >= depth) ok = __all_sync(0xffffffffu, mb_wait(empty + slot, (unsigned)(n / depth - 1) & 1u, s_fail, a.wait_clocks));
                    if (!ok) break;
                    const bool there = k < K;
                    const uint32_t into = to + slot * kSlot;
                    for (int i = loader; i < rows_here; i += kLoaders) {
                        const T* x = (const T*)__shfl_sync(0xffffffffu, row, i) + (there ? k : 0);
#pragma unroll
                        for (int l = 0; l < PL; ++l) copy16(into + l * (kStageK / 64 * kColumnBox) + i * 128 + ((uint32_t)(lane ^ i) % 8) * 16, x + l * plane, there);
                    }
                    arrive_copies(full + slot);
                }
            }
            asm volatile("cp.async.wait_all;\n" ::: "memory");
            return;
        }
        if (!kUp) pdl_wait();
        const int g = lane / 4, piece = lane % 4 * 8, row_g = g / 2 + g % 2 * 4;
        // the columns of the stage that comes next: its unit, number and k, and where this lane's are
        int xu = blockIdx.x, xs = 0, x_end = 0;
        const T* xp[NT];
        auto aim = [&]() {
            if (kCopied || xu >= units) return;
            const Group q = p[xu / parts / tiles];
            xs = begin_of(xu), x_end = end_of(xu);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int pair = p.pairs[q.first + min(8 * t + g, q.n - 1)];
                xp[t] = (kUp ? (const T*)a.x + (int64_t)(pair / a.k) * a.x_stride : (const T*)a.h + (int64_t)pair * a.f) + xs * kStageK + warp * kChunk + piece;
            }
        };
        auto load_columns = [&](uint4 (&x)[PL][NT]) {
            if (kCopied || xu >= units) return;
            if (xs * kStageK + kStageK <= K) {
#pragma unroll
                for (int l = 0; l < PL; ++l)
#pragma unroll
                    for (int t = 0; t < NT; ++t) x[l][t] = __ldcg(reinterpret_cast<const uint4*>(xp[t] + l * plane));
            } else {  // (zeros past the end, as in the weights' boxes)
                const bool there = xs * kStageK + warp * kChunk + piece < K;
#pragma unroll
                for (int l = 0; l < PL; ++l)
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        x[l][t] = make_uint4(0u, 0u, 0u, 0u);
                        if (there) x[l][t] = __ldcg(reinterpret_cast<const uint4*>(xp[t] + l * plane));
                    }
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) xp[t] += kStageK;
            if (++xs == x_end) {
                xu += gridDim.x;
                aim();
            }
        };
        // where this lane's 16 bytes of a row are in a box (swizzled), and its box in the stage
        const uint32_t mine = ring + warp / 2 * kBox + row_g * 128 + ((uint32_t)(warp % 2 * 4 + lane % 4) ^ (uint32_t)row_g) * 16;
        const uint32_t columns = ring + kStage + warp / 2 * kColumnBox + (mine - ring - warp / 2 * kBox);
        int u = blockIdx.x, stage = begin_of(u), end = end_of(u), slot = 0;
        unsigned phase = 0;
        int buffer = 0, turn = 0;
        float acc[NT][kTiles][4] = {};
        // one stage: columns x, and those of the next one asked for; false after the last
        auto one = [&](uint4 (&x)[PL][NT], uint4 (&next)[PL][NT]) {
            load_columns(next);
            ok = ok && __all_sync(0xffffffffu, mb_wait(full + slot, phase, s_fail, a.wait_clocks));
            if (ok) {
                uint4 w[kTiles][2];
#pragma unroll
                for (int m = 0; m < kTiles; ++m)
#pragma unroll
                    for (int r = 0; r < 2; ++r) w[m][r] = load_shared(mine + slot * kSlot + (kUp ? r * (kBox / 2) + m * 1024 : (2 * m + r) * 1024));
                if (kCopied) {
#pragma unroll
                    for (int l = 0; l < PL; ++l)
#pragma unroll
                        for (int t = 0; t < NT; ++t) x[l][t] = load_shared(columns + slot * kSlot + l * (kStageK / 64 * kColumnBox) + t * 1024);
                }
                auto multiply = [&](float (&sum)[kTiles][4], const uint4& v) {
#pragma unroll
                    for (int m = 0; m < kTiles; ++m) mma(sum[m], w[m][0].x, w[m][1].x, w[m][0].y, w[m][1].y, v.x, v.y, T());
#pragma unroll
                    for (int m = 0; m < kTiles; ++m) mma(sum[m], w[m][0].z, w[m][1].z, w[m][0].w, w[m][1].w, v.z, v.w, T());
                };
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    float sum[kTiles][4] = {};
#pragma unroll
                    for (int l = PL - 1; l >= 0; --l) {
                        if (l + 1 < PL && kRestScale<T> != 1.f) {
#pragma unroll
                            for (int m = 0; m < kTiles; ++m)
#pragma unroll
                                for (int i = 0; i < 4; ++i) sum[m][i] *= 1.f / kRestScale<T>;
                        }
                        multiply(sum, x[l][t]);
                    }
#pragma unroll
                    for (int m = 0; m < kTiles; ++m)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[t][m][i] += sum[m][i];
                }
            }
            __syncwarp();
            if (lane == 0) arrive(empty + slot);
            if (++slot == depth) slot = 0, phase ^= 1u;
            if (++stage < end) return true;
            // the warps' sums, in order: [warp][tile][lane], one tile of columns after the other.  With one tile the buffers take turns,
            // so that the warps that do not add go on (what they write next is read by then: there is a barrier in between).
            const int part = u % parts, rest = u / parts, row0 = rest % tiles * kRows;
            const Group q = p[rest / tiles];
            const float lost = ok ? 0.f : __int_as_float(0x7fffffff);  // (what misses something is NaN, so that it is seen without `status`, too)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float4* red = s_red + buffer * kSums;
#pragma unroll
                for (int m = 0; m < kTiles; ++m) red[(warp * kTiles + m) * 32 + lane] = make_float4(acc[t][m][0] + lost, acc[t][m][1] + lost, acc[t][m][2] + lost, acc[t][m][3] + lost);
                sums_sync();
                const int m = (warp + turn) % kMoeWarps;  // (tiles go to other warps from unit to unit)
                if (m < kTiles) {
                    float4 v = red[m * 32 + lane];
#pragma unroll
                    for (int j = 1; j < kMoeWarps; ++j) {
                        const float4 o = red[(j * kTiles + m) * 32 + lane];
                        v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
                    }
                    finish(a, p, q, row0 + m * (kUp ? 8 : 16) + row_g, rows, t * 8 + (kCopied ? lane % 4 : lane % 4 * 2), part, plane, v);
                }
                if (kSumBuffers == 1) sums_sync();
                else buffer ^= 1;
                turn += kTiles;
#pragma unroll
                for (int i = 0; i < kTiles; ++i) acc[t][i][0] = acc[t][i][1] = acc[t][i][2] = acc[t][i][3] = 0.f;
            }
            u += gridDim.x;
            if (u >= units) return false;
            stage = begin_of(u), end = end_of(u);
            return true;
        };
        uint4 x0[PL][NT], x1[PL][NT];
        if (u < units) {
            aim();
            load_columns(x0);
            if (kCopied) {
                while (one(x0, x0)) {
                }
            } else {
                while (one(x0, x1) && one(x1, x0)) {
                }
            }
        }
        if (!ok && lane == 0) say(a.status, SSD_STATUS_TIMEOUT);
    }

    // sums of output rows `row` (up: of gate and up) and `row` + 8 (down), columns col and col + 1 (of copied columns: col + 4, in the order of row_g)
    static __device__ __forceinline__ void finish(const MoeArgs& a, const Plan& p, const Group& q, int row, int rows, int col, int part, int64_t plane, const float4& v) {
        constexpr int kNext = kCopied ? 4 : 1;
        if (kUp) {
            const float h[2] = {v.x / (1.f + expf(-v.x)) * v.z, v.y / (1.f + expf(-v.y)) * v.w};
#pragma unroll
            for (int j = 0; j < 2; ++j)
                if (row < rows && col + j * kNext < q.n) {
                    T* to = (T*)a.h + (int64_t)p.pairs[q.first + col + j * kNext] * a.f + row;
                    float left = h[j];
#pragma unroll
                    for (int l = 0; l < kPlanes<T>; ++l) {
                        const T v = (T)left;
                        to[l * plane] = v;
                        left = isfinite((float)v) ? (left - (float)v) * kRestScale<T> : 0.f;
                    }
                }
        } else {
            const float y[2][2] = {{v.x, v.y}, {v.z, v.w}};
#pragma unroll
            for (int j = 0; j < 2; ++j)
                if (col + j * kNext < q.n) {
                    const int pair = p.pairs[q.first + col + j * kNext];
                    const float w = __ldcg(a.weights + pair);
                    float* to = a.y + ((int64_t)pair * a.parts + part) * a.d + row;
                    if (row < rows) to[0] = w * y[0][j];
                    if (row + 8 < rows) to[8] = w * y[1][j];
                }
        }
    }
};

// the ring's barriers, and the plan behind the ring
template <typename P>
__device__ __forceinline__ void set_barriers(uint64_t* full, uint64_t* empty, int* s_fail) {
    if (threadIdx.x == 0) {
        for (int i = 0; i < P::kDepth; ++i) {
            tc::mb_init(full + i, 1 + 32 * P::kLoaders);
            tc::mb_init(empty + i, kMoeWarps);
        }
        *s_fail = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
}

template <typename T, int NT>
__global__ void __launch_bounds__(Products<T, NT, true>::kThreads, Products<T, NT, true>::kCtas)
    moe_up_kernel(const __grid_constant__ MoeArgs a, const __grid_constant__ CUtensorMap gate, const __grid_constant__ CUtensorMap up) {
    using P = Products<T, NT, true>;
    extern __shared__ unsigned char s_dyn[];
    __shared__ float4 s_red[P::kSumBuffers * P::kSums];
    __shared__ uint64_t full[P::kDepth], empty[P::kDepth];
    __shared__ int s_scan[kMoeWarps], s_fail;
    static_assert(sizeof(s_red) >= kMaxExperts * sizeof(int), "a count for each expert");
    const uint32_t pad = (1024u - smem_u32(s_dyn) % 1024u) % 1024u;
    set_barriers<P>(full, empty, &s_fail);
    pdl_wait();
    pdl_launch_dependents();  // (only here: the next kernel reads ids before it waits)
    const Plan p = make_plan<P::kThreads>(a, P::kColumns, s_dyn + pad + a.up_depth * P::kSlot, reinterpret_cast<int*>(s_red), s_scan);
    P::run(a, &gate, &up, p, smem_u32(s_dyn) + pad, s_red, full, empty, &s_fail);
}

template <typename T, int NT>
__global__ void __launch_bounds__(Products<T, NT, false>::kThreads, Products<T, NT, false>::kCtas) moe_down_kernel(const __grid_constant__ MoeArgs a, const __grid_constant__ CUtensorMap down) {
    using P = Products<T, NT, false>;
    extern __shared__ unsigned char s_dyn[];
    __shared__ float4 s_red[P::kSumBuffers * P::kSums];
    __shared__ uint64_t full[P::kDepth], empty[P::kDepth];
    __shared__ int s_scan[kMoeWarps], s_fail;
    const uint32_t pad = (1024u - smem_u32(s_dyn) % 1024u) % 1024u;
    set_barriers<P>(full, empty, &s_fail);
    pdl_launch_dependents();
    // ids were complete before the kernel before this one let it start; weights need not wait for h, and the warps that multiply do
    const Plan p = make_plan<P::kThreads>(a, P::kColumns, s_dyn + pad + a.down_depth * P::kSlot, reinterpret_cast<int*>(s_red), s_scan);
    P::run(a, &down, nullptr, p, smem_u32(s_dyn) + pad, s_red, full, empty, &s_fail);
}

// out = residual + the rows' slots and their parts, in order
constexpr int kSumThreads = 128, kSumAhead = 8;
template <typename T>
__global__ void __launch_bounds__(kSumThreads) moe_sum_kernel(const __grid_constant__ MoeArgs a) {
    pdl_launch_dependents();
    pdl_wait();
    __shared__ bool s_has[kMaxSlots];
    const int row = blockIdx.y, dim = (blockIdx.x * kSumThreads + threadIdx.x) * 4;
    if (threadIdx.x < a.k) {
        const int e = __ldcg(a.ids + (int64_t)row * a.k + threadIdx.x);
        s_has[threadIdx.x] = e >= 0 && e < a.n_experts;
    }
    __syncthreads();
    if (dim >= a.d) return;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    const int n = a.k * a.parts;
    const float* y = a.y + (int64_t)row * n * a.d + dim;
    for (int i = 0; i < n; i += kSumAhead) {
        float4 v[kSumAhead];
#pragma unroll
        for (int j = 0; j < kSumAhead; ++j) {
            v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (i + j < n && s_has[(i + j) / a.parts]) v[j] = __ldcg(reinterpret_cast<const float4*>(y + (int64_t)(i + j) * a.d));
        }
#pragma unroll
        for (int j = 0; j < kSumAhead; ++j) s.x += v[j].x, s.y += v[j].y, s.z += v[j].z, s.w += v[j].w;
    }
    uint2 r = make_uint2(0u, 0u);
    if (a.residual) r = __ldcg(reinterpret_cast<const uint2*>((const T*)a.residual + (int64_t)row * a.residual_stride + dim));
    const float2 r0 = unpack2(r.x, T()), r1 = unpack2(r.y, T());
    *reinterpret_cast<uint2*>((T*)a.out + (int64_t)row * a.out_stride + dim) = make_uint2(pack2(r0.x + s.x, r0.y + s.y, T()), pack2(r1.x + s.z, r1.y + s.w, T()));
}

std::mutex g_mu;  // guards what follows, and what is set up
// ssd_debug_moe_stall, for one call
int g_stall = -1;
double g_stall_wait_s = 0.0;

size_t plan_bytes(int n_pairs, int n_experts, int size) { return 4 * ((size_t)max_groups(n_pairs, n_experts, size) + (size_t)n_pairs); }

// parts of f: until there are units of down for two waves of CTAs and more (as many experts met as can be), four stages each at least
constexpr int kMaxParts = 8, kDownUnits = 2000;
int parts_of(const ssd_moe& m, int64_t pairs) {
    const int64_t tiles = (m.d + 31) / 32, met = std::min<int64_t>(m.n_experts, pairs);
    int parts = 1;
    while (parts < kMaxParts && met * tiles * parts < kDownUnits && m.f >= 8 * kStageK * parts) parts *= 2;
    return parts;
}
// The most that pairs * parts comes to for up to this many pairs.  (More pairs have fewer parts, so that few of them can need
// more than many do; a workspace for the largest round is enough for all.)
int64_t most_sums(const ssd_moe& m, int64_t pairs) {
    const int64_t tiles = (m.d + 31) / 32;
    int64_t most = pairs;
    for (int parts = 2; parts <= kMaxParts && m.f >= 8 * kStageK * (parts / 2); parts *= 2) {
        const int64_t met = (kDownUnits - 1) / (tiles * (parts / 2));  // as many experts at most have so many parts
        most = std::max(most, parts * (m.n_experts <= met ? pairs : std::min(pairs, met)));
    }
    return most;
}

struct Workspace {
    size_t y, total;  // offset behind h, bytes
};
Workspace workspace_of(const ssd_moe& m, int n_rows, int k) {
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    const size_t pairs = (size_t)n_rows * k;
    Workspace w;
    w.y = up(2 * (size_t)(m.dtype == SSD_BF16 ? kPlanes<bf16> : kPlanes<f16>) * pairs * m.f);
    w.total = w.y + up(4 * (size_t)most_sums(m, (int64_t)pairs) * m.d);
    return w;
}

int check_experts(const char* call, const ssd_moe* m, int n_rows, int k) {
    if (!m) return refuse_arg(call, "NULL experts");
    if (m->dtype != SSD_F16 && m->dtype != SSD_BF16) return refuse_arg(call, "the experts must be fp16 or bf16");
    if (m->n_experts < 1 || m->n_experts > kMaxExperts || m->d < 8 || m->d > 65536 || m->d % 8 || m->f < 8 || m->f > 65536 || m->f % 8)
        return refuse_arg(call, "need 1 <= n_experts <= 1024, d and f multiples of 8, 8 .. 65536");
    if (n_rows < 0 || n_rows > kMaxMoeRows || k < 1 || k > kMaxSlots) return refuse_arg(call, "need 0 <= n_rows <= 1024 and 1 <= k <= 16");
    return SSD_OK;
}

PFN_cuTensorMapEncodeTiled_v12000 g_encode = nullptr;
// dynamic shared memory of a CTA, and of one of two on an SM (of 228 KB each has 17 KB static and 1 KB for the system.  With
// more of it for the pairs of 512 rows, 8 of 1024 experts, one CTA an SM had to end before the next began)
constexpr int kMostShared = 209 * 1024, kMostOfTwo = 96 * 1024;

// the experts' matrices [expert][rows][width] as {width, rows, experts}, box 64 x box_rows
int encode(const char* call, CUtensorMap* m, const void* base, int dtype, int width, int rows, int n_experts, int64_t stride, int box_rows) {
    const cuuint64_t dims[3] = {(cuuint64_t)width, (cuuint64_t)rows, (cuuint64_t)n_experts};
    const cuuint64_t strides[2] = {(cuuint64_t)width * 2, (cuuint64_t)(n_experts > 1 ? stride : (int64_t)width * rows) * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1}, step[3] = {1, 1, 1};
    const CUresult r = g_encode(m, dtype == SSD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(base), dims, strides, box,
                                step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? SSD_OK : refuse(SSD_ERR_CUDA, call, "cuTensorMapEncodeTiled failed (%d)", (int)r);
}

// all kernels of the call, so that a first use with one row prepares captures with any
template <typename T, int NT>
cudaError_t set_up_moe() {
    const cudaError_t e = cudaFuncSetAttribute(moe_up_kernel<T, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared);
    return e == cudaSuccess ? cudaFuncSetAttribute(moe_down_kernel<T, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared) : e;
}
template <typename T>
cudaError_t set_up_moe() {
    cudaError_t e = set_up_moe<T, 1>();
    if (e == cudaSuccess) e = set_up_moe<T, 2>();
    if (e == cudaSuccess) e = set_up_moe<T, 4>();
    return e == cudaSuccess ? loaded({(const void*)moe_sum_kernel<T>}) : e;
}
int set_up_moe(const char* call) {
    static bool ready[kMaxDevices] = {};
    int dev = 0;
    if (int rc = device_of(call, &dev)) return rc;
    std::lock_guard<std::mutex> lock(g_mu);
    if (ready[dev]) return SSD_OK;
    cudaError_t e = set_up_moe<f16>();
    if (e == cudaSuccess) e = set_up_moe<bf16>();
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    if (e == cudaSuccess) e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found);
    if (e != cudaSuccess) return refuse(SSD_ERR_CUDA, call, "set-up: %s", cudaGetErrorString(e));
    if (!fn || found != cudaDriverEntryPointSuccess) return refuse(SSD_ERR_CUDA, call, "cuTensorMapEncodeTiled unavailable");
    g_encode = (PFN_cuTensorMapEncodeTiled_v12000)fn;
    ready[dev] = true;
    return SSD_OK;
}

template <typename T, int NT>
int launch_moe(const char* call, MoeArgs& a, const ssd_moe& m, int sms, void* stream) {
    using U = Products<T, NT, true>;
    using D = Products<T, NT, false>;
    CUtensorMap gate, up, down;
    if (int rc = encode(call, &gate, m.gate, m.dtype, m.d, m.f, m.n_experts, m.gate_stride, U::kWeightRows / 2)) return rc;
    if (int rc = encode(call, &up, m.up, m.dtype, m.d, m.f, m.n_experts, m.up_stride, U::kWeightRows / 2)) return rc;
    if (int rc = encode(call, &down, m.down, m.dtype, m.f, m.d, m.n_experts, m.down_stride, D::kWeightRows)) return rc;
    const int more = 1024 + (int)plan_bytes(a.n_rows * a.k, a.n_experts, 8 * NT);
    constexpr int kRoom = U::kCtas == 2 ? kMostOfTwo : kMostShared;
    a.up_depth = std::min((int)U::kDepth, (kRoom - more) / U::kSlot);
    a.down_depth = std::min((int)D::kDepth, (kRoom - more) / D::kSlot);
    const dim3 grid((unsigned)(U::kCtas * sms));
    if (int rc = launch(call, moe_up_kernel<T, NT>, grid, U::kThreads, (size_t)(a.up_depth * U::kSlot + more), stream, a, gate, up)) return rc;
    if (int rc = launch(call, moe_down_kernel<T, NT>, grid, D::kThreads, (size_t)(a.down_depth * D::kSlot + more), stream, a, down)) return rc;
    return launch(call, moe_sum_kernel<T>, dim3((unsigned)((a.d + 4 * kSumThreads - 1) / (4 * kSumThreads)), (unsigned)a.n_rows), kSumThreads, 0, stream, a);
}

template <typename T>
int start_moe(const char* call, MoeArgs& a, const ssd_moe& m, void* stream) {
    if (int rc = set_up_moe(call)) return rc;
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return refuse(SSD_ERR_CUDA, call, "%s", cudaGetErrorString(e));
    a.parts = parts_of(m, (int64_t)a.n_rows * a.k);
    // rows of an expert that its weights are read for at once: as many as it has on average, or all of a few
    const int64_t pairs = (int64_t)a.n_rows * a.k;
    if (a.n_rows <= 8 || pairs <= 4 * (int64_t)a.n_experts) return launch_moe<T, 1>(call, a, m, sms, stream);
    if (a.n_rows <= 16 || pairs <= 12 * (int64_t)a.n_experts) return launch_moe<T, 2>(call, a, m, sms, stream);
    return launch_moe<T, 4>(call, a, m, sms, stream);
}

}  // namespace step
}  // namespace ssd

using namespace ssd;
using namespace ssd::step;

extern "C" void ssd_debug_moe_stall(int cta, double wait_limit_s) {
    std::lock_guard<std::mutex> lock(g_mu);
    g_stall = cta >= 0 && wait_limit_s > 0.0 && wait_limit_s <= 10.0 ? cta : -1;
    g_stall_wait_s = wait_limit_s;
}

extern "C" int ssd_moe_route(int dtype, int n_rows, int d, int n_experts, int k, const void* x, int64_t x_stride, const void* w_router,
                             const float* favour, int score, int renorm, float scale, int32_t* ids, float* weights, void* cuda_stream) {
    static const char call[] = "ssd_moe_route";
    if (dtype != SSD_F16 && dtype != SSD_BF16) return refuse_arg(call, "rows and router must be fp16 or bf16");
    if (n_rows < 0 || n_rows > 65535 || d < 8 || d > 65536 || d % 8) return refuse_arg(call, "need 0 <= n_rows <= 65535, d a multiple of 8, 8 .. 65536");
    if (n_experts < 1 || n_experts > kMaxExperts || k < 1 || k > kMaxSlots || k > n_experts)
        return refuse_arg(call, "need 1 <= k <= 16 and k <= n_experts <= 1024");
    if ((score != SSD_MOE_SOFTMAX && score != SSD_MOE_SIGMOID) || (renorm != 0 && renorm != 1)) return refuse_arg(call, "unknown score, or renorm not 0 or 1");
    if (!std::isfinite(scale)) return refuse_arg(call, "scale must be finite");
    if (n_rows == 0) return SSD_OK;
    if (!x || !w_router || !ids || !weights) return refuse_arg(call, "NULL pointer");
    if (int rc = check_rows(call, "x", x, x_stride, dtype, d)) return rc;
    if ((uintptr_t)w_router & 15u) return refuse_arg(call, "w_router must be 16-byte aligned");
    if (!aligned(4, {favour, ids, weights})) return refuse_arg(call, "favour, ids and weights must be aligned to their type");
    const size_t picked = 4 * (size_t)n_rows * k;
    const Range i1[1] = {{ids, picked}}, w1[1] = {{weights, picked}};
    const Range in[3] = {{x, span(n_rows, x_stride, d, dtype)}, {w_router, 2 * (size_t)n_experts * d}, {favour, 4 * (size_t)n_experts}};
    if (meet(i1, w1) || meet(i1, in) || meet(w1, in)) return refuse_arg(call, "ids and weights must overlap neither each other nor an input");
    if (int rc = check_device(call, x)) return rc;
    if (int rc = set_up_once<route_kernel<f16>, route_kernel<bf16>>(call)) return rc;
    RouteArgs a{};
    a.x = x;
    a.w = w_router;
    a.favour = favour;
    a.ids = ids;
    a.weights = weights;
    a.x_stride = x_stride;
    a.d = d;
    a.n_experts = n_experts;
    a.k = k;
    a.score = score;
    a.renorm = renorm;
    a.scale = scale;
    cudaLaunchConfig_t cfg = {};
    // as many CTAs a row as are there at once, two an SM
    unsigned split = kRouteSplit;
    while (split > 2 && (long long)n_rows * split > 304) split /= 2;
    cfg.gridDim = dim3(split, (unsigned)n_rows, 1);
    cfg.blockDim = dim3(kRouteThreads, 1, 1);
    cfg.stream = (cudaStream_t)cuda_stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = split, attr[1].val.clusterDim.y = 1, attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const cudaError_t e = dtype == SSD_F16 ? cudaLaunchKernelEx(&cfg, route_kernel<f16>, a) : cudaLaunchKernelEx(&cfg, route_kernel<bf16>, a);
    return e == cudaSuccess ? SSD_OK : refuse(SSD_ERR_CUDA, call, "%s", cudaGetErrorString(e));
}

extern "C" int ssd_moe_workspace(const ssd_moe* experts, int n_rows, int k, size_t* bytes) {
    static const char call[] = "ssd_moe_workspace";
    if (!bytes) return refuse_arg(call, "NULL pointer");
    if (int rc = check_experts(call, experts, n_rows, k)) return rc;
    *bytes = workspace_of(*experts, n_rows, k).total;
    return SSD_OK;
}

extern "C" int ssd_moe_mlp(const ssd_moe* experts, int n_rows, int k, const void* x, int64_t x_stride, const int32_t* ids,
                           const float* weights, const void* residual, int64_t residual_stride, void* out, int64_t out_stride,
                           void* workspace, size_t workspace_bytes, int32_t* status, void* cuda_stream) {
    static const char call[] = "ssd_moe_mlp";
    if (int rc = check_experts(call, experts, n_rows, k)) return rc;
    const ssd_moe& m = *experts;
    if (!m.gate || !m.up || !m.down || ((uintptr_t)m.gate | (uintptr_t)m.up | (uintptr_t)m.down) & 15u)
        return refuse_arg(call, "gate, up and down must be 16-byte aligned and not NULL");
    const int64_t size = (int64_t)m.d * m.f, strides[3] = {m.gate_stride, m.up_stride, m.down_stride};
    for (int64_t s : strides)
        if (m.n_experts > 1 && (s < size || s % 8 || s > (int64_t(1) << 37))) return refuse_arg(call, "experts must be multiples of 8 elements apart and not overlap");
    if (n_rows == 0) return SSD_OK;
    if (!x || !ids || !weights || !out || !workspace) return refuse_arg(call, "NULL pointer");
    if (int rc = check_rows(call, "x", x, x_stride, m.dtype, m.d)) return rc;
    if (int rc = check_rows(call, "out", out, out_stride, m.dtype, m.d)) return rc;
    if (residual)
        if (int rc = check_rows(call, "residual", residual, residual_stride, m.dtype, m.d)) return rc;
    if (!aligned(4, {ids, weights, status})) return refuse_arg(call, "ids, weights and status must be aligned to their type");
    if (residual == out && residual_stride != out_stride) return refuse_arg(call, "out in the residual's place needs its stride");
    const Workspace w = workspace_of(m, n_rows, k);
    const size_t picked = 4 * (size_t)n_rows * k, rows = span(n_rows, out_stride, m.d, m.dtype);
    const Range o[1] = {{out, rows}}, ws[1] = {{workspace, w.total}}, st[1] = {{status, 4}};
    auto matrices = [&](int64_t stride) { return 2 * ((size_t)(m.n_experts - 1) * (size_t)(m.n_experts > 1 ? stride : 0) + (size_t)size); };
    const Range in[6] = {{x, span(n_rows, x_stride, m.d, m.dtype)}, {ids, picked}, {weights, picked}, {m.gate, matrices(m.gate_stride)}, {m.up, matrices(m.up_stride)}, {m.down, matrices(m.down_stride)}}, re[1] = {{residual, residual ? span(n_rows, residual_stride, m.d, m.dtype) : 0}};
    if (meet(o, in) || (out != residual && meet(o, re))) return refuse_arg(call, "out must be the residual with its stride or overlap no input");
    if (meet(ws, o) || meet(ws, in) || meet(ws, re) || meet(st, o) || meet(st, ws) || meet(st, in) || meet(st, re))
        return refuse_arg(call, "workspace and status must not overlap other tensors");
    if ((uintptr_t)workspace & 15u) return refuse_arg(call, "the workspace must be 16-byte aligned");
    if (workspace_bytes < w.total) return refuse(SSD_ERR_CAPACITY, call, "the workspace needs %zu bytes", w.total);
    if (int rc = check_device(call, x)) return rc;
    MoeArgs a{};
    a.x = x;
    a.x_stride = x_stride;
    a.residual = residual;
    a.residual_stride = residual_stride;
    a.out = out;
    a.out_stride = out_stride;
    a.ids = ids;
    a.weights = weights;
    a.h = workspace;
    a.y = (float*)((char*)workspace + w.y);
    a.n_rows = n_rows;
    a.k = k;
    a.n_experts = m.n_experts;
    a.d = m.d;
    a.f = m.f;
    a.status = status;
    a.wait_clocks = (long long)(kWaitSeconds * kClocksPerSecond);
    a.stall = -1;
    {
        std::lock_guard<std::mutex> lock(g_mu);
        if (g_stall >= 0) {
            a.stall = g_stall;
            a.wait_clocks = (long long)(g_stall_wait_s * kClocksPerSecond);
            g_stall = -1;
        }
    }
    return m.dtype == SSD_F16 ? start_moe<f16>(call, a, m, cuda_stream) : start_moe<bf16>(call, a, m, cuda_stream);
}
