// step_moe.cu - a mixture-of-experts layer for the rows of a decoding step:
// the router (ssd_moe_route) and the experts' products (ssd_moe_mlp) of ssd_step.h.
#include <algorithm>
#include <cmath>

#include "step_ops.cuh"

namespace ssd {
namespace step {

constexpr int kMaxExperts = 1024, kMaxSlots = 16, kMaxMoeRows = 1024;

// ---------------------------------------------------------------------------
// ssd_moe_route
// ---------------------------------------------------------------------------
constexpr int kRouteThreads = 256, kRouteWarps = kRouteThreads / 32, kRouteSplit = 8;
constexpr int kRouteShare = kMaxExperts / kRouteSplit;  // experts of a CTA at most

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

// A cluster of 8 CTAs takes a row, each an eighth of the experts.  Which of two experts comes first must not hang on the order of a sum,
// so the products (exact in fp32: two values of 8 or 11 bits) are added without loss to a pair of floats, 6 additions each
// (Knuth's two-sum), and pairs are joined in fp64.  fp64 sums would be slower by an order: the chip has two fp64 units an SM.
// Scores decide by z itself where that is the same order, in fp64 where something is added to them.  The rank of an
// expert is the number of better ones, counted by the CTA that has it; the winners go to the first CTA.
template <typename T>
__global__ void __launch_bounds__(kRouteThreads) route_kernel(const __grid_constant__ RouteArgs a) {
    __shared__ double s_part[kRouteWarps * kRouteShare];  // [warp of an expert][expert]
    __shared__ double s_z[kRouteShare];
    __shared__ uint64_t s_key[kRouteShare], s_all[kMaxExperts];
    __shared__ double s_top[kMaxSlots];  // the winners' z and expert, in the first CTA
    __shared__ uint64_t s_who[kMaxSlots], s_stat[kRouteSplit];
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, rank = blockIdx.x, row = blockIdx.y;
    const int share = (a.n_experts + kRouteSplit - 1) / kRouteSplit, e0 = min(rank * share, a.n_experts), mine = min(share, a.n_experts - e0);
    // warps of an expert, each a part of d
    const int per = share <= 1 ? 8 : share <= 2 ? 4 : share <= 4 ? 2 : 1, part = warp % per;
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
                for (int j = 0; j < 8; ++j) {
                    const float q = __fmul_rn(f[j], g[j]), t = __fadd_rn(s, q), b = __fsub_rn(t, s);
                    c = __fadd_rn(c, __fadd_rn(__fsub_rn(s, __fsub_rn(t, b)), __fsub_rn(q, b)));
                    s = t;
                }
            }
        }
        double z = isfinite(s) ? (double)s + (double)c : (double)s;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
        if (lane == 0) s_part[part * kRouteShare + e] = z;
    }
    __syncthreads();
    for (int e = tid; e < mine; e += kRouteThreads) {
        double z = 0.0;
        for (int i = 0; i < per; ++i) z += s_part[i * kRouteShare + e];
        s_z[e] = z;
    }
    __syncthreads();
    // softmax over all experts where the scores or the weights need it: the row's maximum and sum
    const bool whole = a.score == SSD_MOE_SOFTMAX && (a.favour || !a.renorm);
    if (whole) {
        cluster_sync();  // (every CTA has started)
        double m = -INFINITY;
        if (warp == 0) {
            for (int e = lane; e < mine; e += 32) m = fmax(m, s_z[e]);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) m = fmax(m, __shfl_xor_sync(0xffffffffu, m, o));
            if (lane < kRouteSplit) peer_store(&s_stat[rank], lane, (uint64_t)__double_as_longlong(m));
        }
        cluster_sync();
        m = -INFINITY;
        for (int i = 0; i < kRouteSplit; ++i) m = fmax(m, __longlong_as_double((long long)s_stat[i]));
        double sum = 0.0;
        if (warp == 0) {
            for (int e = lane; e < mine; e += 32) sum += exp(s_z[e] - m);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        }
        cluster_sync();  // (the maxima are read)
        if (warp == 0 && lane < kRouteSplit) peer_store(&s_stat[rank], lane, (uint64_t)__double_as_longlong(sum));
        cluster_sync();
        sum = 0.0;
        for (int i = 0; i < kRouteSplit; ++i) sum += __longlong_as_double((long long)s_stat[i]);
        for (int e = tid; e < mine; e += kRouteThreads) {
            const double p = exp(s_z[e] - m) / sum;
            s_z[e] = p;  // (from here on the score)
            s_key[e] = order_of(a.favour ? p + (double)__ldcg(a.favour + e0 + e) : p);
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
    for (int e = tid; e < mine; e += kRouteThreads) {
        const uint64_t key = s_key[e];
        int better = 0;
        for (int i = 0; i < a.n_experts; ++i) better += s_all[i] > key || (s_all[i] == key && i < e0 + e);
        if (better < a.k) {
            peer_store(&s_top[better], 0, (uint64_t)__double_as_longlong(s_z[e]));
            peer_store(&s_who[better], 0, (uint64_t)(e0 + e));
        }
    }
    cluster_sync();
    if (rank || warp) return;
    // weights of the winners, a lane each
    float p = 0.f;
    if (lane < a.k) {
        // (what rounding the exponent to fp32 leaves is a factor)
        const double z = a.score == SSD_MOE_SIGMOID ? -s_top[lane] : s_top[lane] - s_top[0];
        const float near = (float)z, rest = (float)(z - (double)near), e = expf(near) * (1.f + (isfinite(near) ? rest : 0.f));
        if (whole) p = (float)s_top[lane];
        else if (a.score == SSD_MOE_SIGMOID) p = 1.f / (1.f + e);
        else p = e;  // (renormalised below)
    }
    if (a.renorm) p /= warp_sum(p);
    if (lane < a.k) {
        a.ids[(int64_t)row * a.k + lane] = (int)s_who[lane];
        a.weights[(int64_t)row * a.k + lane] = p * a.scale;
    }
}

// ---------------------------------------------------------------------------
// ssd_moe_mlp
// ---------------------------------------------------------------------------
constexpr int kMoeThreads = 256, kMoeWarps = kMoeThreads / 32;
// rows of an expert that its weights are read for at once (MT: tiles of 16 weight rows in a warp)
__host__ __device__ constexpr int group_of(int MT) { return MT == 1 ? 8 : 32; }
constexpr int kMaxGroup = 32;
constexpr int kChunk = 32;  // k of a chunk: 4 lanes have 16 bytes each of a row

struct MoeArgs {
    const void *gate, *up, *down, *x, *residual;
    void* out;
    const int32_t* ids;
    const float* weights;
    int64_t gate_stride, up_stride, down_stride, x_stride, residual_stride, out_stride;
    void* h;             // [2][pair][f]: silu(gate x) * (up x) as hi + lo
    float* y;            // [pair][d]: weights * down h
    unsigned* arrived;   // [tile of d]: groups that have written their part of y
    int n_rows, k, n_experts, d, f;
};

__device__ __forceinline__ uint4 load_weights(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
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

// The rows' experts, as every CTA of both kernels works them out for itself from ids: the (row, slot) pairs of an expert in
// order, in groups of 8 or 32; a unit of work is a group and a tile of output rows.
template <int kGroup>
struct Plan {
    int n_groups;
    uint16_t* of_pair;  // [pair] expert, 0xffff: none
    uint16_t* expert;   // [group]
    uint16_t* first;    // [group] its number among its expert's groups
};
__host__ __device__ inline int max_groups(int n_pairs, int n_experts, int size) { return (n_experts < n_pairs ? n_experts : n_pairs) + n_pairs / size; }

template <int kGroup>
__device__ __forceinline__ Plan<kGroup> make_plan(const MoeArgs& a, unsigned char* smem, int* s_count, int* s_scan) {
    const int tid = threadIdx.x, n = a.n_rows * a.k;
    Plan<kGroup> p;
    p.of_pair = reinterpret_cast<uint16_t*>(smem);
    p.expert = p.of_pair + n;
    p.first = p.expert + max_groups(n, a.n_experts, kGroup);
    for (int e = tid; e < kMaxExperts; e += kMoeThreads) s_count[e] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kMoeThreads) {
        const int e = __ldcg(a.ids + i);
        const bool ok = e >= 0 && e < a.n_experts;
        p.of_pair[i] = ok ? (uint16_t)e : (uint16_t)0xffff;
        if (ok) atomicAdd(s_count + e, 1);
    }
    __syncthreads();
    // groups of experts before: 4 experts a thread, summed over the warps
    constexpr int kEach = kMaxExperts / kMoeThreads;
    int mine[kEach], sum = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        mine[i] = (s_count[tid * kEach + i] + kGroup - 1) / kGroup;
        sum += mine[i];
    }
    int upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int v = __shfl_up_sync(0xffffffffu, upto, o);
        if (tid % 32 >= o) upto += v;
    }
    if (tid % 32 == 31) s_scan[tid / 32] = upto;
    __syncthreads();
    int at = upto - sum;
    p.n_groups = 0;
    for (int w = 0; w < kMoeWarps; ++w) {
        if (w < tid / 32) at += s_scan[w];
        p.n_groups += s_scan[w];
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        for (int g = 0; g < mine[i]; ++g, ++at) p.expert[at] = (uint16_t)(tid * kEach + i), p.first[at] = (uint16_t)g;
    __syncthreads();
    return p;
}

// warp 0: the pairs of a group, and how many
template <int kGroup>
__device__ __forceinline__ void find_pairs(const Plan<kGroup>& p, int n_pairs, int group, int* s_pairs, int* s_n) {
    const int lane = threadIdx.x, e = p.expert[group], from = p.first[group] * kGroup;
    int seen = 0;
    for (int i = 0; i < n_pairs && seen < from + kGroup; i += 32) {
        const bool is = i + lane < n_pairs && p.of_pair[i + lane] == e;
        const unsigned m = __ballot_sync(0xffffffffu, is);
        const int at = seen + __popc(m & ((1u << lane) - 1u)) - from;
        if (is && at >= 0 && at < kGroup) s_pairs[at] = i + lane;
        seen += __popc(m);
    }
    if (lane == 0) *s_n = min(seen - from, kGroup);
}

// Sums of a warp's MT tiles of 16 weight rows and NT tiles of 8 columns over k0 .. k1 (pieces of 8 past k1 count as zeros).
// wp: this lane's two rows of each tile, xp: its column of each tile and plane, all at their lane % 4 th piece.  The k that a lane
// holds go to the matrix instruction in an order of their own, the same for both operands, so that every load is 16
// bytes straight into the fragments.  The next kAhead chunks of weights are under way while those before are multiplied:
// 16 warps an SM of 4 KB each, which covers HBM's latency.
template <typename T, int MT, int NT, int PL>
struct Products {
    static constexpr int kAhead = 4 / MT;
    uint4 w[2][kAhead][MT][2];
    __device__ __forceinline__ void load(int b, const T* const (&wp)[MT][2], int k, int k1) {
        const int piece = threadIdx.x % 4 * 8;
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < 2; ++r)
                    w[b][i][m][r] = k + i * kChunk + piece < k1 ? load_weights(wp[m][r] + k + i * kChunk) : make_uint4(0u, 0u, 0u, 0u);
    }
    __device__ __forceinline__ void multiply(int b, float (&acc)[MT][NT][4], const T* const (&xp)[PL][NT], int k, int k1) {
        const int piece = threadIdx.x % 4 * 8;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (k + i * kChunk >= k1) break;
            const bool in = k + i * kChunk + piece < k1;
#pragma unroll
            for (int l = 0; l < PL; ++l)
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const uint4 x = in ? *reinterpret_cast<const uint4*>(xp[l][t] + k + i * kChunk) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        const uint4 &u = w[b][i][m][0], &v = w[b][i][m][1];
                        mma(acc[m][t], u.x, v.x, u.y, v.y, x.x, x.y, T());
                        mma(acc[m][t], u.z, v.z, u.w, v.w, x.z, x.w, T());
                    }
                }
        }
    }
    __device__ __forceinline__ void run(float (&acc)[MT][NT][4], const T* const (&wp)[MT][2], const T* const (&xp)[PL][NT], int k0, int k1) {
        constexpr int kStep = kAhead * kChunk;
        load(0, wp, k0, k1);
        for (int k = k0; k < k1; k += 2 * kStep) {
            load(1, wp, k + kStep, k1);
            multiply(0, acc, xp, k, k1);
            load(0, wp, k + 2 * kStep, k1);
            multiply(1, acc, xp, k + kStep, k1);
        }
    }
};

// h = silu(gate x) * (up x).  A tile of 16 weight rows is 8 of gate and the same 8 of up, so that both sums of an output are in
// one lane.  The CTA's 8 warps take parts of d, added in order through shared memory.
template <typename T, int MT, int NT>
__device__ __forceinline__ void up_unit(const MoeArgs& a, int e, int f0, int n, const int* s_pairs, float4* s_red) {
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, g = lane / 4, piece = lane % 4 * 8;
    const int chunks = (a.d + kChunk - 1) / kChunk, each = (chunks + kMoeWarps - 1) / kMoeWarps;
    const T *wp[MT][2], *xp[1][NT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int64_t at = (int64_t)min(f0 + 8 * m + g, a.f - 1) * a.d + piece;
        wp[m][0] = (const T*)a.gate + (int64_t)e * a.gate_stride + at;
        wp[m][1] = (const T*)a.up + (int64_t)e * a.up_stride + at;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) xp[0][t] = (const T*)a.x + (int64_t)(s_pairs[min(8 * t + g, n - 1)] / a.k) * a.x_stride + piece;
    float acc[MT][NT][4] = {};
    Products<T, MT, NT, 1> p;
    p.run(acc, wp, xp, warp * each * kChunk, min((warp + 1) * each * kChunk, a.d));
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t) s_red[((warp * MT + m) * NT + t) * 32 + lane] = make_float4(acc[m][t][0], acc[m][t][1], acc[m][t][2], acc[m][t][3]);
    __syncthreads();
    for (int i = tid; i < MT * NT * 32; i += kMoeThreads) {
        float4 s = s_red[i];
#pragma unroll
        for (int w = 1; w < kMoeWarps; ++w) {
            const float4 v = s_red[w * MT * NT * 32 + i];
            s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
        }
        const int f = f0 + i / (NT * 32) * 8 + lane / 4, col = i / 32 % NT * 8 + lane % 4 * 2;
        const float h[2] = {s.x / (1.f + expf(-s.x)) * s.z, s.y / (1.f + expf(-s.y)) * s.w};
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (f < a.f && col + j < n) {
                T* to = (T*)a.h + (int64_t)s_pairs[col + j] * a.f + f;
                const T hi = (T)h[j];
                to[0] = hi;
                to[(int64_t)a.n_rows * a.k * a.f] = isfinite((float)hi) ? (T)(h[j] - (float)hi) : (T)0.f;
            }
    }
}

template <typename T, int MT>
__global__ void __launch_bounds__(kMoeThreads, 2) moe_up_kernel(const __grid_constant__ MoeArgs a) {
    extern __shared__ __align__(16) unsigned char s_plan[];
    __shared__ int s_count[kMaxExperts], s_scan[kMoeWarps], s_pairs[kMaxGroup], s_n;
    __shared__ float4 s_red[kMoeWarps * MT * (group_of(MT) / 8) * 32];
    pdl_wait();
    pdl_launch_dependents();  // (only here: the next kernel reads ids before it waits)
    const Plan<group_of(MT)> p = make_plan<group_of(MT)>(a, s_plan, s_count, s_scan);
    const int tiles = (a.f + 8 * MT - 1) / (8 * MT);
    for (int i = blockIdx.x * kMoeThreads + threadIdx.x; i < (a.d + 15) / 16; i += gridDim.x * kMoeThreads) a.arrived[i] = 0u;
    int last = -1;
    for (int64_t u = blockIdx.x; u < (int64_t)p.n_groups * tiles; u += gridDim.x) {
        const int group = (int)(u / tiles), f0 = (int)(u % tiles) * 8 * MT;
        if (group != last) {
            __syncthreads();
            if (threadIdx.x < 32) find_pairs(p, a.n_rows * a.k, group, s_pairs, &s_n);
            last = group;
        }
        __syncthreads();  // (the sums of the unit before are read, too)
        const int e = p.expert[group], n = s_n;
        if (MT == 1 || n <= 8) up_unit<T, MT, 1>(a, e, f0, n, s_pairs, s_red);
        else if (n <= 16) up_unit<T, MT, MT == 1 ? 1 : 2>(a, e, f0, n, s_pairs, s_red);
        else up_unit<T, MT, MT == 1 ? 1 : 4>(a, e, f0, n, s_pairs, s_red);
    }
}

// y = weights * (down h), h as two planes
template <typename T, int MT, int NT>
__device__ __forceinline__ void down_unit(const MoeArgs& a, int e, int d0, int n, const int* s_pairs, float4* s_red, bool& waited) {
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, g = lane / 4, piece = lane % 4 * 8;
    const int chunks = (a.f + kChunk - 1) / kChunk, each = (chunks + kMoeWarps - 1) / kMoeWarps;
    const T *wp[MT][2], *xp[2][NT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < 2; ++r) wp[m][r] = (const T*)a.down + (int64_t)e * a.down_stride + (int64_t)min(d0 + 16 * m + 8 * r + g, a.d - 1) * a.f + piece;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        xp[0][t] = (const T*)a.h + (int64_t)s_pairs[min(8 * t + g, n - 1)] * a.f + piece;
        xp[1][t] = xp[0][t] + (int64_t)a.n_rows * a.k * a.f;
    }
    float acc[MT][NT][4] = {};
    Products<T, MT, NT, 2> p;
    if (!waited) {
        pdl_wait();
        waited = true;
    }
    p.run(acc, wp, xp, warp * each * kChunk, min((warp + 1) * each * kChunk, a.f));
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t) s_red[((warp * MT + m) * NT + t) * 32 + lane] = make_float4(acc[m][t][0], acc[m][t][1], acc[m][t][2], acc[m][t][3]);
    __syncthreads();
    for (int i = tid; i < MT * NT * 32; i += kMoeThreads) {
        float4 s = s_red[i];
#pragma unroll
        for (int w = 1; w < kMoeWarps; ++w) {
            const float4 v = s_red[w * MT * NT * 32 + i];
            s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
        }
        const int dim = d0 + i / (NT * 32) * 16 + lane / 4, col = i / 32 % NT * 8 + lane % 4 * 2;
        const float v[2][2] = {{s.x, s.y}, {s.z, s.w}};
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (col + j < n) {
                const int pair = s_pairs[col + j];
                const float w = __ldcg(a.weights + pair);
                float* y = a.y + (int64_t)pair * a.d;
                if (dim < a.d) y[dim] = w * v[0][j];
                if (dim + 8 < a.d) y[dim + 8] = w * v[1][j];
            }
    }
}

// The CTA that writes the last part of a tile of y adds the rows' slots in order, whoever wrote them.
template <typename T, int MT>
__global__ void __launch_bounds__(kMoeThreads, 2) moe_down_kernel(const __grid_constant__ MoeArgs a) {
    extern __shared__ __align__(16) unsigned char s_plan[];
    __shared__ int s_count[kMaxExperts], s_scan[kMoeWarps], s_pairs[kMaxGroup], s_n, s_last;
    __shared__ float4 s_red[kMoeWarps * MT * (group_of(MT) / 8) * 32];
    pdl_launch_dependents();
    // ids were complete before the kernel before this one let it start
    const Plan<group_of(MT)> p = make_plan<group_of(MT)>(a, s_plan, s_count, s_scan);
    constexpr int kTile = 16 * MT;
    const int tiles = (a.d + kTile - 1) / kTile, groups = max(p.n_groups, 1);
    bool waited = false;
    int last = -1;
    for (int64_t u = blockIdx.x; u < (int64_t)groups * tiles; u += gridDim.x) {
        const int group = (int)(u / tiles), tile = (int)(u % tiles), d0 = tile * kTile;
        if (p.n_groups) {
            if (group != last) {
                __syncthreads();
                if (threadIdx.x < 32) find_pairs(p, a.n_rows * a.k, group, s_pairs, &s_n);
                last = group;
            }
            __syncthreads();
            const int e = p.expert[group], n = s_n;
            if (MT == 1 || n <= 8) down_unit<T, MT, 1>(a, e, d0, n, s_pairs, s_red, waited);
            else if (n <= 16) down_unit<T, MT, MT == 1 ? 1 : 2>(a, e, d0, n, s_pairs, s_red, waited);
            else down_unit<T, MT, MT == 1 ? 1 : 4>(a, e, d0, n, s_pairs, s_red, waited);
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) s_last = atomicAdd(a.arrived + tile, 1u) == (unsigned)p.n_groups - 1u;
            __syncthreads();
            if (!s_last) continue;
            __threadfence();
        } else if (!waited) {
            pdl_wait();
            waited = true;
        }
        const int width = min(kTile, a.d - d0);
        for (int i = threadIdx.x; i < a.n_rows * width; i += kMoeThreads) {
            const int row = i / width, dim = d0 + i % width;
            float s = a.residual ? (float)((const T*)a.residual)[(int64_t)row * a.residual_stride + dim] : 0.f;
            float t = 0.f;
            for (int j = 0; j < a.k; ++j)
                if (p.of_pair[row * a.k + j] != 0xffff) t += __ldcg(a.y + ((int64_t)row * a.k + j) * a.d + dim);
            ((T*)a.out)[(int64_t)row * a.out_stride + dim] = (T)(s + t);
        }
    }
    if (!waited) pdl_wait();
}

size_t plan_bytes(int n_pairs, int n_experts, int size) { return 2 * ((size_t)n_pairs + 2 * (size_t)max_groups(n_pairs, n_experts, size)); }

struct Workspace {
    size_t h, y, total;  // offsets behind the counters, bytes
};
Workspace workspace_of(const ssd_moe& m, int n_rows, int k) {
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    const size_t pairs = (size_t)n_rows * k;
    Workspace w;
    w.h = up(4 * (((size_t)m.d + 15) / 16));
    w.y = w.h + up(2 * 2 * pairs * m.f);
    w.total = w.y + up(4 * pairs * m.d);
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

template <typename T>
int launch_moe(const char* call, const MoeArgs& a, void* stream) {
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    static bool ready[64] = {};  // (set once a device and type; setting it twice is harmless)
    if (e == cudaSuccess && !(dev < 64 && ready[dev])) {
        // (static and dynamic shared memory may pass 48 KB together)
        const int most = (int)plan_bytes(kMaxMoeRows * kMaxSlots, kMaxExperts, kMaxGroup);
        e = cudaFuncSetAttribute(moe_up_kernel<T, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(moe_down_kernel<T, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
        if (e == cudaSuccess && dev < 64) ready[dev] = true;
    }
    if (e != cudaSuccess) return refuse(SSD_ERR_CUDA, call, "%s", cudaGetErrorString(e));
    const size_t smem = plan_bytes(a.n_rows * a.k, a.n_experts, a.n_rows <= 8 ? group_of(1) : group_of(2));
    const dim3 grid((unsigned)(2 * sms));
    // up to 8 rows an expert has one tile of columns at most: tiles of 16 weight rows, more chunks under way
    if (a.n_rows <= 8) {
        if (int rc = launch(call, moe_up_kernel<T, 1>, grid, kMoeThreads, smem, stream, a)) return rc;
        return launch(call, moe_down_kernel<T, 1>, grid, kMoeThreads, smem, stream, a);
    }
    if (int rc = launch(call, moe_up_kernel<T, 2>, grid, kMoeThreads, smem, stream, a)) return rc;
    return launch(call, moe_down_kernel<T, 2>, grid, kMoeThreads, smem, stream, a);
}

}  // namespace step
}  // namespace ssd

using namespace ssd;
using namespace ssd::step;

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
    const size_t picked = 4 * (size_t)n_rows * k;
    if (meet(ids, picked, weights, picked) || meet(ids, picked, x, span(n_rows, x_stride, d, dtype)) || meet(weights, picked, x, span(n_rows, x_stride, d, dtype)))
        return refuse_arg(call, "ids and weights must overlap neither each other nor x");
    if (int rc = check_device(call, x)) return rc;
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
    cfg.gridDim = dim3(kRouteSplit, (unsigned)n_rows, 1);
    cfg.blockDim = dim3(kRouteThreads, 1, 1);
    cfg.stream = (cudaStream_t)cuda_stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kRouteSplit, attr[1].val.clusterDim.y = 1, attr[1].val.clusterDim.z = 1;
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
                           void* workspace, size_t workspace_bytes, void* cuda_stream) {
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
    if (residual == out && residual_stride != out_stride) return refuse_arg(call, "out in the residual's place needs its stride");
    const Workspace w = workspace_of(m, n_rows, k);
    const size_t picked = 4 * (size_t)n_rows * k, rows = span(n_rows, out_stride, m.d, m.dtype);
    if (x == out || meet(out, rows, ids, picked) || meet(out, rows, weights, picked)) return refuse_arg(call, "out must not overlap x, ids or weights");
    if (meet(workspace, w.total, out, rows) || meet(workspace, w.total, x, span(n_rows, x_stride, m.d, m.dtype)) || meet(workspace, w.total, ids, picked) ||
        meet(workspace, w.total, weights, picked) || meet(workspace, w.total, residual, span(n_rows, residual_stride, m.d, m.dtype)))
        return refuse_arg(call, "the workspace must not overlap other tensors");
    if ((uintptr_t)workspace & 15u) return refuse_arg(call, "the workspace must be 16-byte aligned");
    if (workspace_bytes < w.total) return refuse(SSD_ERR_CAPACITY, call, "the workspace needs %zu bytes", w.total);
    if (int rc = check_device(call, x)) return rc;
    MoeArgs a{};
    a.gate = m.gate;
    a.up = m.up;
    a.down = m.down;
    a.gate_stride = m.gate_stride;
    a.up_stride = m.up_stride;
    a.down_stride = m.down_stride;
    a.x = x;
    a.x_stride = x_stride;
    a.residual = residual;
    a.residual_stride = residual_stride;
    a.out = out;
    a.out_stride = out_stride;
    a.ids = ids;
    a.weights = weights;
    a.arrived = (unsigned*)workspace;
    a.h = (char*)workspace + w.h;
    a.y = (float*)((char*)workspace + w.y);
    a.n_rows = n_rows;
    a.k = k;
    a.n_experts = m.n_experts;
    a.d = m.d;
    a.f = m.f;
    return m.dtype == SSD_F16 ? launch_moe<f16>(call, a, cuda_stream) : launch_moe<bf16>(call, a, cuda_stream);
}
