// tree_few.cu - ssd_tree_attention for tiles of few rows (single tokens of heads that
// share little or nothing), in fp32 on the CUDA cores.
//
// With R rows a position costs 4 hd bytes, whatever R is, and R (2 hd multiply-adds and an
// exponential): up to some rows HBM is the bound without matrix instructions, whose tile
// of 128 rows would be almost empty, and q and the weights need no rounding.
//
// A CTA (one per SM) walks its range (tree_sched.cuh).  Each warp takes every W-th block of an
// item: 16 positions (head_dim 64: 32), of whose K a lane holds 16 bytes of 8 of them (W
// blocks' K and V are what keeps HBM busy: the next block's K is asked for before the
// weights, V with the scores).  The lanes' products are added by a transposing
// reduction - 8 sums of 16 lanes in 8 exchanges - which leaves a lane one position's score; each
// warp has its own reference for the weights, which moves when a score exceeds it by more than
// kSlack.  At the end of an item the warps' sums meet in shared memory, with the next
// item's first K on its way; parts of items that other CTAs share go to the workspace for
// join_kernel.
//
// Measured (with join_kernel), against the tensor cores' kernel: single tokens of 16
// requests, 262 to 2100 positions, 32 heads of 128 dims, fp32 64 us (5.5 TB/s, 81 % of the copy rate)
// against 88, fp16 64 against 77; two heads a KV head 71 against 88 and 71 against 77; head_dim 64, 32 requests 69
// against 99 (fp16) and 136 (fp32); one request of 4000 positions 17 against 27, of 200 9.6 against 16.  Four rows a tile:
// 96 against 88 (fp32) and 74 (fp16), as the arithmetic of a block then takes as long as its loads; so
// two rows are the most.  What is left: 7 us until the first block is there, 3 to join, uneven blocks.
#include "tree_attn.cuh"

namespace ssd {
namespace tree {
namespace {

// threads of a CTA: as many as have the registers for R rows (one row: 512 threads 64 us, 384 65;
// two: 384 70 us, 256 83, 512 with spilled registers 81)
template <int R>
constexpr int kThreadsOf = R == 1 ? 512 : 384;
constexpr int kLoads = 8;  // 16-byte loads of K (V) that a lane has in flight (4: 67 us)
constexpr float kSlack = 8.f;  // log2: weights up to 2^8 of the reference's

__device__ __forceinline__ void cp_async16(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}

// fp32 pairs of 8 values of the cache
template <typename C>
__device__ __forceinline__ void pairs_of(const uint4& u, f32x2 (&p)[4]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 v = unpack2(w[i], C());
        p[i] = two(v.x, v.y);
    }
}

// p[0 .. M-1] of N lanes -> the sum over them of p[i], i = the upper bits of the lane's place
template <int N, int M>
__device__ __forceinline__ float sums_of(float (&p)[M], int lane) {
    int off = N / 2;
#pragma unroll
    for (int half = M / 2; half; half /= 2, off /= 2) {
        const bool up = lane & off;
#pragma unroll
        for (int i = 0; i < half; ++i) {
            const float give = up ? p[i] : p[i + half], keep = up ? p[i + half] : p[i];
            p[i] = keep + __shfl_xor_sync(0xffffffffu, give, off);
        }
    }
#pragma unroll
    for (; off; off /= 2) p[0] += __shfl_xor_sync(0xffffffffu, p[0], off);
    return p[0];
}

template <typename T, int HD, int R>
__global__ void __launch_bounds__(kThreadsOf<R>, 1) few_kernel(const __grid_constant__ AttnOpArgs a) {
    using C = typename Types<T>::C;
    constexpr int THREADS = kThreadsOf<R>, W = THREADS / 32, LANES = HD / 8, AT_ONCE = 32 / LANES;
    constexpr int M = kLoads, BLOCK = M * AT_ONCE, PIECES = BLOCK <= 16 ? 1 : BLOCK / 16, SAME = LANES / M;  // (SAME lanes get the same sums)
    constexpr int QROW = HD * (int)sizeof(T) / 16;  // 16-byte pieces of a row of q
    extern __shared__ __align__(16) float s_o[];    // [segment & 1][W][R][HD]
    __shared__ float2 s_end[2][W][R];               // reference and sum of weights
    __shared__ __align__(16) uint4 s_q[2][R * QROW];
    __shared__ Seg s_seg[4];
    __shared__ int s_has[4];
    __shared__ RangeOf<THREADS> s_range;
    __shared__ Walk s_walk;  // (what few threads need now and then is kept out of the registers)
    __shared__ long long s_units;
    __shared__ int s_ctas;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x;
    pdl_launch_dependents();
    pdl_wait();  // everything below may come from the previous kernel
    if (tid == 0) a.cuts[cta].last = -1;
    const Shape& sh = a.shape;
    // one thread walks, two segments ahead
    const bool walker = tid == THREADS - 1;
    auto walk_on = [&](unsigned n) {
        Walk w = s_walk;
        s_has[n & 3] = walk_next(w, sh, R, s_seg[n & 3]);
        s_walk = w;
    };
    {
        Walk w;
        int ctas;
        const long long units = range_of<THREADS>(a, R, s_range, w, ctas);
        if (walker) {
            s_walk = w;
            s_units = units;
            s_ctas = ctas;
        }
    }
    if (walker) {
        walk_on(0);
        walk_on(1);
    }
    __syncthreads();

    const int in_load = lane / LANES, dim = lane % LANES * 8;
    const int64_t step = a.pos_stride * (2 * AT_ONCE), lane_off = (in_load * a.pos_stride + dim) * 2;
    auto ask_q = [&](unsigned n) {
        const Seg& g = s_seg[n & 3];
        if (tid < R * QROW) {
            const int r = min(g.mt * R + tid / QROW, g.q.n * sh.group - 1), node = r / sh.group, head = g.kvh * sh.group + r - node * sh.group;
            cp_async16(&s_q[n & 1][tid], (const T*)a.q + (int64_t)(g.q.r0 + node) * a.q_stride + head * HD + tid % QROW * (16 / (int)sizeof(T)));
        }
    };
    // where the warp's block i0 + lane of a segment lies: bytes behind the layer's K (V) of each 16 positions; -1: outside, reads as zeros
    auto find = [&](unsigned n, int i0, int64_t (&at)[PIECES]) {
        const Seg& g = s_seg[n & 3];
        const long long x0 = (long long)g.u0 * kUnit + (long long)(warp + W * (i0 + lane)) * BLOCK;
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            const long long x = x0 + 16 * k;
            at[k] = -1;
            if (x < min((long long)g.u1 * kUnit, (long long)g.q.total)) {
                const int in_table = (int)x / sh.page_size, page = __ldcg(a.block_table + (size_t)g.b * sh.max_blocks + in_table);
                if (page >= 0 && page < a.n_pages) at[k] = (page * a.page_stride + g.kvh * a.head_stride + ((int)x - in_table * sh.page_size) * a.pos_stride) * 2;
            }
        }
    };
    auto ask = [&](const void* base, const int64_t (&at)[PIECES], int i, int left, uint4 (&r)[M]) {  // left: positions from the block's first on
        int64_t o[PIECES];
        bool all = left >= BLOCK;
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            o[k] = __shfl_sync(0xffffffffu, at[k], i & 31);
            all = all && o[k] >= 0;
        }
        const char* p = (const char*)base + lane_off;
        if (all) {
#pragma unroll
            for (int k = 0; k < M; ++k) r[k] = __ldcg(reinterpret_cast<const uint4*>(p + o[k * PIECES / M] + (k % (M / PIECES)) * step));
        } else {
#pragma unroll
            for (int k = 0; k < M; ++k) {
                r[k] = make_uint4(0, 0, 0, 0);
                if (o[k * PIECES / M] >= 0 && k * AT_ONCE + in_load < left) r[k] = __ldcg(reinterpret_cast<const uint4*>(p + o[k * PIECES / M] + (k % (M / PIECES)) * step));
            }
        }
    };
    auto end_of = [&](const Seg& g) { return min(g.u1 * kUnit, g.q.total); };
    auto blocks_of = [&](const Seg& g) { return (end_of(g) - g.u0 * kUnit - warp * BLOCK + W * BLOCK - 1) / (W * BLOCK); };  // of this warp (rounds towards 0)

    int64_t at[PIECES], at_next[PIECES];
    uint4 k8[M];
    // the first block's K of segment n
    auto first_k = [&](unsigned n, const int64_t (&where)[PIECES]) {
        const Seg& g = s_seg[n & 3];
        if (blocks_of(g) > 0) ask(a.kc, where, 0, end_of(g) - g.u0 * kUnit - warp * BLOCK, k8);
    };
    if (s_has[0]) {
        ask_q(0);
        find(0, 0, at);
        first_k(0, at);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    for (unsigned n = 0; s_has[n & 3]; ++n) {
        const bool more = s_has[(n + 1) & 3];
        if (more) {
            ask_q(n + 1);
            find(n + 1, 0, at_next);
        }
        if (walker) {
            if (more) walk_on(n + 2);
            else s_has[(n + 2) & 3] = 0;
        }
        const int len = s_seg[n & 3].q.len, end = end_of(s_seg[n & 3]), blocks = blocks_of(s_seg[n & 3]);
        const int row0 = s_seg[n & 3].mt * R, rows = min(s_seg[n & 3].q.n * sh.group - row0, R);  // rows that exist
        const int node0 = row0 / sh.group, all_seen = min(sh.chain ? len + node0 + 1 : len, end);  // positions below it are seen by every row
        f32x2 q[R][4], o[R][4];
        float ref[R], l[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            ref[r] = -INFINITY;
            l[r] = 0.f;
            const T* from = reinterpret_cast<const T*>(s_q[n & 1]) + r * HD + dim;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                q[r][i] = two((float)from[2 * i], (float)from[2 * i + 1]);
                o[r][i] = 0;
            }
        }
        const int x0 = s_seg[n & 3].u0 * kUnit + warp * BLOCK;
#pragma unroll 1
        for (int i = 0; i < blocks; ++i) {
            const int x = x0 + i * (W * BLOCK);
            uint4 v8[M];
            ask(a.vc, at, i, end - x, v8);
            float s[R], p[R][M];
#pragma unroll
            for (int k = 0; k < M; ++k) {
                f32x2 kk[4];
                pairs_of<C>(k8[k], kk);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const f32x2 d = fma2(q[r][3], kk[3], fma2(q[r][2], kk[2], fma2(q[r][1], kk[1], mul2(q[r][0], kk[0]))));
                    float d0, d1;
                    of_two(d, d0, d1);
                    p[r][k] = d0 + d1;
                }
            }
            if (i + 1 < blocks) {
                if (!((i + 1) & 31)) find(n, i + 1, at);
                ask(a.kc, at, i + 1, end - x - W * BLOCK, k8);
            } else if (more) {
                first_k(n + 1, at_next);
            }
            const int mine = x + lane % LANES / SAME * AT_ONCE + in_load;  // the position whose scores this lane has
            const bool edge = x + BLOCK > all_seen;
            unsigned hidden = 0;  // rows that do not see it
#pragma unroll
            for (int r = 0; r < R; ++r) s[r] = sums_of<LANES, M>(p[r], lane) * a.scale2;
            if (edge) {
                const int j = mine - len;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int node = (row0 + min(r, rows - 1)) / sh.group;
                    const bool seen = mine < end && (j < 0 || (sh.chain ? j <= node : j < 64 * a.words && (__ldcg(a.masks + (size_t)(s_seg[n & 3].q.r0 + node) * a.words + (j >> 6)) >> (j & 63) & 1)));
                    if (!seen) {
                        s[r] = -INFINITY;
                        hidden |= 1u << r;
                    }
                }
            }
            bool grown = false;
#pragma unroll
            for (int r = 0; r < R; ++r) grown = grown || s[r] > ref[r] + kSlack;
            if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    if (R > 1 && !__any_sync(0xffffffffu, s[r] > ref[r] + kSlack)) continue;  // (what one row sees moves no other's)
                    float top = fmaxf(ref[r], s[r]);
#pragma unroll
                    for (int off = 16; off; off /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
                    const float f = ref[r] == -INFINITY ? 0.f : ex2(ref[r] - top);
                    l[r] *= f;
#pragma unroll
                    for (int k = 0; k < 4; ++k) o[r][k] = mul2(o[r][k], two(f, f));
                    ref[r] = top;
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                s[r] = ex2(s[r] - (ref[r] == -INFINITY ? 0.f : ref[r]));
                l[r] += s[r];
                if (hidden >> r & 1) s[r] = -1.f;  // (no weight is)
            }
            // the weights' lane of load k
            const int from = lane / LANES * LANES;
#pragma unroll
            for (int k = 0; k < M; ++k) {
                f32x2 vv[4];
                pairs_of<C>(v8[k], vv);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float w = __shfl_sync(0xffffffffu, s[r], from + k * SAME);
                    if (edge && w < 0.f) continue;  // not seen: its values may be anything
#pragma unroll
                    for (int c = 0; c < 4; ++c) o[r][c] = fma2(two(w, w), vv[c], o[r][c]);
                }
            }
        }
        if (blocks <= 0 && more) first_k(n + 1, at_next);

        // the warps' parts
        float* to = s_o + ((n & 1) * W + warp) * R * HD;
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int off = 16; off >= LANES; off /= 2)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    o[r][c] = add2(o[r][c], __shfl_xor_sync(0xffffffffu, o[r][c], off));
                }
#pragma unroll
            for (int off = 16; off >= SAME; off /= 2) l[r] += __shfl_xor_sync(0xffffffffu, l[r], off);
            if (lane < LANES) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float4 x4;
                    of_two(o[r][2 * c], x4.x, x4.y);
                    of_two(o[r][2 * c + 1], x4.z, x4.w);
                    *reinterpret_cast<float4*>(to + r * HD + dim + 4 * c) = x4;
                }
            }
            if (lane == 0) s_end[n & 1][warp][r] = make_float2(ref[r], l[r]);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();
        const int r = (warp + W - (int)(n * R % W)) % W;  // this warp's row (in turn)
        if (r < rows) {
            const Seg& g = s_seg[n & 3];
            float top = -INFINITY, sum = 0.f;
            float4 x4 = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < W; ++w) top = fmaxf(top, s_end[n & 1][w][r].x);
            const int c = lane % (HD / 4);
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float2 e = s_end[n & 1][w][r];
                const float f = e.x == -INFINITY ? 0.f : ex2(e.x - top);  // (0 x NaN stays NaN)
                const float4 y = *reinterpret_cast<const float4*>(s_o + (((n & 1) * W + w) * R + r) * HD + 4 * c);
                sum += e.y * f;
                x4 = make_float4(x4.x + y.x * f, x4.y + y.y * f, x4.z + y.z * f, x4.w + y.w * f);
            }
            if (lane < HD / 4) {
                if (g.u0 == 0 && g.u1 == g.n) {
                    const int node = (row0 + r) / sh.group, head = g.kvh * sh.group + row0 + r - node * sh.group;
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;
                    T* out = (T*)a.out + (int64_t)(g.q.r0 + node) * a.out_stride + head * HD + 4 * c;
                    x4 = make_float4(x4.x * inv, x4.y * inv, x4.z * inv, x4.w * inv);
                    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(out) = x4;
                    else *reinterpret_cast<uint2*>(out) = make_uint2(pack2(x4.x, x4.y, T()), pack2(x4.z, x4.w, T()));
                } else {
                    const int slot = n ? 1 : 0;
                    a.part[((size_t)(cta * 2 + slot) * (HD / 4) + c) * kTile + r] = x4;
                    if (lane == 0) {
                        float* st = a.stats + (size_t)(cta * 2 + slot) * 2 * kTile + r;
                        st[0] = top;
                        st[kTile] = sum;
                    }
                }
            }
            if (r == 0 && lane == 0 && g.u1 < g.n) {
                Cut cut;
                holders(g, s_units, s_ctas, cut.first, cut.last, cut.first_slot);
                cut.row0 = row0;
                cut.rows = rows;
                cut.r0 = g.q.r0;
                cut.kvh = g.kvh;
                cut.pad = 0;
                a.cuts[cta] = cut;
            }
        }
#pragma unroll
        for (int k = 0; k < PIECES; ++k) at[k] = at_next[k];
    }
}

template <int HD, int R>
constexpr size_t few_bytes() { return 2 * (kThreadsOf<R> / 32) * R * HD * sizeof(float); }

template <typename T, int HD>
int launch_hd(const char* call, const AttnOpArgs& a, void* stream) {
    const dim3 grid((unsigned)a.grid);
    if (a.tile == 1) return launch(call, few_kernel<T, HD, 1>, grid, kThreadsOf<1>, few_bytes<HD, 1>(), stream, a);
    return launch(call, few_kernel<T, HD, 2>, grid, kThreadsOf<2>, few_bytes<HD, 2>(), stream, a);
}
template <typename T>
int launch_type(const char* call, const AttnOpArgs& a, int hd, void* stream) {
    return hd == 64 ? launch_hd<T, 64>(call, a, stream) : launch_hd<T, 128>(call, a, stream);
}
}  // namespace

int launch_few(const char* call, const AttnOpArgs& a, int dtype, int hd, void* stream) {
    if (dtype == SSD_F32) return launch_type<float>(call, a, hd, stream);
    if (dtype == SSD_F16) return launch_type<f16>(call, a, hd, stream);
    return launch_type<bf16>(call, a, hd, stream);
}

}  // namespace tree
}  // namespace ssd
