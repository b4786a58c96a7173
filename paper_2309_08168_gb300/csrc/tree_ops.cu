// tree_ops.cu - the parts of a tree round around its attention (ssd_ops.h):
// pages, slots, positions and masks of a round's rows (ssd_tree_plan), rotary
// positions with the write of keys and values (ssd_rope_kv), and the walk along
// the accepted path with the move of its keys and values (ssd_tree_commit).
#include <algorithm>
#include <cmath>

#include "tree_ops.cuh"

namespace ssd {
namespace tree {
namespace {

// ---------------------------------------------------------------------------
// ssd_tree_plan
// ---------------------------------------------------------------------------
constexpr int kPlanThreads = 128, kNodesPerThread = kMaxNodes / kPlanThreads;

struct PlanArgs {
    int n_requests, n_rows, max_blocks, page_size, n_pages, words;
    const int32_t *row_start, *lens, *parents, *held;
    int32_t *block_table, *held_out, *ring;
    const int64_t* ends;
    int64_t* ends_out;
    int32_t *slots, *positions;
    uint64_t* masks;
    int32_t* status;
};

// what a request needs beyond what it holds, and gives back
struct Want {
    int len, held, fresh, back;
    bool live, fits;
};
__device__ __forceinline__ Want want_of(const PlanArgs& a, int b, const Rows& rows) {
    Want w;
    w.len = __ldcg(a.lens + b);
    w.held = min(max(__ldcg(a.held + b), 0), a.max_blocks);
    w.live = w.len >= 0;
    // (divided in 32 bits; what needs more does not fit, as a cache has less than 2^31 positions)
    const unsigned long long last = (unsigned long long)(w.live ? w.len : 0) + (unsigned)rows.n + (unsigned)a.page_size - 1u;
    const unsigned need = !w.live ? 0u : last >> 32 ? 0xffffffffu : (unsigned)last / (unsigned)a.page_size;
    w.fits = need <= (unsigned)a.max_blocks;
    w.fresh = w.live && w.fits ? max((int)need - w.held, 0) : 0;
    w.back = w.live ? 0 : w.held;
    return w;
}

// One CTA per request; a chain's rows are shared by gridDim.y of them.  Bound by latency: a request's place in the queue of free pages
// is a sum over those before it, which every CTA forms for itself (three words a
// request, from L2, all threads at once) rather than wait for another launch, while its own
// rows' parents are on their way; masks and depths of a tree come from pointer
// doubling: after step s a node knows its ancestors up to 2^s levels above.
// 128 threads, so that a thousand requests run at once: with 256, and a scan over
// all requests in every CTA, 1000 trees of 33 to 64 nodes took 19.0 us; now 12.0 (0.9 MB, 0.08 TB/s), one
// tree of 5 nodes 4.3.  A chain of 8191 rows: one CTA 24.3, shared 5.5.
__global__ void __launch_bounds__(kPlanThreads, 10) plan_kernel(const PlanArgs a) {
    __shared__ long long s_sum[2][kPlanThreads / 32], s_top[kPlanThreads / 32];
    __shared__ int s_up[kMaxNodes], s_depth[kMaxNodes];
    __shared__ uint64_t s_mask[4][kMaxNodes];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, b = blockIdx.x;
    pdl_launch_dependents();
    pdl_wait();
    const Rows rows = rows_of(a.row_start, b, a.n_rows);
    const int nodes = a.parents ? min(rows.n, 64 * a.words) : 0;
    int up[kNodesPerThread];
#pragma unroll
    for (int k = 0; k < kNodesPerThread; ++k) {
        const int i = tid + k * kPlanThreads;
        up[k] = i < nodes ? __ldcg(a.parents + rows.r0 + i) : -1;
    }
    const Want w = want_of(a, b, rows);
    long long sums[2] = {0, 0};  // pages taken and given back by the requests before
#pragma unroll 2
    for (int i = tid; i < b; i += kPlanThreads) {
        const Want o = want_of(a, i, rows_of(a.row_start, i, a.n_rows));
        sums[0] += o.fresh;
        sums[1] += o.back;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sums[k] += __shfl_xor_sync(0xffffffffu, sums[k], o);
        if (lane == 0) s_sum[k][warp] = sums[k];
    }
    const long long head = __ldcg(a.ends), tail = __ldcg(a.ends + 1);
    const long long avail = min(max(tail - head, 0ll), (long long)a.n_pages);
    __syncthreads();
    long long first = 0, returned = 0;
#pragma unroll
    for (int k = 0; k < kPlanThreads / 32; ++k) first += s_sum[0][k], returned += s_sum[1][k];
    const bool given = w.live && w.fits && (w.fresh == 0 || first + w.fresh <= avail);
    // ring[(head + x) mod n_pages]; x stays below n_pages where the counts are sound
    const int h0 = (int)(((head % a.n_pages) + a.n_pages) % a.n_pages), t0 = (int)(((tail % a.n_pages) + a.n_pages) % a.n_pages);
    auto ring_at = [&](int base, long long x) {
        const long long y = base + x;
        return (int)(y < a.n_pages ? y : y < 2ll * a.n_pages ? y - a.n_pages : y % a.n_pages);
    };
    int32_t* table = a.block_table + (size_t)b * a.max_blocks;
    if (tid == 0 && blockIdx.y == 0) {
        a.held_out[b] = !w.live ? 0 : given ? w.held + w.fresh : w.held;
        if (w.live && !w.fits) say(a.status, SSD_STATUS_TABLE);
        if (w.live && w.fits && !given) say(a.status, SSD_STATUS_PAGES);
    }
    if (given && blockIdx.y == 0)
        for (int j = tid; j < w.fresh; j += kPlanThreads) table[w.held + j] = __ldcg(a.ring + ring_at(h0, first + j));
    if (!w.live && blockIdx.y == 0)
        for (int j = tid; j < w.back; j += kPlanThreads) a.ring[ring_at(t0, returned + j)] = __ldcg(table + j);

    // the rows: depths and masks of a tree first
    if (a.parents && rows.n > 0) {
        bool bad = tid == 0 && rows.n > nodes;
#pragma unroll
        for (int k = 0; k < kNodesPerThread; ++k) {
            const int i = tid + k * kPlanThreads;
            if (up[k] < -1 || up[k] >= i) {
                bad = true;
                up[k] = -1;
            }
            s_up[i] = up[k];
            s_depth[i] = up[k] >= 0;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint64_t m = 0;
                if (i < nodes && i >> 6 == q) m |= 1ull << (i & 63);
                if (up[k] >= 0 && up[k] >> 6 == q) m |= 1ull << (up[k] & 63);
                if (q < a.words) s_mask[q][i] = m;
            }
        }
        if (bad) say(a.status, SSD_STATUS_PARENT);
        // (a node's words hold itself and the next 2^s ancestors, s_up the one after those)
        auto more = [&] {
            bool any = false;
#pragma unroll
            for (int k = 0; k < kNodesPerThread; ++k) any = any || up[k] >= 0;
            return any;
        };
        while (__syncthreads_or(more())) {
            uint64_t m[kNodesPerThread][4];
            int d[kNodesPerThread], next[kNodesPerThread];
#pragma unroll
            for (int k = 0; k < kNodesPerThread; ++k)
                if (up[k] >= 0) {
                    next[k] = s_up[up[k]];
                    d[k] = s_depth[up[k]];
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (q < a.words) m[k][q] = s_mask[q][up[k]];
                }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kNodesPerThread; ++k)
                if (up[k] >= 0) {
                    const int i = tid + k * kPlanThreads;
                    s_up[i] = next[k];
                    s_depth[i] += d[k];
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (q < a.words) s_mask[q][i] |= m[k][q];
                    up[k] = next[k];
                }
        }
    }
#pragma unroll 2
    for (int i = blockIdx.y * kPlanThreads + tid; i < rows.n; i += kPlanThreads * gridDim.y) {
        const unsigned at = (unsigned)w.len + (unsigned)i;
        int slot = -1;
        if (given) {
            const int j = (int)(at / (unsigned)a.page_size);  // < the pages needed <= max_blocks
            const int page = j < w.held ? __ldcg(table + j) : __ldcg(a.ring + ring_at(h0, first + j - w.held));
            if (page >= 0 && page < a.n_pages) slot = page * a.page_size + (int)(at - (unsigned)j * (unsigned)a.page_size);
        }
        a.slots[rows.r0 + i] = slot;
        a.positions[rows.r0 + i] = a.parents ? w.len + (i < nodes ? s_depth[i] : 0) : (int)at;
        if (a.parents)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k < a.words) a.masks[(size_t)(rows.r0 + i) * a.words + k] = i < nodes ? s_mask[k][i] : 0ull;
    }
    if (b || blockIdx.y) return;
    // The first CTA also leaves the queue's new ends: the pages taken are the largest sum over
    // the first requests, in order, that the queue covers (a run of requests per thread).
    const int per = (a.n_requests + kPlanThreads - 1) / kPlanThreads;
    const int b0 = min(tid * per, a.n_requests), b1 = min(b0 + per, a.n_requests);
    long long fresh = 0, back = 0;
    for (int i = b0; i < b1; ++i) {
        const Want o = want_of(a, i, rows_of(a.row_start, i, a.n_rows));
        fresh += o.fresh;
        back += o.back;
    }
    long long run = fresh;  // inclusive over the warp, then exclusive over the block
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += x;
        back += __shfl_xor_sync(0xffffffffu, back, o);
    }
    __syncthreads();
    if (lane == 31) s_sum[0][warp] = run;
    if (lane == 0) s_sum[1][warp] = back;
    __syncthreads();
    run -= fresh;
    for (int k = 0; k < warp; ++k) run += s_sum[0][k];
    long long top = 0;
    for (int i = b0; i < b1; ++i) {
        run += want_of(a, i, rows_of(a.row_start, i, a.n_rows)).fresh;
        if (run <= avail) top = run;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (lane == 0) s_top[warp] = top;
    __syncthreads();
    if (tid == 0) {
        long long total = 0;
        top = 0;
        for (int k = 0; k < kPlanThreads / 32; ++k) {
            top = max(top, s_top[k]);
            total += s_sum[1][k];
        }
        a.ends_out[0] = head + top;
        a.ends_out[1] = tail + total;
    }
}

// ---------------------------------------------------------------------------
// ssd_rope_kv
// ---------------------------------------------------------------------------
constexpr int kRopeThreads = 128;

struct RopeArgs {
    const void *q, *k, *v;
    void* q_out;
    int64_t q_stride, k_stride, v_stride, q_out_stride;  // elements
    const int32_t *positions, *slots;
    void *kc, *vc;  // the layer's cache
    int64_t page_stride, head_stride, pos_stride;
    int n_heads, n_kv_heads, hd, page_size, n_pages;
    ssd_rope rope;
};

// A CTA takes a row (blockIdx.x), or with gridDim.y > 1 a share of its heads.  A thread has
// one place in a head - 16 bytes, or the two halves of 16 bytes of pairs - and goes
// through the heads, kRopeAhead at a time, all loads before the first store: the kernel is
// bound by HBM (or L2) and by the loads under way.  Measured: 8191 fp16 rows of 32 + 2 x 32 heads of
// 128 71 us (402 MB, 5.7 TB/s, 84 % of the copy rate); 400 bf16 rows of 64 + 2 x 8 heads, in L2, 5.3
// us (3.1 TB/s); one row 2.4.
//
// The angle of pair i at position p is p f_i.  f_i / 2 pi is held as a fraction
// of 2^64, so the product modulo 2^64 is the angle's fraction of a turn exactly,
// at any position; fp32 (p f_i) would be off by 0.06 radians at p = 10^6.
//
// Of two CTAs that write one cache row nothing orders the stores.  In calls of up to kLastStays rows a CTA compares its slot with those of the rows
// behind it, one a thread, and leaves the cache alone if one has it (33 fp16 rows of 32 + 2 x 8 heads 3.1 us, without 2.8; one row and
// large calls the same).
//
// T: rows, C: cache
constexpr int kRopeAhead = 4, kLastStays = 129;
static_assert(kRopeThreads >= kLastStays - 1, "a thread for each row behind the first");
template <typename T, typename C>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const __grid_constant__ RopeArgs a) {
    constexpr int V = Vec<T>::N;
    __shared__ float2 s_cs[64];
    pdl_launch_dependents();
    pdl_wait();
    const int row = blockIdx.x, half = a.rope.rot_dim / 2;
    const int slot = __ldcg(a.slots + row);
    if (threadIdx.x < half) {
        const uint64_t turn = (uint64_t)(int64_t)__ldcg(a.positions + row) * a.rope.turns[threadIdx.x];
        float s, c;
        sincospif((float)((int64_t)turn >> 32) * 0x1p-31f, &s, &c);
        s_cs[threadIdx.x] = make_float2(c * a.rope.amplitude, s * a.rope.amplitude);
    }
    auto later_has_it = [&]() {
        const int n_rows = gridDim.x, other = row + 1 + (int)threadIdx.x;
        if (n_rows == 1 || n_rows > kLastStays) return false;
        return __syncthreads_or(other < n_rows && __ldcg(a.slots + other) == slot) != 0;
    };
    const bool cached = !later_has_it() && slot >= 0 && slot < a.n_pages * a.page_size;
    const int64_t at = cached ? (int64_t)(slot / a.page_size) * a.page_stride + (int64_t)(slot % a.page_size) * a.pos_stride : 0;
    auto to_cache = [&](void* base, int head, int e, const float (&f)[V]) {
        C* p = (C*)base + at + (int64_t)head * a.head_stride + e;
        if constexpr (V == 8) *reinterpret_cast<uint4*>(p) = Vec<C>::put(f);
        else *reinterpret_cast<uint2*>(p) = make_uint2(pack2(f[0], f[1], C()), pack2(f[2], f[3], C()));
    };
    const int lines = kRopeThreads * gridDim.y, line = blockIdx.y * kRopeThreads + threadIdx.x;  // threads of the row
    // values first: they need no angles
    const int n_pass = a.hd / V;
    if (cached) {
        const int c = line % n_pass, step = lines / n_pass;
        const T* v = (const T*)a.v + (int64_t)row * a.v_stride + c * V;
        for (int h = line / n_pass; h < a.n_kv_heads; h += kRopeAhead * step) {
            uint4 x[kRopeAhead];
#pragma unroll
            for (int i = 0; i < kRopeAhead; ++i)
                if (h + i * step < a.n_kv_heads) x[i] = __ldcg(reinterpret_cast<const uint4*>(v + (h + i * step) * a.hd));
#pragma unroll
            for (int i = 0; i < kRopeAhead; ++i)
                if (h + i * step < a.n_kv_heads) {
                    float f[V];
                    Vec<T>::get(x[i], f);
                    to_cache(a.vc, h + i * step, c * V, f);
                }
        }
    }
    __syncthreads();
    // queries and keys, heads 0 .. n_heads - 1 and n_heads .. ; a head's pairs first, then what passes
    const int n_pair = a.rope.interleaved ? a.rope.rot_dim / V : half / V, n_rot = n_pair + (a.hd - a.rope.rot_dim) / V;
    const int c = line % n_rot, step = lines / n_rot, heads = a.n_heads + (cached ? a.n_kv_heads : 0);
    if (line >= step * n_rot) return;  // (no whole head is left for these threads)
    const bool pair = c < n_pair, two = pair && !a.rope.interleaved;
    const int e = pair ? c * V : a.rope.rot_dim + (c - n_pair) * V;
    const T* q = (const T*)a.q + (int64_t)row * a.q_stride + e;
    const T* k = (const T*)a.k + (int64_t)row * a.k_stride + e;
    T* qo = (T*)a.q_out + (int64_t)row * a.q_out_stride + e;
    for (int h0 = line / n_rot; h0 < heads; h0 += kRopeAhead * step) {
        uint4 x[kRopeAhead], y[kRopeAhead];
#pragma unroll
        for (int i = 0; i < kRopeAhead; ++i) {
            const int h = h0 + i * step;
            if (h < heads) {
                const T* src = h < a.n_heads ? q + (int64_t)h * a.hd : k + (int64_t)(h - a.n_heads) * a.hd;
                x[i] = __ldcg(reinterpret_cast<const uint4*>(src));
                if (two) y[i] = __ldcg(reinterpret_cast<const uint4*>(src + half));
            }
        }
#pragma unroll
        for (int i = 0; i < kRopeAhead; ++i) {
            const int h = h0 + i * step;
            if (h >= heads) break;
            auto store = [&](int more, const float (&f)[V]) {
                if (h < a.n_heads) *reinterpret_cast<uint4*>(qo + (int64_t)h * a.hd + more) = Vec<T>::put(f);
                else to_cache(a.kc, h - a.n_heads, e + more, f);
            };
            float f[V];
            Vec<T>::get(x[i], f);
            if (two) {
                float g[V], o[V], p[V];
                Vec<T>::get(y[i], g);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float2 cs = s_cs[c * V + j];
                    o[j] = f[j] * cs.x - g[j] * cs.y;
                    p[j] = g[j] * cs.x + f[j] * cs.y;
                }
                store(0, o);
                store(half, p);
            } else if (pair) {
                float o[V];
#pragma unroll
                for (int j = 0; j < V / 2; ++j) {
                    const float2 cs = s_cs[c * (V / 2) + j];
                    o[2 * j] = f[2 * j] * cs.x - f[2 * j + 1] * cs.y;
                    o[2 * j + 1] = f[2 * j + 1] * cs.x + f[2 * j] * cs.y;
                }
                store(0, o);
            } else {
                store(0, f);
            }
        }
    }
}

// ---------------------------------------------------------------------------
// ssd_tree_commit
// ---------------------------------------------------------------------------
constexpr int kCommitThreads = 256, kCommitAhead = 4, kCommitColumns = 2;
static_assert(kCommitThreads >= kMaxNodes, "a thread per node");

struct CommitArgs {
    int n_rows, max_blocks;
    const int32_t *row_start, *lens, *block_table, *parents, *tokens, *target;
    int32_t *accepted, *next_token, *lens_out, *path, *emitted;
    void *kc, *vc;  // nullptr: no cache
    int n_layers, n_pages, page_size, n_kv_heads, chunks;  // chunks: 16-byte pieces of a head
    int64_t layer_stride, page_stride, head_stride, pos_stride;
};

// A request's CTAs (gridDim.y) each walk its path - a warp, eight nodes a lane -
// and move their share of (K or V, layer, head, 16 bytes) columns.  A thread takes two
// columns along the whole path in order, four rows at a time: path[j] >= j and
// the path rises, so nothing is overwritten before it is read.  Measured: 48 trees of
// 64 nodes, 32 layers of 8 heads of 128 12.5 us (44 MB with the accepted paths, 3.5 TB/s: bound by the
// chain path - page - rows of a few thousand scattered 16-byte columns); one tree 2.8 us.
__global__ void __launch_bounds__(kCommitThreads) commit_kernel(const CommitArgs a) {
    __shared__ int s_parent[kMaxNodes], s_token[kMaxNodes], s_target[kMaxNodes], s_path[kMaxNodes], s_n;
    __shared__ int64_t s_off[kMaxNodes];  // cache row at lens + i, -1: none
    const int b = blockIdx.x, tid = threadIdx.x;
    pdl_launch_dependents();
    pdl_wait();
    const Rows rows = rows_of(a.row_start, b, a.n_rows);
    const int len = __ldcg(a.lens + b), nodes = min(rows.n, kMaxNodes);
    if (nodes == 0 || len < 0) {
        if (blockIdx.y == 0 && tid == 0) {
            a.accepted[b] = -1;
            a.next_token[b] = -1;
            a.lens_out[b] = len;
        }
        return;
    }
    if (tid < nodes) {
        s_parent[tid] = a.parents ? __ldcg(a.parents + rows.r0 + tid) : tid - 1;
        s_token[tid] = __ldcg(a.tokens + rows.r0 + tid);
        s_target[tid] = __ldcg(a.target + rows.r0 + tid);
        int64_t off = -1;
        if (a.kc) {
            const long long at = (long long)len + tid, j = at / a.page_size;
            if (j < a.max_blocks) {
                const int page = __ldcg(a.block_table + (size_t)b * a.max_blocks + j);
                if (page >= 0 && page < a.n_pages) off = page * a.page_stride + (at - j * a.page_size) * a.pos_stride;
            }
        }
        s_off[tid] = off;
    }
    __syncthreads();
    if (tid < 32) {
        int cur = 0, n = 0;
        if (tid == 0) s_path[0] = 0;
        for (;;) {
            const int want = s_target[cur];
            unsigned best = 0xffffffffu;
#pragma unroll
            for (int k = kMaxNodes / 32 - 1; k >= 0; --k) {
                const int i = tid + 32 * k;
                if (i > cur && i < nodes && s_parent[i] == cur && s_token[i] == want) best = (unsigned)i;
            }
            best = __reduce_min_sync(0xffffffffu, best);
            if (best == 0xffffffffu) break;
            cur = (int)best;
            ++n;
            if (tid == 0) s_path[n] = cur;
        }
        if (tid == 0) s_n = n;
    }
    __syncthreads();
    const int n = s_n;
    if (blockIdx.y == 0) {
        const int next = s_target[s_path[n]];
        if (tid <= n) {
            a.path[rows.r0 + tid] = s_path[tid];
            a.emitted[rows.r0 + tid] = tid < n ? s_token[s_path[tid + 1]] : next;
        }
        if (tid == 0) {
            a.accepted[b] = n;
            a.next_token[b] = next;
            a.lens_out[b] = len + 1 + n;
        }
    }
    if (!a.kc) return;
    const unsigned per_layer = 2u * a.n_kv_heads * a.chunks, per_kv = (unsigned)(a.n_kv_heads * a.chunks);
    const unsigned columns = (unsigned)a.n_layers * per_layer, lines = gridDim.y * kCommitThreads;
    for (unsigned col = blockIdx.y * kCommitThreads + tid; col < columns; col += kCommitColumns * lines) {
        char* base[kCommitColumns];
#pragma unroll
        for (int k = 0; k < kCommitColumns; ++k) {
            const unsigned x = min(col + k * lines, columns - 1);
            const unsigned layer = x / per_layer, r = x - layer * per_layer, kv = r >= per_kv, r2 = r - kv * per_kv;
            const unsigned head = r2 / (unsigned)a.chunks, c = r2 - head * (unsigned)a.chunks;
            base[k] = (char*)(kv ? a.vc : a.kc) + 2 * (layer * a.layer_stride + head * a.head_stride + c * 8);
        }
        for (int j = 1; j <= n; j += kCommitAhead) {
            uint4 x[kCommitColumns][kCommitAhead];
            int64_t src[kCommitAhead], dst[kCommitAhead];
#pragma unroll
            for (int i = 0; i < kCommitAhead; ++i) {
                src[i] = dst[i] = -1;
                if (j + i <= n && s_path[j + i] != j + i) src[i] = s_off[s_path[j + i]], dst[i] = s_off[j + i];
                if (src[i] >= 0)
#pragma unroll
                    for (int k = 0; k < kCommitColumns; ++k)
                        if (col + k * lines < columns) x[k][i] = __ldcg(reinterpret_cast<const uint4*>(base[k] + 2 * src[i]));
            }
#pragma unroll
            for (int i = 0; i < kCommitAhead; ++i)
                if (src[i] >= 0 && dst[i] >= 0)
#pragma unroll
                    for (int k = 0; k < kCommitColumns; ++k)
                        if (col + k * lines < columns) *reinterpret_cast<uint4*>(base[k] + 2 * dst[i]) = x[k][i];
        }
    }
}

}  // namespace
}  // namespace tree
}  // namespace ssd

using namespace ssd;
using namespace ssd::tree;

extern "C" int ssd_tree_plan(const ssd_batch* batch, int page_size, int n_pages, const int32_t* parents, const int32_t* held,
                             int32_t* held_out, int32_t* ring, const int64_t* ends, int64_t* ends_out, int32_t* slots,
                             int32_t* positions, uint64_t* masks, int mask_words, int32_t* status, void* cuda_stream) {
    static const char call[] = "ssd_tree_plan";
    if (int rc = check_batch(call, batch)) return rc;
    if (int rc = check_page_size(call, page_size, n_pages)) return rc;
    if (!held || !held_out || !ring || !ends || !ends_out) return refuse_arg(call, "NULL pointer");
    if (held == held_out || ends == ends_out) return refuse_arg(call, "held_out and ends_out must be arrays of their own");
    if (batch->n_rows > 0 && (!slots || !positions)) return refuse_arg(call, "slots and positions must not be NULL");
    if (parents ? mask_words < 1 || mask_words > 4 || (batch->n_rows > 0 && !masks) : mask_words != 0 || masks != nullptr)
        return refuse_arg(call, "trees need masks and 1 <= mask_words <= 4, chains (parents = NULL) neither");
    if (int rc = check_device(call, batch->lens)) return rc;
    PlanArgs a{};
    a.n_requests = batch->n_requests;
    a.n_rows = batch->n_rows;
    a.max_blocks = batch->max_blocks;
    a.page_size = page_size;
    a.n_pages = n_pages;
    a.words = mask_words;
    a.row_start = batch->row_start;
    a.lens = batch->lens;
    a.parents = parents;
    a.held = held;
    a.block_table = batch->block_table;
    a.held_out = held_out;
    a.ring = ring;
    a.ends = ends;
    a.ends_out = ends_out;
    a.slots = slots;
    a.positions = positions;
    a.masks = masks;
    a.status = status;
    // a tree is one CTA's (its threads are its nodes), a chain's rows are several CTAs', four a thread
    const int lines = parents ? 1 : (int)std::min(64ll, ((long long)batch->max_rows + 4 * kPlanThreads - 1) / (4 * kPlanThreads));
    return launch(call, plan_kernel, dim3((unsigned)a.n_requests, (unsigned)lines), kPlanThreads, 0, cuda_stream, a);
}

extern "C" int ssd_rope_init(int rot_dim, int interleaved, int scaling, double theta, double factor, double original_len,
                             double slow, double fast, double amplitude, ssd_rope* out) {
    static const char call[] = "ssd_rope_init";
    if (!out) return refuse_arg(call, "NULL pointer");
    if (rot_dim < 16 || rot_dim > 128 || rot_dim % 16) return refuse_arg(call, "rot_dim must be a multiple of 16, 16 .. 128");
    if (interleaved != 0 && interleaved != 1) return refuse_arg(call, "interleaved must be 0 or 1");
    if (scaling < SSD_ROPE_PLAIN || scaling > SSD_ROPE_BY_PARTS) return refuse_arg(call, "unknown scaling");
    if (!(theta > 1.0) || !std::isfinite(theta) || !(factor >= 1.0) || !std::isfinite(factor) || !(amplitude > 0.0) ||
        !std::isfinite((float)amplitude))
        return refuse_arg(call, "need theta > 1, factor >= 1 and amplitude > 0, all finite");
    if (scaling == SSD_ROPE_BY_PARTS &&
        (!(original_len >= 1.0) || !std::isfinite(original_len) || !(slow >= 0.0) || !(fast > slow) || !std::isfinite(fast)))
        return refuse_arg(call, "scaling by parts needs original_len >= 1 and 0 <= slow < fast");
    ssd_rope r{};
    r.rot_dim = rot_dim;
    r.interleaved = interleaved;
    r.amplitude = (float)amplitude;
    const double two_pi = 6.283185307179586476925;
    for (int i = 0; i < rot_dim / 2; ++i) {
        double t = std::pow(theta, -2.0 * i / rot_dim) / two_pi;  // turns a position, < 1/6
        if (scaling == SSD_ROPE_LINEAR) t /= factor;
        if (scaling == SSD_ROPE_BY_PARTS) {
            const double g = std::fmin(std::fmax((original_len * t - slow) / (fast - slow), 0.0), 1.0);
            t *= g + (1.0 - g) / factor;
        }
        r.turns[i] = (uint64_t)std::nearbyint(std::ldexp(t, 64));
    }
    *out = r;
    return SSD_OK;
}

extern "C" int ssd_rope_kv(const ssd_pages* cache, int layer, const ssd_rope* rope, int dtype, int n_rows, int n_heads,
                           const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                           const int32_t* positions, const int32_t* slots, void* q_out, int64_t q_out_stride,
                           void* cuda_stream) {
    static const char call[] = "ssd_rope_kv";
    if (int rc = check_pages(call, cache)) return rc;
    if (layer < 0 || layer >= cache->n_layers) return refuse_arg(call, "no such layer");
    if (int rc = check_rows_type(call, dtype, cache)) return rc;
    if (!rope || rope->rot_dim < 16 || rope->rot_dim % 16 || rope->rot_dim > cache->head_dim)
        return refuse_arg(call, "rope must come from ssd_rope_init, with rot_dim <= head_dim");
    if (n_rows < 0 || n_heads < 1 || n_heads > 65536) return refuse_arg(call, "need n_rows >= 0 and 1 <= n_heads <= 65536");
    if (n_rows == 0) return SSD_OK;
    if (!q || !k || !v || !positions || !slots || !q_out) return refuse_arg(call, "NULL pointer");
    const int hd = cache->head_dim;
    if (int rc = check_rows(call, "q", q, q_stride, dtype, (int64_t)n_heads * hd)) return rc;
    if (int rc = check_rows(call, "q_out", q_out, q_out_stride, dtype, (int64_t)n_heads * hd)) return rc;
    if (int rc = check_rows(call, "k", k, k_stride, dtype, (int64_t)cache->n_kv_heads * hd)) return rc;
    if (int rc = check_rows(call, "v", v, v_stride, dtype, (int64_t)cache->n_kv_heads * hd)) return rc;
    if (q == q_out && q_stride != q_out_stride) return refuse_arg(call, "q_out in q's place needs its stride");
    if (int rc = check_device(call, cache->k)) return rc;
    RopeArgs a{};
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_out = q_out;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.q_out_stride = q_out_stride;
    a.positions = positions;
    a.slots = slots;
    a.kc = (char*)cache->k + 2 * layer * cache->layer_stride;
    a.vc = (char*)cache->v + 2 * layer * cache->layer_stride;
    a.page_stride = cache->page_stride;
    a.head_stride = cache->head_stride;
    a.pos_stride = cache->pos_stride;
    a.n_heads = n_heads;
    a.n_kv_heads = cache->n_kv_heads;
    a.hd = hd;
    a.page_size = cache->page_size;
    a.n_pages = cache->n_pages;
    a.rope = *rope;
    // few rows: a row's units over several CTAs, until there are four per SM (400 rows: split in two 5.3 us,
    // whole 6.8; 200 rows: in four 3.8, two 4.6, whole 5.2, eight 5.5; 50 rows: all 3.1 to 3.7)
    const int per16 = dtype == SSD_F32 ? 4 : 8;
    const long long units = (long long)(n_heads + 2 * cache->n_kv_heads) * hd / per16;
    int split = 1;
    while (split < 64 && (long long)n_rows * split < 608 && units > (long long)kRopeThreads * split) split *= 2;
    const dim3 grid((unsigned)n_rows, (unsigned)split);
    if (dtype == SSD_F32) return launch(call, rope_kernel<float, f16>, grid, kRopeThreads, 0, cuda_stream, a);
    if (dtype == SSD_F16) return launch(call, rope_kernel<f16, f16>, grid, kRopeThreads, 0, cuda_stream, a);
    return launch(call, rope_kernel<bf16, bf16>, grid, kRopeThreads, 0, cuda_stream, a);
}

extern "C" int ssd_tree_commit(const ssd_batch* batch, const ssd_pages* cache, const int32_t* parents, const int32_t* tokens,
                               const int32_t* target, int32_t* accepted, int32_t* next_token, int32_t* lens_out, int32_t* path,
                               int32_t* emitted, void* cuda_stream) {
    static const char call[] = "ssd_tree_commit";
    if (int rc = check_batch(call, batch)) return rc;
    if (cache)
        if (int rc = check_pages(call, cache)) return rc;
    if (!accepted || !next_token || !lens_out) return refuse_arg(call, "NULL pointer");
    if (batch->n_rows > 0 && (!tokens || !target || !path || !emitted)) return refuse_arg(call, "NULL pointer");
    // (a request's CTAs each walk the path from what they read, while one of them writes the results)
    const void* const in[] = {batch->row_start, batch->lens, batch->block_table, parents, tokens, target};
    const void* const out[] = {accepted, next_token, lens_out, path, emitted};
    for (int i = 0; i < 5; ++i) {
        for (const void* p : in)
            if (out[i] && out[i] == p) return refuse_arg(call, "the results must be arrays of their own");
        for (int j = 0; j < i; ++j)
            if (out[i] && out[i] == out[j]) return refuse_arg(call, "the results must be arrays of their own");
    }
    if (int rc = check_device(call, batch->lens)) return rc;
    CommitArgs a{};
    a.n_rows = batch->n_rows;
    a.max_blocks = batch->max_blocks;
    a.row_start = batch->row_start;
    a.lens = batch->lens;
    a.block_table = batch->block_table;
    a.parents = parents;
    a.tokens = tokens;
    a.target = target;
    a.accepted = accepted;
    a.next_token = next_token;
    a.lens_out = lens_out;
    a.path = path;
    a.emitted = emitted;
    int split = 1;
    if (cache) {
        a.kc = cache->k;
        a.vc = cache->v;
        a.n_layers = cache->n_layers;
        a.n_pages = cache->n_pages;
        a.page_size = cache->page_size;
        a.n_kv_heads = cache->n_kv_heads;
        a.chunks = cache->head_dim / 8;
        a.layer_stride = cache->layer_stride;
        a.page_stride = cache->page_stride;
        a.head_stride = cache->head_stride;
        a.pos_stride = cache->pos_stride;
        const long long columns = 2ll * cache->n_layers * cache->n_kv_heads * a.chunks;
        if (columns >= (1ll << 30)) return refuse_arg(call, "need n_layers * n_kv_heads * head_dim < 2^32");
        // (48 requests: in eight 13.0 us, in four 17.4, in 16 13.5, in 32 18.4; one request: all 3.6)
        while (split < 64 && columns > (long long)kCommitThreads * split && (long long)batch->n_requests * split < 304) split *= 2;
    }
    return launch(call, commit_kernel, dim3((unsigned)batch->n_requests, (unsigned)split), kCommitThreads, 0, cuda_stream, a);
}
