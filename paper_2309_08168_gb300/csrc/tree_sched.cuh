// tree_sched.cuh - how ssd_tree_attention's work is spread over its CTAs.
//
// An item is a tile of query rows of one request against one KV head; a unit is
// kUnit positions of its cache.  Items stand in a row - request by request, KV head
// by KV head, tile by tile - and their units are cut into equal ranges, one per
// CTA, whatever the lengths are.  An item counts kItemCost units more than it has,
// in front of them: the time that its q, first scores and output take (16 requests of 32 heads,
// 262 to 2100 positions each, one row a tile: 64 us, with none 72, one 68, five 65; 1024 items of 90 to 270
// positions, 9 fp32 rows: 74 us when it was chosen, with two 76).  An item that lies in one CTA's range is finished there;
// one that a range end cuts leaves a partial sum per CTA, joined afterwards in
// the order of the CTAs.  A CTA has at most two of those: the item that its range
// starts in and the one that it ends in.
//
// Row r of a request and KV head is node r / group, query head r % group of the
// head's group.
#pragma once

#include <stdint.h>

#include "ssd_internal.cuh"

namespace ssd {
namespace tree {

constexpr int kUnit = 128;  // positions
constexpr int kItemCost = 3;

struct Shape {
    int n_requests, n_rows, max_blocks, page_size, n_kv_heads, group, chain;
    const int32_t *row_start, *lens;
};
__host__ __device__ __forceinline__ int sched_load(const int32_t* p) {
#ifdef __CUDA_ARCH__
    return __ldcg(p);
#else
    return *p;
#endif
}

// A request; rows stay inside [0, n_rows) whatever row_start holds.
struct Req {
    int r0, n, len;  // first row, rows (0: nothing to do), cached positions
    int total;       // positions that its rows may see
    int clipped;     // some are not in the table
};
__host__ __device__ __forceinline__ Req req_of(const Shape& s, int b) {
    Req q;
    int e = sched_load(s.row_start + b + 1);
    q.r0 = sched_load(s.row_start + b);
    q.len = sched_load(s.lens + b);
    q.r0 = q.r0 < 0 ? 0 : q.r0 > s.n_rows ? s.n_rows : q.r0;
    e = e < q.r0 ? q.r0 : e > s.n_rows ? s.n_rows : e;
    q.n = q.len < 0 ? 0 : e - q.r0;
    const long long most = (1ll << 31) - 2 * kUnit, cap = (long long)s.max_blocks * s.page_size;
    const long long room = cap < most ? cap : most, want = (long long)q.len + q.n;
    q.clipped = want > room;
    q.total = (int)(want < room ? want : room);
    return q;
}
__host__ __device__ __forceinline__ int tiles_of(const Shape& s, const Req& q, int tile) {
    return (q.n * s.group + tile - 1) / tile;
}
// units of a tile: of a chain, up to the position of its last row
__host__ __device__ __forceinline__ int units_of(const Shape& s, const Req& q, int tile, int mt) {
    int keys = q.total;
    if (s.chain) {
        const int row = (mt + 1) * tile - 1, last = s.group == 1 ? row : row / s.group;  // the tile's last node
        const long long seen = (long long)q.len + (last < q.n - 1 ? last : q.n - 1) + 1;
        if (seen < keys) keys = (int)seen;
    }
    return (keys + kUnit - 1) / kUnit;
}
// units of one KV head of a request, with what its items count more.  (No unrolling, here and
// below: these run once or a few times in a CTA's life, and their instructions come from
// L2 at first use.)
__host__ __device__ __forceinline__ long long head_units(const Shape& s, const Req& q, int tile) {
    const int n = tiles_of(s, q, tile);
    if (!s.chain) return (long long)n * (n ? units_of(s, q, tile, 0) + kItemCost : 0);
    long long u = (long long)n * kItemCost;
#pragma unroll 1
    for (int mt = 0; mt < n; ++mt) u += units_of(s, q, tile, mt);
    return u;
}

// CTAs that take part, the first unit of a CTA's range, the CTA that a unit belongs to
__host__ __device__ __forceinline__ int ctas_of(long long units, int grid) {
    return units < 1 ? 1 : units < grid ? (int)units : grid;
}
// (in 32 bits where that is enough: a 64-bit division is some 100 instructions)
__host__ __device__ __noinline__ inline long long range_start(long long units, int ctas, int c) {
    const long long x = units * c;
    return x >> 32 ? x / ctas : (long long)((uint32_t)x / (uint32_t)ctas);
}
__host__ __device__ __noinline__ inline int cta_of(long long units, int ctas, long long u) {
    const long long x = (u + 1) * ctas - 1;
    return (x | units) >> 32 ? (int)(x / units) : (int)((uint32_t)x / (uint32_t)units);
}

// One CTA's share of an item: units [u0, u1) of n, u0 < u1.
struct Seg {
    int b, kvh, mt, u0, u1, n;
    long long item;  // of all units, the first that the item counts
    Req q;
};
// A walk through a CTA's range.
struct Walk {
    int b, kvh, mt, u;  // u: units of the item before the range, counted ones too
    long long at, left;
    Req q;
};
// `off`: units of request b (q; `per` for each KV head) before the range [at, at + left)
__host__ __device__ __forceinline__ void walk_init(Walk& w, const Shape& s, int tile, int b, const Req& q, long long off, long long at, long long left, long long per) {
    w.at = at;
    w.left = left;
    if (left <= 0) return;
    w.b = b;
    w.q = q;
    w.kvh = (off | per) >> 32 ? (int)(off / per) : (int)((uint32_t)off / (uint32_t)per);
    off -= w.kvh * per;
    w.mt = 0;
#pragma unroll 1
    for (int n; off >= (n = units_of(s, w.q, tile, w.mt) + kItemCost); ++w.mt) off -= n;
    w.u = (int)off;
}
__host__ __device__ __forceinline__ void walk_init(Walk& w, const Shape& s, int tile, int b, const Req& q, long long off, long long at, long long left) {
    walk_init(w, s, tile, b, q, off, at, left, head_units(s, q, tile));
}
__host__ __device__ __forceinline__ bool walk_next(Walk& w, const Shape& s, int tile, Seg& g) {
#pragma unroll 1
    while (w.left > 0) {
        const int n = units_of(s, w.q, tile, w.mt), rest = n + kItemCost - w.u;
        const int take = rest < w.left ? rest : (int)w.left, from = w.u - kItemCost, to = from + take;
        g.b = w.b;
        g.kvh = w.kvh;
        g.mt = w.mt;
        g.q = w.q;
        g.n = n;
        g.u0 = from > 0 ? from : 0;
        g.u1 = to;
        g.item = w.at - w.u;
        w.at += take;
        w.left -= take;
        w.u = 0;
        if (w.left > 0 && ++w.mt == tiles_of(s, w.q, tile)) {
            w.mt = 0;
            if (++w.kvh == s.n_kv_heads) {
                w.kvh = 0;
#pragma unroll 1
                do w.q = req_of(s, ++w.b);
                while (w.q.n == 0);  // (units are left, so there is one)
            }
        }
        if (to > 0) return true;  // (else the range ends before the item's units)
    }
    return false;
}
// The CTAs that hold parts of a segment's item, and whether the first one's is its
// first segment (the others' is).
__host__ __device__ __forceinline__ void holders(const Seg& g, long long units, int ctas, int& first, int& last, int& later) {
    first = cta_of(units, ctas, g.item + kItemCost);
    last = cta_of(units, ctas, g.item + kItemCost + g.n - 1);
    later = range_start(units, ctas, first) < g.item;
}

}  // namespace tree
}  // namespace ssd
