// tree_attn.cu - ssd_tree_attention (ssd_ops.h): attention of a batch's rows
// over a paged cache, with the masks of their trees.
#include <cmath>

#include "tree_ops.cuh"

namespace ssd {
namespace tree {
namespace {

struct AttnOpArgs {
    int n_requests, n_rows, max_blocks, words;
    const int32_t *row_start, *lens, *block_table;
    const void* q;
    void* out;
    int64_t q_stride, out_stride;
    const uint64_t* masks;
    const void *kc, *vc;  // the layer's cache
    int64_t page_stride, head_stride, pos_stride;
    int n_heads, n_kv_heads, page_size, n_pages;
    float scale2;  // log2(e) * scale
    int32_t* status;
};

// One warp per (row, head), position by position with the running maximum and
// sum of the softmax.
template <typename T, typename C, int HD>
__global__ void __launch_bounds__(128) attn_simple_kernel(const AttnOpArgs a) {
    constexpr int E = HD / 32;
    pdl_launch_dependents();
    pdl_wait();
    const int row = blockIdx.x, head = blockIdx.y * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (head >= a.n_heads) return;
    int b = 0;
    Rows rows{0, 0};
    for (; b < a.n_requests; ++b) {
        rows = rows_of(a.row_start, b, a.n_rows);
        if (row >= rows.r0 && row < rows.r0 + rows.n) break;
    }
    if (b == a.n_requests) return;
    const int len = __ldcg(a.lens + b), node = row - rows.r0;
    if (len < 0) return;
    const long long room = (long long)a.max_blocks * a.page_size, want = (long long)len + rows.n;
    if (want > room && lane == 0) say(a.status, SSD_STATUS_TABLE);
    const long long total = min(want, room);
    const int kvh = head / (a.n_heads / a.n_kv_heads);
    const T* q = (const T*)a.q + (int64_t)row * a.q_stride + head * HD + lane * E;
    float qf[E], o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) qf[e] = (float)q[e], o[e] = 0.f;
    float mx = -INFINITY, sum = 0.f;
    for (long long x = 0; x < total; ++x) {
        if (x >= len) {
            const int j = (int)(x - len);
            if (a.masks) {
                if (j >= 64 * a.words || !(__ldcg(a.masks + (size_t)row * a.words + (j >> 6)) >> (j & 63) & 1)) continue;
            } else if (j > node) {
                break;
            }
        }
        const int blk = (int)(x / a.page_size), page = __ldcg(a.block_table + (size_t)b * a.max_blocks + blk);
        const bool has = page >= 0 && page < a.n_pages;
        const int64_t at = has ? page * a.page_stride + kvh * a.head_stride + (x - (long long)blk * a.page_size) * a.pos_stride + lane * E : 0;
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) s += qf[e] * (has ? (float)((const C*)a.kc)[at + e] : 0.f);
        s = warp_sum(s) * a.scale2;
        if (s == -INFINITY) continue;
        const float m2 = fmaxf(mx, s), f = exp2f(mx - m2), p = exp2f(s - m2);
        mx = m2;
        sum = sum * f + p;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = o[e] * f + p * (has ? (float)((const C*)a.vc)[at + e] : 0.f);
    }
    T* out = (T*)a.out + (int64_t)row * a.out_stride + head * HD + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) out[e] = (T)(sum == 0.f ? 0.f : o[e] / sum);
}

size_t workspace_need() { return 16; }

}  // namespace
}  // namespace tree
}  // namespace ssd

using namespace ssd;
using namespace ssd::tree;

extern "C" int ssd_tree_attention_workspace(int head_dim, size_t* bytes) {
    static const char call[] = "ssd_tree_attention_workspace";
    if (!bytes) return refuse_arg(call, "NULL pointer");
    if (head_dim != 64 && head_dim != 128) return refuse_arg(call, "head_dim must be 64 or 128");
    *bytes = workspace_need();
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
    if (!(scale > 0.f) || !std::isfinite(scale)) return refuse_arg(call, "scale must be positive and finite");
    if (masks ? mask_words < 1 || mask_words > 4 : mask_words != 0)
        return refuse_arg(call, "masks need 1 <= mask_words <= 4, chains (masks = NULL) 0");
    if (batch->n_rows == 0) return SSD_OK;
    if (!q || !out || !workspace) return refuse_arg(call, "NULL pointer");
    if (int rc = check_rows(call, "q", q, q_stride, dtype, (int64_t)n_heads * cache->head_dim)) return rc;
    if (int rc = check_rows(call, "out", out, out_stride, dtype, (int64_t)n_heads * cache->head_dim)) return rc;
    if (q == out) return refuse_arg(call, "out must be memory of its own");
    if ((uintptr_t)workspace & 15u) return refuse_arg(call, "the workspace must be 16-byte aligned");
    if (workspace_bytes < workspace_need()) return refuse(SSD_ERR_CAPACITY, call, "the workspace needs %zu bytes", workspace_need());
    if (int rc = check_device(call, cache->k)) return rc;
    AttnOpArgs a{};
    a.n_requests = batch->n_requests;
    a.n_rows = batch->n_rows;
    a.max_blocks = batch->max_blocks;
    a.words = mask_words;
    a.row_start = batch->row_start;
    a.lens = batch->lens;
    a.block_table = batch->block_table;
    a.q = q;
    a.out = out;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.masks = masks;
    a.kc = (const char*)cache->k + 2 * layer * cache->layer_stride;
    a.vc = (const char*)cache->v + 2 * layer * cache->layer_stride;
    a.page_stride = cache->page_stride;
    a.head_stride = cache->head_stride;
    a.pos_stride = cache->pos_stride;
    a.n_heads = n_heads;
    a.n_kv_heads = cache->n_kv_heads;
    a.page_size = cache->page_size;
    a.n_pages = cache->n_pages;
    a.scale2 = (float)(1.4426950408889634 * scale);
    a.status = status;
    const dim3 grid((unsigned)batch->n_rows, (unsigned)((n_heads + 3) / 4));
    const bool wide = cache->head_dim == 128;
    if (dtype == SSD_F32)
        return wide ? launch(call, attn_simple_kernel<float, f16, 128>, grid, 128, 0, cuda_stream, a)
                    : launch(call, attn_simple_kernel<float, f16, 64>, grid, 128, 0, cuda_stream, a);
    if (dtype == SSD_F16)
        return wide ? launch(call, attn_simple_kernel<f16, f16, 128>, grid, 128, 0, cuda_stream, a)
                    : launch(call, attn_simple_kernel<f16, f16, 64>, grid, 128, 0, cuda_stream, a);
    return wide ? launch(call, attn_simple_kernel<bf16, bf16, 128>, grid, 128, 0, cuda_stream, a)
                : launch(call, attn_simple_kernel<bf16, bf16, 64>, grid, 128, 0, cuda_stream, a);
}
