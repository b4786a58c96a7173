/*
 * ssd_ops.h - operators of libssd on the caller's own device tensors: a round
 * of decoding over a tree of drafted tokens, for a batch of requests that
 * share a paged KV cache.
 *
 * ssd.h decodes one sequence, one chain of drafts a round.  A program that
 * serves several requests, or drafts several continuations at once, runs its
 * own forward; these calls are the parts of its round that touch the cache:
 *
 *   ssd_tree_plan       pages for the round's rows; every row's slot in the
 *                       cache, position and ancestor mask
 *   ssd_rope_kv         (each layer) queries and keys turned to their
 *                       positions, keys and values written to their slots
 *   ssd_tree_attention  (each layer) the rows' attention over the cache
 *   ssd_tree_commit     the path that the target model's tokens take through
 *                       each tree; its keys and values moved behind the
 *                       prefix, len <- len + 1 + n (the KV rollback of ssd.h)
 *
 * Like ssd_linear_noalloc they allocate nothing, launch on the given stream
 * (NULL: the legacy default stream) of the current device and return once the
 * work is enqueued.  All tensors are the caller's, in memory of the current
 * device.  Lengths and tables are read on the device: a captured call replays
 * with whatever they hold then.  Calls on several streams do not disturb each
 * other as long as they share no output and no workspace.
 *
 * Return value: SSD_OK or a negative SSD_ERR_* code of ssd.h, with the message
 * in ssd_last_error().  The first use of a call on a device sets its kernels
 * up; make it before any stream capture.  Host-side errors are found before
 * anything is launched.  What only the device can see is kept inside the
 * tensors' bounds: rows outside [0, n_rows), slots outside the cache and pages
 * outside [0, n_pages) are not touched (a page outside reads as zeros), and
 * where a call takes `status` it ORs an SSD_STATUS_* bit into it.
 */
#ifndef SSD_OPS_H
#define SSD_OPS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Types of the rows that an operator reads and writes.  fp32 and fp16 rows go
 * with an fp16 cache (ssd.h's), bf16 rows with a bf16 cache. */
typedef enum { SSD_F32 = 0, SSD_F16 = 1, SSD_BF16 = 2 } ssd_dtype;

/* Bits of a status word (device int32, set by the caller to 0; may be NULL). */
#define SSD_STATUS_PAGES 1   /* ssd_tree_plan: too few free pages; some requests got none */
#define SSD_STATUS_TABLE 2   /* a request is longer than its row of the block table */
#define SSD_STATUS_PARENT 4  /* a parent is not an earlier node of the same tree, or a tree has more nodes than its masks have bits */
#define SSD_STATUS_TIMEOUT 8 /* ssd_tree_attention: a bounded wait gave up; its output is not valid */

/* A paged KV cache.  Element (layer, page, kv_head, position in the page, dim)
 * of K lies layer * layer_stride + page * page_stride + kv_head * head_stride +
 * position * pos_stride + dim elements behind k, and the same of V behind v.
 * Strides are multiples of 8 elements (pos_stride >= head_dim), k and v 16-byte
 * aligned, dtype SSD_F16 or SSD_BF16, head_dim 64 or 128, page_size a multiple of 16
 * of at most 65536, n_pages * page_size < 2^31.  (A contiguous cache is one of n_pages
 * requests with one page each.)  Keys and values behind a request's last
 * position may be anything, NaN included. */
typedef struct {
    void* k;
    void* v;
    int dtype, n_layers, n_pages, n_kv_heads, page_size, head_dim;
    int64_t layer_stride, page_stride, head_stride, pos_stride;
} ssd_pages;

/* The rows of a round.  Request b owns rows row_start[b] .. row_start[b + 1] - 1
 * (row_start: n_requests + 1 values that do not decrease): node i of its tree is
 * row row_start[b] + i, and will sit at cache index lens[b] + i, behind its lens[b]
 * cached positions, which are in pages block_table[b][0 ..] (rows of max_blocks
 * entries).  lens[b] < 0: the request has ended.  n_rows: rows that the row
 * tensors have; those that no request owns are left as they were.  max_rows: the
 * largest number of rows of a request; it only chooses between kernels.
 * 1 <= n_requests <= 4096; n_rows >= 0 (0: nothing but ssd_tree_plan's pages
 * is done); 1 <= max_rows; 1 <= max_blocks. */
typedef struct {
    int n_requests, n_rows, max_rows, max_blocks;
    const int32_t* row_start;
    const int32_t* lens;
    int32_t* block_table;
} ssd_batch;

/* Pages, slots, positions and masks of a round.
 * Free pages are a queue in a ring: ring[x mod n_pages] for x from ends[0] up to
 * (not including) ends[1]; a page is in the queue or with one request, so the ring never overflows.
 *   - Request b needs ceil((lens[b] + rows) / page_size) pages and holds held[b].
 *     What is missing is taken from the queue's front, requests in order, and
 *     written to block_table[b][held[b] ..].  The first request that does not get
 *     all it needs and those after it that need any get nothing (SSD_STATUS_PAGES); a request that
 *     needs more than max_blocks gets nothing and the others go on
 *     (SSD_STATUS_TABLE).  A request never gives pages back while it runs.
 *     A request that got nothing has no place for this round's rows: they are not written (slots of -1), its attention is not
 *     valid, and the caller keeps lens[b] and leaves its commit's results.  ssd_tree_attention and ssd_tree_commit go by block_table
 *     alone, so entries behind the pages that a request holds must be -1 (or outside [0, n_pages)) for them not to
 *     read, and move rows in, pages of others: this call leaves those entries as they are, of ended requests too.
 *   - One with lens[b] < 0 gives its pages back: they are appended to the queue,
 *     requests in order, and can be taken from the next call on.
 *   - held_out and ends_out get the new counts (arrays of their own: held and
 *     ends are only read, so that a call can be repeated).
 * For each row (node i of request b with parent p):
 *   - slots[row] = its cache row, page * page_size + position in the page; -1 if the page is not one of the cache's, or
 *     its request got no pages or has ended;
 *   - positions[row] = lens[b] + depth, with depth 0 for a root, depth of the parent + 1 else;
 *   - masks[row][0 .. mask_words-1]: bit j % 64 of word j / 64 is set for node j = i and its ancestors.
 * parents: per row, the index within its tree of an earlier node, or -1 for a
 * root; any other value is taken for -1 (SSD_STATUS_PARENT).  A tree has at most
 * 64 * mask_words nodes (further nodes: depth as of a root, no bits, and
 * SSD_STATUS_PARENT); 1 <= mask_words <= 4.  parents = NULL: every request is a
 * chain of any length; masks must be NULL and mask_words 0.
 * status may be NULL; slots, positions and masks may be NULL if n_rows = 0.
 * Errors: INVALID_ARG, CUDA. */
int ssd_tree_plan(const ssd_batch* batch, int page_size, int n_pages, const int32_t* parents, const int32_t* held,
                  int32_t* held_out, int32_t* ring, const int64_t* ends, int64_t* ends_out, int32_t* slots,
                  int32_t* positions, uint64_t* masks, int mask_words, int32_t* status, void* cuda_stream);

/* Rotary frequencies: the first rot_dim dims of a head form pairs i = 0 ..
 * rot_dim / 2 - 1, dims (i, i + rot_dim / 2), or (2i, 2i + 1) with interleaved = 1;
 * pair i turns by f_i = theta^(-2i / rot_dim) radians a position; the other dims pass.
 *   SSD_ROPE_PLAIN     f_i
 *   SSD_ROPE_LINEAR    f_i / factor (position interpolation)
 *   SSD_ROPE_BY_PARTS  f_i (g + (1 - g) / factor), g = clamp((r - slow) / (fast - slow), 0, 1), r = original_len
 *                      f_i / 2 pi: pairs that turn often within the original context keep their
 *                      frequency, the slow ones are interpolated (YaRN, Peng et al. 2023)
 * The rotated dims are multiplied by amplitude (1 if nothing else is wanted). */
typedef enum { SSD_ROPE_PLAIN = 0, SSD_ROPE_LINEAR = 1, SSD_ROPE_BY_PARTS = 2 } ssd_rope_scaling;
typedef struct {
    int rot_dim, interleaved;
    float amplitude;
    uint64_t turns[64]; /* f_i / 2 pi, as a fraction of 2^64 */
} ssd_rope;

/* Fills *out (host only; keep it as long as you like).  rot_dim: a multiple of 16, 16 ..
 * 128; theta > 1; factor >= 1; BY_PARTS: original_len >= 1, 0 <= slow < fast; amplitude > 0.
 * Errors: INVALID_ARG. */
int ssd_rope_init(int rot_dim, int interleaved, int scaling, double theta, double factor, double original_len,
                  double slow, double fast, double amplitude, ssd_rope* out);

/* Turns n_rows rows of queries [row][n_heads][head_dim] and keys
 * [row][n_kv_heads][head_dim] to positions[row] >= 0; writes the queries to q_out
 * (which may be q; else it overlaps no input) and the keys and the values v [row][n_kv_heads][head_dim] to rows
 * slots[row] of the cache's layer.  A row whose slot is negative or outside the cache
 * leaves the cache alone.  Slots are distinct: of rows with the same slot the last stays in calls
 * of up to 129 rows; in larger ones any may, K and V and each head by itself.  Rows are q_stride, k_stride, v_stride and q_out_stride elements
 * apart (so q, k and v may be parts of one projection's output), heads
 * head_dim; pointers 16-byte aligned, strides multiples of 16 bytes.  rot_dim <= head_dim.
 * Angles are exact to 2^-24 of a turn at any position; sums in fp32, one rounding.
 * Errors: INVALID_ARG, CUDA. */
int ssd_rope_kv(const ssd_pages* cache, int layer, const ssd_rope* rope, int dtype, int n_rows, int n_heads,
                const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                const int32_t* positions, const int32_t* slots, void* q_out, int64_t q_out_stride, void* cuda_stream);

/* Attention of the rows over their requests' cache:
 *   out[row][h] = sum_x w_x V[x][g] / sum_x w_x,  w_x = exp(scale q[row][h] . K[x][g] - max),  g = h n_kv_heads / n_heads,
 * over the positions x that the row sees: the lens[b] cached ones and, of its own
 * round's rows (which ssd_rope_kv has put at lens[b] + j), node j if bit j of masks[row] is set,
 * or, with masks = NULL, nodes 0 .. i of a chain.  Nodes from 64 * mask_words on are not seen
 * (SSD_STATUS_PARENT).
 * A row that sees nothing, or whose scores are all -inf, gets zeros.  What a row does
 * not see does not change its output, be it NaN; an infinite value that it sees comes out as
 * infinity or NaN.  Positions that max_blocks pages do not hold are
 * not seen (SSD_STATUS_TABLE).  Rows of a request with lens[b] < 0 are left as they were.
 * q and out: [row][n_heads][head_dim] of dtype, rows q_stride and out_stride
 * elements apart, 16-byte aligned, strides multiples of 16 bytes; no overlap.  n_heads is a
 * multiple of n_kv_heads; 0 < scale, finite.
 * Scores, statistics and sums are fp32.  If no request has more than two rows a KV head
 * (max_rows n_heads / n_kv_heads <= 2) everything is fp32.  Else the weights, and q of fp32 rows, enter
 * the products as pairs of the cache's type (fp16 22 bits, bf16 16).
 * Measured against 64 bits, values around 1, at any length: fp32 rows 1e-6; 16-bit rows what rounding the exact result to the type
 * costs, and up to 4e-5 of the result more (tensor cores sum up to 3072 positions and cut off what their sums do not hold).
 * A wait inside the call that has not ended after two seconds gives up (SSD_STATUS_TIMEOUT): the call ends, and
 * without `status` no one can tell that its output is not valid.
 * workspace: ssd_tree_attention_workspace() bytes, 16-byte aligned; its contents
 * mean nothing between calls.  The same inputs give the same bits; the order of
 * sums depends on the whole batch's lengths.
 * Errors: INVALID_ARG, CAPACITY (workspace too small), CUDA. */
int ssd_tree_attention(const ssd_batch* batch, const ssd_pages* cache, int layer, int dtype, int n_heads,
                       const void* q, int64_t q_stride, const uint64_t* masks, int mask_words, float scale, void* out,
                       int64_t out_stride, void* workspace, size_t workspace_bytes, int32_t* status,
                       void* cuda_stream);

/* Bytes of workspace for a cache of this head_dim on the current device, whatever the batch.
 * Errors: INVALID_ARG, CUDA. */
int ssd_tree_attention_workspace(int head_dim, size_t* bytes);

/* Test hook for the bounded waits of ssd_tree_attention: in the next call of the process whose tiles have
 * more than two rows, CTA `cta` never asks for its keys, and waits give up after wait_limit_s (0 < wait_limit_s <= 10; else 2 s).  The call ends with
 * SSD_STATUS_TIMEOUT, its output is not valid, and the calls after it are not affected.  cta < 0 disarms. */
void ssd_debug_tree_stall(int cta, double wait_limit_s);

/* The end of a round.  tokens[row]: the drafted token of each node (that of a root,
 * node 0, is the last token of the sequence, which no cache row holds yet);
 * target[row]: the token that the target model chose after the node (argmax or a
 * sample).  From node 0 the path goes to the lowest child whose token is the
 * node's target, until there is none: n nodes accepted.  For request b:
 *   accepted[b] = n;  next_token[b] = target of the last node on the path;
 *   lens_out[b] = lens[b] + 1 + n;
 *   path[row_start[b] + j] = node at step j = 0 .. n (path[row_start[b]] = 0);
 *   emitted[row_start[b] + j] = token of step j + 1, j < n, and next_token at j = n;
 * and in every layer the keys and values at lens[b] + path[j] move to lens[b] + j.
 * A request without rows, or with lens[b] < 0, gets accepted = -1, next_token = -1,
 * lens_out = lens.  The walk goes over the first 256 nodes of a request: a path ends
 * there at the latest, with what the target chose after its last node, so what is accepted is still the target's own text.  A
 * child has a higher index than its parent (others are not reached); parents = NULL: chains.
 * cache = NULL: tokens only, nothing moves.  The results are arrays of their own: none overlaps another or an input.
 * Errors: INVALID_ARG, CUDA. */
int ssd_tree_commit(const ssd_batch* batch, const ssd_pages* cache, const int32_t* parents, const int32_t* tokens,
                    const int32_t* target, int32_t* accepted, int32_t* next_token, int32_t* lens_out, int32_t* path,
                    int32_t* emitted, void* cuda_stream);

#ifdef __cplusplus
}
#endif

#endif /* SSD_OPS_H */
