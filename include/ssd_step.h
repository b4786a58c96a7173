/*
 * ssd_step.h - operators of libssd on the caller's own device tensors: the
 * parts of a decoding step that stand next to the tree operators of ssd_ops.h,
 * for programs that run their own forward.
 *
 *   ssd_norm_rope_kv    (each layer, in the place of ssd_rope_kv) queries and keys
 *                       normalised head by head and turned to positions on one
 *                       or several axes, keys and values written to their slots
 *   ssd_moe_route       (each layer) the experts of every row and their weights
 *   ssd_moe_mlp         (each layer) the rows through their experts
 *   ssd_logits_adjust   penalties for tokens that were said before, biases and
 *                       masks of allowed tokens on the logits of a round's rows
 *   ssd_logits_choose   the same without writing them: every row's best tokens and
 *                       their log probabilities - the `target` of ssd_tree_commit,
 *                       or the children of a drafted tree's nodes
 *
 * They keep the manner of ssd_ops.h: they allocate nothing, launch on the given
 * stream (NULL: the legacy default stream) of the current device and return once
 * the work is enqueued.  All tensors are the caller's, in memory of the current
 * device.  Lengths, ids and row starts are read on the device: a captured call replays
 * with whatever they hold then.  Calls on several streams do not disturb each
 * other as long as they share no output and no workspace.
 *
 * Return value: SSD_OK or a negative SSD_ERR_* code of ssd.h, with the message
 * in ssd_last_error().  Tensors are aligned to their type at least (refused if not).  The first use of a call on a device sets its kernels up;
 * make it before any stream capture.  Host-side errors are found before anything
 * is launched.  What only the device can see is kept inside the tensors' bounds:
 * rows outside [0, n_rows), slots outside the cache, tokens outside [0, vocab),
 * experts outside [0, n_experts) and sets outside their table are passed over.
 */
#ifndef SSD_STEP_H
#define SSD_STEP_H

#include "ssd_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Which axis of its positions turns each pair of a head (ssd_rope): pair i turns by
 * turns[i] * positions[axis[i]].  Text has the same position on every axis; pieces of
 * an image or a video have a time, a height and a width. */
typedef struct {
    int n_axes; /* 1 .. 4 */
    uint8_t axis[64];
} ssd_rope_axes;

/*   SSD_AXES_SECTIONS  the first pairs[0] pairs go with axis 0, the next pairs[1] with axis 1, ..
 *   SSD_AXES_IN_TURNS  pair i goes with axis i mod n_axes while that axis has had fewer than its
 *                      pairs[.] of them, and with axis 0 from then on: every axis gets
 *                      fast and slow pairs */
typedef enum { SSD_AXES_SECTIONS = 0, SSD_AXES_IN_TURNS = 1 } ssd_axes_layout;

/* Fills *out (host only).  pairs: n_axes counts >= 0 that add up to rot_dim / 2 of the rope.
 * Errors: INVALID_ARG. */
int ssd_rope_axes_init(const ssd_rope* rope, int layout, int n_axes, const int* pairs, ssd_rope_axes* out);

/* RMS norms of the heads: x <- x / sqrt(mean(x^2) + eps) * gain, over the head_dim dims of a head.
 * Gains are head_dim fp32 values on the device (16-byte aligned), the same for all heads; NULL: that side is not
 * normalised.  0 < eps, finite. */
typedef struct {
    const float* q_gain;
    const float* k_gain;
    float eps;
} ssd_head_norm;

/* ssd_rope_kv (ssd_ops.h: its tensors, strides and slots) with norms before the rotation and
 * positions on several axes.  Without both it gives what ssd_rope_kv gives, up to the last place, and that call is the faster one but for
 * many rows of 16 bits (403 rows of 32 + 16 heads 4.2 against 6.5 us, 4095 of 32 + 64 51 against 57).
 * norm = NULL: no norms.  axes = NULL: one axis.  positions: [n_axes][n_rows], any
 * int32.  Of two rows with the same slot either may stay, K and V and each head by itself.  Values are copied.  Angles are exact to 2^-24 of a turn at any position; squares, sums and products in
 * fp32, one rounding to the rows' and the cache's type.
 * Errors: INVALID_ARG, CUDA. */
int ssd_norm_rope_kv(const ssd_pages* cache, int layer, const ssd_rope* rope, const ssd_rope_axes* axes,
                     const ssd_head_norm* norm, int dtype, int n_rows, int n_heads, const void* q, int64_t q_stride,
                     const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int32_t* positions,
                     const int32_t* slots, void* q_out, int64_t q_out_stride, void* cuda_stream);

/* What is done to the logits of a round's rows.  Every part may be left out (NULL).
 * Request b owns rows row_start[b] .. row_start[b + 1] - 1 as in ssd_batch (rows that no request
 * owns are left as they were); row_start = NULL: n_requests = n_rows, one row each.  1 <= n_requests <= 4096.
 *
 * What a row's text has said:
 *   - history[b * history_stride ..]: the request's tokens so far, the first clamp(history_len[b], 0, max_history) of them
 *     (without the round's nodes); the first prompt_len[b] are the prompt's, the others the model's own
 *     (prompt_len = NULL: all are the model's);
 *   - of the round's nodes, tokens[row_start[b] + j] for the nodes j that the row's mask shows (masks of
 *     mask_words 64-bit words a row as ssd_tree_plan gives them, 1 .. 4), or with masks = NULL nodes 0 .. i of a chain.  They
 *     count as the model's own.
 * With c the number of times that the model itself has said token x, a row's logit l of x becomes, in fp32 with a
 * rounding after each step,
 *   l > 0 ? l / repetition[b] : l * repetition[b]   if x is in the prompt or c > 0,
 *   l - frequency[b] * c,
 *   l - presence[b]                                 if c > 0,
 *   l + bias[bias_of[b]][x]                         (bias_of = NULL: bias[0]; outside [0, n_bias): none),
 *   -inf                                            if bit x % 32 of word x / 32 of allowed[allowed_of[row]] is 0
 *                                                   (allowed_of = NULL: allowed[row]; outside [0, n_allowed): all are allowed).
 * repetition, presence, frequency: fp32 [n_requests]; NULL leaves that step out.  bias rows are bias_stride floats
 * apart (>= vocab), those of allowed allowed_stride words (>= ceil(vocab / 32)).
 * 1 <= vocab <= 262144; max_rows: the largest number of rows of a request, which only says how
 * many rows may share one count of what their text has said. */
typedef struct {
    int vocab, n_requests, n_rows, max_rows;
    const int32_t* row_start;
    const int32_t* history;
    const int32_t* history_len;
    const int32_t* prompt_len;
    int64_t history_stride;
    int max_history, mask_words;
    const int32_t* tokens;
    const uint64_t* masks;
    const float* repetition;
    const float* presence;
    const float* frequency;
    const float* bias;
    const int32_t* bias_of;
    const uint32_t* allowed;
    const int32_t* allowed_of;
    int64_t bias_stride, allowed_stride;
    int n_bias, n_allowed;
} ssd_logit_rules;

/* out[row][x] = the logits of type dtype after the rules, rounded to dtype once.  Rows are stride and out_stride elements apart
 * (>= vocab; any alignment that the type has); out may be logits with its stride, else it overlaps no input.
 * A NaN that is allowed stays NaN.
 * Errors: INVALID_ARG, CUDA. */
int ssd_logits_adjust(const ssd_logit_rules* rules, int dtype, const void* logits, int64_t stride, void* out,
                      int64_t out_stride, void* cuda_stream);

/* The k (1 .. 16) largest logits l of each row after the rules, largest first, of equal ones the lowest token first:
 *   tokens[row][j]   the token, -1 where fewer than j + 1 tokens are left (those at -inf and NaN are never chosen);
 *   logprob[row][j]  l - logsumexp of all of the row's, -inf where there is no token;
 *   total[row]       that logsumexp (-inf for a row with nothing left); may be NULL.
 * A NaN counts as -inf, in the sum too.  A logit of +inf takes all of the probability, shared with others of +inf.  Sums in fp32; logprob and total are off by some 1e-7
 * of the larger of 1 and the largest logit.  The same inputs and sizes give the same bits.
 * Errors: INVALID_ARG, CUDA. */
int ssd_logits_choose(const ssd_logit_rules* rules, int dtype, const void* logits, int64_t stride, int k, int32_t* tokens,
                      float* logprob, float* total, void* cuda_stream);

/* How the router's products z = w_router x become scores p: softmax over the experts, or 1 / (1 + exp(-z)). */
typedef enum { SSD_MOE_SOFTMAX = 0, SSD_MOE_SIGMOID = 1 } ssd_moe_score;

/* The experts of each row: the k with the largest p + favour[e] (favour fp32 [n_experts], NULL: 0), largest first, of equal ones the
 * lowest first:  ids[row][j] = e,  weights[row][j] = scale p  (renorm = 1: divided by the sum of the row's k p's).
 * x: [row][d], rows x_stride elements apart, and w_router [n_experts][d], of dtype SSD_F16 or SSD_BF16, 16-byte aligned, d and
 * x_stride multiples of 8.  1 <= k <= 16, k <= n_experts <= 1024; d <= 65536.  Products are summed to about 48 bits and scored in fp64: two experts come in their exact
 * order unless their sums are within some 1e-11 of the sum of their products' absolute values.  An expert whose score is NaN comes after all others; one
 * whose product is NaN has no part in the sums, and weight NaN where it is among the k all the same.  +inf takes all of the softmax, shared with others of +inf.
 * Without favour the order is that of the products.
 * Errors: INVALID_ARG, CUDA. */
int ssd_moe_route(int dtype, int n_rows, int d, int n_experts, int k, const void* x, int64_t x_stride, const void* w_router,
                  const float* favour, int score, int renorm, float scale, int32_t* ids, float* weights, void* cuda_stream);

/* The experts' matrices: gate and up [n_experts][f][d], down [n_experts][d][f], of dtype SSD_F16 or SSD_BF16; an expert's lie
 * *_stride elements behind the one's before (so gate and up may be halves of one tensor).  16-byte aligned, strides, d and f
 * multiples of 8; d, f <= 65536, n_experts <= 1024. */
typedef struct {
    const void* gate;
    const void* up;
    const void* down;
    int64_t gate_stride, up_stride, down_stride;
    int dtype, n_experts, d, f;
} ssd_moe;

/* out[row] = residual[row] + sum_j weights[row][j] * down[e] (silu(gate[e] x[row]) * (up[e] x[row])),  e = ids[row][j],
 * silu(a) = a / (1 + exp(-a)); a slot with ids outside [0, n_experts) adds nothing (experts that are elsewhere).  Made for the rows of a
 * decoding or verification step: an expert that some row goes to is read once for up to 8, 16 or 32 of its rows, by how many go to one on average.  From some 64
 * rows on its time grows with the rows (64, 128, 256 and 1024 rows, 2 of 16 experts of 5120 x 13824: 1.05, 1.5, 2.2 and 7.3 ms): for a prompt, matrix
 * products of an expert's rows are the better way.
 * x, residual and out: [row][d] of the experts' dtype, 16-byte aligned, rows *_stride elements apart, multiples of 8; residual may be
 * NULL; out may be residual with its stride, and overlaps nothing else.  n_rows <= 1024, 1 <= k <= 16.
 * Sums in fp32, slots in order; silu(..) * (..) enters the product with down in all bits of fp32 (bf16), or off by 2^-22 of it and 2^-36 at most
 * (fp16, where it is infinite beyond 65504).  The same inputs give the same bits.
 * A wait inside the call that has not ended after two seconds gives up: the call ends with SSD_STATUS_TIMEOUT in `status` (which may be NULL),
 * and results that miss something are NaN.
 * workspace: ssd_moe_workspace() bytes, 16-byte aligned; its contents mean nothing between calls.
 * Errors: INVALID_ARG, CAPACITY (workspace too small), CUDA. */
int ssd_moe_mlp(const ssd_moe* experts, int n_rows, int k, const void* x, int64_t x_stride, const int32_t* ids,
                const float* weights, const void* residual, int64_t residual_stride, void* out, int64_t out_stride,
                void* workspace, size_t workspace_bytes, int32_t* status, void* cuda_stream);

/* Test hook for the bounded waits of ssd_moe_mlp: in the next call of the process CTA `cta` never asks for its weights, and waits give
 * up after wait_limit_s (0 < wait_limit_s <= 10; else 2 s).  The call ends with SSD_STATUS_TIMEOUT, the rows that the CTA had a part in are NaN, and the
 * calls after it are not affected.  cta < 0 disarms. */
void ssd_debug_moe_stall(int cta, double wait_limit_s);

/* Bytes of workspace for this many rows and slots; never fewer than for fewer rows or slots.  Errors: INVALID_ARG. */
int ssd_moe_workspace(const ssd_moe* experts, int n_rows, int k, size_t* bytes);

#ifdef __cplusplus
}
#endif

#endif /* SSD_STEP_H */
