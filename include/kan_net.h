/*
 * kan_net.h - operators around the layers of kan.h in a residual network on tokens.
 *
 * What a stack of KAN layers needs beside them: the norms before and after a block with its gate
 * and residual scale, the rows of an embedding table with their gradient, log probabilities of
 * tokens with the gradient of a loss on them, and the norm of all gradients with the gradients
 * scaled to it.  Same library (libkan_hip.so) and same conventions as kan.h (device memory owned by
 * the caller, descriptors and lists on the host and read during the call, nothing allocated, nothing
 * kept between calls, work enqueued on `stream`, a kan_status returned and nothing thrown), except:
 *   - data are fp32 or bf16 (kan_type); what is computed is held in 32 bits or more and rounded once,
 *     to nearest even, where it is written;
 *   - arrays need the alignment of their elements only, workspaces 256 bytes;
 *   - infinities and NaN are ordinary values here: what they lead to is said at each operator.
 * None of these calls synchronises, so all can be captured in a HIP graph.  All sums run in a fixed
 * order: repeated calls give the same bits.
 */
#ifndef KAN_NET_H
#define KAN_NET_H

#include "kan.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum kan_type { KAN_F32 = 0, KAN_BF16 = 1 } kan_type;

/* ---- norms at a block boundary -------------------------------------------------------------- */

enum { KAN_NORM_RMS = 0, KAN_NORM_LAYER = 1 };

/* One boundary between two blocks of a residual network, rows of n channels (n <= 16384):
     u     = norm(f) * w_post + b_post                    f: what the block before has computed
     x_out = residual_scale * x + gate * u                x: the residual stream in front of it
     h     = norm(x_out) * w_pre + b_pre                  what the block behind reads
   norm(v) = (v - mean(v)) / sqrt(mean((v - mean(v))^2) + eps), without the mean for KAN_NORM_RMS; eps > 0.  The norm of
   x_out is that of its 32-bit value, not of the one rounded to stream_type.  Rows of any finite values keep their digits, also where
   squares or sums of them are not in a float's range.  A NaN in a row makes its norm NaN; an infinity makes a layer norm NaN and an
   RMS norm NaN in its place and 0 in the others.
   Row b takes row b / gate_rows of the gate; gate_rows = 0: all rows share one.
   stream_type is the type of x, x_out and their gradients, branch_type that of f, h and theirs: KAN_BF16 branches need a
   KAN_BF16 stream (KAN_ERR_UNSUPPORTED otherwise).  Parameters and their gradients are fp32. */
typedef struct kan_block_norm_desc {
    int32_t n;
    int32_t norm;
    float eps;
    float residual_scale;
    int64_t gate_rows;
    int32_t stream_type, branch_type;
} kan_block_norm_desc;

/* w_post[n] b_post[n] w_pre[n] b_pre[n], gate[ceil(B / gate_rows)][n] ([1][n] for gate_rows = 0).  A NULL weight or gate stands for
   ones, a NULL bias for zeros. */
typedef struct kan_block_norm_params {
    const float *w_post, *b_post, *gate, *w_pre, *b_pre;
} kan_block_norm_params;

/* Gradients of the above, same shapes; any member may be NULL. */
typedef struct kan_block_norm_grads {
    float *gw_post, *gb_post, *ggate, *gw_pre, *gb_pre;
} kan_block_norm_grads;

/* f NULL: the first norm of a network (x_out = x, which is not written; x_out, w_post, b_post, gate and residual_scale are not looked
   at).  h NULL: the last block, without a norm behind it.  Not both.  x_out may be x and h may be f (in place); other overlaps are not
   allowed.  stats[B][4] (mean and 1/sigma of f, mean and 1/sigma of x_out; unused ones 0) is for the backward pass and may
   be NULL. */
int kan_block_norm_forward(const kan_block_norm_desc *desc, int64_t B, const void *x, const void *f,
                           const kan_block_norm_params *p, void *x_out, void *h, float *stats, void *stream);

/* Gradients given gx_out = dL/dx_out and gh = dL/dh (either may be NULL: zero), with x, f, p and stats as the forward call had
   and left them:
     d  = gx_out + back(gh * w_pre; x_out)      gx = residual_scale * d      gw_pre = sum gh * norm(x_out)     gb_pre = sum gh
     gf = back(d * gate * w_post; f)            ggate = sum d * u            gw_post = sum d * gate * norm(f)  gb_post = sum d * gate
     back(q; v) = (q - mean(q) - norm(v) * mean(q * norm(v))) / sigma, without mean(q) for KAN_NORM_RMS
   sums over the rows (those of its gate row for ggate).  f NULL as in the forward call: gx = d, and no gf, gw_post, gb_post, ggate (KAN_ERR_INVALID_ARG).  gx, gf may be NULL; gx may be
   gx_out and gf may be gh.  Gradients of parameters that are NULL (ones, zeros) can be had as well.  B == 0 gives
   parameters zero gradients (the gate of gate_rows > 0 has no rows then). */
size_t kan_block_norm_workspace_bytes(const kan_block_norm_desc *desc, int64_t B);
int kan_block_norm_backward(const kan_block_norm_desc *desc, int64_t B, const void *x, const void *f,
                            const kan_block_norm_params *p, const float *stats, const void *gx_out, const void *gh,
                            void *gx, void *gf, const kan_block_norm_grads *g, void *ws, size_t ws_bytes, void *stream);

/* ---- embedding ------------------------------------------------------------------------------ */

/* y[t] = scale * table[ids[t]], t < T: rows of n <= 2^30 channels of a table of V < 2^31 - 1 rows; a fp32 table gives fp32 rows, a bf16
   table either.  An id outside 0 .. V-1 (-1 for a place without a token) gives a row of zeros. */
int kan_embedding_forward(int64_t T, int64_t V, int32_t n, const int64_t *ids, const void *table, int32_t table_type, float scale,
                          void *y, int32_t y_type, void *stream);

/* gtable[v] = scale * sum over the t with ids[t] = v of gy[t], for every v < V (zeros where there is none); ids outside the table
   count nowhere.  The tokens are sorted by id first, stably, so that a row's sum has a fixed order; fp32 sums, rounded once.
   T < 2^31 - 65536 (KAN_ERR_UNSUPPORTED otherwise); T == 0 writes zeros. */
size_t kan_embedding_workspace_bytes(int64_t T, int64_t V, int32_t n);
int kan_embedding_backward(int64_t T, int64_t V, int32_t n, const int64_t *ids, const void *gy, int32_t y_type, float scale,
                           void *gtable, int32_t table_type, void *ws, size_t ws_bytes, void *stream);

/* ---- log probabilities of tokens ------------------------------------------------------------ */

/* For R rows of V < 2^31 - 1 logits, row r at logits + r * row_stride elements (row_stride >= V), z = logits / temperature:
     logp[r]    = z[ids[r]] - log sum_v exp(z[v])          an id outside 0 .. V-1 gives 0
     entropy[r] = - sum_v p_v log p_v,  p = softmax(z)
     top_ids[r][j], top_logp[r][j], j < top: the most likely tokens, best first, equal ones by the lowest index
   top <= KAN_TOP_MAX and top <= V.  Masked tokens are logits of -infinity (p = 0, no part of the entropy) or of the type's lowest
   value.  A row that is -infinity throughout has logp = -infinity (0 for an id outside), entropy 0, and for alternatives the tokens
   0 .. top-1 at -infinity.  A NaN or a +infinity in a row makes its logp, entropy and top_logp NaN (an id outside still gives 0);
   for top_ids a NaN counts as larger than +infinity.  stats[R][2] (largest logit of the row; sum of exp(z - its z) over the other tokens) is for
   the backward pass.  logp, entropy and the gradients keep their digits, not only their places, in rows of one likely token.
   logp, entropy, stats and the pair of top_* may be NULL; ids is read for logp only.  1e-30 <= temperature <= 1e30. */
#define KAN_TOP_MAX 64
int kan_token_logprob_forward(int64_t R, int64_t V, const void *logits, int32_t type, int64_t row_stride, const int64_t *ids,
                              float temperature, int32_t top, float *logp, float *entropy, float *stats, int64_t *top_ids,
                              float *top_logp, void *ws, size_t ws_bytes, void *stream);
size_t kan_token_logprob_workspace_bytes(int64_t R, int64_t V, int32_t top);

/* glogits[r][v] = ( g_logp[r] (1[v = ids[r]] - p_v) - g_entropy[r] p_v (log p_v + entropy[r]) ) / temperature, contiguous rows of V in
   the type of the logits, from the forward call's stats and entropy.  g_logp or g_entropy may be NULL (zero), not both; ids and
   g_logp, entropy and g_entropy go together.  Rows whose id is outside have no part of g_logp; rows that are -infinity throughout get
   zeros, rows with a NaN or +infinity NaN.  glogits may be logits where row_stride is V. */
int kan_token_logprob_backward(int64_t R, int64_t V, const void *logits, int32_t type, int64_t row_stride, const int64_t *ids,
                               float temperature, const float *stats, const float *entropy, const float *g_logp,
                               const float *g_entropy, void *glogits, void *stream);

/* ---- norm of all gradients ------------------------------------------------------------------ */

/* One tensor of a list: `count` elements of `type` at `data`; `out` receives the scaled ones and may be data (in place). */
typedef struct kan_tensor_ref {
    const void *data;
    void *out;
    int64_t count;
    int32_t type;
} kan_tensor_ref;

/* *norm = sqrt(sum of the squares of all elements), summed in 64 bits; one float of device memory.  out is not looked at. */
int kan_gradient_norm(int32_t n, const kan_tensor_ref *list, float *norm, void *ws, size_t ws_bytes, void *stream);

/* The same, and out = data * min(1, max_norm / norm) for every tensor.  A norm that is not finite leaves the values as they are
   (out = data), for the caller to see in *norm.  max_norm >= 0, finite.  Outputs must not overlap other tensors of the list. */
int kan_clip_gradients(int32_t n, const kan_tensor_ref *list, float max_norm, float *norm, void *ws, size_t ws_bytes, void *stream);
size_t kan_clip_workspace_bytes(int32_t n);

#ifdef __cplusplus
}
#endif
#endif /* KAN_NET_H */
