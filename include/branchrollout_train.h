/*
 * libbranchrollout -- the operators of a policy update: what a program needs after br_prune to take one optimizer
 * step on the velocity network.  Conventions as in branchrollout.h; nothing here allocates, and every call only
 * enqueues kernels on `stream`.
 *
 * Samples of different lengths lie one behind the other ("documents" of a packed batch): document d owns rows
 * off[d] .. off[d + 1] - 1 of a matrix of tokens, off being a device array of n_docs + 1 ascending offsets.  The
 * host does not read it; offsets outside [0, rows] are taken as the nearest end, a document that ends before it
 * begins as empty, so that no offset makes a kernel leave its buffers.
 */
#ifndef BRANCHROLLOUT_TRAIN_H
#define BRANCHROLLOUT_TRAIN_H

#include "branchrollout.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------- *
 * Attention over packed documents.
 *   out[i, h] = sum_j p_ij v[j, g(h)],  p_ij = exp(scale q[i, h] . k[j, g(h)] - lse[h, i]),
 *   lse[h, i] = log sum_j exp(scale q[i, h] . k[j, g(h)])
 * over the keys j of the document that holds query i; g(h) = h / (n_heads / n_kv_heads).  A query without
 * keys (an empty document, or a row of no document) has out = 0, lse = -inf and no gradients; a key row of no document
 * gets zeros as its gradient.  A key whose products with all queries are -inf counts as none: probability 0, dk = dv = 0 (dq of these
 * queries is 0 x -inf, not a number, as the formula says).
 * Sums, exponentials and log-sum-exps are fp32.  BR_BF16: the probabilities and their gradients ds are rounded to bf16 as operands of the matrix products, and
 * the results once more; dout . out is taken from out as it was rounded, in documents of one tile of keys (32; 64 past 4 GiB of a matrix) from the probabilities.
 * Together 0.0023 of the results' norm, where a single rounding of exact results is 0.0017.
 * q dev [q_tokens, n_heads, head_dim], k, v dev [k_tokens, n_kv_heads, head_dim] in `dtype`, tokens *_stride
 * elements apart (so that the three may be parts of one QKV matrix), heads adjacent.
 * BR_ESHAPE unless head_dim is 64 or 128 (BR_BF16) or 16, 32, 64 or 128 (BR_F32), strides are multiples of 8 (BR_BF16) or 4
 * elements and pointers 16-byte aligned.
 * ------------------------------------------------------------------------- */
typedef struct {
  int32_t dtype, n_heads, n_kv_heads, head_dim;
  int32_t n_docs;
  int32_t q_tokens, k_tokens;
  float scale;                         /* > 0; 0: 1 / sqrt(head_dim) */
  int64_t q_stride, k_stride, v_stride, o_stride;     /* elements between tokens of q, k, v and of out / dout */
  int64_t dq_stride, dk_stride, dv_stride;            /* of the gradients (backward only) */
  const int32_t *q_off, *k_off;        /* dev [n_docs + 1] */
} br_attn_shape;

/* Workspace of the two calls below (0 on invalid arguments). */
size_t br_attention_workspace_bytes(const br_attn_shape* shape, int32_t backward);

/* out dev out, tokens o_stride apart; lse dev out [n_heads, q_tokens] fp32. */
br_status br_attention_forward(const br_attn_shape* shape, const void* q, const void* k, const void* v, void* out,
                               float* lse, void* workspace, size_t workspace_bytes, void* stream);

/* Gradients of a loss with respect to q, k and v, given dout = its gradient with respect to out and what the
 * forward call wrote:
 *   dv_j = sum_i p_ij dout_i,  ds_ij = scale p_ij (dout_i . v_j - dout_i . out_i),  dq_i = sum_j ds_ij k_j,  dk_j = sum_i ds_ij q_i
 * (dk, dv also summed over the heads of queries that share a head of keys).  dq, dk, dv dev out in `dtype`; they may be
 * parts of one matrix.  Sums are taken in a fixed order: equal inputs give equal bits. */
br_status br_attention_backward(const br_attn_shape* shape, const void* dout, const void* q, const void* k,
                                const void* v, const void* out, const float* lse, void* dq, void* dk, void* dv,
                                void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------- *
 * LayerNorm modulated by each document's condition (the network's LN(x)(1 + scale) + shift, eps 1e-6, no affine).
 *   y[r] = (x[r] - mean[r]) rstd[r],  out[r] = y[r] (1 + scale[g]) + shift[g],  g = group[document of r]
 * shift and scale of group g are mods + g*mods_stride + {shift_off, scale_off}, hidden values each.  With one group
 * this is the LayerNorm with weight 1 + scale and bias shift.  Rows of no document are left alone.
 * BR_ESHAPE unless hidden, mods_stride and the offsets are multiples of 4 and pointers 16-byte aligned; hidden <= 16384,
 * n_groups <= 65535, backward n_groups (n_docs + 2050) <= 2^28.
 * ------------------------------------------------------------------------- */
typedef struct {
  int32_t dtype;                       /* of out and dout; everything else is fp32 */
  int32_t rows, hidden, n_docs, n_groups;
  int32_t mods_stride, shift_off, scale_off;
  const int32_t* row_off;              /* dev [n_docs + 1] */
  const int32_t* group;                /* dev [n_docs], each in [0, n_groups); the document is left alone otherwise */
} br_norm_shape;

/* Of the backward call; at most 8 max(hidden, 64) (rows / 16 + 2 n_docs + 1024) bytes. */
size_t br_layer_norm_workspace_bytes(const br_norm_shape* shape);

/* x dev [rows, hidden] fp32; out dev out [rows, hidden]; mean, rstd dev out [rows] or both NULL. */
br_status br_layer_norm_forward(const br_norm_shape* shape, const float* x, const float* mods, void* out,
                                float* mean, float* rstd, void* stream);

/* dx[r] = residual[r] + rstd (g - mean(g) - y mean(g y)),  g = dout[r] (1 + scale);
 * dmods at shift_off = sum over the group's rows of dout, at scale_off = that of dout y (0 for a group without rows).
 *   residual dev [rows, hidden] fp32 or NULL (0): the gradient that reaches x past the norm; dx may be the same memory
 *   dmods    dev out [n_groups, mods_stride]: the two vectors of every group are written, the rest is not touched
 * Sums are taken in a fixed order. */
br_status br_layer_norm_backward(const br_norm_shape* shape, const void* dout, const float* x, const float* mean,
                                 const float* rstd, const float* mods, const float* residual, float* dx,
                                 float* dmods, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------- *
 * The clipped objective of Eq. 5 over kept edges, and its gradient with respect to the velocities.
 * ------------------------------------------------------------------------- */

/* Tables of a set of edges (host only): its rows are the distinct parents of the edges in ascending order, which are
 * the samples that a training pass of the network evaluates.  Row r: node row_parent[r]; edges row_first[r] ..
 * row_first[r + 1] - 1 of edge_ids; coefficients row_coef[4 r ..]: a_z, a_v, h, c0 with
 *   mu = a_z z + a_v v,   log-density of a child z_c = c0 - h |z_c - mu|^2   (h = c0 = 0 on steps without noise)
 * of the parent's step (as br_logprob defines them, divided by D if MEAN).
 *   edge_ids host [n_edges], strictly ascending global child ids, none a root
 *   row_parent host out [n_edges], row_first host out [n_edges + 1], row_coef host out [4 n_edges]: n_rows entries are written
 *   n_rows host out [1] */
br_status br_edge_rows(const br_tree* tree, const br_sched* sched, int64_t D, const int32_t* edge_ids, int32_t n_edges,
                       int32_t* row_parent, int32_t* row_first, double* row_coef, int32_t* n_rows);

typedef struct {
  int64_t D;                           /* values of a latent, a multiple of 4 */
  int32_t n_nodes;                     /* rows of z_nodes, logp_old_nodes and adv_nodes */
  int32_t n_rows, n_edges;             /* n_rows = n_edges = 0: J = 0 */
  int32_t n_total;                     /* divisor of the mean, >= 1 (several calls may share one objective); 0: n_edges */
  float clip_eps;                      /* >= 0 */
  const int32_t *edge_ids, *row_parent, *row_first;   /* dev [n_edges], [n_rows], [n_rows + 1] */
  const double* row_coef;              /* dev [n_rows, 4] */
} br_edge_set;

size_t br_grpo_backward_workspace_bytes(const br_edge_set* edges);

/* For every edge e with child c, row r and rho = exp(logp_new[e] - logp_old_nodes[c]):
 *   J = 1/n sum_e min(rho A_c, clip(rho, 1 - clip_eps, 1 + clip_eps) A_c)
 *   grad_v[r] = d(-J)/dv[r] = -1/n sum over the row's edges, those left out where the clipped term is the smaller one, of
 *               rho A_c 2 h a_v (z_c - mu)
 *   z_nodes dev [n_nodes, D] fp32; v_rows dev [n_rows, D]; logp_old_nodes, adv_nodes dev [n_nodes]
 *   J dev out [1]; logp_new dev out [n_edges]; grad_v dev out [n_rows, D]
 *   clipped dev out [n_edges] or NULL: 1 for an edge left out, else 0
 * Node ids outside [0, n_nodes) and edges outside [0, n_edges) are taken as the nearest valid ones. */
br_status br_grpo_backward(const br_edge_set* edges, const float* z_nodes, const float* v_rows,
                           const float* logp_old_nodes, const float* adv_nodes, float* J, float* logp_new,
                           float* grad_v, uint8_t* clipped, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------- *
 * AdamW over many tensors at once (decoupled weight decay):
 *   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2,
 *   p = p (1 - lr weight_decay) - lr / (1 - beta1^step) m / (sqrt(v / (1 - beta2^step)) + eps)
 * States in 8 bits hold m and sqrt(v) in blocks of 256 elements of a tensor, each with the scale that takes the block's
 * largest value to the largest code.  A code has 4 bits of exponent e and M bits of mantissa f (M = 3 behind a sign bit
 * for m, 4 for sqrt(v)) and stands for f at e = 0, (f + 2^M) 2^(e - 1) above, times the scale.  Values go to one of the two
 * neighbouring codes at random, with probabilities that keep their mean: a change of 0.1 % a step, which rounding to the
 * nearest would never see, moves a second moment as it should.  The random bits of elements 4 q .. 4 q + 3 of tensor
 * number i are the words of Philox4x32-10 at counter (q, i, step, 4) keyed by `seed`, low halves for m, high ones for sqrt(v).
 * A block with a value that is not finite becomes NaN; one without a value above 2^-96 is held as zeros.
 * ------------------------------------------------------------------------- */
typedef struct {
  float* param;                        /* dev [n] */
  const void* grad;                    /* dev [n] in grad_dtype */
  void *m, *v;                         /* dev [n]: fp32, or uint8 codes of m and of sqrt(v) */
  float *m_scale, *v_scale;            /* dev [ceil(n / 256)] (8 bits) or NULL */
  void* copy;                          /* dev [n] bf16 or NULL: the parameter rounded, as the network reads it */
  int64_t n;                           /* >= 0 */
  double weight_decay;
} br_adamw_tensor;

typedef struct {
  double lr, beta1, beta2, eps;        /* 0 <= beta < 1, eps >= 0 */
  int64_t step;                        /* >= 1: number of this step */
  uint64_t seed;
  int32_t grad_dtype;                  /* BR_F32 / BR_BF16 */
  int32_t state_bits;                  /* 32 or 8 */
  const float* grad_scale;             /* dev [1] or NULL: a factor of every gradient (clipping by a norm, loss scaling) */
} br_adamw_cfg;

/* tensors host [n_tensors]; one launch for 48 of them.
 * The step's number, learning rate and corrections travel with the launch: a graph that has captured a call (states in 32 bits) takes the same step
 * again on every replay, reading gradients and *grad_scale anew.  States in 8 bits cannot be captured (BR_EINVAL): replays would draw the same random bits. */
br_status br_adamw_step(const br_adamw_cfg* cfg, const br_adamw_tensor* tensors, int32_t n_tensors, void* stream);

/* The values that 8-bit states stand for (m, and the second moment v itself), as 32-bit states hold them: for checkpoints
 * and checks.  m_out, v_out host [n_tensors] of dev out [n] fp32. */
br_status br_adamw_state_values(const br_adamw_tensor* tensors, int32_t n_tensors, float* const* m_out,
                                float* const* v_out, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* BRANCHROLLOUT_TRAIN_H */
