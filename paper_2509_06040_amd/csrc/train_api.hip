// C-ABI entry points of the operators of a policy update: argument checks, host tables.
#include <math.h>

#include "../../include/branchrollout_train.h"
#include "common.h"
#include "kernels.h"
#include "train.h"

using namespace br;

static bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// ------------------------------------------------------------------ attention
static br_status attn_check(const br_attn_shape* s, const char* who, bool backward) {
  const std::string w = who;
  BR_REQUIRE(s, BR_EINVAL, w + ": NULL shape");
  BR_REQUIRE(s->dtype == BR_F32 || s->dtype == BR_BF16, BR_EINVAL, w + ": unknown dtype");
  BR_REQUIRE(s->n_heads >= 1 && s->n_kv_heads >= 1 && s->n_heads % s->n_kv_heads == 0, BR_EINVAL, w + ": n_heads must be a multiple of n_kv_heads");
  BR_REQUIRE(s->n_docs >= 0 && s->q_tokens >= 0 && s->k_tokens >= 0, BR_EINVAL, w + ": bad sizes");
  BR_REQUIRE(s->q_off && s->k_off, BR_EINVAL, w + ": NULL offsets");
  BR_REQUIRE(s->scale >= 0.f && isfinite(s->scale), BR_EINVAL, w + ": scale must be finite and not negative");
  const int d = s->head_dim;
  BR_REQUIRE(d == 64 || d == 128 || (s->dtype == BR_F32 && (d == 16 || d == 32)), BR_ESHAPE, w + ": head_dim must be 64 or 128 (fp32: 16, 32 too)");
  BR_REQUIRE(s->n_heads <= 65535 && s->n_docs <= (1 << 24) && s->q_tokens <= 0x7FFFFF00 && s->k_tokens <= 0x7FFFFF00, BR_ESHAPE, w + ": too many heads, documents or tokens");
  const int64_t nq = (int64_t)s->n_heads * d, nk = (int64_t)s->n_kv_heads * d, unit = s->dtype == BR_BF16 ? 8 : 4;
  auto stride = [&](int64_t v, int64_t least) { return v >= least && v % unit == 0 && v < (1LL << 31); };
  BR_REQUIRE(stride(s->q_stride, nq) && stride(s->o_stride, nq) && stride(s->k_stride, nk) && stride(s->v_stride, nk), BR_ESHAPE,
             w + ": strides must hold all heads of a token and be multiples of 16 bytes");
  if (backward)
    BR_REQUIRE(stride(s->dq_stride, nq) && stride(s->dk_stride, nk) && stride(s->dv_stride, nk), BR_ESHAPE,
               w + ": strides of the gradients must hold all heads of a token and be multiples of 16 bytes");
  return BR_OK;
}

extern "C" size_t br_attention_workspace_bytes(const br_attn_shape* s, int32_t backward) {
  return attn_check(s, "br_attention_workspace_bytes", backward != 0) == BR_OK ? attn_train_workspace(*s, backward != 0) : 0;
}

extern "C" br_status br_attention_forward(const br_attn_shape* s, const void* q, const void* k, const void* v, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  const br_status ok = attn_check(s, "br_attention_forward", false);
  if (ok != BR_OK) return ok;
  if (s->q_tokens == 0) return BR_OK;
  BR_REQUIRE(q && out && lse && (s->k_tokens == 0 || (k && v)), BR_EINVAL, "br_attention_forward: NULL argument");
  BR_REQUIRE(aligned16(q) && aligned16(k) && aligned16(v) && aligned16(out), BR_ESHAPE, "br_attention_forward: pointers must be 16-byte aligned");
  const size_t need = attn_train_workspace(*s, false);
  BR_REQUIRE(need == 0 || (ws && ws_bytes >= need && aligned16(ws)), BR_EWORKSPACE, "br_attention_forward: workspace too small");
  return launch_attn_train_forward(*s, q, k, v, out, lse, ws, (hipStream_t)stream);
}

extern "C" br_status br_attention_backward(const br_attn_shape* s, const void* dout, const void* q, const void* k, const void* v, const void* out, const float* lse, void* dq, void* dk,
                                           void* dv, void* ws, size_t ws_bytes, void* stream) {
  const br_status ok = attn_check(s, "br_attention_backward", true);
  if (ok != BR_OK) return ok;
  BR_REQUIRE((s->q_tokens == 0 || (dout && q && out && lse && dq)) && (s->k_tokens == 0 || (k && v && dk && dv)), BR_EINVAL, "br_attention_backward: NULL argument");
  BR_REQUIRE(aligned16(dout) && aligned16(q) && aligned16(k) && aligned16(v) && aligned16(out) && aligned16(dq) && aligned16(dk) && aligned16(dv), BR_ESHAPE,
             "br_attention_backward: pointers must be 16-byte aligned");
  const size_t need = attn_train_workspace(*s, true);
  BR_REQUIRE(need == 0 || (ws && ws_bytes >= need && aligned16(ws)), BR_EWORKSPACE, "br_attention_backward: workspace too small");
  return launch_attn_train_backward(*s, dout, q, k, v, out, lse, dq, dk, dv, ws, (hipStream_t)stream);
}

// ----------------------------------------------------------------- layer norm
static br_status norm_check(const br_norm_shape* s, const char* who, bool backward) {
  const std::string w = who;
  BR_REQUIRE(s, BR_EINVAL, w + ": NULL shape");
  BR_REQUIRE(s->dtype == BR_F32 || s->dtype == BR_BF16, BR_EINVAL, w + ": unknown dtype");
  BR_REQUIRE(s->rows >= 0 && s->n_docs >= 0 && s->n_groups >= 1 && s->hidden >= 4, BR_EINVAL, w + ": bad sizes");
  BR_REQUIRE(s->row_off && (s->n_docs == 0 || s->group), BR_EINVAL, w + ": NULL offsets or groups");
  BR_REQUIRE(s->hidden % 4 == 0 && s->mods_stride % 4 == 0 && s->shift_off % 4 == 0 && s->scale_off % 4 == 0, BR_ESHAPE, w + ": hidden, mods_stride and offsets must be multiples of 4");
  BR_REQUIRE(s->hidden <= 16384 && s->n_docs <= (1 << 24) && s->n_groups <= 65535 && s->rows <= 0x7FFFFF00, BR_ESHAPE, w + ": hidden above 16384, or too many documents, groups or rows");
  BR_REQUIRE(s->shift_off >= 0 && s->scale_off >= 0 && (int64_t)s->shift_off + s->hidden <= s->mods_stride && (int64_t)s->scale_off + s->hidden <= s->mods_stride, BR_EINVAL,
             w + ": shift and scale must lie within a group's vectors");
  // (each group's join reads the groups of all tiles: 15 360 groups of one document each take 37 ms at hidden = 1024)
  BR_REQUIRE(!backward || (int64_t)s->n_groups * (s->n_docs + 2050LL) <= (1LL << 28), BR_ESHAPE, w + ": too many groups for so many documents");
  return BR_OK;
}

extern "C" size_t br_layer_norm_workspace_bytes(const br_norm_shape* s) {
  return norm_check(s, "br_layer_norm_workspace_bytes", true) == BR_OK ? norm_train_workspace(*s) : 0;
}

extern "C" br_status br_layer_norm_forward(const br_norm_shape* s, const float* x, const float* mods, void* out, float* mean, float* rstd, void* stream) {
  const br_status ok = norm_check(s, "br_layer_norm_forward", false);
  if (ok != BR_OK) return ok;
  if (s->rows == 0) return BR_OK;
  BR_REQUIRE(x && mods && out && (mean != nullptr) == (rstd != nullptr), BR_EINVAL, "br_layer_norm_forward: NULL argument");
  BR_REQUIRE(aligned16(x) && aligned16(mods) && aligned16(out), BR_ESHAPE, "br_layer_norm_forward: pointers must be 16-byte aligned");
  return launch_norm_forward(*s, x, mods, out, mean, rstd, (hipStream_t)stream);
}

extern "C" br_status br_layer_norm_backward(const br_norm_shape* s, const void* dout, const float* x, const float* mean, const float* rstd, const float* mods, const float* residual,
                                            float* dx, float* dmods, void* ws, size_t ws_bytes, void* stream) {
  const br_status ok = norm_check(s, "br_layer_norm_backward", true);
  if (ok != BR_OK) return ok;
  BR_REQUIRE(dmods && (s->rows == 0 || (dout && x && mean && rstd && mods && dx)), BR_EINVAL, "br_layer_norm_backward: NULL argument");
  const int gap = s->shift_off > s->scale_off ? s->shift_off - s->scale_off : s->scale_off - s->shift_off;
  BR_REQUIRE(gap >= s->hidden, BR_EINVAL, "br_layer_norm_backward: the gradients of shift and scale overlap");
  BR_REQUIRE(aligned16(dout) && aligned16(x) && aligned16(mods) && aligned16(residual) && aligned16(dx) && aligned16(dmods), BR_ESHAPE,
             "br_layer_norm_backward: pointers must be 16-byte aligned");
  const size_t need = norm_train_workspace(*s);
  BR_REQUIRE(ws && ws_bytes >= need && aligned16(ws), BR_EWORKSPACE, "br_layer_norm_backward: workspace too small");
  return launch_norm_backward(*s, dout, x, mean, rstd, mods, residual, dx, dmods, ws, (hipStream_t)stream);
}

// ------------------------------------------------------------------ objective
extern "C" br_status br_edge_rows(const br_tree* t, const br_sched* sched, int64_t D, const int32_t* ids, int32_t n, int32_t* row_parent, int32_t* row_first, double* row_coef,
                                  int32_t* n_rows) {
  BR_REQUIRE(t && sched && row_first && n_rows && (n == 0 || (ids && row_parent && row_coef)), BR_EINVAL, "br_edge_rows: NULL argument");
  BR_REQUIRE(n >= 0 && D >= 1 && sched->t && sched->sigma && sched->T == t->T, BR_EINVAL, "br_edge_rows: bad sizes, or a schedule of another length than the tree");
  BR_REQUIRE(sched->logp_reduce == BR_LOGP_SUM || sched->logp_reduce == BR_LOGP_MEAN, BR_EINVAL, "br_edge_rows: unknown logp_reduce");
  for (int i = 0; i < t->T; ++i)
    BR_REQUIRE(sched->t[i] > sched->t[i + 1] && sched->t[i] > 0.f && sched->sigma[i] >= 0.f && isfinite(sched->sigma[i]), BR_EINVAL,
               "br_edge_rows: times must descend and stay above 0, sigma must not be negative");
  const int64_t nodes = (int64_t)t->n_tree * t->n_nodes;
  int rows = 0;
  for (int e = 0; e < n; ++e) {
    const int id = ids[e];
    BR_REQUIRE(id >= 0 && id < nodes && (e == 0 || id > ids[e - 1]) && id % t->n_nodes != 0, BR_EINVAL, "br_edge_rows: edge ids must ascend strictly and name children");
    const int local = id % t->n_nodes, parent = id - local + t->parent[local];
    if (rows > 0 && row_parent[rows - 1] == parent) continue;
    const StepCoef c = step_coef(sched, t->depth[local] - 1, D);
    const double sd = c.noise ? (double)sched->sigma[t->depth[local] - 1] * sqrt((double)sched->t[t->depth[local] - 1] - (double)sched->t[t->depth[local]]) : 0.0;
    row_parent[rows] = parent;
    row_first[rows] = e;
    row_coef[4 * rows] = c.a_z;
    row_coef[4 * rows + 1] = c.a_v;
    row_coef[4 * rows + 2] = c.noise ? 0.5 / (sd * sd) * c.inv_div : 0.0;
    row_coef[4 * rows + 3] = c.c0 * c.inv_div;
    ++rows;
  }
  row_first[rows] = n;
  *n_rows = rows;
  return BR_OK;
}

static br_status edges_check(const br_edge_set* e, const char* who) {
  const std::string w = who;
  BR_REQUIRE(e, BR_EINVAL, w + ": NULL edge set");
  BR_REQUIRE(e->D >= 4 && e->n_rows >= 0 && e->n_edges >= e->n_rows && (e->n_edges == 0) == (e->n_rows == 0) && e->n_total >= 0 && e->n_nodes >= 1, BR_EINVAL, w + ": bad sizes");
  BR_REQUIRE(e->D % 4 == 0, BR_ESHAPE, w + ": D must be a multiple of 4");
  BR_REQUIRE(e->clip_eps >= 0.f && isfinite(e->clip_eps), BR_EINVAL, w + ": clip_eps must be finite and not negative");
  BR_REQUIRE(e->n_edges == 0 || (e->edge_ids && e->row_parent && e->row_first && e->row_coef), BR_EINVAL, w + ": NULL table");
  return BR_OK;
}

extern "C" size_t br_grpo_backward_workspace_bytes(const br_edge_set* e) {
  return edges_check(e, "br_grpo_backward_workspace_bytes") == BR_OK ? objective_grad_workspace(*e) : 0;
}

extern "C" br_status br_grpo_backward(const br_edge_set* e, const float* z, const float* v, const float* logp_old, const float* adv, float* J, float* logp_new, float* grad,
                                      uint8_t* clipped, void* ws, size_t ws_bytes, void* stream) {
  const br_status ok = edges_check(e, "br_grpo_backward");
  if (ok != BR_OK) return ok;
  BR_REQUIRE(J && (e->n_edges == 0 || (z && v && logp_old && adv && logp_new && grad)), BR_EINVAL, "br_grpo_backward: NULL argument");
  BR_REQUIRE(aligned16(z) && aligned16(v) && aligned16(grad), BR_ESHAPE, "br_grpo_backward: pointers must be 16-byte aligned");
  if (e->n_edges == 0) return launch_fill_zero(J, 1, (hipStream_t)stream);
  const size_t need = objective_grad_workspace(*e);
  BR_REQUIRE(ws && ws_bytes >= need && aligned16(ws), BR_EWORKSPACE, "br_grpo_backward: workspace too small");
  return launch_objective_grad(*e, z, v, logp_old, adv, J, logp_new, grad, clipped, ws, (hipStream_t)stream);
}

// ---------------------------------------------------------------------- AdamW
extern "C" br_status br_adamw_step(const br_adamw_cfg* c, const br_adamw_tensor* t, int32_t n, void* stream) {
  BR_REQUIRE(c && (n == 0 || t) && n >= 0, BR_EINVAL, "br_adamw_step: NULL argument or negative count");
  BR_REQUIRE(c->grad_dtype == BR_F32 || c->grad_dtype == BR_BF16, BR_EINVAL, "br_adamw_step: unknown grad_dtype");
  BR_REQUIRE(c->state_bits == 32 || c->state_bits == 8, BR_EINVAL, "br_adamw_step: state_bits is 32 or 8");
  BR_REQUIRE(c->step >= 1 && c->beta1 >= 0 && c->beta1 < 1 && c->beta2 >= 0 && c->beta2 < 1 && c->eps >= 0 && isfinite(c->eps) && isfinite(c->lr), BR_EINVAL,
             "br_adamw_step: step starts at 1, 0 <= beta < 1, eps >= 0, lr finite");
  if (c->state_bits == 8) {
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing((hipStream_t)stream, &capture) != hipSuccess) (void)hipGetLastError();  // (no device here, or a stream that the launch itself will refuse)
    BR_REQUIRE(capture == hipStreamCaptureStatusNone, BR_EINVAL, "br_adamw_step: a captured step would draw the same random bits on every replay: states in 8 bits cannot be captured");
  }
  for (int i = 0; i < n; ++i) {
    BR_REQUIRE(t[i].n >= 0 && isfinite(t[i].weight_decay), BR_EINVAL, "br_adamw_step: negative size or weight decay that is not finite");
    BR_REQUIRE(t[i].n < (1LL << 34), BR_ESHAPE, "br_adamw_step: more than 2^34 elements in a tensor");
    if (t[i].n == 0) continue;
    BR_REQUIRE(t[i].param && t[i].grad && t[i].m && t[i].v && (c->state_bits == 32 || (t[i].m_scale && t[i].v_scale)), BR_EINVAL, "br_adamw_step: NULL tensor");
    auto aligned = [](const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; };
    BR_REQUIRE(aligned(t[i].param, 4) && aligned(t[i].grad, c->grad_dtype == BR_F32 ? 4 : 2) && aligned(t[i].copy, 2) && aligned(t[i].m_scale, 4) && aligned(t[i].v_scale, 4) &&
                   (c->state_bits == 8 || (aligned(t[i].m, 4) && aligned(t[i].v, 4))), BR_ESHAPE, "br_adamw_step: a tensor is not aligned to its elements");
  }
  return launch_adamw(*c, t, n, (hipStream_t)stream);
}

extern "C" br_status br_adamw_state_values(const br_adamw_tensor* t, int32_t n, float* const* m, float* const* v, void* stream) {
  BR_REQUIRE(n >= 0 && (n == 0 || (t && m && v)), BR_EINVAL, "br_adamw_state_values: NULL argument or negative count");
  for (int i = 0; i < n; ++i) {
    BR_REQUIRE(t[i].n >= 0 && t[i].n < (1LL << 34), BR_EINVAL, "br_adamw_state_values: bad size");
    BR_REQUIRE(t[i].n == 0 || (t[i].m && t[i].v && t[i].m_scale && t[i].v_scale && m[i] && v[i]), BR_EINVAL, "br_adamw_state_values: NULL tensor");
    BR_REQUIRE(t[i].n == 0 || (((reinterpret_cast<uintptr_t>(m[i]) | reinterpret_cast<uintptr_t>(v[i])) & 3) == 0), BR_ESHAPE, "br_adamw_state_values: outputs must be aligned");
  }
  return launch_adamw_values(t, n, m, v, (hipStream_t)stream);
}
