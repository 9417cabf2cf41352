// Launch wrappers of the operators of a policy update; internal.
#pragma once
#include "../../include/branchrollout_train.h"
#include "common.h"

namespace br {

// ---- attn_train.hip
size_t attn_train_workspace(const br_attn_shape& s, bool backward);
br_status launch_attn_train_forward(const br_attn_shape& s, const void* q, const void* k, const void* v, void* out, float* lse, void* ws, hipStream_t st);
br_status launch_attn_train_backward(const br_attn_shape& s, const void* dout, const void* q, const void* k, const void* v, const void* out, const float* lse, void* dq, void* dk,
                                     void* dv, void* ws, hipStream_t st);

// ---- norm_train.hip
size_t norm_train_workspace(const br_norm_shape& s);
br_status launch_norm_forward(const br_norm_shape& s, const float* x, const float* mods, void* out, float* mean, float* rstd, hipStream_t st);
br_status launch_norm_backward(const br_norm_shape& s, const void* dout, const float* x, const float* mean, const float* rstd, const float* mods, const float* residual, float* dx,
                               float* dmods, void* ws, hipStream_t st);

// ---- objective_grad.hip
size_t objective_grad_workspace(const br_edge_set& e);
br_status launch_objective_grad(const br_edge_set& e, const float* z, const float* v, const float* logp_old, const float* adv, float* J, float* logp_new, float* grad,
                                unsigned char* clipped, void* ws, hipStream_t st);

// ---- adamw.hip
br_status launch_adamw(const br_adamw_cfg& c, const br_adamw_tensor* t, int n, hipStream_t st);
br_status launch_adamw_values(const br_adamw_tensor* t, int n, float* const* m, float* const* v, hipStream_t st);

}  // namespace br
