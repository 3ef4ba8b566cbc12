// Host side of the stateless operators around the step: checks of arguments, then the launches, three at most, on the caller's stream.
// Nothing here allocates, waits, keeps anything between calls or throws.
#include "../../include/xsv.h"

#include <cmath>

#include "operators.h"

using namespace xsv;

namespace {

bool operand_ok(const xsv_tensor& t) {
  return t.ptr != nullptr && t.stride_token >= kD && t.stride_token <= (1ll << 24) && t.stride_head >= 0 &&
         (reinterpret_cast<uintptr_t>(t.ptr) % 16 == 0) && t.stride_token % 8 == 0 && t.stride_head % 8 == 0;
}

bool aligned_to(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

int launched(hipError_t e) { return e == hipSuccess ? XSV_OK : XSV_ERR_HIP; }

int check_rotate(const xsv_rotate_config* c) {
  if (!c || c->n < 0 || c->heads_q < 0 || c->heads_k < 0 || c->heads_q + (long long)c->heads_k == 0) return XSV_ERR_ARG;
  if (c->norm < XSV_NORM_NONE || c->norm > XSV_NORM_LAYER || c->axes < 0 || c->axes > 2) return XSV_ERR_ARG;
  if (c->norm != XSV_NORM_NONE && !(c->eps > 0.0f && std::isfinite(c->eps))) return XSV_ERR_ARG;
  if (c->axes > 0 && !(c->base >= 1.0 && std::isfinite(c->base))) return XSV_ERR_ARG;
  if (c->axes > 0 && c->n > 0 && (!c->positions || !aligned_to(c->positions, 4))) return XSV_ERR_ARG;
  for (const float* p : {c->q_weight, c->q_bias, c->k_weight, c->k_bias})
    if (!aligned_to(p, 4)) return XSV_ERR_ARG;
  if (c->heads_q > (1 << 16) || c->heads_k > (1 << 16)) return XSV_ERR_UNSUPPORTED;
  return XSV_OK;
}

RotateArgs rotate_args(const xsv_rotate_config& c) {
  RotateArgs a{};
  a.t[0].weight = c.q_weight; a.t[0].bias = c.q_bias; a.t[0].heads = c.heads_q;
  a.t[1].weight = c.k_weight; a.t[1].bias = c.k_bias; a.t[1].heads = c.heads_k;
  a.positions = c.positions;
  a.eps = c.eps;
  a.n = c.n;
  const int half = c.axes ? kAngles / c.axes : 1;  // pairs of one axis
  for (int i = 0; c.axes && i < kAngles; ++i) a.turns[i] = i < half ? std::pow(c.base, -(double)i / half) / (2.0 * M_PI) : a.turns[i - half];
  return a;
}

int check_seq(const xsv_seq_config* c) {
  if (!c || c->heads < 1 || c->kv_heads < 1 || c->heads % c->kv_heads != 0 || c->sequences < 0 || c->rows_q < 0 || c->rows_k < 0) return XSV_ERR_ARG;
  if (c->longest_q < 0 || c->longest_k < 0 || c->longest_q > c->rows_q || c->longest_k > c->rows_k || c->causal < 0) return XSV_ERR_ARG;
  if (c->softmax_scale != 0.0f && !(c->softmax_scale >= 1e-20f && c->softmax_scale <= 1e20f)) return XSV_ERR_ARG;
  if (c->sequences > 0 && (!c->q_begin || !c->k_begin || !aligned_to(c->q_begin, 4) || !aligned_to(c->k_begin, 4))) return XSV_ERR_ARG;
  if (c->heads > (1 << 16)) return XSV_ERR_UNSUPPORTED;
  return XSV_OK;
}

SeqArgs seq_args(const xsv_seq_config& c) {
  SeqArgs a{};
  a.q_begin = c.q_begin; a.k_begin = c.k_begin;
  a.heads = c.heads; a.kv_heads = c.kv_heads; a.sequences = c.sequences;
  a.rows_q = c.rows_q; a.rows_k = c.rows_k; a.longest_q = c.longest_q; a.longest_k = c.longest_k;
  a.causal = c.causal;
  a.scale = c.softmax_scale == 0.0f ? 1.0f / std::sqrt((float)kD) : c.softmax_scale;
  return a;
}

// A tensor of `rows` rows; one without rows is not looked at.
bool rows_of(const xsv_tensor& t, int rows, SeqRows* r) {
  if (rows > 0 && !operand_ok(t)) return false;
  r->p = static_cast<const uint16_t*>(t.ptr); r->sh = t.stride_head; r->st = t.stride_token;
  return true;
}

}  // namespace

extern "C" {

int xsv_norm_rotate(void* hip_stream, const xsv_rotate_config* c, xsv_tensor q, xsv_tensor k, xsv_tensor q_out, xsv_tensor k_out) {
  const int rc = check_rotate(c);
  if (rc != XSV_OK) return rc;
  if (c->n == 0) return XSV_OK;
  RotateArgs a = rotate_args(*c);
  const xsv_tensor in[2] = {q, k}, out[2] = {q_out, k_out};
  for (int i = 0; i < 2; ++i) {
    if (a.t[i].heads == 0) continue;
    if (!operand_ok(in[i]) || !operand_ok(out[i])) return XSV_ERR_ARG;
    a.t[i].x = static_cast<const uint16_t*>(in[i].ptr); a.t[i].x_sh = in[i].stride_head; a.t[i].x_st = in[i].stride_token;
    a.t[i].y = static_cast<uint16_t*>(const_cast<void*>(out[i].ptr)); a.t[i].y_sh = out[i].stride_head; a.t[i].y_st = out[i].stride_token;
  }
  return launched(launch_rotate(a, c->norm, c->axes, c->interleaved != 0, static_cast<hipStream_t>(hip_stream)));
}

int xsv_norm_rotate_grad_workspace(const xsv_rotate_config* c, int64_t* bytes) {
  const int rc = check_rotate(c);
  if (rc != XSV_OK) return rc;
  if (!bytes) return XSV_ERR_ARG;
  *bytes = (int64_t)rotate_grad_workgroups(c->n, c->heads_q, c->heads_k) * 4 * kD * (int64_t)sizeof(float);
  return XSV_OK;
}

int xsv_norm_rotate_grad(void* hip_stream, const xsv_rotate_config* c, xsv_tensor q, xsv_tensor k, xsv_tensor dq_out, xsv_tensor dk_out,
                         xsv_tensor dq, xsv_tensor dk, float* weight_grads, void* workspace, int64_t workspace_bytes) {
  int64_t need = 0;
  const int rc = xsv_norm_rotate_grad_workspace(c, &need);
  if (rc != XSV_OK) return rc;
  if (weight_grads && (!aligned_to(weight_grads, 4) || (need > 0 && !workspace) || !aligned_to(workspace, 16) || workspace_bytes < need))
    return XSV_ERR_ARG;
  RotateArgs a = rotate_args(*c);
  const xsv_tensor in[2] = {q, k}, dy[2] = {dq_out, dk_out}, out[2] = {dq, dk};
  for (int i = 0; i < 2 && c->n > 0; ++i) {
    if (a.t[i].heads == 0) continue;
    if (!operand_ok(in[i]) || !operand_ok(dy[i]) || !operand_ok(out[i])) return XSV_ERR_ARG;
    a.t[i].x = static_cast<const uint16_t*>(in[i].ptr); a.t[i].x_sh = in[i].stride_head; a.t[i].x_st = in[i].stride_token;
    a.t[i].dy = static_cast<const uint16_t*>(dy[i].ptr); a.t[i].dy_sh = dy[i].stride_head; a.t[i].dy_st = dy[i].stride_token;
    a.t[i].y = static_cast<uint16_t*>(const_cast<void*>(out[i].ptr)); a.t[i].y_sh = out[i].stride_head; a.t[i].y_st = out[i].stride_token;
  }
  if (weight_grads) {
    a.partials = static_cast<float*>(workspace);
    a.weight_grads = weight_grads;
  }
  return launched(launch_rotate_grad(a, c->norm, c->axes, c->interleaved != 0, static_cast<hipStream_t>(hip_stream)));
}

int xsv_seq_attend_workspace(const xsv_seq_config* c, int64_t* bytes) {
  const int rc = check_seq(c);
  if (rc != XSV_OK) return rc;
  if (!bytes) return XSV_ERR_ARG;
  *bytes = seq_attend_workspace(seq_args(*c));
  return XSV_OK;
}

int xsv_seq_attend(void* hip_stream, const xsv_seq_config* c, xsv_tensor q, xsv_tensor k, xsv_tensor v, xsv_tensor out, float* lse, void* workspace,
                   int64_t workspace_bytes) {
  int64_t need = 0;
  const int rc = xsv_seq_attend_workspace(c, &need);
  if (rc != XSV_OK) return rc;
  SeqArgs a = seq_args(*c);
  if (!rows_of(q, c->rows_q, &a.q) || !rows_of(k, c->rows_k, &a.k) || !rows_of(v, c->rows_k, &a.v) || !rows_of(out, c->rows_q, &a.out)) return XSV_ERR_ARG;
  if (c->rows_q > 0 && (!lse || !aligned_to(lse, 4))) return XSV_ERR_ARG;
  if (need > 0 && (!workspace || !aligned_to(workspace, 16) || workspace_bytes < need)) return XSV_ERR_ARG;
  a.lse = lse;
  a.part = static_cast<float*>(workspace);
  if (!seq_attend_fits(a)) return XSV_ERR_UNSUPPORTED;
  return launched(launch_seq_attend(a, static_cast<hipStream_t>(hip_stream)));
}

// delta, then the parts
static int64_t delta_bytes(const xsv_seq_config& c) { return ((int64_t)c.heads * c.rows_q * (int64_t)sizeof(float) + 15) / 16 * 16; }

int xsv_seq_attend_grad_workspace(const xsv_seq_config* c, int64_t* bytes) {
  const int rc = check_seq(c);
  if (rc != XSV_OK) return rc;
  if (!bytes) return XSV_ERR_ARG;
  *bytes = delta_bytes(*c) + seq_attend_grad_parts(seq_args(*c));
  return XSV_OK;
}

int xsv_seq_attend_grad(void* hip_stream, const xsv_seq_config* c, xsv_tensor q, xsv_tensor k, xsv_tensor v, xsv_tensor out, const float* lse,
                        xsv_tensor dout, xsv_tensor dq, xsv_tensor dk, xsv_tensor dv, void* workspace, int64_t workspace_bytes) {
  int64_t need = 0;
  const int rc = xsv_seq_attend_grad_workspace(c, &need);
  if (rc != XSV_OK) return rc;
  SeqArgs a = seq_args(*c);
  if (!rows_of(q, c->rows_q, &a.q) || !rows_of(k, c->rows_k, &a.k) || !rows_of(v, c->rows_k, &a.v) || !rows_of(out, c->rows_q, &a.out) ||
      !rows_of(dout, c->rows_q, &a.dout) || !rows_of(dq, c->rows_q, &a.dq) || !rows_of(dk, c->rows_k, &a.dk) || !rows_of(dv, c->rows_k, &a.dv))
    return XSV_ERR_ARG;
  if (c->rows_q > 0 && (!lse || !aligned_to(lse, 4))) return XSV_ERR_ARG;
  if (need > 0 && (!workspace || !aligned_to(workspace, 16) || workspace_bytes < need)) return XSV_ERR_ARG;
  a.lse = const_cast<float*>(lse);
  a.delta = static_cast<float*>(workspace);
  a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + delta_bytes(*c));
  if (!seq_attend_fits(a)) return XSV_ERR_UNSUPPORTED;
  return launched(launch_seq_attend_grad(a, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
