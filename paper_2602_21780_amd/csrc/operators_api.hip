// Host side of the stateless operators around the step: checks of arguments, then the launches, three at most, on the caller's stream.
// Nothing here allocates, waits, keeps anything between calls or throws.
#include "../../include/xsv.h"

#include <algorithm>
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

bool check_pages(const xsv_pages* p) {
  if (!p || p->pages < 0 || p->kv_heads < 1 || p->sequences < 0 || p->table_width < 0) return false;
  if (p->pages > 0 && (!p->k || !p->v || !p->k_scale || !p->v_scale)) return false;
  if (!aligned_to(p->k, 16) || !aligned_to(p->v, 16) || !aligned_to(p->k_bounds, 16) || !aligned_to(p->k_scale, 4) || !aligned_to(p->v_scale, 4)) return false;
  if (p->sequences > 0 && (!p->lengths || (p->table_width > 0 && !p->table))) return false;
  return aligned_to(p->table, 4) && aligned_to(p->lengths, 4);
}
bool pages_supported(const xsv_pages& p) { return p.kv_heads <= (1 << 16) && p.table_width <= (1 << 24); }

PagesArgs pages_args(const xsv_pages& p) {
  PagesArgs a{};
  a.k = static_cast<uint8_t*>(p.k); a.v = static_cast<uint8_t*>(p.v);
  a.k_scale = p.k_scale; a.v_scale = p.v_scale;
  a.bounds = static_cast<uint16_t*>(p.k_bounds);
  a.table = p.table; a.lengths = p.lengths;
  a.pages = p.pages; a.kv_heads = p.kv_heads; a.sequences = p.sequences; a.width = p.table_width;
  a.longest_k = 1 << 30;  // (the most that a table holds)
  return a;
}

int check_query(const xsv_pages* p, const xsv_pages_query* c) {
  if (!check_pages(p) || !c || c->heads < 1 || c->heads % p->kv_heads != 0 || c->rows < 0 || c->longest_q < 0 || c->longest_q > c->rows || c->longest_k < 0)
    return XSV_ERR_ARG;
  if (c->causal < 0 || c->count < 0 || c->first < 0 || c->last < 0) return XSV_ERR_ARG;
  if (c->softmax_scale != 0.0f && !(c->softmax_scale >= 1e-20f && c->softmax_scale <= 1e20f)) return XSV_ERR_ARG;
  if (!aligned_to(c->q_begin, 4) || !aligned_to(c->chosen, 4) || (p->sequences > 0 && !c->q_begin)) return XSV_ERR_ARG;
  if (!pages_supported(*p) || c->heads > (1 << 16) || c->count > (1 << 24)) return XSV_ERR_UNSUPPORTED;
  return XSV_OK;
}

PagesArgs query_args(const xsv_pages& p, const xsv_pages_query& c) {
  PagesArgs a = pages_args(p);
  a.begin = c.q_begin;
  a.rows = c.rows; a.longest = c.longest_q;
  a.longest_k = std::min(c.longest_k, p.table_width * 64);
  a.heads = c.heads; a.causal = c.causal;
  a.scale = c.softmax_scale == 0.0f ? 1.0f / std::sqrt((float)kD) : c.softmax_scale;
  a.count = c.count; a.first = c.first; a.last = c.last;
  a.chosen = c.count > 0 ? c.chosen : nullptr;
  return a;
}

// A tensor of `rows` rows; one without rows is not looked at.
bool rows_of(const xsv_tensor& t, int rows, SeqRows* r) {
  if (rows > 0 && !operand_ok(t)) return false;
  r->p = static_cast<const uint16_t*>(t.ptr); r->sh = t.stride_head; r->st = t.stride_token;
  return true;
}

// The rows that a call writes or reads.
int move_args(const xsv_pages* p, const int32_t* begin, int rows, int longest, const xsv_tensor& k, const xsv_tensor& v, PagesArgs* a) {
  if (!check_pages(p) || rows < 0 || longest < 0 || longest > rows || !aligned_to(begin, 4) || (p->sequences > 0 && !begin)) return XSV_ERR_ARG;
  if (!pages_supported(*p)) return XSV_ERR_UNSUPPORTED;
  *a = pages_args(*p);
  a->begin = begin;
  a->rows = rows; a->longest = longest;
  if (!rows_of(k, rows, &a->keys) || !rows_of(v, rows, &a->values)) return XSV_ERR_ARG;
  return pages_move_fits(*a) ? XSV_OK : XSV_ERR_UNSUPPORTED;
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

int xsv_pages_write(void* hip_stream, const xsv_pages* p, const int32_t* begin, int rows, int longest, xsv_tensor k, xsv_tensor v) {
  PagesArgs a;
  const int rc = move_args(p, begin, rows, longest, k, v, &a);
  return rc != XSV_OK ? rc : launched(launch_pages_write(a, static_cast<hipStream_t>(hip_stream)));
}

int xsv_pages_read(void* hip_stream, const xsv_pages* p, const int32_t* begin, int rows, int longest, xsv_tensor k, xsv_tensor v) {
  PagesArgs a;
  const int rc = move_args(p, begin, rows, longest, k, v, &a);
  return rc != XSV_OK ? rc : launched(launch_pages_read(a, static_cast<hipStream_t>(hip_stream)));
}

int xsv_pages_attend_workspace(const xsv_pages* p, const xsv_pages_query* c, int64_t* bytes) {
  const int rc = check_query(p, c);
  if (rc != XSV_OK) return rc;
  if (!bytes) return XSV_ERR_ARG;
  const PagesArgs a = query_args(*p, *c);
  if (!pages_attend_fits(a)) return XSV_ERR_UNSUPPORTED;
  *bytes = pages_attend_workspace(a);
  return XSV_OK;
}

int xsv_pages_attend(void* hip_stream, const xsv_pages* p, const xsv_pages_query* c, xsv_tensor q, xsv_tensor out, float* lse, void* workspace,
                     int64_t workspace_bytes) {
  int64_t need = 0;
  const int rc = xsv_pages_attend_workspace(p, c, &need);
  if (rc != XSV_OK) return rc;
  PagesArgs a = query_args(*p, *c);
  if (!rows_of(q, c->rows, &a.q) || !rows_of(out, c->rows, &a.out)) return XSV_ERR_ARG;
  if (c->rows > 0 && (!lse || !aligned_to(lse, 4))) return XSV_ERR_ARG;
  if (need > 0 && (!workspace || !aligned_to(workspace, 16) || workspace_bytes < need)) return XSV_ERR_ARG;
  a.lse = lse;
  a.part = static_cast<float*>(workspace);
  return launched(launch_pages_attend(a, static_cast<hipStream_t>(hip_stream)));
}

int xsv_pages_select(void* hip_stream, const xsv_pages* p, const xsv_pages_query* c, xsv_tensor q, int32_t* chosen) {
  const int rc = check_query(p, c);
  if (rc != XSV_OK) return rc;
  if ((long long)c->first + c->last > c->count || c->count < 1 || (p->pages > 0 && !p->k_bounds)) return XSV_ERR_ARG;
  PagesArgs a = query_args(*p, *c);
  if (!rows_of(q, c->rows, &a.q) || (c->rows > 0 && (!chosen || !aligned_to(chosen, 4)))) return XSV_ERR_ARG;
  a.choice = chosen;
  if (!pages_select_fits(a)) return XSV_ERR_UNSUPPORTED;
  return launched(launch_pages_select(a, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
