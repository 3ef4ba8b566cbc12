// Internal interface of the stateless operators around the step (not part of the ABI): what operators_api.hip has checked and
// hands to the kernels of rotate.hip, seq_attend.hip, pages.hip, pages_attend.hip and pages_select.hip.
#pragma once

#include "xsv_internal.h"

namespace xsv {

constexpr int kAngles = kD / 2;  // rotated pairs of a row: 32 on one axis, 16 on each of two

// One of the two tensors a rotate launch works on (queries or keys), strides in elements.
struct RotateTensor {
  const uint16_t* x;    // rows before the norm
  const uint16_t* dy;   // gradient only: of the rotated rows
  uint16_t* y;          // rotated rows; gradient: of x
  int64_t x_sh, x_st, dy_sh, dy_st, y_sh, y_st;
  const float* weight;  // [64] or null
  const float* bias;
  int heads;
};
struct RotateArgs {
  RotateTensor t[2];
  const int32_t* positions;  // [n][axes]
  float* partials;           // gradient: [workgroups][4][64], null without weight gradients
  float* weight_grads;       // [4][64]
  float eps;
  int n;
  double turns[kAngles];     // revolutions per position of every pair
};
hipError_t launch_rotate(const RotateArgs& a, int norm, int axes, bool interleaved, hipStream_t stream);
hipError_t launch_rotate_grad(const RotateArgs& a, int norm, int axes, bool interleaved, hipStream_t stream);
int rotate_grad_workgroups(int n, int heads_q, int heads_k);

// Rows of one tensor of a seq_attend call, strides in elements.
struct SeqRows {
  const uint16_t* p;
  int64_t sh, st;
};
struct SeqArgs {
  SeqRows q, k, v, out, dout;  // out: written by the forward pass, read by the gradient
  SeqRows dq, dk, dv;
  float* lse;    // [heads][rows_q]
  float* delta;  // gradient: [heads][rows_q] sums of dout * out, written by the first launch, read by the others
  const int32_t* q_begin;
  const int32_t* k_begin;
  int heads, kv_heads, sequences, rows_q, rows_k, longest_q, longest_k;
  int causal;
  float scale;
  float* part;       // small launches: what workgroups that share the tiles of a block leave, [part][head][row][64]
  float* part_sums;  // and their references and sums, [part][head][row][2]
  int parts;         // workgroups that do so (set by the launchers)
};
int64_t seq_attend_workspace(const SeqArgs& a);   // bytes of SeqArgs::part
int64_t seq_attend_grad_parts(const SeqArgs& a);
hipError_t launch_seq_attend(const SeqArgs& a, hipStream_t stream);
hipError_t launch_seq_attend_grad(const SeqArgs& a, hipStream_t stream);
bool seq_attend_fits(const SeqArgs& a);  // its grids stay within what a launch can have

// A pool of pages in 8 bits, the sequences that it holds, and the rows that a call writes, reads or asks with.
struct PagesArgs {
  uint8_t* k;         // [pages][kv_heads][64 tokens][64 channels]
  uint8_t* v;         // [pages][kv_heads][64 channels][64 tokens]
  float* k_scale;     // [pages][kv_heads]
  float* v_scale;
  uint16_t* bounds;   // fp16 [pages][kv_heads][2][64]
  const int32_t* table;
  const int32_t* lengths;
  const int32_t* begin;
  int pages, kv_heads, sequences, width;
  int rows, longest, longest_k;  // of `begin`; bounds on a sequence's rows and tokens: those behind them are left out
  SeqRows keys, values;          // written or read
  SeqRows q, out;
  float* lse;                    // [heads][rows]
  int heads, causal;
  float scale;
  const int32_t* chosen;         // [rows][kv_heads][count]; null: all pages
  int32_t* choice;               // the same, written
  int count, first, last;
  float* part;                   // attention cut over workgroups: what each leaves, [part][head][row][64]
  float* part_sums;              // and its reference and sum, [part][head][row][2]
  int parts, chunk, group;       // how many share a block of rows, pages for each; queries that share a list of pages (set by the launchers)
  int ranked;                    // blocks are numbered over all sequences
};
hipError_t launch_pages_write(PagesArgs a, hipStream_t stream);
hipError_t launch_pages_read(PagesArgs a, hipStream_t stream);
hipError_t launch_pages_attend(const PagesArgs& a, hipStream_t stream);
hipError_t launch_pages_select(const PagesArgs& a, hipStream_t stream);
int64_t pages_attend_workspace(const PagesArgs& a);  // bytes of PagesArgs::part
bool pages_move_fits(const PagesArgs& a);            // their grids stay within what a launch can have
bool pages_attend_fits(const PagesArgs& a);
bool pages_select_fits(const PagesArgs& a);

}  // namespace xsv
