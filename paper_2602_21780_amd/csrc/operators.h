// Internal interface of the stateless operators around the step (not part of the ABI): what operators_api.hip has checked and
// hands to the kernels of rotate.hip and seq_attend.hip.
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

}  // namespace xsv
