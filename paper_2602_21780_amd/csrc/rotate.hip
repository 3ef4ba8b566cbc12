// Norms of queries and keys per head with the position rotation in the same pass, and its gradient.
//
//   hat = x | x / sqrt(mean(x^2) + eps) | (x - mean(x)) / sqrt(var(x) + eps),   y = R(position) (hat * weight + bias)
//
// R turns 32 pairs of a row's 64 channels; pair i of an axis' section of w channels turns by position * base^(-2 i / w).
//   gradient:  g = R^T dy,  d weight = sum g * hat,  d bias = sum g,  u = g * weight,
//              dx = (u - [layer] mean(u) - hat * mean(u * hat)) / sqrt(..)
// Everything between the load and the one rounding of the result is fp32.  What bounds both is memory: 4 (6) bytes per
// element against a few operations.  Measured: 40000 tokens of 40 heads (410 MB) 81 us, 5.1 TB/s; the gradient of 32976 tokens of 32 heads
// (405 MB) 91 us and 5 us for the sums, 4.5 TB/s; a large copy reaches 4.8.  One frame of 1374 tokens takes 5 us, one token 2.6: a launch
// and two waits for memory.
//
// A wave takes one token and eight of its heads at a time: 8 lanes hold a row, 16 bytes each, so that a load
// instruction covers eight whole rows, the sums over a row are three steps among its lanes, and the 32 angles of the
// token are worked out once per wave - one per lane, the cosines in the lower half of the wave and the sines in the upper -
// and handed round, for all heads that the wave takes.  The angle is reduced in fp64: position * turns is exact to 2^-50 of itself, a
// fraction of a revolution is taken of that, and only the rest goes through fp32, so far positions lose nothing.
#include "operators.h"

#include <algorithm>

namespace xsv {
namespace {

constexpr int kWaves = 4;       // waves of a workgroup; they share nothing in the forward pass
constexpr int kRowsAtOnce = 8;  // heads a wave loads with one instruction

using u32x4 = __attribute__((ext_vector_type(4))) uint32_t;

__device__ inline void unpack8(const u32x4 raw, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(raw[i] << 16);
    x[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
  }
}

using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
__device__ inline u32x4 pack8(const float* x) {  // to bf16, nearest even
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bf16x2 p = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
    r[i] = __builtin_bit_cast(uint32_t, p);
  }
  return r;
}

// A value of another lane of the same row, without a round trip through LDS.
template <int CTRL>
__device__ inline float from_lane(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
constexpr int kLane1 = 0xb1, kLane2 = 0x4e, kReverse4 = 0x1b, kReverse8 = 0x141;  // lane ^ 1, lane ^ 2, 3 - lane in four, 7 - lane in eight
template <int MASK>
__device__ inline float mate_of(float v) {  // of lane ^ MASK
  static_assert(MASK == 2 || MASK == 4);
  if (MASK == 2) return from_lane<kLane2>(v);
  return from_lane<kReverse4>(from_lane<kReverse8>(v));
}
__device__ inline float row_sum(float v) {  // over the 8 lanes of a row
  v += from_lane<kLane1>(v);
  v += from_lane<kLane2>(v);
  return v + from_lane<kReverse8>(v);  // (the four lanes of either half hold the same)
}

// Cosine and sine of the pairs that this lane's channels 8c .. 8c + 7 belong to.
template <int AXES, bool INTERLEAVED>
struct Turn {
  static constexpr int kOwn = INTERLEAVED ? 4 : 8;
  float cos_[kOwn], sin_[kOwn];

  __device__ inline void load(const RotateArgs& a, long long token, int lane) {
    const int i = lane % kAngles;
    const int axis = i / (kAngles / AXES);
    double rev = (double)a.positions[token * AXES + axis] * a.turns[i] + (lane < 32 ? 0.25 : 0.0);
    rev -= rint(rev);
    const float v = sinpif(2.0f * (float)rev);  // sin(2 pi (x + 1/4)) = cos(2 pi x)
    const int c = lane % 8;
    int first;  // pair of the lane's first channel
    if (INTERLEAVED) first = 4 * c;
    else if (AXES == 1) first = 8 * (c % 4);
    else first = 16 * (c / 4) + 8 * (c % 2);
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      cos_[j] = __shfl(v, first + j);
      sin_[j] = __shfl(v, 32 + first + j);
    }
  }

  // x turned by +angle (SIGN = 1) or -angle (the transposed rotation)
  template <int SIGN>
  __device__ inline void apply(float* x, int lane) const {
    if (INTERLEAVED) {
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const float u = x[2 * p], w = x[2 * p + 1], s = SIGN * sin_[p];
        x[2 * p] = u * cos_[p] - w * s;
        x[2 * p + 1] = w * cos_[p] + u * s;
      }
      return;
    }
    constexpr int kMate = AXES == 1 ? 4 : 2;  // the lane with the pairs' other channels
    const bool upper = (lane & kMate) != 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float mate = mate_of<kMate>(x[j]);
      const float s = SIGN * sin_[j];
      x[j] = x[j] * cos_[j] + (upper ? mate * s : -(mate * s));
    }
  }
};
template <bool INTERLEAVED>
struct Turn<0, INTERLEAVED> {
  __device__ inline void load(const RotateArgs&, long long, int) {}
  template <int SIGN>
  __device__ inline void apply(float*, int) const {}
};

__device__ inline void load_param(const float* p, int c, float otherwise, float* v) {
  if (p) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = p[8 * c + j];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = otherwise;
  }
}

// x -> hat, returns 1 / sqrt(..)
template <int NORM>
__device__ inline float normalize(float* x, float eps) {
  if (NORM == 0) return 1.0f;
  if (NORM == 2) {
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s += x[j];
    const float mean = row_sum(s) * (1.0f / kD);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] -= mean;
  }
  float s = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) s += x[j] * x[j];
  const float r = 1.0f / sqrtf(row_sum(s) * (1.0f / kD) + eps);
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] *= r;
  return r;
}

// A unit is one token and AT_ONCE batches of eight heads of its queries and keys (queries' batches first).
template <int NORM, int AXES, bool INTERLEAVED, int AT_ONCE>
__global__ __launch_bounds__(64 * kWaves) void rotate_kernel(RotateArgs a, int batches_q, int batches, long long units, int units_per_token) {
  const int lane = threadIdx.x % 64, g = lane / 8, c = lane % 8;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  for (long long unit = (long long)blockIdx.x * kWaves + wave; unit < units; unit += (long long)gridDim.x * kWaves) {
    const long long token = unit / units_per_token;
    const int first = (int)(unit % units_per_token) * AT_ONCE;
    u32x4 raw[AT_ONCE];
#pragma unroll
    for (int b = 0; b < AT_ONCE; ++b) {
      const int batch = first + b;
      if (batch >= batches) break;
      const RotateTensor& t = a.t[batch < batches_q ? 0 : 1];
      const int head = 8 * (batch < batches_q ? batch : batch - batches_q) + g;
      raw[b] = u32x4{};
      if (head < t.heads) raw[b] = *reinterpret_cast<const u32x4*>(t.x + head * t.x_sh + token * t.x_st + 8 * c);
    }
    Turn<AXES, INTERLEAVED> turn;
    turn.load(a, token, lane);
#pragma unroll
    for (int b = 0; b < AT_ONCE; ++b) {
      const int batch = first + b;
      if (batch >= batches) break;
      const RotateTensor& t = a.t[batch < batches_q ? 0 : 1];
      const int head = 8 * (batch < batches_q ? batch : batch - batches_q) + g;
      float x[8], w[8], bias[8];
      load_param(t.weight, c, 1.0f, w);
      load_param(t.bias, c, 0.0f, bias);
      unpack8(raw[b], x);
      normalize<NORM>(x, a.eps);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = x[j] * w[j] + bias[j];
      turn.template apply<1>(x, lane);
      if (head < t.heads) *reinterpret_cast<u32x4*>(t.y + head * t.y_sh + token * t.y_st + 8 * c) = pack8(x);
    }
  }
}

// The gradient: as above, with a lane's sums for the weights' gradients carried over all units of the wave, added up over the
// workgroup at the end and written as one partial of it; rotate_grad_sum adds the partials in their order (no atomics:
// the same bits every time).
template <int NORM, int AXES, bool INTERLEAVED, int AT_ONCE>
__global__ __launch_bounds__(64 * kWaves) void rotate_grad_kernel(RotateArgs a, int batches_q, int batches, long long units, int units_per_token) {
  __shared__ float part[kWaves][4][kD];
  const int lane = threadIdx.x % 64, g = lane / 8, c = lane % 8;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  float dw[2][8] = {}, db[2][8] = {};
  for (long long unit = (long long)blockIdx.x * kWaves + wave; unit < units; unit += (long long)gridDim.x * kWaves) {
    const long long token = unit / units_per_token;
    const int first = (int)(unit % units_per_token) * AT_ONCE;
    u32x4 raw[AT_ONCE], raw_dy[AT_ONCE];
#pragma unroll
    for (int b = 0; b < AT_ONCE; ++b) {
      const int batch = first + b;
      if (batch >= batches) break;
      const RotateTensor& t = a.t[batch < batches_q ? 0 : 1];
      const int head = 8 * (batch < batches_q ? batch : batch - batches_q) + g;
      raw[b] = raw_dy[b] = u32x4{};
      if (head < t.heads) {
        raw[b] = *reinterpret_cast<const u32x4*>(t.x + head * t.x_sh + token * t.x_st + 8 * c);
        raw_dy[b] = *reinterpret_cast<const u32x4*>(t.dy + head * t.dy_sh + token * t.dy_st + 8 * c);
      }
    }
    Turn<AXES, INTERLEAVED> turn;
    turn.load(a, token, lane);
#pragma unroll
    for (int b = 0; b < AT_ONCE; ++b) {
      const int batch = first + b;
      if (batch >= batches) break;
      const int which = batch < batches_q ? 0 : 1;
      const RotateTensor& t = a.t[which];
      const int head = 8 * (which == 0 ? batch : batch - batches_q) + g;
      float x[8], u[8], w[8];
      load_param(t.weight, c, 1.0f, w);
      unpack8(raw[b], x);
      unpack8(raw_dy[b], u);
      turn.template apply<-1>(u, lane);
      const float r = normalize<NORM>(x, a.eps);
      float su = 0.0f, sux = 0.0f;
      auto add = [&](float* to_w, float* to_b) {  // (a lane without a head holds zeros and adds nothing)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          to_w[j] += u[j] * x[j];
          to_b[j] += u[j];
        }
      };
      if (which == 0) add(dw[0], db[0]);
      else add(dw[1], db[1]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        u[j] *= w[j];
        su += u[j];
        sux += u[j] * x[j];
      }
      if (NORM != 0) {
        const float mean_u = NORM == 2 ? row_sum(su) * (1.0f / kD) : 0.0f;
        const float mean_ux = row_sum(sux) * (1.0f / kD);
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] = r * (u[j] - mean_u - x[j] * mean_ux);
      }
      if (head < t.heads) *reinterpret_cast<u32x4*>(t.y + head * t.y_sh + token * t.y_st + 8 * c) = pack8(u);
    }
  }
  if (!a.partials) return;
#pragma unroll
  for (int which = 0; which < 2; ++which)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float sw = dw[which][j], sb = db[which][j];
#pragma unroll
      for (int m = 8; m < 64; m *= 2) {
        sw += __shfl_xor(sw, m);
        sb += __shfl_xor(sb, m);
      }
      if (g == 0) {
        part[wave][2 * which][8 * c + j] = sw;
        part[wave][2 * which + 1][8 * c + j] = sb;
      }
    }
  __syncthreads();
  const int i = threadIdx.x;  // 4 x 64 sums, one a thread
  float s = 0.0f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) s += (&part[w][0][0])[i];
  a.partials[(size_t)blockIdx.x * 4 * kD + i] = s;
}

constexpr int kSumColumns = 16, kSumSlices = 64;
__global__ __launch_bounds__(kSumColumns * kSumSlices) void rotate_grad_sum(const float* partials, float* weight_grads, int n_partials) {
  __shared__ float part[kSumSlices][kSumColumns];
  const int col = threadIdx.x % kSumColumns, slice = threadIdx.x / kSumColumns;
  const int at = blockIdx.x * kSumColumns + col;
  float s = 0.0f;
#pragma unroll 8
  for (int p = slice; p < n_partials; p += kSumSlices) s += partials[(size_t)p * 4 * kD + at];
  part[slice][col] = s;
  __syncthreads();
  if (slice == 0) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kSumSlices; ++i) sum += part[i][col];
    weight_grads[at] = sum;
  }
}

int batches_of(int heads) { return (heads + kRowsAtOnce - 1) / kRowsAtOnce; }

// Batches of eight heads in a launch from which on a wave takes several of a token: their loads are in flight together and they share one
// set of angles, but there are fewer waves.  us with one and with four, 32 heads in all: 1 token 2.6 and 4.2, 1000 (4000 batches) 4.1 and 6.0, 10000
// (40000) 19.2 and 20.0, 32976 (131904) 56.5 and 48.9.  The gradient, with one and with two: 100 tokens 7.9 and 8.3, 500 (2000) 11.0 and
// 9.8, 1000 14.8 and 12.0, 32976 101 and 94; it has each wave's sums to add up too.
constexpr long long kManyUnits = 65536, kManyGradUnits = 1024;
bool many_units(int n, int batches) { return (long long)n * batches > kManyUnits; }
bool many_grad_units(int n, int batches) { return (long long)n * batches > kManyGradUnits; }

#define XSV_ROTATE_CASES(KERNEL, AT_ONCE)                                                           \
  [&]() {                                                                                           \
    using F = decltype(&KERNEL<0, 0, false, AT_ONCE>);                                              \
    static const F table[3][5] = {                                                                  \
        {KERNEL<0, 0, false, AT_ONCE>, KERNEL<0, 1, false, AT_ONCE>, KERNEL<0, 1, true, AT_ONCE>,   \
         KERNEL<0, 2, false, AT_ONCE>, KERNEL<0, 2, true, AT_ONCE>},                                \
        {KERNEL<1, 0, false, AT_ONCE>, KERNEL<1, 1, false, AT_ONCE>, KERNEL<1, 1, true, AT_ONCE>,   \
         KERNEL<1, 2, false, AT_ONCE>, KERNEL<1, 2, true, AT_ONCE>},                                \
        {KERNEL<2, 0, false, AT_ONCE>, KERNEL<2, 1, false, AT_ONCE>, KERNEL<2, 1, true, AT_ONCE>,   \
         KERNEL<2, 2, false, AT_ONCE>, KERNEL<2, 2, true, AT_ONCE>}};                               \
    return table[norm][axes == 0 ? 0 : 2 * axes - 1 + (interleaved ? 1 : 0)];                       \
  }()

}  // namespace

hipError_t launch_rotate(const RotateArgs& a, int norm, int axes, bool interleaved, hipStream_t stream) {
  const int batches_q = batches_of(a.t[0].heads), batches = batches_q + batches_of(a.t[1].heads);
  const bool many = many_units(a.n, batches);
  const int at_once = many ? 4 : 1;
  const int units_per_token = (batches + at_once - 1) / at_once;
  const long long units = (long long)a.n * units_per_token;
  const int blocks = (int)std::min<long long>((units + kWaves - 1) / kWaves, 1 << 22);
  auto kernel = many ? XSV_ROTATE_CASES(rotate_kernel, 4) : XSV_ROTATE_CASES(rotate_kernel, 1);
  kernel<<<blocks, 64 * kWaves, 0, stream>>>(a, batches_q, batches, units, units_per_token);
  return hipGetLastError();
}

int rotate_grad_workgroups(int n, int heads_q, int heads_k) {
  const int batches = batches_of(heads_q) + batches_of(heads_k);
  const bool many = many_grad_units(n, batches);
  const long long units = (long long)n * (many ? (batches + 1) / 2 : batches);
  return (int)std::min<long long>((units + kWaves - 1) / kWaves, 1024);
}

hipError_t launch_rotate_grad(const RotateArgs& a, int norm, int axes, bool interleaved, hipStream_t stream) {
  const int batches_q = batches_of(a.t[0].heads), batches = batches_q + batches_of(a.t[1].heads);
  const bool many = many_grad_units(a.n, batches);
  const int at_once = many ? 2 : 1;
  const int units_per_token = (batches + at_once - 1) / at_once;
  const long long units = (long long)a.n * units_per_token;
  const int blocks = rotate_grad_workgroups(a.n, a.t[0].heads, a.t[1].heads);
  if (blocks > 0) {
    auto kernel = many ? XSV_ROTATE_CASES(rotate_grad_kernel, 2) : XSV_ROTATE_CASES(rotate_grad_kernel, 1);
    kernel<<<blocks, 64 * kWaves, 0, stream>>>(a, batches_q, batches, units, units_per_token);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!a.weight_grads) return hipSuccess;
  rotate_grad_sum<<<4 * kD / kSumColumns, kSumColumns * kSumSlices, 0, stream>>>(a.partials, a.weight_grads, blocks);  // (no tokens: zeros)
  return hipGetLastError();
}

}  // namespace xsv
