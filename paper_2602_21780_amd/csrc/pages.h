// What the kernels of the paged cache share: a sequence's rows and tokens, what a query sees, e4m3 codes.
#pragma once

#include "operators.h"

namespace xsv {

using u32x2 = __attribute__((ext_vector_type(2))) uint32_t;
using u32x4 = __attribute__((ext_vector_type(4))) uint32_t;
using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using f32x2 = __attribute__((ext_vector_type(2))) float;
using f32x4 = __attribute__((ext_vector_type(4))) float;

constexpr int kPage = 64;             // tokens per page
constexpr int kPageBytes = kPage * kD;  // codes of a page's keys (or values) of one head
constexpr float kInf = __builtin_inff();
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;

struct Held {
  int row0, n;  // rows of the call, within the bound
  int m;        // tokens, within theirs
  int ahead;    // the place of row 0 among them: rows stand at the end of their sequence, whatever the bounds leave out
};
// Offsets and lengths are device data: whatever they hold, no row outside the tensors and no entry outside the table is touched.
__device__ __forceinline__ Held held(const PagesArgs& a, int s) {
  Held h;
  h.row0 = min(max(a.begin[s], 0), a.rows);
  const int n = min(max(a.begin[s + 1], h.row0), a.rows) - h.row0;
  const int m = min(max(a.lengths[s], 0), a.width * kPage);
  h.m = min(m, a.longest_k);
  h.ahead = m - n;
  h.n = min(n, a.longest);
  return h;
}

// Tokens that row i of a sequence sees: all, or up to the end of the block of `causal` tokens that it stands in.
__device__ __forceinline__ int tokens_seen(const PagesArgs& a, const Held& h, int i) {
  const int at = i + h.ahead;
  if (at < 0) return 0;
  if (a.causal == 0) return h.m;  // (of a row in front of the first token: nothing, whatever the mask)
  return (int)min((int64_t)h.m, ((int64_t)(at / a.causal) + 1) * a.causal);
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const bf16x2 p = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, p);
}

__device__ __forceinline__ float bf16_low(uint32_t two) { return __uint_as_float(two << 16); }
__device__ __forceinline__ float bf16_high(uint32_t two) { return __uint_as_float(two & 0xffff0000u); }

__device__ __forceinline__ uint32_t wave_largest(uint32_t x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x = max(x, (uint32_t)__shfl_xor((int)x, d));
  return x;
}

}  // namespace xsv
