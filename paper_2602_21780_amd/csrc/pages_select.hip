// Which pages of a paged cache a query looks at: those whose keys could have the largest logits, by the bounds of their channels.
//
//   q' = q 2^-t rounded to whole numbers, t = floor(log2 max |q|) - 7, so |q'| <= 255 (and the largest are exact)
//   I_j = sum_c max(q'_c hi_c, q'_c lo_c),   score_j = max over the key head's query heads of I_j 2^(t + e_j - 1)
//
// hi, lo are whole numbers up to 896 and I_j below 64 * 255 * 896 < 2^24, so every sum is exact in fp32 in any order: the same pages whatever
// computes them, and equal scores are equal.  A row's `first` and `last` pages are chosen whatever their scores; equal scores go to the lower page.
#include <algorithm>

#include "pages.h"

namespace xsv {
namespace {

constexpr int kThreads = 256;
constexpr int kMostPages = 32768;  // scores of a row's pages are held in LDS

__device__ __forceinline__ uint32_t ordered(float x) {  // larger numbers, larger keys; 0 and the largest are for other uses
  const uint32_t b = __float_as_uint(x == 0.0f ? 0.0f : x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float power(int e) { return __int_as_float((e + 127) << 23); }

__device__ __forceinline__ float channel_sum(float x) {  // over a wave
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
  return x;
}

__global__ __launch_bounds__(kThreads) void pages_select_kernel(PagesArgs a) {
  extern __shared__ __align__(16) uint32_t keys[];
  __shared__ float whole[kD];
  __shared__ int unit_of, hist[256], found[2], counts[kThreads / 64], all;
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int rep = a.heads / a.kv_heads;
  const int kv = blockIdx.x % a.kv_heads, i = blockIdx.x / a.kv_heads % a.longest, s = blockIdx.x / a.kv_heads / a.longest;
  const Held h = held(a, s);
  if (i >= h.n) return;
  const int pages = (tokens_seen(a, h, i) + kPage - 1) / kPage;
  const int64_t row = h.row0 + i;
  const int32_t* table = a.table + (int64_t)s * a.width;
  int32_t* out = a.choice + (row * a.kv_heads + kv) * a.count;
  for (int r = 0; r < rep; ++r) {
    __syncthreads();
    if (tid < 64) {
      const uint16_t bits = a.q.p[(int64_t)(kv * rep + r) * a.q.sh + row * a.q.st + tid];
      const bool finite = (bits & 0x7f80u) != 0x7f80u;
      const float x = finite ? __uint_as_float((uint32_t)bits << 16) : 0.0f;
      float m = fabsf(x);
      for (int d = 1; d < 64; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
      const int t = max((int)(__float_as_uint(m) >> 23) - 127, -119) - 7;  // (below 2^-119: as if it were 2^-119, which fp32 can turn round)
      whole[tid] = rintf(x * power(-t));
      if (tid == 0) unit_of = t;
    }
    __syncthreads();
    for (int j = tid; j < pages; j += kThreads) {
      const int page = table[j];
      uint32_t key = 0;
      if (page >= 0 && page < a.pages) {
        const int64_t unit = (int64_t)page * a.kv_heads + kv;
        const _Float16* b = reinterpret_cast<const _Float16*>(a.bounds) + unit * 2 * kD;
        float sum = 0.0f;
        for (int c = 0; c < kD; ++c) sum += whole[c] * (float)(whole[c] > 0.0f ? b[c] : b[kD + c]);
        const int e = unit_of + (int)((__float_as_uint(a.k_scale[unit]) >> 23) & 0xffu) - 128;
        key = ordered(sum * power(min(max(e, -100), 100)));
        if (j < a.first || j >= pages - a.last) key = 0xffffffffu;
      }
      keys[j] = r ? max(keys[j], key) : key;
    }
  }
  // The `want`-th largest key, a byte at a time.
  __syncthreads();
  if (tid == 0) all = 0;
  __syncthreads();
  for (int j = tid; j < pages; j += kThreads)
    if (keys[j]) atomicAdd(&all, 1);
  __syncthreads();
  int want = min(a.count, all), left = want;  // left: how many of the keys that begin as the `want`-th does
  uint32_t prefix = 0;
  for (int shift = 24; shift >= 0 && want > 0; shift -= 8) {
    hist[tid] = 0;
    __syncthreads();
    for (int j = tid; j < pages; j += kThreads)
      if (keys[j] && (shift == 24 || keys[j] >> (shift + 8) == prefix >> (shift + 8))) atomicAdd(&hist[keys[j] >> shift & 255], 1);
    __syncthreads();
    if (tid == 0) {
      int n = 0, bin = 255;
      while (n + hist[bin] < left) n += hist[bin--];
      found[0] = bin;
      found[1] = left - n;
    }
    __syncthreads();
    prefix |= (uint32_t)found[0] << shift;
    left = found[1];
  }
  // In order: keys above it, and the first `left` that equal it.
  int done = 0, equal = 0;
  for (int j0 = 0; j0 < pages; j0 += kThreads) {
    const int j = j0 + tid;
    const uint32_t key = j < pages ? keys[j] : 0;
    const bool same = want > 0 && key == prefix && key;
    __syncthreads();
    if (lane == 0) counts[wave] = 0;
    const uint64_t ties = __ballot(same);
    if (lane == 0) counts[wave] = __popcll(ties);
    __syncthreads();
    int before = equal + __popcll(ties & ((1ull << lane) - 1));
    for (int w = 0; w < kThreads / 64; ++w) {
      if (w < wave) before += counts[w];
      equal += counts[w];
    }
    const bool take = want > 0 && (key > prefix || (same && before < left));
    const uint64_t takes = __ballot(take);
    __syncthreads();
    if (lane == 0) counts[wave] = __popcll(takes);
    __syncthreads();
    int at = done + __popcll(takes & ((1ull << lane) - 1));
    for (int w = 0; w < kThreads / 64; ++w) {
      if (w < wave) at += counts[w];
      done += counts[w];
    }
    if (take) out[at] = j;
  }
  for (int j = done + tid; j < a.count; j += kThreads) out[j] = -1;
}

int pages_held(const PagesArgs& a) { return std::min(a.width, (int)(((long long)a.longest_k + kPage - 1) / kPage)); }

}  // namespace

bool pages_select_fits(const PagesArgs& a) {
  const long long most = (1ll << 32) / kThreads - 1;
  return pages_held(a) <= kMostPages && (long long)a.longest * a.kv_heads <= most && (long long)a.longest * a.kv_heads * a.sequences <= most;
}

hipError_t launch_pages_select(const PagesArgs& a, hipStream_t stream) {
  if (a.sequences == 0 || a.longest == 0 || a.count == 0) return hipSuccess;
  const int bytes = std::max(pages_held(a), 1) * (int)sizeof(uint32_t);
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(pages_select_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != hipSuccess) return e;
  pages_select_kernel<<<a.sequences * a.longest * a.kv_heads, kThreads, bytes, stream>>>(a);
  return hipGetLastError();
}

}  // namespace xsv
