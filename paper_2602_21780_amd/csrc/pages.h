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
  int m;        // tokens, within theirs and the table
  int ahead;    // the place of row 0 among them: rows stand at the end of their sequence, whatever the bounds and the table leave out
};
// Offsets and lengths are device data: whatever they hold, no row outside the tensors and no entry outside the table is touched.
__device__ __forceinline__ Held held(const PagesArgs& a, int s) {
  Held h;
  h.row0 = min(max(a.begin[s], 0), a.rows);
  const int n = min(max(a.begin[s + 1], h.row0), a.rows) - h.row0;
  const int m = max(a.lengths[s], 0);
  h.m = min(min(m, a.width * kPage), a.longest_k);
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

// Blocks of rows numbered over all sequences: launches are sized by the rows and the sequences, not by the longest sequence that there may be times the
// sequences.  Block number `*block` becomes its number within its sequence.
// Up to 64 sequences: `blocks_of(h)` of each, those of the sequences that see the most pages first.  A lane looks a sequence up.
template <typename F>
__device__ __forceinline__ bool ranked_block(const PagesArgs& a, F blocks_of, int* block, int* sequence, Held* h) {
  const int lane = threadIdx.x % 64;
  Held own{};
  int blocks = 0, cost = -1, before = 0;
  if (lane < a.sequences) {
    own = held(a, lane);
    blocks = blocks_of(own);
    cost = own.n > 0 ? tokens_seen(a, own, own.n - 1) : 0;
  }
  for (int s = 0; s < a.sequences; ++s) {
    const int other = __builtin_amdgcn_readlane(cost, s), n = __builtin_amdgcn_readlane(blocks, s);
    before += other > cost || (other == cost && s < lane) ? n : 0;
  }
  const uint64_t here = __ballot(lane < a.sequences && before <= *block && *block < before + blocks);
  if (!here) return false;
  const int s = __builtin_ctzll(here);
  *sequence = s;
  *block -= __builtin_amdgcn_readlane(before, s);
  *h = Held{__builtin_amdgcn_readlane(own.row0, s), __builtin_amdgcn_readlane(own.n, s), __builtin_amdgcn_readlane(own.m, s), __builtin_amdgcn_readlane(own.ahead, s)};
  return true;
}

// More sequences, in their order: those in front of row r have at most `whole(r)` blocks, and `extra` more each; at that number the blocks of the sequence
// that begins with r begin, so that it is found by 64 offsets at a time.  (Numbers between one sequence's last block and the next one's first are nobody's.)
template <typename W>
__device__ __forceinline__ bool numbered_block(const PagesArgs& a, W whole, int extra, int* block, int* sequence, Held* h) {
  const int lane = threadIdx.x % 64;
  int s = 0;
  for (int n = a.sequences; n > 1;) {
    const int step = (n + 63) / 64, at = s + min(lane * step, n - 1);
    const int64_t number = (int64_t)whole(min(max(a.begin[at], 0), a.rows)) + (int64_t)at * extra;
    const int i = 63 - __builtin_clzll(__ballot(lane * step < n && number <= *block) | 1ull);
    s += i * step;
    n = min(step, n - i * step);
  }
  *sequence = s;
  *h = held(a, s);
  const int64_t number = *block - ((int64_t)whole(h->row0) + (int64_t)s * extra);
  *block = (int)number;
  return number >= 0;
}
constexpr int kRanked = 64;
// More than kRanked sequences: is the launch of all blocks by number, `numbered`, taken, or that of as many for each sequence as the longest may
// have, `each`? Empty workgroups cost less than the search; both sides, us, each and numbered, 500 sequences of a row and one of L, 16 heads:
// written, L = 100 (each 1.5 times numbered) 38 and 45, L = 300 (2.9) 67 and 45; choice of 4 pages, L = 300 142 and 42, L = 1000 388 and 51;
// attention 186 and 149, 313 and 155.
inline bool by_number(double each, long long numbered) { return (double)numbered <= each / 2; }  // (the product may pass 64 bits)

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
