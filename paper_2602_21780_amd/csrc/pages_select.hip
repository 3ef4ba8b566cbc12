// Which pages of a paged cache a query looks at: those whose keys could have the largest logits, by the bounds of their channels.
//
//   q' = q 2^-t rounded to whole numbers, t = floor(log2 max |q|) - 7, so |q'| <= 255 (and the largest are exact)
//   I_j = sum_c max(q'_c hi_c, q'_c lo_c),   score_j = max over the key head's query heads of I_j 2^(t + e_j - 1)
//
// Since hi >= lo, I_j = max(q', 0) . hi_j + min(q', 0) . lo_j: a product of 128 numbers for matrix instructions in fp16.  hi, lo are whole numbers up to 896
// and all partial sums below 64 * 255 * 896 < 2^24, so that fp32 holds each exactly in any order: the same pages whatever
// computes them, and equal scores are equal.  A row's `first` and `last` pages are chosen whatever their scores; equal scores go to the lower page.
//
// A workgroup has some queries of one key head, 32 rows (query, head) of a product if it can, whose pages it scores together, 32 a wave and turn, from
// the pool into keys in LDS; then a wave takes a query, its keys in registers, and halves the interval of keys that its last chosen one lies in
// until as many keys as wanted lie above it.
#include <algorithm>
#include <type_traits>

#include "pages.h"

namespace xsv {
namespace {

using f16x2 = __attribute__((ext_vector_type(2))) _Float16;
using f16x8 = __attribute__((ext_vector_type(8))) _Float16;
using f32x16 = __attribute__((ext_vector_type(16))) float;

constexpr int kMostPages = 32768;  // scores of a row's pages are held in LDS
constexpr int kMostKeys = 32768;   // of a workgroup
constexpr int kHole = INT32_MIN;

__device__ __forceinline__ uint32_t ordered(float x) {  // larger numbers, larger keys; 0 and the largest are for other uses
  const uint32_t b = __float_as_uint(x + 0.0f);         // (0 of either sign is +0)
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float power(int e) { return __int_as_float((e + 127) << 23); }

__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const f16x2 p = {(_Float16)a, (_Float16)b};
  return __builtin_bit_cast(uint32_t, p);
}

// Over a wave, in every lane.
template <typename F>
__device__ __forceinline__ uint32_t over_wave(uint32_t x, F f) {
  auto from = [](uint32_t v, auto ctrl) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, decltype(ctrl)::value, 0xf, 0xf, true); };
  x = f(x, from(x, std::integral_constant<int, 0xb1>{}));   // lane ^ 1
  x = f(x, from(x, std::integral_constant<int, 0x4e>{}));   // lane ^ 2
  x = f(x, from(x, std::integral_constant<int, 0x141>{}));  // 7 - lane of eight: the other four
  x = f(x, from(x, std::integral_constant<int, 0x140>{}));  // 15 - lane of sixteen: the other eight
  const auto p = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = f(p[0], p[1]);
  const auto q = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return f(q[0], q[1]);
}

// A number that n of a wave's keys, one a lane, are at least (n keys that there are), or more only if they equal it: the n-th largest, or one
// between it and the next.  Bit by bit, those that the keys have in common left out.
__device__ __forceinline__ uint32_t nth_largest(uint32_t key, int n) {
  const uint32_t any = __builtin_amdgcn_readfirstlane(over_wave(key, [](uint32_t x, uint32_t y) { return x | y; }));
  const uint32_t all = __builtin_amdgcn_readfirstlane(over_wave(key, [](uint32_t x, uint32_t y) { return x & y; }));
  uint32_t x = all;
  for (uint32_t left = any & ~all; left;) {
    const uint32_t bit = 0x80000000u >> __builtin_clz(left);
    left ^= bit;
    const int c = __popcll(__ballot(key >= (x | bit)));
    if (c >= n) x |= bit;
    if (c == n) break;
  }
  return x;
}

// N: keys of a query that a lane holds (0: as many as there are, from LDS each time).
template <int WAVES, int N>
__global__ __launch_bounds__(64 * WAVES) void pages_select_kernel(PagesArgs a, int queries, int pitch) {
  extern __shared__ __align__(16) uint32_t keys[];  // [queries][pitch]
  __shared__ __align__(16) int exponents[WAVES][32];
  const int lane = threadIdx.x % 64, g = lane / 32, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int rep = a.heads / a.kv_heads, groups = (a.longest + queries - 1) / queries;
  const int kv = blockIdx.x % a.kv_heads, group = blockIdx.x / a.kv_heads % groups, s = blockIdx.x / a.kv_heads / groups;
  const Held h = held(a, s);
  const int query0 = group * queries, n = min(queries, h.n - query0);
  if (n <= 0) return;
  const int32_t* table = a.table + (int64_t)s * a.width;
  const int pages = (tokens_seen(a, h, query0 + n - 1) + kPage - 1) / kPage;  // (queries ascend, and so does what they see)
  const int turns = a.pages > 0 ? (pages + 31) / 32 : 0;
  if (rep > 1 || turns == 0) {
    for (int i = threadIdx.x; i < n * pitch; i += 64 * WAVES) keys[i] = 0;
    __syncthreads();
  }
  auto id_of = [&](int turn) {  // the page that the lane looks up for a turn, or none
    const int ordinal = turn * 32 + lane % 32;
    const int id = ordinal < pages ? table[ordinal] : -1;
    return id < a.pages ? id : -1;
  };
  for (int c0 = 0; c0 < n * rep; c0 += 32) {
    int id = id_of(wave), id_next = id_of(wave + WAVES);
    // The lane's column, a query of a head, and its channels 32 g .. (columns behind the last are copies of it that change nothing)
    const int col = min(c0 + lane % 32, n * rep - 1), query = col / rep;
    f16x8 above[4], below[4];
    int t;
    {
      const uint16_t* q = a.q.p + (int64_t)(kv * rep + col % rep) * a.q.sh + (h.row0 + query0 + query) * a.q.st + 32 * g;
      float x[32], m = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(q + 8 * i);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[8 * i + 2 * j] = (w[j] & 0x7f80u) == 0x7f80u ? 0.0f : bf16_low(w[j]);
          x[8 * i + 2 * j + 1] = (w[j] & 0x7f800000u) == 0x7f800000u ? 0.0f : bf16_high(w[j]);
        }
      }
#pragma unroll
      for (int i = 0; i < 32; ++i) m = fmaxf(m, fabsf(x[i]));
      m = fmaxf(m, __shfl_xor(m, 32));
      t = max((int)(__float_as_uint(m) >> 23) - 127, -119) - 7;  // (below 2^-119: as if it were 2^-119, which fp32 can turn round)
      const float f = power(-t);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u32x4 up, down;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float y = rintf(x[8 * i + 2 * j] * f), z = rintf(x[8 * i + 2 * j + 1] * f);
          up[j] = pack_f16(fmaxf(y, 0.0f), fmaxf(z, 0.0f));
          down[j] = pack_f16(fminf(y, 0.0f), fminf(z, 0.0f));
        }
        above[i] = __builtin_bit_cast(f16x8, up);
        below[i] = __builtin_bit_cast(f16x8, down);
      }
    }
    for (int turn = wave; turn < turns; turn += WAVES) {
      const bool some = id >= 0;
      const size_t unit = (size_t)(some ? id : 0) * a.kv_heads + kv;
      const u32x4* b = reinterpret_cast<const u32x4*>(a.bounds + unit * 2 * kD) + 4 * g;
      u32x4 hi[4], lo[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        hi[i] = b[i];
        lo[i] = b[8 + i];
      }
      const int e = some ? (int)((__float_as_uint(a.k_scale[unit]) >> 23) & 0xffu) - 128 : kHole;
      id = id_next;
      id_next = id_of(turn + 2 * WAVES);
      if (g == 0) exponents[wave][lane] = e;  // (read by this wave alone, whose LDS accesses stay in order)
      f32x16 sum = {};
#pragma unroll
      for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, hi[i]), above[i], sum, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, lo[i]), below[i], sum, 0, 0, 0);
      __builtin_amdgcn_wave_barrier();
      // the lane has pages 8 i + 4 g + 0..3 of the 32 for its column
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u32x4 key;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int e = exponents[wave][8 * i + 4 * g + j];
          const uint32_t k = ordered(sum[4 * i + j] * power(min(max(t + max(e, -1000), -100), 100)));
          key[j] = e == kHole ? 0u : k;
        }
        uint32_t* to = keys + query * pitch + turn * 32 + 8 * i + 4 * g;
        if (rep == 1) {
          *reinterpret_cast<u32x4*>(to) = key;
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) atomicMax(to + j, key[j]);
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
  __syncthreads();
  for (int query = wave; query < n; query += WAVES) {
    const int np = (tokens_seen(a, h, query0 + query) + kPage - 1) / kPage, steps = (np + 63) / 64;
    uint32_t* row = keys + query * pitch;
    // Forced pages' keys are the largest, those behind the last are none.
    for (int j = lane; j < min(a.first, np); j += 64)
      if (row[j]) row[j] = 0xffffffffu;
    for (int j = max(np - a.last, 0) + lane; j < 64 * steps; j += 64) row[j] = j < np && row[j] ? 0xffffffffu : 0u;
    uint32_t held_keys[N ? N : 1];
    auto key_at = [&](int i) { return row[64 * i + lane]; };  // of page 64 i + lane
    int32_t* out = a.choice + ((int64_t)(h.row0 + query0 + query) * a.kv_heads + kv) * a.count;
    const uint64_t before = (1ull << lane) - 1;
    if (steps == 0) {
      for (int j = lane; j < a.count; j += 64) out[j] = -1;
      continue;
    }
    if constexpr (N > 0) {
      uint32_t most = 0;  // of this lane's keys
#pragma unroll
      for (int i = 0; i < N; ++i) {
        held_keys[i] = key_at(min(i, steps - 1)) & (i < steps ? 0xffffffffu : 0u);
        most = max(most, held_keys[i]);
      }
      // As many lanes as pages are wanted have a key of at least `least`, so what is below it is not chosen; what is not is rarely more than a key a lane.
      const int some = __popcll(__ballot(most > 0));
      if (steps == 1 || some >= a.count) {
        const int want = min(a.count, some);
        uint32_t key = most;
        int page = lane, found = some;
        if (steps > 1) {
          const uint32_t least = nth_largest(most, want);
          found = 0;
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const uint64_t some = __ballot(held_keys[i] >= least);
            if (some) {
              const int place = found + __popcll(some & before);
              if ((some >> lane & 1) && place < 64) {
                row[place] = held_keys[i];  // (its keys are all in registers)
                row[64 + place] = 64 * i + lane;
              }
              found += __popcll(some);
            }
          }
          if (found <= 64) {
            key = lane < found ? row[lane] : 0u;
            page = (int)row[64 + lane];
          }
        }
        if (found <= 64) {
          const uint32_t nth = want > 0 ? nth_largest(key, want) : 0xffffffffu;
          const int ties = want - __popcll(__ballot(key > nth));
          const uint64_t same = __ballot(key == nth && key > 0), takes = __ballot(key > nth || (key == nth && key > 0 && __popcll(same & before) < ties));
          if (takes >> lane & 1) out[__popcll(takes & before)] = page;
          for (int j = want + lane; j < a.count; j += 64) out[j] = -1;
          continue;
        }
      }
    }
    auto over = [&](auto f) {  // f(step, key) for every step of 64 pages
      if constexpr (N > 0) {
#pragma unroll
        for (int i = 0; i < N; ++i)
          f(i, held_keys[i]);
      } else {
        for (int i = 0; i < steps; ++i) f(i, key_at(i));
      }
    };
    auto count_above = [&](uint32_t x) {
      int c = 0;
      over([&](int, uint32_t k) { c += __popcll(__ballot(k > x)); });
      return c;
    };
    // More than `want` keys are above lo, at most `want` above hi, which all forced ones are.
    const int all = count_above(0), want = min(a.count, all);
    uint32_t lo = 0, hi = 0xfffffffeu;
    int above_hi = 0;
    if (all == want) {
      hi = 0;
      above_hi = want;
    } else {
      uint32_t least = 0xfffffffeu, most = 1;
      over([&](int, uint32_t k) {
        if (k && k != 0xffffffffu) {
          least = min(least, k);
          most = max(most, k);
        }
      });
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        least = min(least, (uint32_t)__shfl_xor((int)least, d));
        most = max(most, (uint32_t)__shfl_xor((int)most, d));
      }
      lo = __builtin_amdgcn_readfirstlane(least) - 1;
      hi = __builtin_amdgcn_readfirstlane(most);
      above_hi = count_above(hi);
      while (above_hi != want && hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        const int c = count_above(mid);
        if (c > want) lo = mid;
        else {
          hi = mid;
          above_hi = c;
        }
      }
    }
    // In order: the keys above hi, and of those that equal it as many of the first as are left.
    int done = 0, left = want - above_hi;
    over([&](int i, uint32_t k) {
      uint64_t takes = __ballot(k > hi);
      if (left > 0) {
        const uint64_t ties = __ballot(k == hi);
        const bool tie = k == hi && __popcll(ties & before) < left;
        takes |= __ballot(tie);
        left = max(left - __popcll(ties), 0);
      }
      if (takes >> lane & 1) out[done + __popcll(takes & before)] = 64 * i + lane;
      done += __popcll(takes);
    });
    for (int j = done + lane; j < a.count; j += 64) out[j] = -1;
  }
}

int pages_held(const PagesArgs& a) { return std::min(a.width, (int)(((long long)a.longest_k + kPage - 1) / kPage)); }

struct Plan {
  int queries, pitch;  // of a workgroup; keys of a query (four more than a multiple of 64: queries side by side are in different banks)
};
Plan plan_of(const PagesArgs& a) {
  Plan p;
  p.pitch = (std::max(pages_held(a), 1) + 63) / 64 * 64 + 4;
  p.queries = std::max(std::min({32 / (a.heads / a.kv_heads), a.longest, kMostKeys / (p.pitch - 4)}), 1);
  return p;
}

template <int WAVES, int N>
hipError_t launch(const PagesArgs& a, const Plan& p, hipStream_t stream) {
  const int bytes = p.queries * p.pitch * (int)sizeof(uint32_t), groups = (a.longest + p.queries - 1) / p.queries;
  if (bytes > (48 << 10)) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(pages_select_kernel<WAVES, N>), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  pages_select_kernel<WAVES, N><<<a.sequences * groups * a.kv_heads, 64 * WAVES, bytes, stream>>>(a, p.queries, p.pitch);
  return hipGetLastError();
}

template <int WAVES>
hipError_t launch_for(const PagesArgs& a, const Plan& p, hipStream_t stream) {
  const int held = pages_held(a);
  if (held <= 256) return launch<WAVES, 4>(a, p, stream);
  if (held <= 512) return launch<WAVES, 8>(a, p, stream);
  if (held <= 1024) return launch<WAVES, 16>(a, p, stream);
  if (held <= 2048) return launch<WAVES, 32>(a, p, stream);
  return launch<WAVES, 0>(a, p, stream);
}

}  // namespace

bool pages_select_fits(const PagesArgs& a) {
  const long long most = (1ll << 32) / 1024 - 1;
  return pages_held(a) <= kMostPages && (long long)a.longest * a.kv_heads <= most && (long long)a.longest * a.kv_heads * a.sequences <= most;
}

hipError_t launch_pages_select(const PagesArgs& a, hipStream_t stream) {
  if (a.sequences == 0 || a.longest == 0 || a.count == 0) return hipSuccess;
  const Plan p = plan_of(a);
  if (p.queries <= 4) return launch_for<4>(a, p, stream);
  return launch_for<16>(a, p, stream);
}

}  // namespace xsv
