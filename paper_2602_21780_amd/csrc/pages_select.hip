// Which pages of a paged cache a query looks at: those whose keys could have the largest logits, by the bounds of their channels.
//
//   q' = q 2^-t rounded to whole numbers, t = floor(log2 max |q|) - 7, so |q'| <= 255 (and the largest are exact)
//   I_j = sum_c max(q'_c hi_c, q'_c lo_c),   score_j = max over the key head's query heads of I_j 2^(t + e_j - 1)
//
// Since hi >= lo, I_j = max(q', 0) . hi_j + min(q', 0) . lo_j: a product of 128 numbers for matrix instructions in fp16.  hi, lo are whole numbers up to 896
// and all partial sums below 64 * 255 * 896 < 2^24, so that fp32 holds each exactly in any order: the same pages whatever
// computes them, and equal scores are equal.  A row's `first` and `last` pages are chosen whatever their scores; equal scores go to the lower page.
//
// A workgroup has some queries of one key head, 16 or 32 rows (query, head) of a product if it can, whose pages its waves score together, 16 a wave
// and turn, from the pool into scores in LDS; then a wave takes a query, its scores in registers. The n-th largest of each lane's largest is a bound
// that few more than n scores pass, and those are looked at one a lane: each counts the larger ones. Bounds are read from memory once per workgroup
// and scores never written there; what bounds it are waits: the two halves take some 6 and 5 of a workgroup's 15 us, with one workgroup of 16 waves on
// a compute unit: 1374 queries of 16 heads choose 32 of 1024 pages each in 45 us. A few queries (decoding) are a chain of waits, and have all bounds
// of four products' pages on their way at once: 64 streams choose 32 of up to 512 pages in 10 us.
#include <algorithm>

#include "pages.h"

namespace xsv {
namespace {

using f16x2 = __attribute__((ext_vector_type(2))) _Float16;
using f16x8 = __attribute__((ext_vector_type(8))) _Float16;

// Workgroups of a query or a few have 8 waves, which look up 32 pages at a time (64 streams over up to 512 pages 10.1 us, 64 at a time 13.6).
constexpr int kFewTurns = 2, kFewQueries = 4;
constexpr int kLeastBits = 16;   // of a bound on the scores that are chosen: sign, exponent and 7 more (with 14, 64 streams took 6 us longer, with 18 or 20 as long)
constexpr int kMostPages = 32768;  // scores of a row's pages are held in LDS
constexpr int kMostScores = 32768;   // of a workgroup: 128 KB, and 32 for the waves' pieces
constexpr int kHole = -(1 << 20);  // the exponent of a page that is none

constexpr float kNone = -kInf;  // the score of a page that is none
constexpr float kLowest = -3.402823466e38f;
// Larger numbers, larger keys, and back.  (A sum that begins with +0 is never -0.)
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t k) { return __uint_as_float(k >> 31 ? k ^ 0x80000000u : ~k); }
template <int CTRL>
__device__ __forceinline__ f32x4 larger(f32x4 x) {
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = fmaxf(x[j], __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x[j]), CTRL, 0xf, 0xf, true)));
  return x;
}
// The sum over lanes up to and with this one: rows of 16 by DPP, then what the rows before have.
__device__ __forceinline__ int sum_upto(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // lane 15 of a row to the next, rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31 to rows 2 and 3
  return x;
}
__device__ __forceinline__ float power(int e) { return __int_as_float((e + 127) << 23); }

// Of bits, signed: __popcll is not, and a difference of it and a larger number would be a large one.
__device__ __forceinline__ int ones(uint64_t mask) { return (int)__popcll(mask); }

__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const f16x2 p = {(_Float16)a, (_Float16)b};
  return __builtin_bit_cast(uint32_t, p);
}

constexpr int kPieceWords = 16 * kD / 2;  // of a wave: LDS to bring one of 16 pages' bounds, upper or lower, into the order of a product's rows
// Where a query's scores are turned to, so that what 16 queries side by side write is in different banks.
__device__ __forceinline__ int score_turn(int query) { return query % 16 * 4; }

// The first BITS bits of the n-th largest of a wave's keys, one a lane (0 if there are fewer), two bits at a time: the three counts do not wait for
// one another.
template <int BITS>
__device__ __forceinline__ uint32_t nth_largest(uint32_t key, int n) {
  uint32_t x = 0;
#pragma unroll
  for (int bit = 30; bit > 30 - BITS; bit -= 2) {
    const uint32_t y1 = x | 1u << bit, y2 = x | 2u << bit, y3 = x | 3u << bit;
    const int c1 = ones(__ballot(key >= y1)), c2 = ones(__ballot(key >= y2)), c3 = ones(__ballot(key >= y3));
    x = c3 >= n ? y3 : c2 >= n ? y2 : c1 >= n ? y1 : x;
  }
  return x;
}

// N: scores of a query that a lane holds (0: as many as there are, from LDS each time).
// SETS: of 16 columns of a product, rows (query, head), that a wave has at once.
template <int WAVES, int N, int SETS>
__global__ __launch_bounds__(64 * WAVES) void pages_select_kernel(PagesArgs a, int queries, int pitch) {
  extern __shared__ __align__(16) float scores[];  // [queries][pitch], of page j of query r at j ^ score_turn(r); behind them a piece of each wave
  const int lane = threadIdx.x % 64, u = lane / 16, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int rep = a.heads / a.kv_heads, kv = blockIdx.x % a.kv_heads;
  int group = blockIdx.x / a.kv_heads, s;
  Held h;
  if (a.ranked) {
    auto blocks_of = [&](const Held& h) { return (int)(((int64_t)h.n + queries - 1) / queries); };
    auto whole = [&](int row) { return row / queries; };
    if (!(a.sequences <= kRanked ? ranked_block(a, blocks_of, &group, &s, &h) : numbered_block(a, whole, 1, &group, &s, &h))) return;
  } else {
    const int groups = (int)(((int64_t)a.longest + queries - 1) / queries);
    s = group / groups;
    group %= groups;
    h = held(a, s);
  }
  const int query0 = group * queries, n = min(queries, h.n - query0);
  if (n <= 0) return;
  const int32_t* table = a.table + (int64_t)s * a.width;
  const int pages = (tokens_seen(a, h, query0 + n - 1) + kPage - 1) / kPage;  // (queries ascend, and so does what they see)
  constexpr int kTurns = WAVES < 16 ? kFewTurns : 4, kChunk = 16 * kTurns;  // pages that a wave looks up together
  const int chunks = a.pages > 0 ? (pages + kChunk - 1) / kChunk : 0;
  // The heads of a query are side by side in 16 columns, if their number divides 16: the largest of their scores is what one of them writes.
  const bool side_by_side = rep <= 16 && (rep & (rep - 1)) == 0;
  if (!side_by_side || chunks == 0) {
    for (int i = threadIdx.x; i < n * pitch; i += 64 * WAVES) scores[i] = kNone;
    __syncthreads();
  }
  uint32_t* piece = reinterpret_cast<uint32_t*>(scores + queries * pitch) + wave * kPieceWords;
  auto id_of = [&](int ordinal) {  // a page of the pool, or none
    const int id = ordinal < pages ? table[ordinal] : -1;
    return id < a.pages ? id : -1;
  };
  for (int c0 = 0; c0 < n * rep && wave < min(WAVES, chunks); c0 += 16 * SETS) {
    // A wave takes kChunk pages, one to a lane, that are looked up together while those before them are worked on, and then 16 at a time. Of those,
    // the lane has page lane % 16 in the product, and 16 bytes of one of the bounds of pages lane / 8 and 8 + lane / 8 on their way there: 8 lanes
    // side by side take 128 bytes (with a page to a lane, every lane asks for a line of its own, and a load takes the memory path 59 cycles instead
    // of 16).
    struct Way {
      u32x4 bounds[4];
    };
    auto fetch = [&](int id, int turn) {
      Way w;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w.bounds[i] = *reinterpret_cast<const u32x4*>(a.bounds + ((size_t)max(__shfl(id, 16 * turn + 8 * (i % 2) + lane / 8), 0) * a.kv_heads + kv) * 2 * kD + i / 2 * kD + lane % 8 * 8);
      return w;
    };
    auto exponent_of = [&](int id) {
      return id >= 0 ? (int)((__float_as_uint(a.k_scale[(size_t)id * a.kv_heads + kv]) >> 23) & 0xffu) - 128 : kHole;
    };
    int id = id_of(kChunk * wave + lane);
    // The lane's columns, a query of a head each, and 8 channels of each half (columns behind the last are copies of it that nobody writes)
    int query[SETS], t[SETS];
    bool real[SETS];
    f16x8 rows[SETS][4];  // channels 8 u .., 32 + 8 u .. above zero, and below
#pragma unroll
    for (int c = 0; c < SETS; ++c) {
      const int col = min(c0 + 16 * c + lane % 16, n * rep - 1);
      real[c] = c0 + 16 * c + lane % 16 < n * rep;
      query[c] = col / rep;
      const uint16_t* q = a.q.p + (int64_t)(kv * rep + col % rep) * a.q.sh + (h.row0 + query0 + query[c]) * a.q.st + 8 * u;
      float x[16], m = 0.0f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(q + 32 * i);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[8 * i + 2 * j] = (w[j] & 0x7f80u) == 0x7f80u ? 0.0f : bf16_low(w[j]);
          x[8 * i + 2 * j + 1] = (w[j] & 0x7f800000u) == 0x7f800000u ? 0.0f : bf16_high(w[j]);
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(x[i]));
      m = fmaxf(m, __shfl_xor(m, 16));
      m = fmaxf(m, __shfl_xor(m, 32));
      t[c] = max((int)(__float_as_uint(m) >> 23) - 127, -119) - 7;  // (below 2^-119: as if it were 2^-119, which fp32 can turn round)
      const float f = power(-t[c]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        u32x4 up, down;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float y = rintf(x[8 * i + 2 * j] * f), z = rintf(x[8 * i + 2 * j + 1] * f);
          up[j] = pack_f16(fmaxf(y, 0.0f), fmaxf(z, 0.0f));
          down[j] = pack_f16(fminf(y, 0.0f), fminf(z, 0.0f));
        }
        rows[c][i] = __builtin_bit_cast(f16x8, up);
        rows[c][2 + i] = __builtin_bit_cast(f16x8, down);
      }
    }
    auto score = [&](const Way& w, int exponent, int chunk, int turn) {
      // through this wave's piece of LDS (its accesses stay in order); a page's 16-byte pieces are turned so that lanes that read together are in
      // different banks
      f32x4 sum[SETS] = {};
#pragma unroll
      for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
          *reinterpret_cast<u32x4*>(piece + (8 * i + lane / 8) * (kD / 2) + ((lane % 8) ^ (lane / 8)) * 4) = w.bounds[2 * half + i];
        __builtin_amdgcn_wave_barrier();
        f16x8 b[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) b[s] = *reinterpret_cast<const f16x8*>(piece + lane % 16 * (kD / 2) + ((4 * s + u) ^ (lane % 8)) * 4);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int c = 0; c < SETS; ++c) sum[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[s], rows[c][2 * half + s], sum[c], 0, 0, 0);
      }
      // the lane has pages 4 u + 0..3 of the 16 for its columns
      int e[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) e[j] = __shfl(exponent, 16 * turn + 4 * u + j);
#pragma unroll
      for (int c = 0; c < SETS; ++c) {
        f32x4 key;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          // (of bounds that are no numbers, the lowest score: NaN would be larger than no other and smaller than none)
          const float k = fmaxf(__builtin_amdgcn_ldexpf(sum[c][j], min(max(t[c] + e[j], -100), 100)), kLowest);
          key[j] = e[j] == kHole ? kNone : k;
        }
        float* to = scores + query[c] * pitch + ((kChunk * chunk + 16 * turn + 4 * u) ^ score_turn(query[c]));
        if (rep == 1) {  // (copies write the same)
          *reinterpret_cast<f32x4*>(to) = key;
        } else if (side_by_side) {
          key = larger<0xb1>(key);   // of lane ^ 1
          if (rep > 2) key = larger<0x4e>(key);   // lane ^ 2
          if (rep > 4) key = larger<0x141>(key);  // the other four of eight
          if (rep > 8) key = larger<0x140>(key);  // the other eight of sixteen
          if (real[c] && lane % rep == 0) *reinterpret_cast<f32x4*>(to) = key;
        } else if (real[c]) {
#pragma unroll
          for (int j = 0; j < 4; ++j) __hip_atomic_fetch_max(to + j, key[j], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        }
      }
    };
    constexpr int kAhead = SETS == 1 ? kTurns : 1;  // turns whose bounds are on their way
    Way ways[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ways[i] = fetch(id, i);
    for (int chunk = wave; chunk < chunks; chunk += WAVES) {
      const bool more = chunk + WAVES < chunks;
      const int next = id_of(kChunk * (chunk + WAVES) + lane), exponent = exponent_of(id);
#pragma unroll
      for (int turn = 0; turn < kTurns; ++turn) {
        const Way now = ways[turn % kAhead];
        if (turn + kAhead < kTurns) ways[turn % kAhead] = fetch(id, turn + kAhead);
        else if (more) ways[turn % kAhead] = fetch(next, turn + kAhead - kTurns);
        score(now, exponent, chunk, turn);
      }
      id = next;
    }
  }
  __syncthreads();
  // Then a wave takes a query.
  uint32_t* scratch = piece;
  for (int query = wave; query < n; query += WAVES) {
    const int np = (tokens_seen(a, h, query0 + query) + kPage - 1) / kPage, turned = score_turn(query);
    float* row = scores + query * pitch;
    int32_t* out = a.choice + ((int64_t)(h.row0 + query0 + query) * a.kv_heads + kv) * a.count;
    const uint64_t before = (1ull << lane) - 1;
    auto put = [&](int at, int page) {  // (never behind the row's own entries)
      if (at < a.count) out[at] = page;
    };
    const int begin = min(a.first, np), end = max(np - a.last, begin);  // of the pages that are chosen by their scores
    int done = 0, left = a.count;
    for (int j0 = 0; j0 < begin; j0 += 64) {
      const int j = j0 + lane;
      const uint64_t some = __ballot(j < begin && row[j ^ turned] != kNone);
      if (j < begin) row[j ^ turned] = kNone;
      if (some >> lane & 1) put(done + ones(some & before), j);
      done += ones(some);
    }
    auto last_some = [&](int j0) { return __ballot(j0 + lane < np && row[(j0 + lane) ^ turned] != kNone); };
    const uint64_t last = end < np ? last_some(end) : 0;
    left -= done + ones(last);
    for (int j0 = end + 64; j0 < np; j0 += 64) left -= ones(last_some(j0));
    if (lane == 0 && end % 2) row[end ^ turned] = kNone;  // (scores are read two at a time)

    // The `left` largest scores of pages [begin, end).
    const int steps = (end + 63) / 64;
    bool chosen = left <= 0 || end <= begin;
    const int run = (steps + 1) / 2 * 2;  // pages that a lane has side by side, so that lanes are in the order of pages
    float held_scores[N > 0 ? N : 1], most = kNone;
    uint32_t lower = ordered(kNone);  // at least as many scores as are wanted are larger
    if (!chosen) {
      // As many lanes as pages are wanted have a score of at least `least`, so what is below is not chosen; what is not is rarely more than one a
      // lane, and is then dealt out one a lane.
      float score = kNone;
      int page = lane, found = 0;
      if (steps == 1) {
        score = lane < end ? row[lane ^ turned] : kNone;
        found = 64;
      } else {
        auto two_at = [&](int i) {  // of this lane's pages
          const int at = run * lane + i;
          return i < run && at < end ? *reinterpret_cast<const f32x2*>(row + (at ^ turned)) : f32x2{kNone, kNone};
        };
        if constexpr (N > 0) {
#pragma unroll
          for (int i = 0; i < N; i += 2) {
            const f32x2 two = two_at(i);
            held_scores[i] = two[0];
            held_scores[i + 1] = two[1];
            most = fmaxf(most, fmaxf(two[0], two[1]));
          }
        } else {
#pragma unroll 8
          for (int i = 0; i < run; i += 2) {
            const f32x2 two = two_at(i);
            most = fmaxf(most, fmaxf(two[0], two[1]));
          }
        }
        if (ones(__ballot(most != kNone)) >= left) {
          const uint32_t bits = nth_largest<kLeastBits>(ordered(most), left);
          const float least = unordered(bits);
          // (in front of 0 by its bits is -0, which is not less: the number below 0 here, as scores are 0 or at least 2^-100 in size)
          lower = bits == ordered(0.0f) ? ordered(-1.17549435e-38f) : bits - 1;
          uint32_t those = 0;
          int own = 0;
          if constexpr (N > 0) {
#pragma unroll
            for (int i = N - 1; i >= 0; --i) those = 2 * those + (held_scores[i] >= least);
            own = ones(those);
          } else {
#pragma unroll 8
            for (int i = 0; i < run; i += 2) {
              const f32x2 two = two_at(i);
              own += (two[0] >= least) + (two[1] >= least);
            }
          }
          const int upto = sum_upto(own);
          found = __builtin_amdgcn_readlane(upto, 63);
          if (found <= 64) {
            int to = upto - own;
            auto deal = [&](int at, float x) {
              scratch[to] = __float_as_uint(x);
              scratch[64 + to] = at;
              ++to;
            };
            if constexpr (N > 0) {
              for (; __any(those != 0);)
                if (those) {
                  const int at = run * lane + __builtin_ctz(those);
                  deal(at, row[at ^ turned]);
                  those &= those - 1;
                }
            } else {
              for (int i = 0; i < run; i += 2) {
                const f32x2 two = two_at(i);
#pragma unroll
                for (int k = 0; k < 2; ++k)
                  if (two[k] >= least) deal(run * lane + i + k, two[k]);
              }
            }
            __builtin_amdgcn_wave_barrier();
            score = lane < found ? __uint_as_float(scratch[lane]) : kNone;
            page = (int)scratch[64 + lane];
            __builtin_amdgcn_wave_barrier();
          } else {
            found = 0;
          }
        }
      }
      if (found > 0) {
        uint64_t takes = __ballot(score != kNone);
        if (ones(takes) > left) {
          int rank = 0;  // scores that are larger
          for (int i = 0; i < found; i += 4)  // (behind the last, none)
#pragma unroll
            for (int k = 0; k < 4; ++k) rank += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(score), i + k)) > score;
          takes &= __ballot(rank < left);
          const int over = ones(takes) - left;
          if (over > 0) {  // of equal ones that are not all chosen, those of the first pages
            int most = takes >> lane & 1 ? rank : 0;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) most = max(most, __shfl_xor(most, d));
            uint64_t same = takes & __ballot(rank == most);
            const bool stays = ones(same & before) < ones(same) - over;
            takes &= ~same | __ballot(stays);
          }
        }
        if (takes >> lane & 1) put(done + ones(takes & before), page);
        done += ones(takes);
        chosen = true;
      }
    }
    if (!chosen) {
      if constexpr (N > 0) {
        auto count_above = [&](uint32_t x) {
          const float bound = unordered(x);
          int c = 0;
#pragma unroll
          for (int i = 0; i < N; ++i) c += ones(__ballot(held_scores[i] > bound));
          return c;
        };
        // At least `want` scores are above lo, at most `want` above hi.
        const int all = count_above(lower), want = min(left, all);
        uint32_t lo = lower, hi = lo;
        int above_hi = all;
        if (all > want) {
          hi = __builtin_amdgcn_readfirstlane(wave_largest(ordered(most)));
          above_hi = 0;
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
        // Those above hi, and of those that equal it as many of the first as are wanted.
        const float bound = unordered(hi);
        uint32_t takes = 0, same = 0;
#pragma unroll
        for (int i = N - 1; i >= 0; --i) {
          takes = 2 * takes + (held_scores[i] > bound);
          same = 2 * same + (held_scores[i] == bound);
        }
        if (want > above_hi) {
          const int own = ones(same), rest = want - above_hi - (sum_upto(own) - own);  // that the lanes before leave
          while (ones(same) > max(rest, 0)) same &= ~(0x80000000u >> __builtin_clz(same));
          takes |= same;
        }
        const int own = ones(takes), upto = sum_upto(own);
        for (int to = done + upto - own; __any(takes != 0); ++to)
          if (takes) {
            put(to, run * lane + __builtin_ctz(takes));
            takes &= takes - 1;
          }
        done += __builtin_amdgcn_readlane(upto, 63);
      } else {
        auto over = [&](auto f) {  // f(step, key) for every step of 64 pages; none: 0
          for (int i = 0; i < steps; ++i) {
            const int j = 64 * i + lane;
            const float x = j < end ? row[j ^ turned] : kNone;
            f(i, x == kNone ? 0u : ordered(x));
          }
        };
        auto count_above = [&](uint32_t x) {
          int c = 0;
          over([&](int, uint32_t k) { c += ones(__ballot(k > x)); });
          return c;
        };
        // More than `left` keys are above lo, at most `left` above hi.
        const int all = count_above(0), want = min(left, all);
        uint32_t lo = 0, hi = 0xffffffffu;
        int above_hi = 0;
        if (all == want) {
          hi = 0;
          above_hi = want;
        } else {
          uint32_t least = 0xfffffffeu, most = 1;
          over([&](int, uint32_t k) {
            if (k) {
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
        // In order: the keys above hi, and of those that equal it as many of the first as are wanted.
        int equal = want - above_hi;
        over([&](int i, uint32_t k) {
          uint64_t takes = __ballot(k > hi);
          if (equal > 0) {
            const uint64_t ties = __ballot(k == hi);
            const bool tie = k == hi && ones(ties & before) < equal;
            takes |= __ballot(tie);
            equal = max(equal - ones(ties), 0);
          }
          if (takes >> lane & 1) put(done + ones(takes & before), 64 * i + lane);
          done += ones(takes);
        });
      }
    }
    for (int j0 = end; j0 < np; j0 += 64) {
      const uint64_t some = j0 == end ? last : last_some(j0);
      if (some >> lane & 1) put(done + ones(some & before), j0 + lane);
      done += ones(some);
    }
    for (int j = done + lane; j < a.count; j += 64) out[j] = -1;
  }
}

int pages_held(const PagesArgs& a) { return std::min(a.width, (int)(((long long)a.longest_k + kPage - 1) / kPage)); }

// Rows of a product and waves to a workgroup.  us for 1374 queries that choose 32 pages each:
//                                          16 rows, 4 waves   16 rows, 8 waves   32 rows, 16 waves
//   16 heads on 16, 256 pages                          27.7               28.9                31.3
//                   512                                33.7               34.0                35.3
//                   625                                39.7               37.3                40.4
//                   896                                56.4               42.6                44.6
//                   1024                               60.7               47.0                45.9
//                   1100                               67.5               76.7                69.8
//   64 heads on 16, 256 pages                          50.9               73.7                88.8
//                   896                               101.2                117                 141
// 16 rows, where two workgroups of 16 queries fit a compute unit (kSharedPages) and their queries are 4 or more (kSharedHeads): one's choice runs
// beside the other's scores. Of eight heads to a key head, 16 rows are two queries, a choice for two waves: 700 queries, 128 on 16 heads, 256 pages,
// 32 rows are better with 4 waves (37.5 and 48.4) and with 8 (48.7 and 73.3).
constexpr int kSharedPages = 960, kSharedHeads = 4;
// 4 waves where there are many workgroups, twice as many side by side, if four fit a compute unit's LDS (their scores 32 KB each; 512 and 625 pages
// above): 256 streams of 8192 tokens, 32 on 8 heads, 21.4 and with 8 waves 31.2; eight ragged sequences, 64 on 16 heads, 105 and 173.
constexpr int kManyGroups = 1024, kFourScores = 8192;

struct Plan {
  int queries, pitch;  // of a workgroup; scores of a query
  int columns, waves;
  long long groups;    // of queries of all sequences
  bool ranked;         // numbered over them
};
Plan plan_of(const PagesArgs& a) {
  Plan p;
  const int rep = a.heads / a.kv_heads;
  p.pitch = (std::max(pages_held(a), 1) + 63) / 64 * 64;
  p.columns = p.pitch <= kSharedPages && rep <= kSharedHeads ? 16 : 32;
  p.queries = std::max(std::min({p.columns / rep, a.longest, kMostScores / p.pitch}), 1);
  if (p.queries <= kFewQueries && p.queries * rep <= 16) p.columns = 16;
  const long long of_one = ((long long)a.longest + p.queries - 1) / p.queries, each = of_one * a.sequences;
  const long long all = ((long long)a.rows + p.queries - 1) / p.queries + a.sequences;
  p.ranked = of_one > 1 && a.sequences > 1 && (a.sequences <= kRanked || by_number((double)each, all));
  p.groups = !p.ranked ? each : a.sequences <= kRanked ? std::min(each, all) : all;
  const bool four = p.groups > kManyGroups / a.kv_heads && p.queries * p.pitch <= kFourScores;
  p.waves = p.columns == 32 && p.queries > kFewQueries ? 16 : four ? 4 : 8;
  return p;
}

template <int WAVES, int N, int SETS>
hipError_t launch(PagesArgs a, const Plan& p, hipStream_t stream) {
  const int bytes = (p.queries * p.pitch + WAVES * kPieceWords) * (int)sizeof(uint32_t);
  a.ranked = p.ranked;
  if (bytes > (48 << 10)) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(pages_select_kernel<WAVES, N, SETS>), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  pages_select_kernel<WAVES, N, SETS><<<(int)(p.groups * a.kv_heads), 64 * WAVES, bytes, stream>>>(a, p.queries, p.pitch);
  return hipGetLastError();
}

template <int WAVES, int SETS>
hipError_t launch_for(const PagesArgs& a, const Plan& p, hipStream_t stream) {
  const int held = pages_held(a);
  if (held <= 256) return launch<WAVES, 4, SETS>(a, p, stream);
  if (held <= 512) return launch<WAVES, 8, SETS>(a, p, stream);
  if (held <= 1024) return launch<WAVES, 16, SETS>(a, p, stream);
  if (held <= 2048) return launch<WAVES, 32, SETS>(a, p, stream);
  return launch<WAVES, 0, SETS>(a, p, stream);
}

}  // namespace

bool pages_select_fits(const PagesArgs& a) {
  if (pages_held(a) > kMostPages) return false;
  const Plan p = plan_of(a);
  return p.groups <= ((1ll << 32) / (64 * p.waves) - 1) / a.kv_heads;  // (threads of a launch are counted in 32 bits)
}

hipError_t launch_pages_select(const PagesArgs& a, hipStream_t stream) {
  if (a.sequences == 0 || a.longest == 0 || a.count == 0) return hipSuccess;
  const Plan p = plan_of(a);
  if (p.waves == 16) return launch_for<16, 2>(a, p, stream);
  if (p.columns == 16) return p.waves == 4 ? launch_for<4, 1>(a, p, stream) : launch_for<8, 1>(a, p, stream);
  return p.waves == 4 ? launch_for<4, 2>(a, p, stream) : launch_for<8, 2>(a, p, stream);
}

}  // namespace xsv
