// Attention of a few query rows over a layer's packed cache (single tokens, special tokens, probes): one pass over the cache.
//
//   out = softmax(scale q K~^T) V~,   lse = log sum exp(scale q K~^T),   K~, V~ = bf16((code - zero) * scale)
//
// It reads every packed byte once per block of query rows (0.625 bytes per element at 4 bits and groups of 64), and a few vector instructions per
// element turn it into the same bf16 view that the rest of the library attends to.  Measured at 16 heads, one row over 65536 tokens: a bf16 cache
// 43 us, which is 6.2 TB/s and the memory's bound (the cache fits the last-level one); 4 bits 29 us, 2.8 TB/s, and 2 bits 31 us: there the arithmetic
// of the view bounds it, about 640 vector instructions per wave and 64 tokens, the vector units active in 79 % of the cycles.  One
// row over 4096 tokens takes 9.8 us: the launch, one tile for each wave, 16 parts and their join, each a chain of waits for memory.  17 to 64 rows share
// the view, but the workspace's parts cut their tokens over half of the workgroups that the chip holds: one wave a SIMD, with nothing to hide its loads
// behind (64 rows over 20000 tokens 29 us).
//
// A wave takes 64 tokens at a time straight from memory into registers: keys as the A operand of 16x16x32 MFMAs (transposed
// logits, a lane holds 16 tokens of one query), values, which the cache keeps transposed, as the A operand of the second
// product, and the probabilities, packed, as its B operand.  Operand rows are dealt so that every lane loads runs: its quarter u of the
// wave has channels 16 u .. of a key row and tokens 16 u .. of a value row, and row R of logit block B is token
// 16 (R / 4) + 4 B + R % 4, which puts tokens 16 u .. into the accumulators of quarter u as well.
//
// The tokens are cut over the waves of a workgroup (joined in LDS) and over workgroups, so that few rows still use the whole chip;
// the workgroup of a head that ends last, or a second launch, joins their partial results, in their order.
#include <algorithm>
#include <type_traits>

#include "xsv_internal.h"

namespace xsv {
namespace {

using u32x2 = __attribute__((ext_vector_type(2))) uint32_t;
using u32x4 = __attribute__((ext_vector_type(4))) uint32_t;
using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using f32x4 = __attribute__((ext_vector_type(4))) float;

constexpr int kWaves = 4;
constexpr int kRows = kQueryRows;  // query rows of a column block
constexpr int kJoinRows = 4;       // rows that are joined at a time, one a wave
static_assert(kJoinRows == kWaves);
// A single row whose tokens are cut over a few workgroups is joined by the one that ends last in its head, others by a second launch: the parts, counters and
// fence of many workgroups take longer than a launch.  us on the GPU inside and by a launch, one row: one head over 300 tokens (2 workgroups in all) 5.7 and
// 6.6, 16 heads over 300 (32) 6.5 and 6.8, over 1024 (64) 7.1 and 7.3, over 2048 (128) 8.2 and 7.1, over 4096 (256) 9.7 and 7.5, over 16384 (768) 17.7 and 12.4.
// A launch also costs the host 2 us, which bounds the calls of single tokens from Python: over 4096 tokens 9.7 and 10.1 there, one head over 20000 (79)
// 7.9 and 10.4; so up to a workgroup to each compute unit stays inside.  Two rows inside: 16 heads over 300 tokens 7.6 and 7.1, over 4096 10.9 and 7.4.
constexpr int kInside = 256;
__host__ __device__ bool joins_inside(const QueryArgs& a) { return a.rows == 1 && a.H * a.splits <= kInside; }
// The second launch has a workgroup to a row, and where rows of all heads are many, to four: us with one and with four, 16 heads over 4096 tokens, 1 row
// 7.4 and 8.7, 16 rows 8.1 and 9.4, 64 (1024 in all) 15.0 and 15.1, 200 28.1 and 26.6; one head over 65536, 1 row 9.8 and 15.6, 200 22.9 and 24.7.
constexpr int kJoinApart = 1024;
constexpr float kInf = __builtin_inff();
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ float off_of(float ref) { return ref == -kInf ? 0.0f : ref; }  // (nothing finite seen yet)

__device__ __forceinline__ float column_max(float x) {  // over the four lanes of a query
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float column_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const bf16x2 p = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, p);
}

// 16 codes (or bf16 values) of a row as loaded, and 8 of them as floats / as bf16.
template <int BITS>
struct Run {
  uint32_t w[BITS / 2];
  __device__ __forceinline__ void load(const uint8_t* p) {
    if constexpr (BITS == 16) {
      const u32x4 a = *reinterpret_cast<const u32x4*>(p), b = *reinterpret_cast<const u32x4*>(p + 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[i] = a[i];
        w[4 + i] = b[i];
      }
    } else if constexpr (BITS == 4) {
      const u32x2 a = *reinterpret_cast<const u32x2*>(p);
      w[0] = a[0];
      w[1] = a[1];
    } else {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
  }
  __device__ __forceinline__ void codes(int s, float* x) const {  // 8 s ..
    if constexpr (BITS == 4) {
      uint32_t even = w[s] & 0x0f0f0f0fu, odd = (w[s] >> 4) & 0x0f0f0f0fu;
      // (opaque to the optimizer, which would rather have a bit-field extract for every code than a conversion of a byte)
      asm("" : "+v"(even), "+v"(odd));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = (float)((even >> (8 * i)) & 0xffu);
        x[2 * i + 1] = (float)((odd >> (8 * i)) & 0xffu);
      }
    } else if constexpr (BITS == 2) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t every = (w[0] >> (2 * k)) & 0x03030303u;  // codes k, k + 4, ..
        asm("" : "+v"(every));
        x[k] = (float)((every >> (16 * s)) & 0xffu);
        x[4 + k] = (float)((every >> (16 * s + 8)) & 0xffu);
      }
    }
  }
};

// 8 elements as the cache's dequantized view: an exact difference, one product, one rounding.
template <int BITS>
__device__ __forceinline__ bf16x8 view(const Run<BITS>& r, int s, const float* scale, const float* zero) {
  u32x4 v;
  if constexpr (BITS == 16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = r.w[4 * s + i];
  } else {
    float x[8];
    r.codes(s, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack2((x[2 * i] - zero[2 * i]) * scale[2 * i], (x[2 * i + 1] - zero[2 * i + 1]) * scale[2 * i + 1]);
  }
  return __builtin_bit_cast(bf16x8, v);
}

__device__ __forceinline__ void load16(const float* p, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(p + 4 * i);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[4 * i + j] = v[j];
  }
}

// Over a wave, in every lane: lanes of a row of 16 by DPP, rows by swaps.
template <int CTRL>
__device__ __forceinline__ float from_lane(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
template <typename F>
__device__ __forceinline__ float over_wave(float x, F f) {
  x = f(x, from_lane<0xb1>(x));   // lane ^ 1
  x = f(x, from_lane<0x4e>(x));   // lane ^ 2
  x = f(x, from_lane<0x141>(x));  // 7 - lane of eight: the other four
  x = f(x, from_lane<0x140>(x));  // 15 - lane of sixteen: the other eight
  const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = f(__uint_as_float(p[0]), __uint_as_float(p[1]));
  const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return f(__uint_as_float(q[0]), __uint_as_float(q[1]));
}

// Joins rows r0 .. r0 + n - 1 (n <= 4) of a (head, row block) from its parts, a whole workgroup.  Every wave works out the weights of 64 parts, one a
// lane; thread (g, c) takes the values of the parts g, g + 4, .. of channel c, whose loads do not wait for the weights; the four threads of a
// channel add up in LDS.
// ROWS: as many rows' loads are on their way together; rows from n on are copies of the last and not stored.
using Shares = float[kWaves][kJoinRows][kD];
template <int ROWS>
__device__ __forceinline__ void join(const QueryArgs& a, int unit, int head, int row0, int r0, int n, int rows_wg, Shares& shares) {
  const int lane = threadIdx.x % 64, g = __builtin_amdgcn_readfirstlane(threadIdx.x / kD), c = threadIdx.x % kD;
  const size_t stride = (size_t)rows_wg * kQueryPart;  // between two parts
  float own_top = -kInf, own_sum = 0.0f;  // of row g
  float top_of[ROWS], l_of[ROWS], v_of[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    top_of[r] = -kInf;
    l_of[r] = v_of[r] = 0.0f;
  }
  for (int s0 = 0; s0 < a.splits; s0 += 64) {
    const int last = a.splits - 1;
    float m_of[ROWS], x_of[ROWS], value_of[ROWS][16];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const float* parts = a.parts + (size_t)unit * a.splits * stride + (size_t)(r0 + min(r, n - 1)) * kQueryPart;
      const float* own = parts + min(s0 + lane, last) * stride + kD;
      m_of[r] = s0 + lane <= last ? own[0] : -kInf;
      x_of[r] = own[1];
#pragma unroll
      for (int i = 0; i < 16; ++i) value_of[r][i] = parts[min(s0 + g + i * kWaves, last) * stride + c];
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      float &top = top_of[r], &l = l_of[r], &v = v_of[r];
      const float m = m_of[r], x = x_of[r];
      const float* value = value_of[r];
      const float to = fmaxf(top, over_wave(m, [](float p, float q) { return fmaxf(p, q); })), off = off_of(to);
      const float f = exp2_(top - off), w = exp2_(m - off);
      l = l * f + over_wave(s0 + lane <= last ? x * w : 0.0f, [](float p, float q) { return p + q; });
      v *= f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float part = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), g + i * kWaves));
        v += s0 + g + i * kWaves <= last ? value[i] * part : 0.0f;
      }
      top = to;
    }
  }
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    shares[g][r][c] = v_of[r];
    if (r == g) {
      own_top = top_of[r];
      own_sum = l_of[r];
    }
  }
  __syncthreads();
  if (g < n) {
    float x = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) x += shares[w][g][c];
    const size_t row = (size_t)head * a.rows + row0 + r0 + g;
    a.out[row * kD + c] = (uint16_t)pack2(x / own_sum, 0.0f);
    if (c == 0 && a.lse) a.lse[row] = (off_of(own_top) + log2f(own_sum)) * kLn2;
  }
  __syncthreads();
}

// A workgroup: one head, 16 QB query rows, tiles [begin, end) of 64 tokens.
template <int BITS, int G, int QB>
__global__ __launch_bounds__(64 * kWaves, QB == 1 ? 3 : 2) void query_attend_kernel(QueryArgs a) {
  __shared__ __align__(16) float acc[kWaves][kRows][kD + 4];
  __shared__ float refs[kWaves][kRows], sums[kWaves][kRows];
  __shared__ Shares shares;
  __shared__ int last;
  const int lane = threadIdx.x % 64, col = lane % 16, u = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int split = blockIdx.x % a.splits, unit = blockIdx.x / a.splits, block = unit % a.blocks, head = unit / a.blocks;
  const int row0 = block * kRows * QB;
  const int tiles = (a.T + kTile - 1) / kTile;
  // (at most 2^18 tiles and 2^10 parts)
  const int begin = (int)((uint32_t)tiles * (uint32_t)split / (uint32_t)a.splits), end = (int)((uint32_t)tiles * (uint32_t)(split + 1) / (uint32_t)a.splits);
  constexpr int kRowBytes = kD * BITS / 8, kRunBytes = 2 * BITS, kGroups = kD / G;
  const uint8_t* kc = a.kc + (size_t)head * a.code_head;
  const uint8_t* vc = a.vc + (size_t)head * a.code_head;
  const float* ks = a.ks + (size_t)head * a.kparam_head;
  const float* kz = a.kz + (size_t)head * a.kparam_head;
  const float* vs = a.vs + (size_t)head * a.vparam_head;
  const float* vz = a.vz + (size_t)head * a.vparam_head;

  bf16x8 qf[QB][2];  // (rows behind the last are copies of it that nobody writes)
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const uint16_t* q = a.q + head * a.q_sh + (int64_t)min(row0 + qb * kRows + col, a.rows - 1) * a.q_st + 16 * u;
#pragma unroll
    for (int s = 0; s < 2; ++s) qf[qb][s] = *reinterpret_cast<const bf16x8*>(q + 8 * s);
  }
  f32x4 o[QB][4] = {};
  float ref[QB], sum[QB] = {};
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) ref[qb] = -kInf;

  // A tile's keys are fetched while the values of the wave's tile before are worked on, its values while its keys are.
  Run<BITS> kr[4];
  float kss[16], kzz[16];
  auto fetch_keys = [&](int t) {
#pragma unroll
    for (int b = 0; b < 4; ++b) kr[b].load(kc + ((size_t)t * kTile + 16 * (col / 4) + 4 * b + col % 4) * kRowBytes + u * kRunBytes);
    if constexpr (BITS != 16) {
      const size_t at = ((size_t)t * (kTile / G) + (G == 32 ? col / 8 : 0)) * kD + 16 * u;
      load16(ks + at, kss);
      load16(kz + at, kzz);
    }
  };
  auto tile = [&](int t, auto cut_) {  // cut: some of its tokens lie behind the last
    constexpr bool kCut = decltype(cut_)::value;
    Run<BITS> vr[4];
    float vss[16 * kGroups], vzz[16 * kGroups];
#pragma unroll
    for (int b = 0; b < 4; ++b) vr[b].load(vc + ((size_t)t * kTile + 16 * b + col) * kRowBytes + u * kRunBytes);
    if constexpr (BITS != 16) {
      const size_t at = ((size_t)t * kTile + 16 * u) * kGroups;
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        load16(vs + at + 16 * g, vss + 16 * g);
        load16(vz + at + 16 * g, vzz + 16 * g);
      }
    }
    f32x4 x[QB][4];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) x[qb][b] = f32x4{};
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const bf16x8 k = view<BITS>(kr[b], s, kss + 8 * s, kzz + 8 * s);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) x[qb][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qf[qb][s], x[qb][b], 0, 0, 0);
      }
    }
    if (t + kWaves < end) fetch_keys(t + kWaves);
    const int left = a.T - t * kTile - 16 * u;  // of the lane's 16 tokens
    bool moves = false;
    float top[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      float m = -kInf;
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (kCut) x[qb][b][j] = 4 * b + j < left ? x[qb][b][j] : -kInf;
          m = fmaxf(m, x[qb][b][j]);
        }
      top[qb] = column_max(m) * a.c2;
      moves |= top[qb] > ref[qb];
    }
    if (__any(moves)) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        const float to = fmaxf(top[qb], ref[qb]), f = ref[qb] == -kInf || to == ref[qb] ? 1.0f : exp2_(ref[qb] - to);
        ref[qb] = to;
        sum[qb] *= f;
#pragma unroll
        for (int cb = 0; cb < 4; ++cb) o[qb][cb] *= f;
      }
    }
    bf16x8 p[QB][2];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const float off = off_of(ref[qb]);
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[qb][b][j] = exp2_(x[qb][b][j] * a.c2 - off);
          sum[qb] += x[qb][b][j];
        }
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const u32x4 w = {pack2(x[qb][2 * s][0], x[qb][2 * s][1]), pack2(x[qb][2 * s][2], x[qb][2 * s][3]),
                         pack2(x[qb][2 * s + 1][0], x[qb][2 * s + 1][1]), pack2(x[qb][2 * s + 1][2], x[qb][2 * s + 1][3])};
        p[qb][s] = __builtin_bit_cast(bf16x8, w);
      }
    }
#pragma unroll
    for (int cb = 0; cb < 4; ++cb)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        float sc[8], ze[8];
        if constexpr (BITS != 16) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            sc[e] = vss[(8 * s + e) * kGroups + (kGroups == 2 ? cb / 2 : 0)];
            ze[e] = vzz[(8 * s + e) * kGroups + (kGroups == 2 ? cb / 2 : 0)];
          }
        }
        bf16x8 v = view<BITS>(vr[cb], s, sc, ze);
        if (kCut) {  // rows behind the last token hold whatever the cache held there before
          u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int n = left - (8 * s + 2 * i);
            w[i] &= n >= 2 ? 0xffffffffu : (n == 1 ? 0xffffu : 0u);
          }
          v = __builtin_bit_cast(bf16x8, w);
        }
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) o[qb][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[qb][s], o[qb][cb], 0, 0, 0);
      }
  };
  const int whole = min(end, a.T / kTile);  // (the last tile of all may be cut)
  if (begin + wave < end) fetch_keys(begin + wave);
  for (int t = begin + wave; t < whole; t += kWaves) tile(t, std::false_type{});
  if (whole < end && (whole - begin) % kWaves == wave) tile(whole, std::true_type{});

  // The waves' results, 16 rows at a time: lane (col, u) has channels 16 cb + 4 u + 0..3 of row col.
  float* piece = a.parts + ((size_t)unit * a.splits + split) * kRows * QB * kQueryPart;
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    if (qb > 0) __syncthreads();
    const float total = column_sum(sum[qb]);
#pragma unroll
    for (int cb = 0; cb < 4; ++cb) *reinterpret_cast<f32x4*>(&acc[wave][col][16 * cb + 4 * u]) = o[qb][cb];
    if (u == 0) {
      refs[wave][col] = ref[qb];
      sums[wave][col] = total;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kRows * kD; i += 64 * kWaves) {
      const int r = i / kD, c = i % kD, row = row0 + qb * kRows + r;
      if (row >= a.rows) continue;
      float top = -kInf;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, refs[w][r]);
      const float off = off_of(top);
      float l = 0.0f, v = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = exp2_(refs[w][r] - off);
        l += sums[w][r] * f;
        v += acc[w][r][c] * f;
      }
      if (a.splits == 1) {
        a.out[((size_t)head * a.rows + row) * kD + c] = (uint16_t)pack2(a.T == 0 ? 0.0f : v / l, 0.0f);
        if (c == 0 && a.lse) a.lse[(size_t)head * a.rows + row] = (off + log2f(l)) * kLn2;
      } else {
        float* to = piece + (qb * kRows + r) * kQueryPart;
        __hip_atomic_store(to + c, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (c == 0) {
          __hip_atomic_store(to + kD, top, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          __hip_atomic_store(to + kD + 1, l, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
      }
    }
  }
  if (QB > 1 || a.splits == 1 || !joins_inside(a)) return;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's part has reached memory
  __syncthreads();
  if (threadIdx.x == 0) {
    uint32_t* counter = a.counters + unit;
    last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)a.splits - 1u;
    if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // as the next launch wants it
  }
  __syncthreads();
  if (!last) return;
  // (The fence lets the join read what other XCDs wrote with plain loads, all on their way at once: one after the other, as loads of
  // agent scope are issued, 64 parts took 40 us.)
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  join<1>(a, unit, head, row0, 0, 1, kRows * QB, shares);
}

// The join as a launch of its own, ROWS rows to a workgroup.
template <int ROWS>
__global__ __launch_bounds__(64 * kWaves) void query_join_kernel(QueryArgs a, int rows_wg) {
  __shared__ Shares shares;
  const int groups = (a.rows + ROWS - 1) / ROWS, head = blockIdx.x / groups, row = blockIdx.x % groups * ROWS;
  const int block = row / rows_wg, row0 = block * rows_wg;
  join<ROWS>(a, head * a.blocks + block, head, row0, row - row0, min(ROWS, a.rows - row), rows_wg, shares);
}

template <int BITS, int G>
hipError_t launch(const QueryArgs& a, hipStream_t stream) {
  const int workgroups = a.H * a.blocks * a.splits, rows_wg = a.rows <= kRows ? kRows : kQueryWide * kRows;
  if (a.rows <= kRows) query_attend_kernel<BITS, G, 1><<<workgroups, 64 * kWaves, 0, stream>>>(a);
  else query_attend_kernel<BITS, G, kQueryWide><<<workgroups, 64 * kWaves, 0, stream>>>(a);
  if (a.splits == 1 || joins_inside(a)) return hipGetLastError();
  if ((long long)a.H * a.rows <= kJoinApart) query_join_kernel<1><<<a.H * a.rows, 64 * kWaves, 0, stream>>>(a, rows_wg);
  else query_join_kernel<kJoinRows><<<a.H * ((a.rows + kJoinRows - 1) / kJoinRows), 64 * kWaves, 0, stream>>>(a, rows_wg);
  return hipGetLastError();
}

}  // namespace

// Up to 16 rows one column block; more share the dequantized elements, 64 to a wave (20000 tokens: 16 rows 14.7 us, 17 rows 25, 64 rows 29, so
// two passes of 16 rows would already take longer).  As many workgroups as the chip holds at once, each with a tile for every wave, and no more partial
// results than the workspace holds.
bool plan_query(QueryArgs& a) {
  const int rows_wg = a.rows <= kRows ? kRows : kQueryWide * kRows, tiles = (a.T + kTile - 1) / kTile;
  a.blocks = (a.rows + rows_wg - 1) / rows_wg;
  const long long units = (long long)a.H * a.blocks;
  if (units > (1ll << 32) / (64 * kWaves) - 1) return false;  // threads of a launch are counted in 32 bits
  const long long places = a.rows <= kRows ? 3 * 256 : 2 * 256;  // workgroups that the chip holds at once
  const long long most = std::min(kQueryPieces * (long long)kRows / rows_wg, places) / units;
  a.splits = (int)std::max<long long>(1, std::min<long long>((tiles + kWaves - 1) / kWaves, most));
  return true;
}

hipError_t launch_query_attend(const QueryArgs& a, int bits, int G, hipStream_t stream) {
  if (bits == 16) return launch<16, 64>(a, stream);
  if (bits == 4) return G == 64 ? launch<4, 64>(a, stream) : launch<4, 32>(a, stream);
  return G == 64 ? launch<2, 64>(a, stream) : launch<2, 32>(a, stream);
}

}  // namespace xsv
