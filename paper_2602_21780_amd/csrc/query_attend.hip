// Attention of a few query rows over a layer's packed cache (single tokens, special tokens, probes): one pass over the cache.
//
//   out = softmax(scale q K~^T) V~,   lse = log sum exp(scale q K~^T),   K~, V~ = bf16((code - zero) * scale)
//
// What bounds it is the cache: every packed byte is read once per block of query rows (0.625 bytes per element at 4 bits),
// and a few vector instructions per element turn it into the same bf16 view that the rest of the library attends to.
//
// A wave takes 64 tokens at a time straight from memory into registers: keys as the A operand of 16x16x32 MFMAs (transposed
// logits, a lane holds 16 tokens of one query), values, which the cache keeps transposed, as the A operand of the second
// product, and the probabilities, packed, as its B operand.  Operand rows are dealt so that every lane loads runs: its quarter u of the
// wave has channels 16 u .. of a key row and tokens 16 u .. of a value row, and row R of logit block B is token
// 16 (R / 4) + 4 B + R % 4, which puts tokens 16 u .. into the accumulators of quarter u as well.
//
// The tokens are cut over the waves of a workgroup (joined in LDS) and over workgroups, so that few rows still use the whole chip;
// the workgroup that ends last in a (head, row block) joins their partial results, in their order.
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

// A workgroup: one head, 16 QB query rows, tiles [begin, end) of 64 tokens.
template <int BITS, int G, int QB>
__global__ __launch_bounds__(64 * kWaves, QB == 1 ? 3 : 2) void query_attend_kernel(QueryArgs a) {
  __shared__ __align__(16) float acc[kWaves][kRows][kD + 4];
  __shared__ float refs[kWaves][kRows], sums[kWaves][kRows];
  __shared__ float shares[kWaves][kJoinRows][kD];
  __shared__ int last;
  const int lane = threadIdx.x % 64, col = lane % 16, u = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int split = blockIdx.x % a.splits, unit = blockIdx.x / a.splits, block = unit % a.blocks, head = unit / a.blocks;
  const int row0 = block * kRows * QB;
  const int tiles = (a.T + kTile - 1) / kTile;
  const int begin = (int)((long long)tiles * split / a.splits), end = (int)((long long)tiles * (split + 1) / a.splits);
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
  if (a.splits == 1) return;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's part has reached memory
  __syncthreads();
  if (threadIdx.x == 0) {
    uint32_t* counter = a.counters + unit;
    last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)a.splits - 1u;
    if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // as the next launch wants it
  }
  __syncthreads();
  if (!last) return;
  // Join: thread (g, c) takes the parts g, g + 4, .. of channel c, four rows at a time, all loads independent of each other; the four
  // threads of a channel add up in LDS.  (The fence lets them be plain loads: one after the other, as loads of agent scope are issued, 64
  // parts took 40 us.)
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  const float* parts = a.parts + (size_t)unit * a.splits * kRows * QB * kQueryPart;
  constexpr size_t kPart = (size_t)kRows * QB * kQueryPart;
  const int g = threadIdx.x / kD, c = threadIdx.x % kD, rows = min(kRows * QB, a.rows - row0);
  static_assert(sizeof(acc) >= (size_t)kJoinRows * kQueryPieces * sizeof(float));
  float (*const weight)[kQueryPieces] = reinterpret_cast<float (*)[kQueryPieces]>(&acc[0][0][0]);  // [row][part]
  for (int r0 = 0; r0 < rows; r0 += kJoinRows) {
    const int n = min(kJoinRows, rows - r0);
    if (wave < n) {  // a wave per row: the parts' weights, the reference and the sum of all
      const float* of_row = parts + (size_t)(r0 + wave) * kQueryPart + kD;
      float top = -kInf, l = 0.0f;
#pragma unroll 2
      for (int s = lane; s < a.splits; s += 64) {
        const float m = of_row[s * kPart], n = of_row[s * kPart + 1], to = fmaxf(top, m), off = off_of(to);
        l = l * exp2_(top - off) + n * exp2_(m - off);
        top = to;
        weight[wave][s] = m;
      }
      const float own = top;
#pragma unroll
      for (int m = 1; m < 64; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
      const float off = off_of(top);
      l *= exp2_(own - off);
#pragma unroll
      for (int m = 1; m < 64; m *= 2) l += __shfl_xor(l, m);
      for (int s = lane; s < a.splits; s += 64) weight[wave][s] = exp2_(weight[wave][s] - off);
      if (lane == 0) {
        refs[0][wave] = top;
        sums[0][wave] = l;
      }
    }
    __syncthreads();
    float v[kJoinRows] = {};
    const float* from = parts + (size_t)r0 * kQueryPart + c;
    if (n == kJoinRows) {
#pragma unroll 8
      for (int s = g; s < a.splits; s += kWaves)
#pragma unroll
        for (int r = 0; r < kJoinRows; ++r) v[r] += from[s * kPart + r * kQueryPart] * weight[r][s];
    } else {
#pragma unroll
      for (int r = 0; r < kJoinRows - 1; ++r)
        if (r < n)
#pragma unroll 16
          for (int s = g; s < a.splits; s += kWaves) v[r] += from[s * kPart + r * kQueryPart] * weight[r][s];
    }
#pragma unroll
    for (int r = 0; r < kJoinRows; ++r) shares[g][r][c] = v[r];
    __syncthreads();
    if (g < n) {
      float x = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) x += shares[w][g][c];
      const size_t row = (size_t)head * a.rows + row0 + r0 + g;
      a.out[row * kD + c] = (uint16_t)pack2(x / sums[0][g], 0.0f);
      if (c == 0 && a.lse) a.lse[row] = (off_of(refs[0][g]) + log2f(sums[0][g])) * kLn2;
    }
    __syncthreads();
  }
}

template <int BITS, int G>
hipError_t launch(const QueryArgs& a, hipStream_t stream) {
  const int workgroups = a.H * a.blocks * a.splits;
  if (a.rows <= kRows) query_attend_kernel<BITS, G, 1><<<workgroups, 64 * kWaves, 0, stream>>>(a);
  else query_attend_kernel<BITS, G, kQueryWide><<<workgroups, 64 * kWaves, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

// Up to 16 rows one column block; more share the dequantized elements, 64 to a wave.  As many workgroups as the chip holds at once, each with a tile for every wave, and no more partial results than the workspace holds.
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
