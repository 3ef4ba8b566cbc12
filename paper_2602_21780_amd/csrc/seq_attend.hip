// Attention inside sequences and its gradient, bf16, 64 channels.
//
//   S = scale q k^T over the keys that a query sees,  lse = log sum exp(S),  P = exp(S - lse),  out = P v
//   dv = P^T dout,  dS = P (dout v^T - delta),  delta = sum_c dout out,  dq = scale dS k,  dk = scale dS^T q
//
// Everything is 32x32x16 MFMA products of tiles; logits, probabilities, sums and accumulators are fp32, and what enters a second
// product (P, dS) is rounded to bf16 once, like the inputs.  The probabilities of the gradient are worked out again from lse.
//
// The forward pass and dq compute transposed logits (keys x queries): a lane then holds 16 keys of ONE query, sums over
// keys stay in a lane, lse and delta are one register, and the packed result already is the operand of the second product.
// dk and dv compute them the other way (queries x keys) for the same reason: a lane holds 16 queries of one key.  The second
// product reads its other operand (v, k, dout, q) across its rows with transposing LDS reads.
//
// The gradient is two launches that share nothing but delta, and recompute S and dout v^T each (7 products instead of 5): one
// that owns queries, for dq, and one that owns keys, for dk and dv.  So no gradient is added up by atomics, heads that share
// a key head are summed in registers, in order, and the results are the same bits every time.
//
// A tile is 64 rows of 128 bytes, its 16-byte pieces permuted within the row by bits 1..3 of the row number (`swizzle`): both the
// reads along rows (16 rows, one piece) and the transposing ones (4 rows, 4 pieces) then touch every bank once.
#include "operators.h"

#include <algorithm>
#include <type_traits>

namespace xsv {
namespace {

using u32x2 = __attribute__((ext_vector_type(2))) uint32_t;
using u32x4 = __attribute__((ext_vector_type(4))) uint32_t;
using i16x4 = __attribute__((ext_vector_type(4))) short;
using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using f32x4 = __attribute__((ext_vector_type(4))) float;
using f32x16 = __attribute__((ext_vector_type(16))) float;
using lds_i16x4 = __attribute__((address_space(3))) i16x4;

constexpr int kRow = 128;             // bytes of a row in LDS
constexpr int kTileBytes = 64 * kRow;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_inff();
// Probabilities are taken against a reference logit per query, the largest of its first 32 keys, which moves when the sum over the 16
// keys that a lane has of 32 passes this: probabilities above 1 are as exact as below.
constexpr float kMaxPart = 16777216.0f;

__device__ __forceinline__ int swizzle(int row) { return ((row >> 1) & 1) << 2 | ((row >> 2) & 1) << 1 | ((row >> 3) & 1); }

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ float half_sum(float x) {  // of the two lanes that hold the same column
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const bf16x2 p = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, p);
}

// Eight values of a column block as the operand of 16 rows: accumulator registers 8 ks .. 8 ks + 7.
__device__ __forceinline__ bf16x8 pack8(const f32x16& x, int ks) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = pack2(x[8 * ks + 2 * i], x[8 * ks + 2 * i + 1]);
  return __builtin_bit_cast(bf16x8, r);
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// How a lane reads a tile.  along: 8 channels (16 s + 8 (lane / 32) ..) of row lane % 32 of a block of 32 rows.
// across: channel 32 cb + lane % 32 of the rows 16 ks + 8 r + 4 (lane / 32) + 0..3, r = 0, 1, of such a block: the order in
// which an accumulator's registers hold rows.
struct Reader {
  uint32_t along_, across_;
  __device__ __forceinline__ explicit Reader(int lane) {
    const int row = lane % 32, h = lane / 32;
    along_ = row * kRow + ((h ^ swizzle(row)) << 4);
    const int p = lane % 16, row4 = 4 * h + p / 4;  // transposing reads: 4 lanes give a row, 16 lanes take a channel each
    across_ = row4 * kRow + (((2 * ((lane / 16) % 2) + (p % 4) / 2) ^ swizzle(row4)) << 4) + 8 * (p % 2);
  }
  __device__ __forceinline__ bf16x8 along(const char* tile, int block, int s) const {
    return *reinterpret_cast<const bf16x8*>(tile + block * 32 * kRow + (along_ ^ (s << 5)));
  }
  __device__ __forceinline__ bf16x8 across(const char* tile, int block, int cb, int ks) const {
    const char* base = tile + block * 32 * kRow + ks * 16 * kRow;
    const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(base + (across_ ^ (cb << 6))));
    const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(base + 8 * kRow + (across_ ^ (cb << 6) ^ (1 << 4))));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

__device__ __forceinline__ bool not_finite(uint32_t two) { return (two & 0x7f80u) == 0x7f80u || (two & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ uint32_t finite_or_zero(uint32_t two) {
  return two & (((two & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((two & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u));
}
__device__ __forceinline__ bf16x8 cleaned(bf16x8 x) {
  u32x4 r = __builtin_bit_cast(u32x4, x);
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = finite_or_zero(r[i]);
  return __builtin_bit_cast(bf16x8, r);
}

// Where a mask cuts a tile, a value that is not finite must not reach queries that do not see its row, but 0 * NaN does: the
// second product of such a tile takes its finite values only, and behind the loop this adds the others, of rows [from, to), to
// the columns (queries, or keys) that see their rows.  visible(row) is the lane's answer for its column.
template <typename F>
__device__ __forceinline__ void add_not_finite(const uint16_t* base, int64_t st, int from, int to, int lane, F visible, f32x16* acc) {
#pragma unroll 1
  for (int row = from; row < to; ++row) {
    const bool sees = visible(row);
#pragma unroll
    for (int cb = 0; cb < 2; ++cb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32x2 two = *reinterpret_cast<const u32x2*>(base + row * st + 32 * cb + 8 * i + 4 * (lane / 32));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t bits = (j & 1) ? (two[j / 2] & 0xffff0000u) : (two[j / 2] << 16);
          acc[cb][4 * i + j] += sees && (bits & 0x7f800000u) == 0x7f800000u ? __uint_as_float(bits) : 0.0f;
        }
      }
  }
}

// The pieces of a tile that a thread of a workgroup of THREADS brings to LDS.
template <int THREADS>
struct Stage {
  static constexpr int kPieces = 512 / THREADS;
  u32x4 r[kPieces];
  // rows row0 .. row0 + 63 of a sequence of n rows that begins at `base`; rows behind it are zeros
  __device__ __forceinline__ void load(const uint16_t* base, int64_t st, int row0, int n) {
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      const int at = p * THREADS + threadIdx.x, row = row0 + at / 8;
      r[p] = row < n ? *reinterpret_cast<const u32x4*>(base + row * st + 8 * (at % 8)) : u32x4{};
    }
  }
  __device__ __forceinline__ void store(char* tile) const {
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      const int at = p * THREADS + threadIdx.x, row = at / 8;
      *reinterpret_cast<u32x4*>(tile + row * kRow + (((at % 8) ^ swizzle(row)) << 4)) = r[p];
    }
  }
  __device__ __forceinline__ bool any_not_finite() const {
    bool bad = false;
#pragma unroll
    for (int p = 0; p < kPieces; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i) bad |= not_finite(r[p][i]);
    return bad;
  }
};

struct Sequence {
  int q0, nq, k0, nk;
};
// Offsets are device data: whatever they hold, no row outside the tensors is touched.
__device__ __forceinline__ Sequence sequence_of(const SeqArgs& a, int s) {
  Sequence r;
  r.q0 = min(max(a.q_begin[s], 0), a.rows_q);
  r.nq = min(min(max(a.q_begin[s + 1], r.q0), a.rows_q) - r.q0, a.longest_q);
  r.k0 = min(max(a.k_begin[s], 0), a.rows_k);
  r.nk = min(min(max(a.k_begin[s + 1], r.k0), a.rows_k) - r.k0, a.longest_k);
  return r;
}
// Query i of a sequence sees the keys in front of this one: query i stands at key position i + nk - nq, and sees the keys
// up to the end of the block of `causal` keys that it stands in.
__device__ __forceinline__ int keys_seen(const SeqArgs& a, const Sequence& s, int i) {
  if (a.causal == 0) return s.nk;
  const int pos = i + s.nk - s.nq;
  if (pos < 0) return 0;
  return (int)min((int64_t)s.nk, ((int64_t)(pos / a.causal) + 1) * a.causal);
}
// ... and a key is seen by the queries from this one on.
__device__ __forceinline__ int first_query(const SeqArgs& a, const Sequence& s, int key) {
  if (a.causal == 0) return 0;
  return max(0, key / a.causal * a.causal - (s.nk - s.nq));
}

// Workgroups are dealt to the XCDs one by one; this gives each XCD a run of consecutive ones, which share keys and values
// (or queries) through its L2.
__device__ __forceinline__ int dealt(int wg, int n) {
  const int xcd = wg % 8, q = n / 8, r = n % 8;
  return xcd * q + min(xcd, r) + wg / 8;
}

// ---- what owns queries: forward, and the gradient of the queries ----------------------------------------------------

// A workgroup's place: WAVES x 32 queries of one head of one sequence.  Blocks with many keys to see come first.
struct QueryBlock {
  Sequence s;
  int head, kv, row0;
  int row, seen;              // the lane's query (behind the last: a copy of it that nobody writes) and the keys it sees
  int wave_least, wave_most;  // keys that all, and any, of the wave's queries see; of the workgroup's
  int wg_least, tiles;
  bool any;
  template <int WAVES>
  __device__ __forceinline__ static QueryBlock of(const SeqArgs& a, int blocks, int wave, int lane) {
    QueryBlock b;
    const int id = dealt(blockIdx.x, gridDim.x);
    const int unit = id / blocks;
    b.head = unit / a.sequences;
    b.kv = b.head / (a.heads / a.kv_heads);
    b.s = sequence_of(a, unit % a.sequences);
    b.row0 = (blocks - 1 - id % blocks) * 32 * WAVES;
    b.any = b.row0 < b.s.nq;
    if (!b.any) return b;
    const int last = b.s.nq - 1, first = min(b.row0 + wave * 32, last);
    b.row = b.row0 + wave * 32 + lane % 32;
    b.seen = keys_seen(a, b.s, min(b.row, last));
    b.wave_least = keys_seen(a, b.s, first);  // (rows ascend, and so does what they see)
    b.wave_most = keys_seen(a, b.s, min(first + 31, last));
    b.wg_least = keys_seen(a, b.s, b.row0);
    b.tiles = (keys_seen(a, b.s, min(b.row0 + 32 * WAVES - 1, last)) + 63) / 64;
    return b;
  }
  // the lane's part of a row of queries, outputs or their gradients
  __device__ __forceinline__ const uint16_t* at(const SeqRows& t, int lane) const {
    return t.p + head * t.sh + (int64_t)(s.q0 + min(row, s.nq - 1)) * t.st + 8 * (lane / 32);
  }
};

// Tiles of keys and values through two buffers: the next one's loads are on their way while a tile is worked on.
// work(t, keys, values, masked, dirty): dirty, only where the mask cuts the tile: keys (WATCH = 0) or values (1) that are not finite.
template <int WAVES, int WATCH, typename F>
__device__ __forceinline__ void over_keys(const SeqArgs& a, const QueryBlock& b, char (*lds)[2][kTileBytes], int* dirty, F work) {
  const uint16_t* kb = a.k.p + b.kv * a.k.sh + b.s.k0 * a.k.st;
  const uint16_t* vb = a.v.p + b.kv * a.v.sh + b.s.k0 * a.v.st;
  Stage<64 * WAVES> sk, sv;
  auto fetch = [&](int t) {
    sk.load(kb, a.k.st, 64 * t, b.s.nk);
    sv.load(vb, a.v.st, 64 * t, b.s.nk);
  };
  auto put = [&](int t) {
    sk.store(lds[t & 1][0]);
    sv.store(lds[t & 1][1]);
    if (64 * (t + 1) > b.wg_least && __any((WATCH ? sv : sk).any_not_finite())) dirty[t & 1] = t + 1;
  };
  if (b.tiles <= 0) return;
  if (threadIdx.x < 2) dirty[threadIdx.x] = 0;
  __syncthreads();
  fetch(0);
  put(0);
  __syncthreads();
  for (int t = 0; t < b.tiles; ++t) {
    if (t + 1 < b.tiles) fetch(t + 1);
    if (64 * (t + 1) <= b.wave_least) work(t, lds[t & 1][0], lds[t & 1][1], std::false_type{}, false);
    else if (64 * t < b.wave_most) work(t, lds[t & 1][0], lds[t & 1][1], std::true_type{}, dirty[t & 1] == t + 1);
    if (t + 1 < b.tiles) put(t + 1);
    __syncthreads();
  }
}

__device__ __forceinline__ void write_columns(uint16_t* dst, const f32x16* x, float f, int h) {
#pragma unroll
  for (int cb = 0; cb < 2; ++cb)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x2 w = {pack2(x[cb][4 * i] * f, x[cb][4 * i + 1] * f), pack2(x[cb][4 * i + 2] * f, x[cb][4 * i + 3] * f)};
      *reinterpret_cast<u32x2*>(dst + 32 * cb + 8 * i + 4 * h) = w;
    }
}

template <int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void seq_attend_kernel(SeqArgs a, int blocks) {
  __shared__ __align__(16) char lds[2][2][kTileBytes];  // [buffer][keys, values]
  __shared__ int dirty[2];                             // number + 1 of a cut tile with values that are not finite
  const int lane = threadIdx.x % 64, h = lane / 32;
  const QueryBlock b = QueryBlock::of<WAVES>(a, blocks, __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane);
  if (!b.any) return;
  bf16x8 qf[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) qf[c] = *reinterpret_cast<const bf16x8*>(b.at(a.q, lane) + 16 * c);
  const Reader rd(lane);
  const float c2 = a.scale * kLog2e;
  f32x16 o[2] = {};
  float sum = 0.0f, ref = -kInf;  // ref in powers of two; -inf: no finite logit yet
  bool left_out = false;          // values that are not finite are to be added

  over_keys<WAVES, 1>(a, b, lds, dirty, [&](int t, const char* kt, const char* vt, auto masked_, bool clean_up) {
    constexpr bool kMasked = decltype(masked_)::value;
    if (kMasked) left_out |= clean_up;
    f32x16 x[2];
    auto logits = [&]() {
#pragma unroll
      for (int kh = 0; kh < 2; ++kh) {
        x[kh] = f32x16{};
#pragma unroll
        for (int c = 0; c < 4; ++c) x[kh] = mfma(rd.along(kt, kh, c), qf[c], x[kh]);
        if (kMasked) {
          const int left = b.seen - (64 * t + 32 * kh + 4 * h);
#pragma unroll
          for (int i = 0; i < 16; ++i) x[kh][i] = 8 * (i / 4) + i % 4 < left ? x[kh][i] : -kInf;
        }
      }
    };
    float part;
    auto probabilities = [&]() {
      const float off = ref == -kInf ? 0.0f : ref;
      float p[4] = {};
#pragma unroll
      for (int kh = 0; kh < 2; ++kh)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          x[kh][i] = exp2_(x[kh][i] * c2 - off);
          p[i % 4] += x[kh][i];
        }
      part = (p[0] + p[1]) + (p[2] + p[3]);
    };
    logits();
    probabilities();
    const bool move = !(part <= kMaxPart) || ref == -kInf;
    if (__any(move)) {
      logits();
      float top = x[0][0];
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, fmaxf(x[0][i], x[1][i]));
      // (a query's two lanes move together, and by themselves: its result does not depend on the wave's other queries)
      const bool moves = half_max(move ? 1.0f : 0.0f) > 0.0f;
      const float moved = moves ? fmaxf(ref, half_max(top) * c2) : ref;
      const float f = ref == -kInf || !moves ? 1.0f : exp2_(ref - moved);  // (from no reference: there is nothing to scale)
      ref = moved;
      sum *= f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        o[0][i] *= f;
        o[1][i] *= f;
      }
      probabilities();
    }
    sum += part;
    auto product = [&](auto clean_) {
#pragma unroll
      for (int kh = 0; kh < 2; ++kh)
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          const bf16x8 p = pack8(x[kh], ks);
#pragma unroll
          for (int cb = 0; cb < 2; ++cb) {
            bf16x8 vf = rd.across(vt, kh, cb, ks);
            if (decltype(clean_)::value) vf = cleaned(vf);
            o[cb] = mfma(vf, p, o[cb]);
          }
        }
    };
    if (clean_up) product(std::true_type{});
    else product(std::false_type{});
  });
  if (left_out)
    add_not_finite(a.v.p + b.kv * a.v.sh + b.s.k0 * a.v.st, a.v.st, b.wave_least / 64 * 64, b.wave_most, lane, [&](int r) { return r < b.seen; }, o);
  const float total = half_sum(sum);
  if (b.row >= b.s.nq) return;
  const bool empty = b.seen == 0;
  write_columns(const_cast<uint16_t*>(b.at(a.out, 0)), o, empty ? 0.0f : 1.0f / total, h);
  if (h == 0) a.lse[(int64_t)b.head * a.rows_q + b.s.q0 + b.row] = empty ? -kInf : ((ref == -kInf ? 0.0f : ref) + log2f(total)) * kLn2;
}

template <int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void seq_grad_q_kernel(SeqArgs a, int blocks) {
  __shared__ __align__(16) char lds[2][2][kTileBytes];
  __shared__ int dirty[2];
  const int lane = threadIdx.x % 64, h = lane / 32;
  const QueryBlock b = QueryBlock::of<WAVES>(a, blocks, __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane);
  if (!b.any) return;
  bf16x8 qf[4], df[4];
  float dot = 0.0f;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    qf[c] = *reinterpret_cast<const bf16x8*>(b.at(a.q, lane) + 16 * c);
    df[c] = *reinterpret_cast<const bf16x8*>(b.at(a.dout, lane) + 16 * c);
    const bf16x8 of = *reinterpret_cast<const bf16x8*>(b.at(a.out, lane) + 16 * c);
#pragma unroll
    for (int e = 0; e < 8; ++e) dot += (float)df[c][e] * (float)of[e];
  }
  const float delta = half_sum(dot);
  const int64_t at = (int64_t)b.head * a.rows_q + b.s.q0 + min(b.row, b.s.nq - 1);
  const float lse2 = a.lse[at] * kLog2e;
  if (h == 0 && b.row < b.s.nq) a.delta[at] = delta;
  const Reader rd(lane);
  const float c2 = a.scale * kLog2e;
  f32x16 g[2] = {};
  bool left_out = false;

  over_keys<WAVES, 0>(a, b, lds, dirty, [&](int t, const char* kt, const char* vt, auto masked_, bool clean_up) {
    constexpr bool kMasked = decltype(masked_)::value;
    if (kMasked) left_out |= clean_up;
#pragma unroll
    for (int kh = 0; kh < 2; ++kh) {
      f32x16 x = {}, y = {};
#pragma unroll
      for (int c = 0; c < 4; ++c) x = mfma(rd.along(kt, kh, c), qf[c], x);
#pragma unroll
      for (int c = 0; c < 4; ++c) y = mfma(rd.along(vt, kh, c), df[c], y);
      const int left = b.seen - (64 * t + 32 * kh + 4 * h);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float p = exp2_(x[i] * c2 - lse2);
        x[i] = p * (y[i] - delta);
        if (kMasked) x[i] = 8 * (i / 4) + i % 4 < left ? x[i] : 0.0f;
      }
      auto product = [&](auto clean_) {
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          const bf16x8 ds = pack8(x, ks);
#pragma unroll
          for (int cb = 0; cb < 2; ++cb) {
            bf16x8 kf = rd.across(kt, kh, cb, ks);
            if (decltype(clean_)::value) kf = cleaned(kf);
            g[cb] = mfma(kf, ds, g[cb]);
          }
        }
      };
      if (clean_up) product(std::true_type{});
      else product(std::false_type{});
    }
  });
  if (left_out)
    add_not_finite(a.k.p + b.kv * a.k.sh + b.s.k0 * a.k.st, a.k.st, b.wave_least / 64 * 64, b.wave_most, lane, [&](int r) { return r < b.seen; }, g);
  if (b.row < b.s.nq) write_columns(const_cast<uint16_t*>(b.at(a.dq, 0)), g, a.scale, h);
}

// ---- gradients of the keys and values -------------------------------------------------------------------------------

// A workgroup: WAVES x 32 keys of one key head of one sequence, over the queries of all heads that share it.
template <int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void seq_grad_kv_kernel(SeqArgs a, int blocks) {
  constexpr int kThreads = 64 * WAVES;
  __shared__ __align__(16) char lds[2][2][kTileBytes];  // [buffer][queries, dout]
  __shared__ __align__(16) float stats[2][2][64];       // [buffer][lse in powers of two, delta]
  __shared__ int dirty[2];
  const int lane = threadIdx.x % 64, h = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int id = dealt(blockIdx.x, gridDim.x);
  const int unit = id / blocks, block = id % blocks;
  const int kv = unit / a.sequences;
  const Sequence s = sequence_of(a, unit % a.sequences);
  const int key0 = block * 32 * WAVES;
  if (key0 >= s.nk) return;
  const int rep = a.heads / a.kv_heads;
  // (columns behind the last key are copies of it that nobody writes)
  const int key = key0 + wave * 32 + lane % 32;
  bf16x8 kf[4], vf[4];
  {
    const int i = min(key, s.nk - 1);
    const uint16_t* k = a.k.p + kv * a.k.sh + (int64_t)(s.k0 + i) * a.k.st + 8 * h;
    const uint16_t* v = a.v.p + kv * a.v.sh + (int64_t)(s.k0 + i) * a.v.st + 8 * h;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      kf[c] = *reinterpret_cast<const bf16x8*>(k + 16 * c);
      vf[c] = *reinterpret_cast<const bf16x8*>(v + 16 * c);
    }
  }
  const int from = first_query(a, s, min(key, s.nk - 1));  // queries that see the lane's key begin here
  const int wave_key = min(key0 + wave * 32, s.nk - 1);
  const int wave_from = first_query(a, s, wave_key), wave_all = first_query(a, s, min(wave_key + 31, s.nk - 1));
  const int wg_from = first_query(a, s, key0), wg_all = first_query(a, s, min(key0 + 32 * WAVES - 1, s.nk - 1));
  const int first_tile = wg_from / 64, tiles = max(0, (s.nq + 63) / 64 - first_tile);
  const int steps = tiles * rep;

  const Reader rd(lane);
  const float c2 = a.scale * kLog2e;
  f32x16 dk[2] = {}, dv[2] = {};
  bool left_out = false;  // some of them are to be added
  if (threadIdx.x < 2) dirty[threadIdx.x] = 0;
  Stage<kThreads> sq, sd;
  float st_l = 0.0f, st_d = 0.0f;
  auto fetch = [&](int n) {
    const int head = kv * rep + n / tiles, row = 64 * (first_tile + n % tiles);
    sq.load(a.q.p + head * a.q.sh + s.q0 * a.q.st, a.q.st, row, s.nq);
    sd.load(a.dout.p + head * a.dout.sh + s.q0 * a.dout.st, a.dout.st, row, s.nq);
    if (threadIdx.x < 64) {
      const int i = row + threadIdx.x;
      const int64_t at = (int64_t)head * a.rows_q + s.q0 + i;
      st_l = i < s.nq ? a.lse[at] * kLog2e : kInf;  // (rows behind the last query have no probability at all)
      st_d = i < s.nq ? a.delta[at] : 0.0f;
    }
  };
  auto put = [&](int n) {
    sq.store(lds[n & 1][0]);
    sd.store(lds[n & 1][1]);
    if (threadIdx.x < 64) {
      stats[n & 1][0][threadIdx.x] = st_l;
      stats[n & 1][1][threadIdx.x] = st_d;
    }
    if (64 * (first_tile + n % tiles) < wg_all && __any(sq.any_not_finite() || sd.any_not_finite())) dirty[n & 1] = n + 1;
  };
  auto tile = [&](int n, int row, auto masked_) {
    constexpr bool kMasked = decltype(masked_)::value;
    const char* qt = lds[n & 1][0];
    const char* dt = lds[n & 1][1];
    const bool clean_up = kMasked && dirty[n & 1] == n + 1;
    if (kMasked) left_out |= clean_up;
#pragma unroll
    for (int qh = 0; qh < 2; ++qh) {
      f32x16 x = {}, y = {};
#pragma unroll
      for (int c = 0; c < 4; ++c) x = mfma(rd.along(qt, qh, c), kf[c], x);
#pragma unroll
      for (int c = 0; c < 4; ++c) y = mfma(rd.along(dt, qh, c), vf[c], y);
      const int least = from - (row + 32 * qh + 4 * h), most = s.nq - (row + 32 * qh + 4 * h);
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const f32x4 l = *reinterpret_cast<const f32x4*>(&stats[n & 1][0][32 * qh + 8 * b + 4 * h]);
        const f32x4 d = *reinterpret_cast<const f32x4*>(&stats[n & 1][1][32 * qh + 8 * b + 4 * h]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int i = 4 * b + j;
          float p = exp2_(x[i] * c2 - l[j]);
          float ds = p * (y[i] - d[j]);
          if (kMasked) {
            const bool sees = 8 * b + j >= least && 8 * b + j < most;
            p = sees ? p : 0.0f;
            ds = sees ? ds : 0.0f;
          }
          x[i] = p;
          y[i] = ds;
        }
      }
      auto product = [&](auto clean_) {
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          const bf16x8 p = pack8(x, ks), ds = pack8(y, ks);
#pragma unroll
          for (int cb = 0; cb < 2; ++cb) {
            bf16x8 df = rd.across(dt, qh, cb, ks), qf = rd.across(qt, qh, cb, ks);
            if (decltype(clean_)::value) {
              df = cleaned(df);
              qf = cleaned(qf);
            }
            dv[cb] = mfma(df, p, dv[cb]);
            dk[cb] = mfma(qf, ds, dk[cb]);
          }
        }
      };
      if (clean_up) product(std::true_type{});
      else product(std::false_type{});
    }
  };
  if (steps > 0) {
    __syncthreads();
    fetch(0);
    put(0);
    __syncthreads();
    for (int n = 0; n < steps; ++n) {
      if (n + 1 < steps) fetch(n + 1);
      const int row = 64 * (first_tile + n % tiles);
      if (row >= wave_all) tile(n, row, std::false_type{});
      else if (row + 64 > wave_from) tile(n, row, std::true_type{});
      if (n + 1 < steps) put(n + 1);
      __syncthreads();
    }
  }
  if (left_out) {
    const int to = min(s.nq, (wave_all + 63) / 64 * 64);
    for (int head = kv * rep; head < (kv + 1) * rep; ++head) {
      add_not_finite(a.dout.p + head * a.dout.sh + s.q0 * a.dout.st, a.dout.st, wave_from / 64 * 64, to, lane, [&](int r) { return r >= from; }, dv);
      add_not_finite(a.q.p + head * a.q.sh + s.q0 * a.q.st, a.q.st, wave_from / 64 * 64, to, lane, [&](int r) { return r >= from; }, dk);
    }
  }
  if (key >= s.nk) return;
  write_columns(const_cast<uint16_t*>(a.dk.p) + kv * a.dk.sh + (int64_t)(s.k0 + key) * a.dk.st, dk, a.scale, h);
  write_columns(const_cast<uint16_t*>(a.dv.p) + kv * a.dv.sh + (int64_t)(s.k0 + key) * a.dv.st, dv, 1.0f, h);
}

long long grid_of(int longest, int rows, int heads, int sequences) { return ((long long)longest + rows - 1) / rows * heads * sequences; }

constexpr long long kMostWorkgroups = (1ll << 32) / 512 - 1;  // threads of a launch are counted in 32 bits

}  // namespace

bool seq_attend_fits(const SeqArgs& a) {
  return grid_of(a.longest_q, 128, a.heads, a.sequences) <= kMostWorkgroups && grid_of(a.longest_k, 128, a.kv_heads, a.sequences) <= kMostWorkgroups;
}

// Eight waves read a tile half as often as two workgroups of four; where blocks of 256 rows would leave compute units
// without work, the shorter ones.
hipError_t launch_seq_attend(const SeqArgs& a, hipStream_t stream) {
  const long long small = grid_of(a.longest_q, 128, a.heads, a.sequences), large = grid_of(a.longest_q, 256, a.heads, a.sequences);
  if (small == 0) return hipSuccess;
  if (large >= 256) seq_attend_kernel<8><<<(int)large, 512, 0, stream>>>(a, (a.longest_q + 255) / 256);
  else seq_attend_kernel<4><<<(int)small, 256, 0, stream>>>(a, (a.longest_q + 127) / 128);
  return hipGetLastError();
}

hipError_t launch_seq_attend_grad(const SeqArgs& a, hipStream_t stream) {
  const long long small_q = grid_of(a.longest_q, 128, a.heads, a.sequences), large_q = grid_of(a.longest_q, 256, a.heads, a.sequences);
  const long long small_k = grid_of(a.longest_k, 128, a.kv_heads, a.sequences), large_k = grid_of(a.longest_k, 256, a.kv_heads, a.sequences);
  if (small_q > 0) {
    if (large_q >= 256) seq_grad_q_kernel<8><<<(int)large_q, 512, 0, stream>>>(a, (a.longest_q + 255) / 256);
    else seq_grad_q_kernel<4><<<(int)small_q, 256, 0, stream>>>(a, (a.longest_q + 127) / 128);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (small_k > 0) {
    if (large_k >= 256) seq_grad_kv_kernel<8><<<(int)large_k, 512, 0, stream>>>(a, (a.longest_k + 255) / 256);
    else seq_grad_kv_kernel<4><<<(int)small_k, 256, 0, stream>>>(a, (a.longest_k + 127) / 128);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace xsv
