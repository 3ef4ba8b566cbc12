// Attention inside sequences and its gradient, bf16, 64 channels.
//
//   S = scale q k^T over the keys that a query sees,  lse = log sum exp(S),  P = exp(S - lse),  out = P v
//   dv = P^T dout,  dS = P (dout v^T - delta),  delta = sum_c dout out,  dq = scale dS k,  dk = scale dS^T q
//
// Everything is 32x32x16 MFMA products of tiles; logits, probabilities, sums and accumulators are fp32, and what enters a second
// product (P, dS) is rounded to bf16 once, like the inputs, since the products take bf16: outputs are off by 0.0020 to 0.0023 of themselves (rms) and
// gradients by 0.0025, where the rounding of a result alone makes 0.0016.  The probabilities of the gradient are worked out again from lse.
//
// The forward pass and dq compute transposed logits (keys x queries): a lane then holds 16 keys of ONE query, sums over
// keys stay in a lane, lse and delta are one register, and the packed result already is the operand of the second product.
// dk and dv compute them the other way (queries x keys) for the same reason: a lane holds 16 queries of one key.  The second
// product reads its other operand (v, k, dout, q) across its rows with transposing LDS reads.
//
// The gradient has workgroups that own queries, for dq, and ones that own keys, for dk and dv, which share nothing but delta and
// recompute S and dout v^T each (7 products instead of 5).  So no gradient is added up by atomics, heads that share
// a key head are summed in registers, in order, and the results are the same bits every time.
//
// A tile is 64 rows of 128 bytes, its 16-byte pieces permuted within the row by bits 1..3 of the row number (`swizzle`): both the
// reads along rows (16 rows, one piece) and the transposing ones (4 rows, 4 pieces) then touch every bank once.
//
// What it takes: per 32 x 32 logits the forward pass has 8 MFMAs of 32 cycles and 16 exponentials, 16 multiply-adds, 16 additions and 8
// conversions (16 cycles the one, 4 the others), which overlap across the waves of a SIMD and hardly within one; the gradient 28 MFMAs and twice
// the exponentials.  Besides, to fetch a tile takes 27 vector instructions a wave (13 in workgroups of eight), 12 of them integer multiplies of rows by strides,
// beside some 120 of the softmax, and the waves of a workgroup meet at a barrier in every tile.  Neither unit is full: six frames of 1374 tokens,
// frame-causal, 16 heads, forward 213 us = 760 TFLOP/s, matrix pipe busy 39 % of the cycles, vector units 63 %, where a loop of the bare mix at three waves
// a SIMD would need some 120 to 140 us; gradient 587 us = 690 TFLOP/s of the 10 D operations a pair that it cannot do without, 48 % and 45 %.
// Eight frames apart, gradient: 267 us = 580 TFLOP/s, 44 % and 45 %: keys and queries are padded to 1408, and 1408 workgroups of each kind end unevenly.
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
using f32x2 = __attribute__((ext_vector_type(2))) float;
using f32x4 = __attribute__((ext_vector_type(4))) float;
using f32x16 = __attribute__((ext_vector_type(16))) float;
using lds_i16x4 = __attribute__((address_space(3))) i16x4;
using lds_u32x4 = __attribute__((address_space(3))) u32x4;
using lds_f32x4 = __attribute__((address_space(3))) f32x4;
using lds_char = __attribute__((address_space(3))) const char;

constexpr int kRow = 128;             // bytes of a row in LDS
constexpr int kTileBytes = 64 * kRow;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_inff();
// Probabilities are taken against a reference logit per query, the largest of its first 32 keys, which moves when the sum over the 16
// keys that a lane has of 32 passes this: probabilities above 1 are as exact as below.
constexpr float kMaxPart = 16777216.0f;

__device__ __forceinline__ int swizzle(int row) { return ((row >> 1) & 1) << 2 | ((row >> 2) & 1) << 1 | ((row >> 3) & 1); }

// Operands are kept as four dwords (what lives across a loop as eight bf16 is taken apart into sixteen-bit pieces by the compiler).
__device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

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
__device__ __forceinline__ u32x4 pack8(const f32x16& x, int ks) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = pack2(x[8 * ks + 2 * i], x[8 * ks + 2 * i + 1]);
  return r;
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// How a lane reads a tile, `at` bytes behind `origin`.  along: 8 channels (16 s + 8 (lane / 32) ..) of row lane % 32 of a block of 32
// rows.  across: channel 32 cb + lane % 32 of the rows 16 ks + 8 r + 4 (lane / 32) + 0..3, r = 0, 1, of such a block: the order in
// which an accumulator's registers hold rows.  The permuted addresses are worked out once; with a constant `at` a read is one instruction.
struct Reader {
  uint32_t along_[4], across_[2][2];
  __device__ __forceinline__ Reader(const char* origin, int lane) {
    const uint32_t base = (uint32_t)(size_t)(lds_char*)origin;
    const int row = lane % 32, h = lane / 32;
#pragma unroll
    for (int s = 0; s < 4; ++s) along_[s] = base + row * kRow + (((2 * s + h) ^ swizzle(row)) << 4);
    const int p = lane % 16, row4 = 4 * h + p / 4;  // transposing reads: 4 lanes give a row, 16 lanes take a channel each
#pragma unroll
    for (int cb = 0; cb < 2; ++cb)
#pragma unroll
      for (int r = 0; r < 2; ++r)
        across_[cb][r] = base + (row4 + 8 * r) * kRow + (((4 * cb + 2 * ((lane / 16) % 2) + (p % 4) / 2) ^ swizzle(row4 + 8 * r)) << 4) + 8 * (p % 2);
  }
  __device__ __forceinline__ u32x4 along(int at, int block, int s) const {
    return *(lds_u32x4*)(along_[s] + at + block * 32 * kRow);
  }
  __device__ __forceinline__ u32x4 across(int at, int block, int cb, int ks) const {
    at += (block * 32 + ks * 16) * kRow;
    const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(across_[cb][0] + at));
    const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(across_[cb][1] + at));
    return __builtin_bit_cast(u32x4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

__device__ __forceinline__ bool not_finite(uint32_t two) { return (two & 0x7f80u) == 0x7f80u || (two & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ uint32_t finite_or_zero(uint32_t two) {
  return two & (((two & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((two & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u));
}
__device__ __forceinline__ u32x4 cleaned(u32x4 x) {
  u32x4 r = x;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = finite_or_zero(r[i]);
  return r;
}

// Where a mask cuts a tile, a value that is not finite must not reach queries that do not see its row, but 0 * NaN does: the
// second product of such a tile takes its finite values only, and this adds the others, of rows [from, to), to the columns (queries, or keys) that
// see their rows: to outputs with each such tile, since waves and workgroups that share tiles weigh theirs in the join and a weight of 0 (a query that
// sees no key of theirs) times infinity is NaN; to gradients, which are only added up, behind the loop.  visible(row) is the lane's answer for its column.
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

// The pieces of TILES consecutive tiles that a thread of a workgroup of THREADS brings to LDS.
template <int THREADS, int TILES>
struct Stage {
  static constexpr int kPieces = 512 * TILES / THREADS;
  u32x4 r[kPieces];
  // rows row0 .. of a sequence of n > 0 rows that begins at `base`; those behind it are copies of the last, which no result uses
  __device__ __forceinline__ void load(const uint16_t* base, int64_t st, int row0, int n) {
#pragma unroll
    for (int p = 0; p < kPieces; ++p) load_piece(p, base, st, row0 + p * (THREADS / 8) + threadIdx.x / 8, n);
  }
  __device__ __forceinline__ void load_piece(int p, const uint16_t* base, int64_t st, int row, int n) {
    r[p] = *reinterpret_cast<const u32x4*>(base + min(row, n - 1) * st + 8 * (threadIdx.x % 8));
  }
  // tile j goes to `tiles` + 2 j tiles: the two tensors' tiles take turns
  __device__ __forceinline__ void store(char* tiles) const {
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      const int row = p * (THREADS / 8) + threadIdx.x / 8;
      *reinterpret_cast<u32x4*>(tiles + (row / 64) * 2 * kTileBytes + (row % 64) * kRow + (((threadIdx.x % 8) ^ swizzle(row)) << 4)) = r[p];
    }
  }
  // of tile j, in the pieces that this thread has
  __device__ __forceinline__ bool any_not_finite(int j) const {
    bool bad = false;
#pragma unroll
    for (int p = 0; p < kPieces; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i) bad |= (p * (THREADS / 8) + (int)threadIdx.x / 8) / 64 == j && not_finite(r[p][i]);
    return bad;
  }
};

struct Sequence {
  int q0, nq, k0, nk;  // rows worked on: the bounds on the lengths leave those behind them out
  int ahead;           // the key position of query 0, from the whole lengths: what a bound leaves out moves no other row
};
// Offsets are device data: whatever they hold, no row outside the tensors is touched.
__device__ __forceinline__ Sequence sequence_of(const SeqArgs& a, int s) {
  Sequence r;
  r.q0 = min(max(a.q_begin[s], 0), a.rows_q);
  r.k0 = min(max(a.k_begin[s], 0), a.rows_k);
  const int n = min(max(a.q_begin[s + 1], r.q0), a.rows_q) - r.q0, m = min(max(a.k_begin[s + 1], r.k0), a.rows_k) - r.k0;
  r.nq = min(n, a.longest_q);
  r.nk = min(m, a.longest_k);
  r.ahead = m - n;
  return r;
}
// Query i of a sequence sees the keys in front of this one: it stands at key position i + ahead, and sees the keys
// up to the end of the block of `causal` keys that it stands in.
__device__ __forceinline__ int keys_seen(const SeqArgs& a, const Sequence& s, int i) {
  if (a.causal == 0) return s.nk;
  const int pos = i + s.ahead;
  if (pos < 0) return 0;
  return (int)min((int64_t)s.nk, ((int64_t)(pos / a.causal) + 1) * a.causal);
}
// ... and a key is seen by the queries from this one on (there may be none such within the bound).
__device__ __forceinline__ int first_query(const SeqArgs& a, const Sequence& s, int key) {
  if (a.causal == 0) return 0;
  return max(0, key / a.causal * a.causal - s.ahead);
}

// Workgroups start in the order of their numbers and are dealt to the XCDs one by one.
// Without a mask every XCD takes a run of the blocks of one head and sequence after the other, which share keys and values (or queries)
// through its L2.  Under a mask blocks differ in length and the longest come first, of all heads and sequences: one head after the other
// left the forward pass of a causal clip of 12 heads 212 us that takes 178, and ragged sequences of 12 heads 28 that take 22.  (Without a mask that order
// costs: 84 and 65 us forward.)  Where eight divides the heads, all blocks of a head and sequence are on one XCD then too; otherwise each block's
// heads begin one further on, so that no XCD has all of a long sequence.
struct Dealt {
  int head, sequence, block;
};
__device__ __forceinline__ Dealt dealt(const SeqArgs& a, int number, int heads, int blocks) {
  const int units = heads * a.sequences;
  if (a.causal) {
    const int block = number / units, first = number % units, unit = heads % 8 ? (first + block) % units : first;
    return Dealt{unit % heads, unit / heads, block};
  }
  const int n = units * blocks, xcd = number % 8, id = xcd * (n / 8) + min(xcd, n % 8) + number / 8, unit = id / blocks;
  return Dealt{unit / a.sequences, unit % a.sequences, id % blocks};
}




// A stretch of a pipeline, in this order whatever the compiler's scheduler would rather do: products one by one, behind each some LDS
// reads for later ones and a share of the arithmetic.
template <int N, typename Product, typename Read, typename Arithmetic>
__device__ __forceinline__ void in_order(Product product, Read read, Arithmetic arithmetic) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    product(i);
    read(i);
    arithmetic(i);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// ---- what owns queries: forward, and the gradient of the queries ----------------------------------------------------

// A workgroup's place: ROWS x 32 queries of one head of one sequence, every 32 of them worked on by SPLIT waves, which take the
// workgroup's tiles in turn and join their results in LDS at the end.  In small launches `parts` workgroups share the tiles of such a
// block, and leave results in fp32 that a second launch joins, in their order.  Blocks with many keys to see come first.
struct QueryBlock {
  Sequence s;
  int head, kv, row0, part;
  int row, seen;              // the lane's query (behind the last: a copy of it that nobody writes) and the keys it sees
  int wave_least, wave_most;  // keys that all, and any, of the wave's queries see; of the workgroup's
  int wg_least, tiles;
  bool any;
  template <int ROWS>
  __device__ __forceinline__ static QueryBlock of(const SeqArgs& a, int number, int blocks, int wave, int lane) {
    QueryBlock b;
    const Dealt d = dealt(a, number, a.heads, blocks * a.parts);
    b.head = d.head;
    b.kv = b.head / (a.heads / a.kv_heads);
    b.s = sequence_of(a, d.sequence);
    b.row0 = (blocks - 1 - d.block / a.parts) * 32 * ROWS;
    b.part = d.block % a.parts;
    b.any = b.row0 < b.s.nq;
    if (!b.any) return b;
    const int last = b.s.nq - 1, first = min(b.row0 + wave * 32, last);
    b.row = b.row0 + wave * 32 + lane % 32;
    b.seen = keys_seen(a, b.s, min(b.row, last));
    b.wave_least = keys_seen(a, b.s, first);  // (rows ascend, and so does what they see)
    b.wave_most = keys_seen(a, b.s, min(first + 31, last));
    b.wg_least = keys_seen(a, b.s, b.row0);
    b.tiles = (keys_seen(a, b.s, min(b.row0 + 32 * ROWS - 1, last)) + 63) / 64;
    return b;
  }
  // the lane's part of a row of queries, outputs or their gradients
  __device__ __forceinline__ const uint16_t* at(const SeqRows& t, int lane) const {
    return t.p + head * t.sh + (int64_t)(s.q0 + min(row, s.nq - 1)) * t.st + 8 * (lane / 32);
  }
};

// Steps of tiles through three buffers: while a step's tiles are worked on, the next one's go from registers to LDS and the loads of
// those behind them are on their way.  Of a wave's tiles, `lead` are taken one by one, then `full` as a pipeline over their halves, then the
// rest one by one.  The pipeline: every stretch of vector arithmetic, on the logits of one half, has independent products beside it,
// those of the next half and the second products of the one before, and a stretch's first operands are read in the stretch before.  (Read
// where they are used, by eight waves that a barrier keeps in step, they had the matrix pipe wait for 0.35 us twice a tile.)
//   first(tile):         first products of its first half (a tile is where it begins, from this wave's place in the first buffer)
//   front(tile, before): arithmetic of the first half; first products of the second, second products of the second half of the tile before
//   back(tile, next):    arithmetic of the second half; second products of the first, first products of the first half of the next tile
//   last(tile):          second products of the second half
//   whole(step, tile, buffer): one tile by itself
template <int SPLIT>
using Buffers = char[3][SPLIT][2][kTileBytes];  // [buffer][tile][the two tensors]
template <int SPLIT, typename Fetch, typename Put, typename First, typename Front, typename Back, typename Last, typename Whole>
__device__ __forceinline__ void over_tiles(int steps, int lead, int full, Fetch fetch, Put put, First first, Front front, Back back, Last last, Whole whole) {
  using std::false_type;
  using std::true_type;
  constexpr int kStep = SPLIT * 2 * kTileBytes;  // of a buffer
  if (steps == 0) return;
  auto after = [](int at) { return at == 2 ? 0 : at + 1; };
  int n = 0, buf = (3 - lead % 3) % 3;  // (the pipeline begins in the first buffer)
  fetch(0);
  put(0, buf);
  __syncthreads();
  if (steps > 1) fetch(1);
  auto advance = [&](int at) {
    if (n + 1 < steps) put(n + 1, after(at));
    __syncthreads();
    if (n + 2 < steps) fetch(n + 2);
  };
  for (; n < lead; ++n, buf = after(buf)) {
    advance(buf);
    whole(n, buf * kStep, buf);
  }
  if (full > 0) {
    first(0);
    front(0, 0, false_type{});
    auto step = [&](auto at_) {  // (three steps a round: the buffers' addresses are constants)
      constexpr int kAt = decltype(at_)::value, kNext = kAt == 2 ? 0 : kAt + 1;
      buf = kAt;
      advance(kAt);
      if (n + 1 >= lead + full) return false;
      ++n;
      back(kAt * kStep, kNext * kStep, true_type{});
      front(kNext * kStep, kAt * kStep, true_type{});
      return true;
    };
    while (step(std::integral_constant<int, 0>{}) && step(std::integral_constant<int, 1>{}) && step(std::integral_constant<int, 2>{})) {
    }
    back(buf * kStep, 0, false_type{});
    last(buf * kStep);
    buf = after(buf);
    ++n;
  }
  for (; n < steps; ++n, buf = after(buf)) {
    advance(buf);
    whole(n, buf * kStep, buf);
  }
}

// ... of the keys and values that a block of queries sees; the tiles that the mask cuts for some of the wave's queries come last.
// whole(t, tile, dirty); dirty: keys (WATCH = 0) or values (1) of a tile that the mask cuts are not finite.
template <int WAVES, int SPLIT, int WATCH, typename First, typename Front, typename Back, typename Last, typename Whole>
__device__ __forceinline__ void over_keys(const SeqArgs& a, const QueryBlock& b, int split, Buffers<SPLIT>& lds, int (&dirty)[3][SPLIT], First first,
                                          Front front, Back back, Last last, Whole whole) {
  const uint16_t* kb = a.k.p + b.kv * a.k.sh + b.s.k0 * a.k.st;
  const uint16_t* vb = a.v.p + b.kv * a.v.sh + b.s.k0 * a.v.st;
  Stage<64 * WAVES, SPLIT> sk, sv;
  if (threadIdx.x < 3 * SPLIT) (&dirty[0][0])[threadIdx.x] = 0;
  __syncthreads();
  const int step = SPLIT * a.parts, from = SPLIT * b.part;  // this workgroup's tiles: step n + from + 0 .. SPLIT - 1
  over_tiles<SPLIT>(
      max(0, b.tiles - from + step - 1) / step, 0, max(0, b.wave_least / 64 - (from + split) + step - 1) / step,
      [&](int n) {
        sk.load(kb, a.k.st, 64 * (step * n + from), b.s.nk);
        sv.load(vb, a.v.st, 64 * (step * n + from), b.s.nk);
      },
      [&](int n, int buf) {
        sk.store(lds[buf][0][0]);
        sv.store(lds[buf][0][1]);
#pragma unroll
        for (int j = 0; j < SPLIT; ++j)
          if (64 * (step * n + from + j + 1) > b.wg_least && __any((WATCH ? sv : sk).any_not_finite(j))) dirty[buf][j] = n + 1;
      },
      first, front, back, last,
      [&](int n, int tile, int buf) {
        const int t = step * n + from + split;
        if (64 * t < b.wave_most) whole(t, tile, dirty[buf][split] == n + 1);
      });
}

// Where the waves that share columns join: the others' accumulators in LDS, behind the tiles' last use, added one after the other.
struct Share {
  float acc[32][64];  // [register][lane]
  __device__ __forceinline__ void put(const f32x16* x, int lane) {
#pragma unroll
    for (int i = 0; i < 32; ++i) acc[i][lane] = x[i / 16][i % 16];
  }
  __device__ __forceinline__ void add_to(f32x16* x, int lane, float own, float others) const {
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i / 16][i % 16] = x[i / 16][i % 16] * own + acc[i][lane] * others;
  }
};

__device__ __forceinline__ void write_columns(uint16_t* dst, const f32x16* x, float f, int h) {
#pragma unroll
  for (int cb = 0; cb < 2; ++cb)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x2 w = {pack2(x[cb][4 * i] * f, x[cb][4 * i + 1] * f), pack2(x[cb][4 * i + 2] * f, x[cb][4 * i + 3] * f)};
      *reinterpret_cast<u32x2*>(dst + 32 * cb + 8 * i + 4 * h) = w;
    }
}

// ... and a workgroup's share of them in fp32, [part][head][row][64].
__device__ __forceinline__ void write_part(float* parts, int part, int64_t row, int64_t rows, const f32x16* x, int h) {
  float* dst = parts + (part * rows + row) * kD;
#pragma unroll
  for (int cb = 0; cb < 2; ++cb)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<f32x4*>(dst + 32 * cb + 8 * i + 4 * h) = f32x4{x[cb][4 * i], x[cb][4 * i + 1], x[cb][4 * i + 2], x[cb][4 * i + 3]};
}

template <int ROWS, int SPLIT>
__global__ __launch_bounds__(64 * ROWS * SPLIT, ROWS * SPLIT == 4 ? 3 : 2) void seq_attend_kernel(SeqArgs a, int blocks) {
  constexpr int kWaves = ROWS * SPLIT;
  __shared__ __align__(16) Buffers<SPLIT> lds;
  __shared__ int dirty[3][SPLIT];  // step + 1 with a cut tile that has values that are not finite
  const int lane = threadIdx.x % 64, h = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), split = wave / ROWS;
  const QueryBlock b = QueryBlock::of<ROWS>(a, blockIdx.x, blocks, wave % ROWS, lane);
  if (!b.any) return;
  u32x4 qf[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) qf[c] = *reinterpret_cast<const u32x4*>(b.at(a.q, lane) + 16 * c);
  const Reader rd(lds[0][split][0], lane);
  const float c2 = a.scale * kLog2e;
  f32x16 o[2] = {};
  float sum = 0.0f, ref = -kInf;  // ref in powers of two; -inf: no finite logit yet

  auto logits = [&](int kt, int kh) {
    f32x16 z = {};
#pragma unroll
    for (int c = 0; c < 4; ++c) z = mfma(rd.along(kt, kh, c), qf[c], z);
    return z;
  };
  auto probabilities = [&](f32x16& x) {
    const float off = ref == -kInf ? 0.0f : ref;
    float p0 = 0.0f, p1 = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      x[i] = exp2_(x[i] * c2 - off);
      x[i + 1] = exp2_(x[i + 1] * c2 - off);
      p0 += x[i];
      p1 += x[i + 1];
    }
    return p0 + p1;
  };
  // Where a lane's sum has passed its bound, or there is no reference yet: again with the reference moved.  x: the logits.
  auto again = [&](f32x16& x, bool move) {
    float top = x[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
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
    return probabilities(x);
  };
  auto product = [&](int vt, int kh, const u32x4* p, auto clean_) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int cb = 0; cb < 2; ++cb) {
        u32x4 vf = rd.across(vt, kh, cb, ks);
        if (decltype(clean_)::value) vf = cleaned(vf);
        o[cb] = mfma(vf, p[ks], o[cb]);
      }
  };

  f32x16 x;         // logits of the half whose turn it is
  u32x4 p[2];      // probabilities of the one before
  u32x4 early[4];  // operands read a stretch ahead: keys of a second half, then values of a first half
  auto settle = [&](int tile, int half, float part) {  // the half's probabilities, once its sum is known to be in bounds
    const bool move = !(part <= kMaxPart) || ref == -kInf;
    if (__any(move)) {
      x = logits(tile, half);
      part = again(x, move);
    }
    sum += part;
    p[0] = pack8(x, 0);
    p[1] = pack8(x, 1);
  };
  float off, part0, part1;
  auto begin = [&]() {
    off = ref == -kInf ? 0.0f : ref;
    part0 = part1 = 0.0f;
  };
  auto two = [&](int i) {  // probabilities 2 i and 2 i + 1
    x[2 * i] = exp2_(x[2 * i] * c2 - off);
    x[2 * i + 1] = exp2_(x[2 * i + 1] * c2 - off);
    part0 += x[2 * i];
    part1 += x[2 * i + 1];
  };
  over_keys<kWaves, SPLIT, 1>(
      a, b, split, lds, dirty,
      [&](int tile) {
        x = logits(tile, 0);
#pragma unroll
        for (int c = 0; c < 4; ++c) early[c] = rd.along(tile, 1, c);
      },
      [&](int tile, int before, auto any_) {
        constexpr bool kAny = decltype(any_)::value;
        f32x16 z = {};
        u32x4 f[4];
        begin();
        in_order<8>(
            [&](int i) {
              if (i < 4) z = mfma(early[i], qf[i], z);
              else if (kAny) o[i % 2] = mfma(f[i - 4], p[i / 2 - 2], o[i % 2]);
            },
            [&](int i) {
              if (i >= 4) early[i - 4] = rd.across(tile + kTileBytes, 0, i % 2, i / 2 - 2);
              else if (kAny) f[i] = rd.across(before + kTileBytes, 1, i % 2, i / 2);
            },
            two);
        settle(tile, 0, part0 + part1);
        x = z;
      },
      [&](int tile, int next, auto more_) {
        constexpr bool kMore = decltype(more_)::value;
        f32x16 z = {};
        u32x4 f[4];
        begin();
        in_order<8>(
            [&](int i) {
              if (i < 4) o[i % 2] = mfma(early[i], p[i / 2], o[i % 2]);
              else if (kMore) z = mfma(f[i - 4], qf[i - 4], z);
            },
            [&](int i) {
              if (kMore && i < 2) {
                f[2 * i] = rd.along(next, 0, 2 * i);
                f[2 * i + 1] = rd.along(next, 0, 2 * i + 1);
              }
              if (kMore && i >= 4) early[i - 4] = rd.along(next, 1, i - 4);
            },
            two);
        settle(tile, 1, part0 + part1);
        if (kMore) x = z;
      },
      [&](int tile) { product(tile + kTileBytes, 1, p, std::false_type{}); },
      [&](int t, int tile, bool clean_up) {
#pragma unroll
        for (int kh = 0; kh < 2; ++kh) {
          auto masked = [&]() {
            f32x16 z = logits(tile, kh);
            const int left = b.seen - (64 * t + 32 * kh + 4 * h);
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] = 8 * (i / 4) + i % 4 < left ? z[i] : -kInf;
            return z;
          };
          x = masked();
          float part = probabilities(x);
          const bool move = !(part <= kMaxPart) || ref == -kInf;
          if (__any(move)) {
            x = masked();
            part = again(x, move);
          }
          sum += part;
          p[0] = pack8(x, 0);
          p[1] = pack8(x, 1);
          if (clean_up) product(tile + kTileBytes, kh, p, std::true_type{});
          else product(tile + kTileBytes, kh, p, std::false_type{});
        }
        if (clean_up)
          add_not_finite(a.v.p + b.kv * a.v.sh + b.s.k0 * a.v.st, a.v.st, 64 * t, min(64 * t + 64, b.wave_most), lane, [&](int r) { return r < b.seen; }, o);
      });
  if constexpr (SPLIT > 1) {
    Share* shares = reinterpret_cast<Share*>(lds);
    static_assert(sizeof(Share) * ROWS * (SPLIT - 1) <= sizeof(lds));
    __shared__ float joint[2][kWaves][64];
    __syncthreads();  // (the tiles' last use)
    if (split > 0) {
      shares[wave - ROWS].put(o, lane);
      joint[0][wave][lane] = ref;
      joint[1][wave][lane] = sum;
    }
    __syncthreads();
    if (split > 0) return;
    for (int w = wave + ROWS; w < kWaves; w += ROWS) {
      const float other = joint[0][w][lane], top = fmaxf(ref, other), off = top == -kInf ? 0.0f : top;
      const float f = exp2_(ref - off), g = exp2_(other - off);
      ref = top;
      sum = sum * f + joint[1][w][lane] * g;
      shares[w - ROWS].add_to(o, lane, f, g);
    }
  }
  const float total = half_sum(sum);
  if (b.row >= b.s.nq) return;
  if (a.parts > 1) {
    const int64_t rows = (int64_t)a.heads * a.rows_q, row = (int64_t)b.head * a.rows_q + b.s.q0 + b.row;
    write_part(a.part, b.part, row, rows, o, h);
    if (h == 0) *reinterpret_cast<f32x2*>(a.part_sums + 2 * (b.part * rows + row)) = f32x2{ref, total};
    return;
  }
  const bool empty = b.seen == 0;
  write_columns(const_cast<uint16_t*>(b.at(a.out, 0)), o, empty ? 0.0f : 1.0f / total, h);
  if (h == 0) a.lse[(int64_t)b.head * a.rows_q + b.s.q0 + b.row] = empty ? -kInf : ((ref == -kInf ? 0.0f : ref) + log2f(total)) * kLn2;
}

// Workgroup `number` of those that own ROWS x 32 queries, a wave to every 32: g = sum of dS K with dS = P (dout V^T - delta).
template <int ROWS>
__device__ __forceinline__ void grad_q(const SeqArgs& a, int number, int blocks, Buffers<1>& lds) {
  __shared__ int dirty[3][1];
  const int lane = threadIdx.x % 64, h = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const QueryBlock b = QueryBlock::of<ROWS>(a, number, blocks, wave, lane);
  if (!b.any) return;
  u32x4 qf[4], df[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    qf[c] = *reinterpret_cast<const u32x4*>(b.at(a.q, lane) + 16 * c);
    df[c] = *reinterpret_cast<const u32x4*>(b.at(a.dout, lane) + 16 * c);
  }
  const int64_t at = (int64_t)b.head * a.rows_q + b.s.q0 + min(b.row, b.s.nq - 1);
  const float lse2 = a.lse[at] * kLog2e, delta = a.delta[at];
  const Reader rd(lds[0][0][0], lane);
  const float c2 = a.scale * kLog2e;
  f32x16 g[2] = {};
  bool left_out = false;

  f32x16 x, y;    // logits and dout v^T - delta of the half whose turn it is
  u32x4 ds[2];    // of the one before
  const f32x16 less_delta = f32x16{} - delta;  // dout v^T - delta: the product begins with it
  auto logits = [&](int tile, int kh, f32x16& u, f32x16& w) {
    u = f32x16{};
    w = less_delta;
#pragma unroll
    for (int c = 0; c < 4; ++c) u = mfma(rd.along(tile, kh, c), qf[c], u);
#pragma unroll
    for (int c = 0; c < 4; ++c) w = mfma(rd.along(tile + kTileBytes, kh, c), df[c], w);
  };
  auto product = [&](int kt, int kh, auto clean_) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int cb = 0; cb < 2; ++cb) {
        u32x4 kf = rd.across(kt, kh, cb, ks);
        if (decltype(clean_)::value) kf = cleaned(kf);
        g[cb] = mfma(kf, ds[ks], g[cb]);
      }
  };
  u32x4 early[4];  // operands read a stretch ahead: keys of a second half along rows, then of a first half across them
  uint32_t packed[8];
  auto share = [&](int i) {  // the i-th of 12 shares of the arithmetic on 16 pairs
#pragma unroll
    for (int e = 16 * i / 12; e < 16 * (i + 1) / 12; ++e) {
      x[e] = exp2_(x[e] * c2 - lse2) * y[e];
      if (e % 2) packed[e / 2] = pack2(x[e - 1], x[e]);
    }
  };
  auto packed_to_ds = [&]() {
    ds[0] = (u32x4{packed[0], packed[1], packed[2], packed[3]});
    ds[1] = (u32x4{packed[4], packed[5], packed[6], packed[7]});
  };
  over_keys<ROWS, 1, 0>(
      a, b, 0, lds, dirty,
      [&](int tile) {
        logits(tile, 0, x, y);
#pragma unroll
        for (int c = 0; c < 4; ++c) early[c] = rd.along(tile, 1, c);
      },
      [&](int tile, int before, auto any_) {
        constexpr bool kAny = decltype(any_)::value;
        f32x16 u = {}, w = less_delta;
        u32x4 f[4], e[4];
        in_order<12>(
            [&](int i) {
              if (i < 4) u = mfma(early[i], qf[i], u);
              else if (i < 8) w = mfma(f[i - 4], df[i - 4], w);
              else if (kAny) g[i % 2] = mfma(e[i - 8], ds[i / 2 - 4], g[i % 2]);
            },
            [&](int i) {
              if (i < 2) {
                f[2 * i] = rd.along(tile + kTileBytes, 1, 2 * i);
                f[2 * i + 1] = rd.along(tile + kTileBytes, 1, 2 * i + 1);
              } else if (i < 6) {
                if (kAny) e[i - 2] = rd.across(before, 1, i % 2, i / 2 - 1);
              } else if (i < 10) {
                early[i - 6] = rd.across(tile, 0, i % 2, i / 2 - 3);
              }
            },
            share);
        packed_to_ds();
        x = u;
        y = w;
      },
      [&](int tile, int next, auto more_) {
        constexpr bool kMore = decltype(more_)::value;
        f32x16 u = {}, w = less_delta;
        u32x4 f[4], e[4];
        in_order<12>(
            [&](int i) {
              if (i < 4) g[i % 2] = mfma(early[i], ds[i / 2], g[i % 2]);
              else if (kMore && i < 8) u = mfma(f[i - 4], qf[i - 4], u);
              else if (kMore) w = mfma(e[i - 8], df[i - 8], w);
            },
            [&](int i) {
              if (!kMore) return;
              if (i < 2) {
                f[2 * i] = rd.along(next, 0, 2 * i);
                f[2 * i + 1] = rd.along(next, 0, 2 * i + 1);
              } else if (i < 4) {
                e[2 * i - 4] = rd.along(next + kTileBytes, 0, 2 * i - 4);
                e[2 * i - 3] = rd.along(next + kTileBytes, 0, 2 * i - 3);
              } else if (i >= 6 && i < 10) {
                early[i - 6] = rd.along(next, 1, i - 6);
              }
            },
            share);
        packed_to_ds();
        if (kMore) {
          x = u;
          y = w;
        }
      },
      [&](int tile) { product(tile, 1, std::false_type{}); },
      [&](int t, int tile, bool clean_up) {
        left_out |= clean_up;
#pragma unroll
        for (int kh = 0; kh < 2; ++kh) {
          logits(tile, kh, x, y);
          const int left = b.seen - (64 * t + 32 * kh + 4 * h);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            x[i] = exp2_(x[i] * c2 - lse2) * y[i];
            x[i] = 8 * (i / 4) + i % 4 < left ? x[i] : 0.0f;
          }
          ds[0] = pack8(x, 0);
          ds[1] = pack8(x, 1);
          if (clean_up) product(tile, kh, std::true_type{});
          else product(tile, kh, std::false_type{});
        }
      });
  if (left_out)
    add_not_finite(a.k.p + b.kv * a.k.sh + b.s.k0 * a.k.st, a.k.st, b.wave_least / 64 * 64, b.wave_most, lane, [&](int r) { return r < b.seen; }, g);
  if (b.row >= b.s.nq) return;
  if (a.parts > 1) write_part(a.part, b.part, (int64_t)b.head * a.rows_q + b.s.q0 + b.row, (int64_t)a.heads * a.rows_q, g, h);
  else write_columns(const_cast<uint16_t*>(b.at(a.dq, 0)), g, a.scale, h);
}

// ---- gradients of the keys and values -------------------------------------------------------------------------------

// Workgroup `number` of those that own KEYS x 32 keys of one key head of one sequence, a wave to every 32, over the queries of all
// heads that share it: the tiles that the mask cuts first, those of all heads, then the others.
template <int KEYS>
__device__ __forceinline__ void grad_kv(const SeqArgs& a, int number, int blocks, Buffers<1>& lds) {  // lds: queries and dout
  __shared__ __align__(16) float stats[3][2][64];  // [buffer][-lse / scale, -delta]: where the products begin
  __shared__ int dirty[3];
  const int lane = threadIdx.x % 64, h = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const Dealt d = dealt(a, number, a.kv_heads, blocks * a.parts);
  const int kv = d.head, part = d.block % a.parts;
  const Sequence s = sequence_of(a, d.sequence);
  const int key0 = d.block / a.parts * 32 * KEYS;
  if (key0 >= s.nk) return;
  const int rep = a.heads / a.kv_heads;
  // (columns behind the last key are copies of it that nobody writes)
  const int end = s.nk - 1, key = key0 + wave * 32 + lane % 32;
  u32x4 kf[4], vf[4];
  {
    const uint16_t* k = a.k.p + kv * a.k.sh + (int64_t)(s.k0 + min(key, end)) * a.k.st + 8 * h;
    const uint16_t* v = a.v.p + kv * a.v.sh + (int64_t)(s.k0 + min(key, end)) * a.v.st + 8 * h;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      kf[c] = *reinterpret_cast<const u32x4*>(k + 16 * c);
      vf[c] = *reinterpret_cast<const u32x4*>(v + 16 * c);
    }
  }
  const int from = first_query(a, s, min(key, end));  // queries that see the lane's key begin here
  const int wave_from = first_query(a, s, min(key0 + wave * 32, end));
  const int wg_from = first_query(a, s, key0), wg_all = first_query(a, s, min(key0 + 32 * KEYS - 1, end));
  const int first_tile = min(wg_from, s.nq) / 64, all_tile = min((wg_all + 63) / 64, (s.nq + 63) / 64), end_tile = (s.nq + 63) / 64;
  const int cut = max(0, all_tile - first_tile), uncut = max(0, end_tile - max(all_tile, first_tile));  // tiles of a head
  // this workgroup's of either kind: a.parts n + part
  const int lead = max(0, cut * rep - part + a.parts - 1) / a.parts, full = max(0, uncut * rep - part + a.parts - 1) / a.parts, steps = lead + full;
  struct Place {
    int head, row;  // row 0 of the tile; behind the last query where there is none
  };
  auto place = [&](int n) {
    const bool lead_part = n < lead;
    const int at = a.parts * (lead_part ? n : n - lead) + part, per_head = max(1, lead_part ? cut : uncut), i = at / per_head;
    return Place{kv * rep + min(i, rep - 1), i < rep ? 64 * ((lead_part ? first_tile : max(all_tile, first_tile)) + at % per_head) : s.nq};
  };

  const Reader rd(lds[0][0][0], lane);
  const float c2 = a.scale * kLog2e, per_scale = -1.0f / a.scale;
  f32x16 dk[2] = {}, dv[2] = {};
  bool left_out = false;
  Stage<64 * KEYS, 1> sq, sd;
  float st_l = 0.0f, st_d = 0.0f;
  if (threadIdx.x < 3) dirty[threadIdx.x] = 0;
  __syncthreads();

  f32x16 x, y;         // logits less lse (in units of the scale) and dout v^T - delta of the half whose turn it is
  u32x4 p[2], ds[2];   // of the one before
  u32x4 early[4];      // operands read a stretch ahead
  const uint32_t begins = (uint32_t)(size_t)(lds_char*)(const char*)stats[0][0] + 16 * h;
  constexpr int kStats = 2 * 64 * 4, kStep = 2 * kTileBytes;  // of a buffer
  auto quarter = [&](f32x16& z, int tile, int which, int half, int i) {  // rows 8 i + 4 h .. of where a product begins
    const f32x4 v = *(lds_f32x4*)(begins + tile / kStep * kStats + which * 256 + half * 128 + i * 32);
#pragma unroll
    for (int j = 0; j < 4; ++j) z[4 * i + j] = v[j];
  };
  uint32_t packed[2][8];
  auto share = [&](int e) {  // the arithmetic on the e-th pair
    x[e] = exp2_(x[e] * c2);
    y[e] *= x[e];
    if (e % 2) {
      packed[0][e / 2] = pack2(x[e - 1], x[e]);
      packed[1][e / 2] = pack2(y[e - 1], y[e]);
    }
  };
  auto packed_to_operands = [&]() {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      p[i] = u32x4{packed[0][4 * i], packed[0][4 * i + 1], packed[0][4 * i + 2], packed[0][4 * i + 3]};
      ds[i] = u32x4{packed[1][4 * i], packed[1][4 * i + 1], packed[1][4 * i + 2], packed[1][4 * i + 3]};
    }
  };
  // The i-th of 8 first products of a half (4 of the logits, 4 of dout v^T) and of 8 second ones, and their operands.
  auto first_operand = [&](int tile, int half, int i) { return rd.along(tile + (i < 4 ? 0 : kTileBytes), half, i % 4); };
  auto second_operand = [&](int tile, int half, int i) { return rd.across(tile + (i % 2 ? 0 : kTileBytes), half, i / 2 % 2, i / 4); };
  auto first_product = [&](int i, u32x4 f, f32x16& u, f32x16& w) {
    if (i < 4) u = mfma(f, kf[i], u);
    else w = mfma(f, vf[i - 4], w);
  };
  auto second_product = [&](int i, u32x4 f) {
    if (i % 2 == 0) dv[i / 2 % 2] = mfma(f, p[i / 4], dv[i / 2 % 2]);
    else dk[i / 2 % 2] = mfma(f, ds[i / 4], dk[i / 2 % 2]);
  };
  auto begin = [&](f32x16& z, int tile, int which, int half) {
#pragma unroll
    for (int i = 0; i < 4; ++i) quarter(z, tile, which, half, i);
  };
  f32x16 u, w;  // of the next half

  over_tiles<1>(
      steps, lead, full,
      [&](int n) {
        const Place at = place(n);
        sq.load(a.q.p + at.head * a.q.sh + s.q0 * a.q.st, a.q.st, at.row, s.nq);
        sd.load(a.dout.p + at.head * a.dout.sh + s.q0 * a.dout.st, a.dout.st, at.row, s.nq);
        if (threadIdx.x < 64) {
          const int i = at.row + lane;
          const int64_t in = (int64_t)at.head * a.rows_q + s.q0 + i;
          st_l = i < s.nq ? a.lse[in] * per_scale : -kInf;  // (rows behind the last query have no probability at all)
          st_d = i < s.nq ? -a.delta[in] : 0.0f;
        }
      },
      [&](int n, int buf) {
        sq.store(lds[buf][0][0]);
        sd.store(lds[buf][0][1]);
        if (threadIdx.x < 64) {
          stats[buf][0][lane] = st_l;
          stats[buf][1][lane] = st_d;
        }
        if (n < lead && __any(sq.any_not_finite(0) || sd.any_not_finite(0))) dirty[buf] = n + 1;
      },
      [&](int tile) {
        begin(x, tile, 0, 0);
        begin(y, tile, 1, 0);
#pragma unroll
        for (int i = 0; i < 8; ++i) first_product(i, first_operand(tile, 0, i), x, y);
        begin(u, tile, 0, 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) early[i] = first_operand(tile, 1, i);
      },
      [&](int tile, int before, auto any_) {
        constexpr bool kAny = decltype(any_)::value;
        u32x4 f[16];
        in_order<16>(
            [&](int i) {
              const u32x4 v = i < 4 ? early[i] : f[i];
              if (i < 8) first_product(i, v, u, w);
              else if (kAny) second_product(i - 8, v);
            },
            [&](int i) {
              if (i < 2) {
                quarter(w, tile, 1, 1, 2 * i);
                quarter(w, tile, 1, 1, 2 * i + 1);
              }
              if (i < 4) f[i + 4] = first_operand(tile, 1, i + 4);
              else if (i < 12 && kAny) f[i + 4] = second_operand(before, 1, i - 4);
              else if (i >= 12) early[i - 12] = second_operand(tile, 0, i - 12);
            },
            share);
        packed_to_operands();
        x = u;
        y = w;
      },
      [&](int tile, int next, auto more_) {
        constexpr bool kMore = decltype(more_)::value;
        u32x4 f[16];
        in_order<16>(
            [&](int i) {
              const u32x4 v = i < 4 ? early[i] : f[i];
              if (i < 8) second_product(i, v);
              else if (kMore) first_product(i - 8, v, u, w);
            },
            [&](int i) {
              if (i < 4) f[i + 4] = second_operand(tile, 0, i + 4);
              else if (i < 12 && kMore) f[i + 4] = first_operand(next, 0, i - 4);
              else if (kMore && i >= 12) early[i - 12] = first_operand(next, 1, i - 12);
              if (kMore && i >= 2 && i < 6) {
                quarter(u, next, 0, 0, i - 2);
                quarter(w, next, 1, 0, i - 2);
              }
            },
            share);
        packed_to_operands();
        if (kMore) {
          x = u;
          y = w;
          begin(u, next, 0, 1);
        }
      },
      [&](int tile) {
#pragma unroll
        for (int i = 0; i < 8; ++i) second_product(i, second_operand(tile, 1, i));
      },
      [&](int n, int tile, int buf) {
        const int row = place(n).row;
        if (row >= s.nq || row + 64 <= wave_from) return;
        const bool clean_up = dirty[buf] == n + 1;
        left_out |= clean_up;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          begin(x, tile, 0, half);
          begin(y, tile, 1, half);
#pragma unroll
          for (int i = 0; i < 8; ++i) first_product(i, first_operand(tile, half, i), x, y);
          const int least = from - (row + 32 * half + 4 * h), most = s.nq - (row + 32 * half + 4 * h);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const bool sees = 8 * (e / 4) + e % 4 >= least && 8 * (e / 4) + e % 4 < most;
            x[e] = exp2_(x[e] * c2);
            y[e] = sees ? x[e] * y[e] : 0.0f;
            x[e] = sees ? x[e] : 0.0f;
            if (e % 2) {
              packed[0][e / 2] = pack2(x[e - 1], x[e]);
              packed[1][e / 2] = pack2(y[e - 1], y[e]);
            }
          }
          packed_to_operands();
          if (clean_up) {
#pragma unroll
            for (int i = 0; i < 8; ++i) second_product(i, cleaned(second_operand(tile, half, i)));
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) second_product(i, second_operand(tile, half, i));
          }
        }
      });
  if (left_out) {
    for (int head = kv * rep; head < (kv + 1) * rep; ++head) {
      auto sees = [&](int r) { return r >= from; };
      const int to = min(s.nq, 64 * all_tile);
      add_not_finite(a.dout.p + head * a.dout.sh + s.q0 * a.dout.st, a.dout.st, wave_from / 64 * 64, to, lane, sees, dv);
      add_not_finite(a.q.p + head * a.q.sh + s.q0 * a.q.st, a.q.st, wave_from / 64 * 64, to, lane, sees, dk);
    }
  }
  if (key >= s.nk) return;
  if (a.parts > 1) {  // (dk, then dv)
    const int64_t rows = (int64_t)a.kv_heads * a.rows_k, row = (int64_t)kv * a.rows_k + s.k0 + key;
    write_part(a.part, part, row, rows, dk, h);
    write_part(a.part, a.parts + part, row, rows, dv, h);
    return;
  }
  write_columns(const_cast<uint16_t*>(a.dk.p) + kv * a.dk.sh + (int64_t)(s.k0 + key) * a.dk.st, dk, a.scale, h);
  write_columns(const_cast<uint16_t*>(a.dv.p) + kv * a.dv.sh + (int64_t)(s.k0 + key) * a.dv.st, dv, 1.0f, h);
}

// The gradients in one launch: the workgroups of the kind whose blocks take longer come first (k_first: the number of the first of the keys').
// One launch behind the other ended twice with compute units that wait for the last blocks: us in two launches and in one, the
// six-frame clip 620 and 578, of 12 heads 533 and 470, the eight frames 280 and 255, one frame 53 and 44.
template <int BLOCK>
__global__ __launch_bounds__(64 * BLOCK, 2) void seq_grad_kernel(SeqArgs k, SeqArgs q, int k_blocks, int q_blocks, int k_first, int k_workgroups) {
  __shared__ __align__(16) Buffers<1> lds;
  const int number = blockIdx.x - k_first;
  if (number >= 0 && number < k_workgroups) grad_kv<BLOCK>(k, number, k_blocks, lds);
  else grad_q<BLOCK>(q, k_first > 0 ? blockIdx.x : number - k_workgroups, q_blocks, lds);
}

// delta = sum of dout * out, which both need: 8 lanes a row, all rows of the tensors.
__global__ __launch_bounds__(256) void delta_kernel(SeqArgs a) {
  const int c = 8 * (threadIdx.x % 8);
  for (int64_t at = (int64_t)blockIdx.x * 32 + threadIdx.x / 8; at < (int64_t)a.heads * a.rows_q; at += (int64_t)gridDim.x * 32) {
    const int64_t head = at / a.rows_q, row = at % a.rows_q;
    const u32x4 x = *reinterpret_cast<const u32x4*>(a.dout.p + head * a.dout.sh + row * a.dout.st + c);
    const u32x4 y = *reinterpret_cast<const u32x4*>(a.out.p + head * a.out.sh + row * a.out.st + c);
    float dot = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      dot += __uint_as_float(x[e] << 16) * __uint_as_float(y[e] << 16);
      dot += __uint_as_float(x[e] & 0xffff0000u) * __uint_as_float(y[e] & 0xffff0000u);
    }
#pragma unroll
    for (int i = 1; i < 8; i *= 2) dot += __shfl_xor(dot, i);
    if (c == 0) a.delta[at] = dot;
  }
}

// ---- joining the parts of small launches ------------------------------------------------------------------------------

constexpr int kJoinRows = 32;  // rows of a workgroup; 8 lanes a row

// out and lse from the parts' accumulators, references and sums
__global__ __launch_bounds__(256) void join_out_kernel(SeqArgs a, int blocks) {
  const int unit = blockIdx.x / blocks, head = unit / a.sequences;
  const Sequence s = sequence_of(a, unit % a.sequences);
  const int i = blockIdx.x % blocks * kJoinRows + threadIdx.x / 8, c = 8 * (threadIdx.x % 8);
  if (i >= s.nq) return;
  const int64_t rows = (int64_t)a.heads * a.rows_q, row = (int64_t)head * a.rows_q + s.q0 + i;
  float x[8] = {}, ref = -kInf, sum = 0.0f;
  for (int p = 0; p < a.parts; ++p) {
    const f32x2 st = *reinterpret_cast<const f32x2*>(a.part_sums + 2 * (p * rows + row));
    const f32x4 lo = *reinterpret_cast<const f32x4*>(a.part + (p * rows + row) * kD + c), hi = *reinterpret_cast<const f32x4*>(a.part + (p * rows + row) * kD + c + 4);
    const float top = fmaxf(ref, st[0]), off = top == -kInf ? 0.0f : top, f = exp2_(ref - off), g = exp2_(st[0] - off);
    ref = top;
    sum = sum * f + st[1] * g;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = x[j] * f + (j < 4 ? lo[j % 4] : hi[j % 4]) * g;
  }
  const bool empty = keys_seen(a, s, i) == 0;
  const float r = empty ? 0.0f : 1.0f / sum;
  u32x4 w;
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = pack2(x[2 * j] * r, x[2 * j + 1] * r);
  *reinterpret_cast<u32x4*>(const_cast<uint16_t*>(a.out.p) + head * a.out.sh + (int64_t)(s.q0 + i) * a.out.st + c) = w;
  if (c == 0) a.lse[row] = empty ? -kInf : ((ref == -kInf ? 0.0f : ref) + log2f(sum)) * kLn2;
}

// A gradient from the parts' sums: of the queries (KEYS = false), or of the keys and, behind them, the values.
template <bool KEYS>
__device__ __forceinline__ void join_grad(const SeqArgs& a, int number, int blocks) {
  const int heads = KEYS ? a.kv_heads : a.heads, units = heads * a.sequences;
  const int which = number / (units * blocks), at = number % (units * blocks);
  const int unit = at / blocks, head = unit / a.sequences;
  const Sequence s = sequence_of(a, unit % a.sequences);
  const int i = at % blocks * kJoinRows + threadIdx.x / 8, c = 8 * (threadIdx.x % 8);
  if (i >= (KEYS ? s.nk : s.nq)) return;
  const int64_t in_tensor = (KEYS ? s.k0 : s.q0) + i, all = KEYS ? a.rows_k : a.rows_q, rows = heads * all, row = head * all + in_tensor;
  float x[8] = {};
  for (int p = 0; p < a.parts; ++p) {
    const float* from = a.part + ((which * a.parts + p) * rows + row) * kD + c;
    const f32x4 lo = *reinterpret_cast<const f32x4*>(from), hi = *reinterpret_cast<const f32x4*>(from + 4);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] += j < 4 ? lo[j % 4] : hi[j % 4];
  }
  const float f = which == 0 ? a.scale : 1.0f;
  u32x4 w;
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = pack2(x[2 * j] * f, x[2 * j + 1] * f);
  const SeqRows& t = !KEYS ? a.dq : (which == 0 ? a.dk : a.dv);
  *reinterpret_cast<u32x4*>(const_cast<uint16_t*>(t.p) + head * t.sh + in_tensor * t.st + c) = w;
}
__global__ __launch_bounds__(256) void join_grad_kernel(SeqArgs k, SeqArgs q, int k_blocks, int q_blocks, int k_workgroups) {
  const int number = blockIdx.x;
  if (number < k_workgroups) join_grad<true>(k, number, k_blocks);
  else join_grad<false>(q, number - k_workgroups, q_blocks);
}

long long grid_of(int longest, int rows, int heads, int sequences) { return ((long long)longest + rows - 1) / rows * heads * sequences; }

constexpr long long kMostWorkgroups = (1ll << 32) / 512 - 1;  // threads of a launch are counted in 32 bits

constexpr int kComputeUnits = 256, kMostParts = 8;
// (the offsets of the sequences are device data: how many blocks of 128 rows there are is only estimated)
long long blocks_of(const SeqArgs& a, long long rows, int heads) { return std::max<long long>({1, rows * heads / 128, (long long)heads * a.sequences}); }

// How the forward pass's blocks of 128 rows are worked on.  Four waves of 32 rows, two or three such workgroups to a compute unit, if there
// are blocks enough; else a second wave to every 32 rows, eight waves that fill a compute unit.  us with four and with eight waves,
// 16 heads: one frame of 1374 tokens (171 blocks) 24.0 and 21.2, 20 heads (214) 23.3 and 20.8, 24 heads (257) 32.8 and 39.4,
// two frames (343) 34 and 40.  Under a mask blocks differ in length and the second round is shorter: causal, 2000 tokens (250) 32.7 and
// 29.1, 3000 (375) 45.4 and 37.2.  Where even those leave compute units without work, several workgroups share the tiles of a block and a
// second launch joins them: 4000 causal tokens of one head 44.5 alone, 28.9 with 2, 20.3 with 4, 17.5 with 8, four single tokens over up to
// 4000 keys 45.7, 28.7, 20.3, 25.2; more of them than there are compute units gain nothing (one frame: 21.2 alone, 34.5 with 2).
// Under a mask and with many keys four waves and parts up to four workgroups to a compute unit even the blocks out better than eight
// waves: the six-frame clip of 5 heads (322 blocks) 97 with eight waves, 133 with four, 84 with those and 3 parts, 16000 causal tokens of 4
// heads (500 blocks) 177, 242 and, with 2 parts, 174.
struct Shape {
  bool split;
  int parts;
};
Shape shape_of(const SeqArgs& a) {
  const long long blocks = blocks_of(a, a.rows_q, a.heads), tiles = (a.longest_k + 63) / 64;
  const bool uneven = a.causal && tiles > 64;
  Shape s{!uneven && blocks <= (a.causal ? 400 : kComputeUnits), 1};
  if (s.split || uneven)
    s.parts = (int)std::max<long long>(1, std::min({(long long)kMostParts, kComputeUnits * (uneven ? 4 : 1) / blocks, tiles / 4}));
  return s;
}

// And the gradient's.  A block whose work is more than twice a place's share (two workgroups to a compute unit; under a mask blocks have half
// of what is counted here) is shared by workgroups, and a second launch joins what they leave: the key blocks of grouped heads above all.
// us alone and so: ragged sequences of 12 heads that share 4 keys' 126 and 56, 8000 causal tokens of such heads 665 and 390, 4000 causal tokens of
// one head 100 and 35.  More of them cost (one frame: 44 alone, 57 with blocks over one share in two).
// Eight waves read every tile once for 256 rows, which long sequences gain (six-frame clip: 590 with four, 578 with eight, 20 heads 810
// and 758, four sequences of 4000 490 and 451) and shorter ones lose by padding and unequal work (frames of 1374: 253 and 264; ragged, up to 2000: 120 and
// 139; a few thousand: the same).
struct GradShape {
  int block;  // waves of 32 rows to a workgroup
  int k_parts, q_parts;
  bool q_first;  // the queries' workgroups
};
GradShape grad_shape_of(const SeqArgs& a) {
  const long long k_tiles = (a.longest_k + 63) / 64, q_tiles = (a.longest_q + 63) / 64 * (long long)(a.heads / a.kv_heads);
  const double k_work = 8.0 * q_tiles, q_work = 6.0 * k_tiles;  // of a block: products of 32 x 32 per tile and wave, four of them the unit
  const double all = k_work * blocks_of(a, a.rows_k, a.kv_heads) + q_work * blocks_of(a, a.rows_q, a.heads);
  const double share = all / (2 * kComputeUnits) / (a.causal ? 2 : 1);
  // (an eighth is let go, so that blocks of just two shares are cut)
  const auto parts = [&](double work, long long tiles) {
    return (int)std::max<long long>(1, std::min({(long long)kMostParts, (long long)(1.125 * work / std::max(share, 1.0)), tiles / 4}));
  };
  GradShape s{4, parts(k_work, q_tiles), parts(q_work, k_tiles), false};
  s.q_first = q_work / s.q_parts > k_work / s.k_parts;
  if (std::min(a.rows_q, a.rows_k) / std::max(1, a.sequences) >= 3500) s.block = 8;
  return s;
}

}  // namespace

// Whether every launch of the forward pass and of the gradient has threads that can be counted: without sharing, and with the workgroups that share blocks
// and those that join them.
bool seq_attend_fits(const SeqArgs& a) {
  if (grid_of(a.longest_q, 128, a.heads, a.sequences) + grid_of(a.longest_k, 128, a.kv_heads, a.sequences) > kMostWorkgroups) return false;
  const auto queries = [&](int rows) { return grid_of(a.longest_q, rows, a.heads, a.sequences); };
  const auto keys = [&](int rows) { return grid_of(a.longest_k, rows, a.kv_heads, a.sequences); };
  const auto fits = [](long long workgroups, int threads) { return workgroups < (1ll << 32) / threads; };
  const Shape f = shape_of(a);
  const GradShape g = grad_shape_of(a);
  return fits(queries(128) * f.parts, f.split ? 512 : 256) && (f.parts == 1 || fits(queries(kJoinRows), 256)) &&
         fits(queries(32 * g.block) * g.q_parts + keys(32 * g.block) * g.k_parts, 64 * g.block) &&
         fits((g.q_parts > 1 ? queries(kJoinRows) : 0) + (g.k_parts > 1 ? 2 * keys(kJoinRows) : 0), 256);
}

int64_t seq_attend_workspace(const SeqArgs& a) {
  const int parts = shape_of(a).parts;
  return parts > 1 ? (int64_t)parts * a.heads * a.rows_q * (kD + 2) * (int64_t)sizeof(float) : 0;
}
int64_t seq_attend_grad_parts(const SeqArgs& a) {
  const GradShape s = grad_shape_of(a);
  return ((s.q_parts > 1 ? (int64_t)s.q_parts * a.heads * a.rows_q : 0) + (s.k_parts > 1 ? (int64_t)2 * s.k_parts * a.kv_heads * a.rows_k : 0)) * kD *
         (int64_t)sizeof(float);
}

hipError_t launch_seq_attend(const SeqArgs& args, hipStream_t stream) {
  SeqArgs a = args;
  const Shape s = shape_of(a);
  a.parts = s.parts;
  a.part_sums = a.part + (int64_t)s.parts * a.heads * a.rows_q * kD;
  const int blocks = (a.longest_q + 127) / 128, workgroups = (int)(grid_of(a.longest_q, 128, a.heads, a.sequences) * s.parts);
  if (workgroups == 0) return hipSuccess;
  if (s.split) seq_attend_kernel<4, 2><<<workgroups, 512, 0, stream>>>(a, blocks);
  else seq_attend_kernel<4, 1><<<workgroups, 256, 0, stream>>>(a, blocks);
  if (s.parts > 1) {
    const int joins = (a.longest_q + kJoinRows - 1) / kJoinRows;
    join_out_kernel<<<joins * a.heads * a.sequences, 256, 0, stream>>>(a, joins);
  }
  return hipGetLastError();
}

hipError_t launch_seq_attend_grad(const SeqArgs& args, hipStream_t stream) {
  const GradShape s = grad_shape_of(args);
  SeqArgs k = args, q = args;
  k.parts = s.k_parts;
  q.parts = s.q_parts;
  q.part += s.k_parts > 1 ? (int64_t)2 * s.k_parts * k.kv_heads * k.rows_k * kD : 0;
  const int rows = 32 * s.block, k_blocks = (k.longest_k + rows - 1) / rows, q_blocks = (q.longest_q + rows - 1) / rows;
  const int k_workgroups = k_blocks * k.kv_heads * k.sequences * k.parts, workgroups = k_workgroups + q_blocks * q.heads * q.sequences * q.parts;
  if (workgroups == 0) return hipSuccess;
  const int k_first = s.q_first ? workgroups - k_workgroups : 0;
  const long long delta = std::min(((long long)q.heads * q.rows_q + 31) / 32, kMostWorkgroups);
  if (delta > 0) delta_kernel<<<(int)delta, 256, 0, stream>>>(q);
  if (s.block == 4) seq_grad_kernel<4><<<workgroups, 256, 0, stream>>>(k, q, k_blocks, q_blocks, k_first, k_workgroups);
  else seq_grad_kernel<8><<<workgroups, 512, 0, stream>>>(k, q, k_blocks, q_blocks, k_first, k_workgroups);
  const int k_rows = k.parts > 1 ? (k.longest_k + kJoinRows - 1) / kJoinRows : 0, q_rows = q.parts > 1 ? (q.longest_q + kJoinRows - 1) / kJoinRows : 0;
  const int k_joins = 2 * k_rows * k.kv_heads * k.sequences, joins = k_joins + q_rows * q.heads * q.sequences;
  if (joins > 0) join_grad_kernel<<<joins, 256, 0, stream>>>(k, q, k_rows, q_rows, k_joins);
  return hipGetLastError();
}

}  // namespace xsv
