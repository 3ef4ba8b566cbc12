// Attention over a paged cache in 8 bits, all pages of a sequence or the ones that are chosen for each query and key head.
//
//   S = scale * k_scale * (q . code_k) over the tokens that a row sees,  lse = log sum exp(S),  out = exp(S - lse) (code_v * v_scale)
//
// Codes become bf16 as they are (e4m3 has 4 significant bits, bf16 has 8), one instruction for two; the page's scales are powers of two, so that
// multiplying logits and probabilities by them instead rounds nothing. (Products in 8 bits would spare the keys' conversions, with q as the sum of
// two codes; but those matrix instructions lose what lies 2^-11 below their largest product, also with scales for blocks: measured.) Probabilities
// are rounded to bf16 once, as the second product's operands.
//
// One pass over the pages with a reference logit per row and a sum; a workgroup's four waves take every fourth page and are joined in LDS, and where
// there are too few blocks of rows to fill the card, workgroups share a block's pages and a second launch joins them in their order. Few rows
// (decoding) are bounded by memory: 64 streams of 60 to 32768 tokens, 32 heads on 8, 79 us, 4.5 TB/s of codes. Many rows are bounded by the vector
// unit (below): a frame of 1374 over 5470 tokens, 16 heads, 46 us, 670 TFLOP/s.
#include <algorithm>
#include <type_traits>

#include "pages.h"

namespace xsv {
namespace {

constexpr int kWaves = 4;       // of a workgroup, or all that a compute unit holds
constexpr int kManyWaves = 16;
constexpr int kMostParts = 64;
// Pages that the waves of a workgroup share where every sequence has one block: their lengths are known on the device alone, so a long one is cut as
// if it were alone, and workgroups without a share end at once. 64 streams of 60 to 32768 tokens, 8 key heads, us: 32 pages 78, 48 77, 64 77, 80 77,
// 128 91, 256 91.
constexpr int kLongest = 64;
// Short caches of few blocks: one workgroup of 16 waves to a block instead of parts and their join, which is a launch more. us from Python, one
// workgroup and parts: 16 blocks over 512 to 4096 tokens 12 and 16, over 8192 20 and 16; 64 over 4096 13 and 16, over 8192 20 and 18; 256 over 4096
// 27 and 33 (over 8192 49 and 56, but there sequences of different lengths would leave compute units empty).
constexpr int kManyUnits = 256, kManyPages = 64;
// 64 rows to a wave, if that fills the card: two workgroups on each of 256 compute units. us, 64 rows and 32 (16 heads): 10992 rows over 16384 tokens
// 744 and 857, 2748 over 8192 107 and 122, 2048 behind 6144 of their own (512 blocks) 75 and 79; 1374 over 5470 (352 blocks) 51 and 46. Just above a
// full card they are even (2100 over 8192, 528 blocks: 106 and 102). Fewer blocks if all parts of their pages are long: 512 over 65536 tokens (4
// parts of 256 pages) 169 and 192, 128 over 131072 (16 of 128) 109 and 118, but 256 over 8192 (8 of 16) 40 and 32.
constexpr long long kFull = 512, kLongPart = 128;
// Short lists of many blocks: a wave to a block, without a list in LDS and without a join, if there are this many blocks for each of a block's
// entries (64 at most). us, a wave and a workgroup to a block, 16 heads on 8, rows that choose 4 pages (32 entries): 512 rows, 512 blocks, 14.5 and
// 12, 1024 rows 15 and 18, 2048 rows 19 and 29; 8 pages (64 entries): 1024 rows 38 and 30, 2048 rows 49 and 51; 256 streams, 32 heads on 8, 8 pages
// 30 and 37, 32 pages 102 and 99.
constexpr long long kSoloBlocks = 32;
constexpr int kListRows = 16;  // rows that share a list of chosen pages
// Probabilities are taken against a reference logit per row, which moves when the sum over what a lane has of a page passes this:
// probabilities above 1 are as exact as below.
constexpr float kMaxPart = 16777216.0f;
using f32x16 = __attribute__((ext_vector_type(16))) float;
using lds_byte = __attribute__((address_space(3))) const uint8_t;

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float off_of(float ref) { return ref == -kInf ? 0.0f : ref; }  // (nothing finite seen yet)

// Products of 16 or 32 columns (rows of queries): D = A B with A the keys, or the values' channels, and a lane's `quarter` its 16 (32: half its 32) lanes.
// A lane then has logits of one row: of tokens 16 quarter + e of the page with 16 columns, 32 (e / 16) + 16 quarter + e % 16 with 32, because
// the rows of A are dealt so that they are runs; and the packed probabilities already are the B operand of the second product.
template <int COLS>
struct Shape;

// Pages go through LDS. A lane's pieces are 64 bytes apart, a row of the page each, and the 16 lanes whose loads the memory path takes together would
// ask for eight lines; it then takes 30 cycles for a load of 1 KB that takes 16 in order. In order, each load brings 16 rows to LDS by itself,
// without registers in between, and the lanes read their pieces there. The four 16-byte pieces of a row are turned by an amount that goes by the row,
// so that the eight lanes that read together are in different banks: keys' rows by key_turn(row of 4, which 16 rows), values' by value_turn(row). (64
// streams 82 -> 79 us, a frame over chosen pages 121 -> 115.)
constexpr int kStagedBytes = 2 * kPageBytes;  // of a wave: keys and values of a page
__device__ __forceinline__ int key_turn(int row, int rows) { return row / 2 % 2 + 2 * (rows % 2); }
__device__ __forceinline__ int value_turn(int row) { return row / 2 % 4; }
__device__ __forceinline__ int turned(int piece, int by) { return (piece + by) % 4 * 16; }
// The 64 rows of a page, in four loads of 1 KB, to LDS at `to`; this lane's piece of 16 rows is `even` bytes behind them in the first and third, `odd`
// in the others.  (What is in LDS has been read: the wait.  The scalar operands may come from a vector instruction: the wait states.)
__device__ __forceinline__ void stage(const uint8_t* page, int even, int odd, uint32_t to) {
  asm volatile(
      "s_waitcnt lgkmcnt(0)\n\ts_mov_b32 m0, %0\n\ts_nop 4\n\t"
      "global_load_lds_dwordx4 %1, %3\n\t"
      "global_load_lds_dwordx4 %2, %3 offset:%4\n\t"
      "global_load_lds_dwordx4 %1, %3 offset:%5\n\t"
      "global_load_lds_dwordx4 %2, %3 offset:%6" ::"s"(to), "v"(even), "v"(odd), "s"(page), "i"(16 * kD), "i"(2 * 16 * kD), "i"(3 * 16 * kD) : "memory", "m0");
}
__device__ __forceinline__ void wait_for_all() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void wait_for_all_but_eight() { asm volatile("s_waitcnt vmcnt(8)" ::: "memory"); }
__device__ __forceinline__ void wait_for_all_but_four() { asm volatile("s_waitcnt vmcnt(4)" ::: "memory"); }

template <>
struct Shape<16> {
  using Acc = f32x4;
  __device__ static __forceinline__ Acc mfma(bf16x8 a, bf16x8 b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  // where in a page the lane's piece i of its four 16-byte pieces of keys, or of values, is: of block i of the product's rows
  __device__ static __forceinline__ int key_at(int col, int quarter, int i) { return (16 * (col / 4) + 4 * i + col % 4) * kD + 16 * quarter; }
  __device__ static __forceinline__ int value_at(int col, int quarter, int i) { return (16 * i + col) * kPage + 16 * quarter; }
  // the same pieces in a page that stage() has brought to LDS: `first` and constants
  __device__ static __forceinline__ int staged_key(int col, int quarter, int i) { return col / 4 * 1024 + col % 4 * 64 + turned(quarter, key_turn(col % 4, col / 4)) + 256 * i; }
  __device__ static __forceinline__ int staged_value(int col, int quarter, int i) { return col * 64 + turned(quarter, value_turn(col)) + 1024 * i; }
  __device__ static __forceinline__ int channel(int block, int quarter, int j) { return 16 * block + 4 * quarter + j; }
  __device__ static __forceinline__ float column_max(float x) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
  }
  __device__ static __forceinline__ float column_sum(float x) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(q[0]) + __uint_as_float(q[1]);
  }
};
template <>
struct Shape<32> {
  using Acc = f32x16;
  __device__ static __forceinline__ Acc mfma(bf16x8 a, bf16x8 b, Acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  // pieces 2 h and 2 h + 1 are of tokens 32 h ..: keys by steps of 16 channels of a lane's 32, values by blocks of channels
  __device__ static __forceinline__ int staged_key(int col, int quarter, int i) {
    return col / 4 % 2 * 1024 + (4 * (col / 8) + col % 4) * 64 + turned(2 * quarter + i % 2, key_turn(col % 4, col / 4 % 2)) + 2048 * (i / 2);
  }
  __device__ static __forceinline__ int staged_value(int col, int quarter, int i) { return col * 64 + turned(2 * (i / 2) + quarter, value_turn(col % 16)) + 2048 * (i % 2); }
  __device__ static __forceinline__ int channel(int block, int quarter, int j) { return 32 * block + 8 * (j / 4) + 4 * quarter + j % 4; }
  __device__ static __forceinline__ float column_max(float x) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  }
  __device__ static __forceinline__ float column_sum(float x) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
  }
};

// 8 codes as bf16, times a power of two
__device__ __forceinline__ bf16x8 view8(uint32_t a, uint32_t b, float times = 1.0f) {
  const bf16x2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, times, false), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, times, true);
  const bf16x2 r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, times, false), s = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, times, true);
  const u32x4 w = {__builtin_bit_cast(uint32_t, p), __builtin_bit_cast(uint32_t, q), __builtin_bit_cast(uint32_t, r), __builtin_bit_cast(uint32_t, s)};
  return __builtin_bit_cast(bf16x8, w);
}

// (A page that was never written may have any scale: 0 would leave nothing of its probabilities.)
__device__ __forceinline__ int exponent_of(float scale) { return min(max((int)((__float_as_uint(scale) >> 23) & 0xffu) - 127, -100), 120); }
// The values' scale 2^ev goes into a weight's exponent, and comes out of the sum again.  With less than this in it, weights of 2^(-126 - ev) of the reference
// would be lost from the sum although their logits are ordinary, as in pages whose values are all zeros (2^-100): such pages have this in the weights and
// the rest in the values.  What is lost then is below 2^-66 of the largest weight.
constexpr int kLeastExponent = -60;
constexpr float kLeastScale = 0x1p-60f;
__device__ __forceinline__ float rest_of(int ev) { return __int_as_float((127 + min(ev - kLeastExponent, 0)) << 23); }
// What logits of a page are multiplied by, never 0: masked ones are -inf.
__device__ __forceinline__ float factor_of(float c2, float scale) { return fmaxf(c2 * scale, 1.17549435e-38f); }
// The NaN codes of a dword, as bytes 0xff.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m |= ((w >> (8 * i)) & 0x7fu) == 0x7fu ? 0xffu << (8 * i) : 0u;
  return m;
}

// A block of up to COLS rows of a key head of a sequence.
struct Block {
  Held h;
  int s, kv;
  int64_t row0, rows;  // the first, among the `rows` of its sequence (chosen pages: of its queries)
  int least, pages;    // tokens that all rows see; pages that any row sees one of
  int part, used;      // this workgroup of those that share the pages
  int query0, queries; // chosen pages: the queries of the block
};

// Its row i (behind the last: a copy of it that nobody writes).
struct Row {
  int query, head;
  int seen;  // tokens
  bool real;
};
__device__ __forceinline__ Row row_of(const PagesArgs& a, const Block& b, int i) {
  const int rep = a.heads / a.kv_heads;
  const uint32_t row = (uint32_t)min(b.row0 + i, b.rows - 1);  // (below 2^32: blocks of a launch are fewer than 2^24)
  Row r;
  r.query = b.query0 + (int)(row / (uint32_t)rep);
  r.head = b.kv * rep + (int)(row % (uint32_t)rep);
  r.seen = tokens_seen(a, b.h, r.query);
  r.real = b.row0 + i < b.rows;
  return r;
}

// All pages: rows (query, head) COLS at a time. Chosen pages: `group` queries with their heads, or 16 heads of a query that has more. Sequences'
// blocks are counted from their ends, so that under a mask those that see the most come first, and those of a short sequence behind a long cache,
// which see as much, among them; up to 64 sequences go by what they see (sequences of 0 to 1374 rows over up to 5470 tokens 55 -> 47 us). Workgroups
// are dealt to the XCDs one by one; where eight divides the key heads, each XCD has its own, one after the other, whose pages are then in one L2, and
// all of whose blocks go through them at about the same time. A block's parts are far apart: side by side, with eight of them, those of short
// sequences, which have little or nothing to do, were dealt to the same compute units (64 streams 89 us, 77).
template <int COLS, bool CHOSEN>
__device__ __forceinline__ bool block_of(const PagesArgs& a, int number, int blocks, Block* b) {
  const int rep = a.heads / a.kv_heads;
  const int heads = a.kv_heads % 8 ? a.kv_heads : a.kv_heads / 8, at = a.kv_heads % 8 ? number : number / 8;
  const int sequences = a.ranked ? 1 : a.sequences, units = heads * sequences * blocks, unit = at % units;
  b->part = at / units;
  const int per = CHOSEN && rep > COLS ? (rep + COLS - 1) / COLS : 1;  // blocks of a query
  auto blocks_of = [&](const Held& h) { return CHOSEN ? (int)(((int64_t)h.n + a.group - 1) / a.group) * per : (int)(((int64_t)h.n * rep + COLS - 1) / COLS); };
  int back;  // blocks of the sequence behind this one
  if (a.kv_heads % 8) {
    b->kv = unit % heads;
    b->s = unit / heads % sequences;
    back = unit / heads / sequences;
  } else {
    b->s = unit % sequences;
    back = unit / sequences % blocks;
    b->kv = number % 8 * heads + unit / sequences / blocks;
  }
  if (a.ranked) {
    auto whole = [&](int row) { return CHOSEN ? (int64_t)(row / a.group) * per : (int64_t)row * rep / COLS; };
    if (!(a.sequences <= kRanked ? ranked_block(a, blocks_of, &back, &b->s, &b->h) : numbered_block(a, whole, per, &back, &b->s, &b->h))) return false;
  } else {
    b->h = held(a, b->s);
  }
  const int block = blocks_of(b->h) - 1 - back;
  if (block < 0) return false;
  b->query0 = CHOSEN ? block / per * a.group : 0;
  b->queries = CHOSEN ? min(a.group, b->h.n - b->query0) : b->h.n;
  b->row0 = (int64_t)(CHOSEN ? block % per : block) * COLS;
  b->rows = (int64_t)b->queries * rep;
  if (b->queries <= 0 || b->row0 >= b->rows) return false;
  b->least = row_of(a, *b, 0).seen;
  b->pages = (row_of(a, *b, COLS - 1).seen + kPage - 1) / kPage;
  b->used = CHOSEN ? a.parts : min(max((b->pages + a.chunk - 1) / a.chunk, 1), a.parts);
  return b->part < b->used;
}

// What 64 lanes know of the next 64 pages of a wave, one a lane.
struct Next {
  int page, ordinal;
  uint32_t rows;  // chosen pages: the rows that listed it
  float ks, vs;
  uint64_t mask;  // lanes that have one
};

// The distinct pages that the rows of a block list, in order, with the rows that list each: pages w0 .. w0 + kWindow - 1.
constexpr int kWindow = 2048;
struct Lists {
  uint32_t rows[kWindow];    // by page
  uint32_t found[kWindow];   // by place: page - w0, and rows in the upper half
  int counts[kWaves];
};
__device__ __forceinline__ int list_window(const PagesArgs& a, const Block& b, int w0, Lists& l) {
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, rep = a.heads / a.kv_heads, words = min(kWindow, b.pages - w0);
  for (int i = tid; i < words; i += 64 * kWaves) l.rows[i] = 0;
  __syncthreads();
  // (the lists of all queries at once: one after the other, each would wait for memory)
  const int entries = b.queries * a.count;  // (more than one query: at most 16 times what a table holds)
  for (int i = tid; i < entries; i += 64 * kWaves) {
    const int q = (int)((uint32_t)i / (uint32_t)a.count);
    const int j = a.chosen[((int64_t)(b.h.row0 + b.query0 + q) * a.kv_heads + b.kv) * a.count + (i - q * a.count)];
    const int end = (tokens_seen(a, b.h, b.query0 + q) + kPage - 1) / kPage;
    const uint32_t rows = rep >= kListRows ? 0xffffu : ((1u << rep) - 1u) << (q * rep);
    if (j >= w0 && j < end && j - w0 < words) atomicOr(&l.rows[j - w0], rows);
  }
  __syncthreads();
  constexpr int kEach = kWindow / (64 * kWaves);
  uint32_t mine[kEach];
  int n = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    mine[i] = tid * kEach + i < words ? l.rows[tid * kEach + i] : 0u;
    n += mine[i] != 0;
  }
  int upto = n;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int x = __shfl_up(upto, d);
    upto += lane >= d ? x : 0;
  }
  if (lane == 63) l.counts[wave] = upto;
  __syncthreads();
  int at = upto - n, total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    at += w < wave ? l.counts[w] : 0;
    total += l.counts[w];
  }
#pragma unroll
  for (int i = 0; i < kEach; ++i)
    if (mine[i]) l.found[at++] = (uint32_t)(tid * kEach + i) | mine[i] << 16;
  __syncthreads();
  return total;
}

// The waves' results, each [COLS][64] of `pitch` pieces, 16-byte pieces of row r in the order of their number xor r, put together: a block's, or this
// part of them.
template <int COLS, int WAVES>
__device__ __forceinline__ void leave(const PagesArgs& a, const Block& b, int thread, const f32x4* acc, int pitch, const float* refs, const float* sums) {
  // All rows at once, a thread some channels of one: 4 threads further on the next 4 if it has more than 4, so that 8 side by side read different banks.
  constexpr int kRowThreads = 64 * WAVES / COLS, kChannels = kD / kRowThreads, kWide = std::min(kChannels, 4);
  const int r = thread / kRowThreads, first = thread % kRowThreads;
  const Row to = row_of(a, b, r);
  if (!to.real) return;
  const int64_t row = b.h.row0 + to.query;
  float top = -kInf;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) top = fmaxf(top, refs[w * COLS + r]);
  const float off = off_of(top);
  float l = 0.0f, f[WAVES];
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    f[w] = exp2_(refs[w * COLS + r] - off);
    l += sums[w * COLS + r] * f[w];
  }
  const int64_t at = ((int64_t)b.part * a.heads + to.head) * a.rows + row;  // of the workspace
  const float whole_of = b.used > 1 ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
  for (int j = 0; j < kChannels / kWide; ++j) {
    const int c = kWide * (first + j * kRowThreads);
    float v[kWide] = {};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float* x = reinterpret_cast<const float*>(acc + w * pitch + r * (kD / 4) + ((c / 4) ^ (r % 16))) + c % 4;
#pragma unroll
      for (int i = 0; i < kWide; ++i) v[i] += x[i] * f[w];
    }
#pragma unroll
    for (int i = 0; i < kWide; ++i) v[i] *= whole_of;
    uint16_t* out = const_cast<uint16_t*>(a.out.p) + to.head * a.out.sh + row * a.out.st + c;
    if constexpr (kWide == 4) {
      if (b.used == 1) *reinterpret_cast<u32x2*>(out) = u32x2{pack2(v[0], v[1]), pack2(v[2], v[3])};
      else *reinterpret_cast<f32x4*>(a.part + at * kD + c) = f32x4{v[0], v[1], v[2], v[3]};
    } else {
      *out = (uint16_t)pack2(v[0], 0.0f);  // (16 waves: nobody shares a block)
    }
  }
  if (first == 0) {
    if (b.used == 1) a.lse[(int64_t)to.head * a.rows + row] = (off + log2f(l)) * kLn2;
    else *reinterpret_cast<f32x2*>(a.part_sums + 2 * at) = f32x2{top, l};
  }
}

struct Empty {};

// 16 rows of a key head at a time, by a workgroup or (SOLO) by each of its waves: single tokens, and chosen pages, where each row has its own and a
// page is worked on for all 16 once any has chosen it. Those are bounded by the vector unit, too (66 % of the cycles, and the matrix instructions
// that hold it up): a page is 64 conversions and 16 logits a lane whether one row has it or all. 1374 queries of 16 heads that choose 32 of 1024
// pages, 23 of them the same: 114 us.
template <bool CHOSEN, int WAVES, bool SOLO>
__global__ __launch_bounds__(64 * WAVES, CHOSEN ? 3 : 4) void pages_attend_kernel(PagesArgs a, int blocks) {
  constexpr int COLS = 16;
  using S = Shape<COLS>;
  constexpr bool kStaged = WAVES == kWaves;  // (the destination of such a load has 16 bits: 64 KB)
  union Share {  // of a wave: its page, later its results, 16-byte pieces of row r in the order of their number xor r
    uint8_t page[kStagedBytes];
    f32x4 acc[COLS][kD / 4];
  };
  __shared__ __align__(16) Share shares[WAVES];
  __shared__ float refs[WAVES][COLS], sums[WAVES][COLS];
  __shared__ std::conditional_t<CHOSEN && !SOLO, Lists, Empty> lists;
  const int lane = threadIdx.x % 64, col = lane % COLS, quarter = lane / COLS;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  Block b;
  if (!block_of<COLS, CHOSEN>(a, SOLO ? wave * gridDim.x + blockIdx.x : blockIdx.x, blocks, &b)) return;
  const Row own = row_of(a, b, col);
  const int32_t* table = a.table + (int64_t)b.s * a.width;

  bf16x8 qf[2];  // a lane has 16 channels, and of what it works out of a page, 16 tokens
  {
    const uint16_t* q = a.q.p + own.head * a.q.sh + (int64_t)(b.h.row0 + own.query) * a.q.st + 16 * quarter;
#pragma unroll
    for (int i = 0; i < 2; ++i) qf[i] = *reinterpret_cast<const bf16x8*>(q + 8 * i);
  }
  f32x4 o[4] = {};
  float ref = -kInf, sum = 0.0f;
  const float c2 = a.scale * kLog2e;

  auto look_up = [&](Next& n, bool some) {
    n.page = some ? table[n.ordinal] : -1;
    some = n.page >= 0 && n.page < a.pages;
    const int64_t unit = some ? (int64_t)n.page * a.kv_heads + b.kv : 0;
    n.ks = some ? a.k_scale[unit] : 0.0f;
    n.vs = some ? a.v_scale[unit] : 0.0f;
    n.mask = __ballot(some);
  };
  // Of the pages (or entries of the list) `from`, `from` + WAVES, .. below `end`.
  // Lists from their end: the pages that all rows have listed, the last ones for the most part, then come before those of single rows, and a row's first
  // page is more work.
  auto look = [&](int from, int begin, int end, int w0) {
    Next n;
    const int at = from + WAVES * lane;
    bool some = at < end;
    n.ordinal = at;
    n.rows = 0;
    if constexpr (CHOSEN && !SOLO) {
      const uint32_t entry = some ? lists.found[begin + end - 1 - at] : 0u;
      n.ordinal = w0 + (int)(entry & 0xffffu);
      n.rows = entry >> 16;
    }
    look_up(n, some);
    return n;
  };
  u32x4 kr[4], vr[4];
  [[maybe_unused]] const uint8_t* staged = shares[wave].page;
  [[maybe_unused]] const uint32_t staged_at = (uint32_t)(size_t)(lds_byte*)staged;
  // (what this lane brings: piece lane % 4 of row lane / 4 of 16, which is another one of the row's)
  [[maybe_unused]] const int key_from = lane / 4 * 64 + (lane - key_turn(lane / 4 % 4, 0)) % 4 * 16, value_from = lane / 4 * 64 + (lane + 4 - value_turn(lane / 4)) % 4 * 16;
  auto fetch_keys = [&](int page) {
    const uint8_t* p = a.k + ((size_t)page * a.kv_heads + b.kv) * kPageBytes;
    if constexpr (kStaged) {
      stage(p, key_from, key_from ^ 32, staged_at);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) kr[i] = *reinterpret_cast<const u32x4*>(p + S::key_at(col, quarter, i));
    }
  };
  f32x4 x[4];
  u32x4 pr[2];
  float part;  // sum of the lane's probabilities in a page
  auto fetch_values = [&](int page) {
    const uint8_t* p = a.v + ((size_t)page * a.kv_heads + b.kv) * kPageBytes;
    if constexpr (kStaged) {
      stage(p, value_from, value_from, staged_at + kPageBytes);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) vr[i] = *reinterpret_cast<const u32x4*>(p + S::value_at(col, quarter, i));
    }
  };
  // Staged pages: what is read has been fetched, and at most the last four loads are still on their way.
  auto take_keys = [&] {
    if constexpr (kStaged) {
      wait_for_all_but_four();
#pragma unroll
      for (int i = 0; i < 4; ++i) kr[i] = *reinterpret_cast<const u32x4*>(staged + S::staged_key(col, quarter, i));
    }
  };
  auto take_values = [&] {
    if constexpr (kStaged) {
      wait_for_all_but_four();
#pragma unroll
      for (int i = 0; i < 4; ++i) vr[i] = *reinterpret_cast<const u32x4*>(staged + kPageBytes + S::staged_value(col, quarter, i));
    }
  };
  auto first_products = [&] {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = f32x4{};
#pragma unroll
      for (int k = 0; k < 2; ++k) x[i] = S::mfma(view8(kr[i][2 * k], kr[i][2 * k + 1]), qf[k], x[i]);
    }
  };
  // The values' scale 2^ev, of tiny ones a part of it, goes into the exponent: what enters the second product is in the values' own units.
  auto weigh = [&](float cs, int ev, bool mine) {
    const float off = off_of(ref) - (float)ev;
    float one = 0.0f, other = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
      const float p = exp2_(x[e / 4][e % 4] * cs - off), q = exp2_(x[e / 4][e % 4 + 1] * cs - off);
      one += p;
      other += q;
      pr[e / 8][e % 8 / 2] = pack2(p, q);
    }
    part = (one + other) * __int_as_float((127 - ev) << 23);
    if (CHOSEN) {
      if (!mine) part = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) pr[i / 4][i % 4] = mine ? pr[i / 4][i % 4] : 0u;
    }
  };
  auto second_products = [&](float rest) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int k = 0; k < 2; ++k)
        o[i] = S::mfma(view8(vr[i][2 * k], vr[i][2 * k + 1], rest), __builtin_bit_cast(bf16x8, pr[k]), o[i]);
  };
  // A page with all that may happen: rows that do not see some of it, references that move, values that are NaN.
  auto whole = [&](int ordinal, uint32_t rows, float ks, float vs, int next_page) {
    const bool mine = !CHOSEN || (rows >> col & 1);
    const int left = mine ? own.seen - ordinal * kPage - 16 * quarter : -kPage;  // of the tokens from the lane's first on
    const float cs = factor_of(c2, ks);
    if constexpr (kStaged) wait_for_all();
    take_keys();
    first_products();
    fetch_keys(next_page);
    take_values();
    float m = -kInf;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float y = e < left ? x[e / 4][e % 4] : -kInf;
      x[e / 4][e % 4] = y;
      m = fmaxf(m, y);
    }
    m = S::column_max(m) * cs;
    const float to = fmaxf(m, ref), f = ref == -kInf || to == ref ? 1.0f : exp2_(ref - to);
    ref = to;
    sum *= f;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] *= f;
    const int ev = exponent_of(vs);
    weigh(cs, max(ev, kLeastExponent), mine);
    sum += part;
    if (vs < 0.0f) {
      // 0 times NaN is NaN: values that are NaN are taken out of the product, and reach the rows that see their tokens by one of their own
      f32x4 count[4] = {};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u32x4 nan;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          nan[j] = nan_bytes(vr[i][j]);
          vr[i][j] &= ~nan[j];
          nan[j] &= 0x38383838u;  // 1
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          u32x4 sees;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int e = 8 * k + 2 * j;
            sees[j] = (e < left ? 0x3f80u : 0u) | (e + 1 < left ? 0x3f800000u : 0u);
          }
          count[i] = S::mfma(view8(nan[2 * k], nan[2 * k + 1]), __builtin_bit_cast(bf16x8, sees), count[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[i][j] = count[i][j] > 0.0f ? __builtin_nanf("") : o[i][j];
    }
    second_products(rest_of(ev));
  };
  // Pages one after the other.  The inner loop has those that need nothing but the arithmetic: the accumulators stay where they are (changed on a way of
  // its own inside the loop, they were copied on the others too, in every page).
  auto pass = [&](Next& n) __attribute__((always_inline)) {
    uint64_t mask = n.mask;
    if (!mask) return;
    if constexpr (kStaged) wait_for_all();  // (the last page's keys, fetched again)
    int i = __builtin_ctzll(mask), page = __builtin_amdgcn_readlane(n.page, i);
    fetch_keys(page);
    asm volatile("" : "+v"(n.ks), "+v"(n.vs));  // (what look() loads is there: nothing waits for it, and so for the pages, in the loop)
    while (true) {
      int ordinal;
      uint32_t rows;
      float ks, vs;
      bool fetched = true, done = false;  // `kr` has this page's keys; the last page is behind
      int next, next_page;
      while (true) {
        ordinal = __builtin_amdgcn_readlane(n.ordinal, i);
        rows = CHOSEN ? __builtin_amdgcn_readlane(n.rows, i) : 0u;
        ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(n.ks), i));
        vs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(n.vs), i));
        mask &= mask - 1;
        next = mask ? __builtin_ctzll(mask) : i;  // (the last one's keys are fetched again)
        next_page = __builtin_amdgcn_readlane(n.page, next);
        fetch_values(page);
        if ((ordinal + 1) * kPage > b.least || vs < kLeastScale) break;  // some row does not see some of its tokens, or values that are NaN or tiny
        const bool mine = !CHOSEN || (rows >> col & 1);
        if (__any(mine && ref == -kInf)) break;  // a row's first page
        take_keys();
        first_products();
        __builtin_amdgcn_sched_barrier(0);
        fetch_keys(next_page);
        weigh(factor_of(c2, ks), exponent_of(vs), mine);
        fetched = false;
        if (__any(part > kMaxPart)) break;
        __builtin_amdgcn_sched_barrier(0);
        sum += part;
        take_values();
        second_products(1.0f);
        done = !mask;
        if (done) break;
        i = next;
        page = next_page;
        fetched = true;
      }
      if (done) break;
      if (!fetched) {
        if constexpr (kStaged) wait_for_all();  // (what is on its way there is not this page's)
        fetch_keys(page);
      }
      whole(ordinal, rows, ks, vs, next_page);
      if (!mask) break;
      i = next;
      page = next_page;
    }
  };
  [[maybe_unused]] auto over = [&](int begin, int end, int w0) {
    for (int from = begin + wave; from < end; from += WAVES * 64) {
      Next n = look(from, begin, end, w0);
      pass(n);
    }
  };
  if constexpr (SOLO) {
    // the lists of all queries, an entry a lane; of those of a page the first has them all
    const int rep = a.heads / a.kv_heads, q = min((int)((uint32_t)lane / (uint32_t)a.count), b.queries - 1);
    const bool some = lane < b.queries * a.count;
    Next n;
    n.ordinal = some ? a.chosen[((int64_t)(b.h.row0 + b.query0 + q) * a.kv_heads + b.kv) * a.count + (lane - q * a.count)] : -1;
    n.rows = 0;
    const int end = (tokens_seen(a, b.h, b.query0 + q) + kPage - 1) / kPage;
    const uint32_t bits = rep >= kListRows ? 0xffffu : ((1u << rep) - 1u) << (q * rep);
    for (uint64_t left = __ballot(n.ordinal >= 0 && n.ordinal < end); left;) {
      const int i = __builtin_ctzll(left), page = __builtin_amdgcn_readlane(n.ordinal, i);
      const uint64_t same = left & __ballot(n.ordinal == page);
      uint32_t rows = 0;
      for (uint64_t those = same; those; those &= those - 1) rows |= __builtin_amdgcn_readlane(bits, __builtin_ctzll(those));
      n.rows = lane == i ? rows : n.rows;
      left &= ~same;
    }
    look_up(n, n.rows != 0);
    pass(n);
  } else if constexpr (CHOSEN) {
    for (int w0 = 0; w0 < b.pages; w0 += kWindow) {
      const int total = list_window(a, b, w0, lists);
      over((int)((uint32_t)(total * b.part) / (uint32_t)b.used), (int)((uint32_t)(total * (b.part + 1)) / (uint32_t)b.used), w0);  // (2048 pages, 64 parts)
      __syncthreads();
    }
  } else {
    over(b.part * a.chunk, b.part == b.used - 1 ? b.pages : (b.part + 1) * a.chunk, 0);
  }

  // The waves' results.
  if constexpr (kStaged) wait_for_all();  // (the last page's keys, fetched again)
  const float total = S::column_sum(sum);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    shares[wave].acc[col][(S::channel(i, quarter, 0) / 4) ^ (col % 16)] = o[i];
  if (quarter == 0) {
    refs[wave][col] = ref;
    sums[wave][col] = total;
  }
  if constexpr (SOLO) {
    __builtin_amdgcn_wave_barrier();
    leave<COLS, 1>(a, b, lane, shares[wave].acc[0], 0, refs[wave], sums[wave]);
  } else {
    __syncthreads();
    leave<COLS, WAVES>(a, b, threadIdx.x, shares[0].acc[0], sizeof(Share) / sizeof(f32x4), refs[0], sums[0]);
  }
}

// Many rows of a sequence: kTiles times 32 of them at a time, which share a page's conversion to bf16. A wave goes through units of 32 tokens and 32
// rows; while it works on the weights of one, its matrix instructions make the logits of the next and add up the values of the one before. What
// bounds it are the vector unit's cycles: of a unit 16 logits a lane with a multiplication, exp2, a sum and half a conversion each, 335 with 64 rows
// and 410 with 32 with its part of the page's conversions, and about 16 for each of its eight matrix instructions, which hold up the others that
// long. 10992 rows over 16384 tokens, 16 heads: 744 us, 992 TFLOP/s (32 rows 857); four rows of eight heads each over 32 caches of 4096 tokens: 46 us
// (weights and products one after the other 51).
template <int kTiles>
__global__ __launch_bounds__(64 * kWaves, kTiles == 1 ? 3 : 2) void pages_attend_rows_kernel(PagesArgs a, int blocks) {
  using S = Shape<32>;
  constexpr int kRows = 32 * kTiles, kUnits = 2 * kTiles;
  union Share {  // of a wave: one page or two, later its results
    uint8_t page[kTiles][kStagedBytes];
    f32x4 acc[kRows][kD / 4];
  };
  __shared__ struct {
    Share of[kWaves];  // (the first 64 KB: the destination of a load to LDS has 16 bits)
    float refs[kWaves][kRows], sums[kWaves][kRows];
  } shares;
  const int lane = threadIdx.x % 64, col = lane % 32, quarter = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  Block b;
  if (!block_of<kRows, false>(a, blockIdx.x, blocks, &b)) return;
  const int32_t* table = a.table + (int64_t)b.s * a.width;
  bf16x8 q[kTiles][4];
  int seen[kTiles];
  f32x16 o[kTiles][2] = {};
  float ref[kTiles], sum[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const Row own = row_of(a, b, 32 * t + col);
    const uint16_t* from = a.q.p + own.head * a.q.sh + (int64_t)(b.h.row0 + own.query) * a.q.st + 32 * quarter;
#pragma unroll
    for (int i = 0; i < 4; ++i) q[t][i] = *reinterpret_cast<const bf16x8*>(from + 8 * i);
    seen[t] = own.seen;
    ref[t] = -kInf;
    sum[t] = 0.0f;
  }
  const float c2 = a.scale * kLog2e;

  // Pages go through LDS, two of a wave's at a time: the one at hand is in place `at_hand`, the next on its way to the other.
  int at_hand = 0;
  const uint32_t staged_at = (uint32_t)(size_t)(lds_byte*)shares.of[wave].page[0];
  const int key_from = lane / 4 * 64 + (lane - key_turn(lane / 4 % 4, 0)) % 4 * 16, value_from = lane / 4 * 64 + (lane + 4 - value_turn(lane / 4)) % 4 * 16;
  auto fetch_keys = [&](int page, int place) {
    stage(a.k + ((size_t)page * a.kv_heads + b.kv) * kPageBytes, key_from, key_from ^ 32, staged_at + place * kStagedBytes);
  };
  auto fetch_values = [&](int page, int place) {
    stage(a.v + ((size_t)page * a.kv_heads + b.kv) * kPageBytes, value_from, value_from, staged_at + place * kStagedBytes + kPageBytes);
  };
  auto fetch = [&](int page, int place) {
    fetch_keys(page, place);
    fetch_values(page, place);
  };
  const int staged_key = S::staged_key(col, quarter, 0), staged_key1 = S::staged_key(col, quarter, 1), staged_value = S::staged_value(col, quarter, 0), staged_value1 = S::staged_value(col, quarter, 2);
  u32x4 kr[2], vr[2];   // 32 tokens as they are
  bf16x8 kb[4], vb[4];  // 32 tokens in bf16: keys by steps of channels, values by blocks of channels and steps of tokens
  auto read_keys = [&](int place, int h) {
    const uint8_t* p = shares.of[wave].page[place] + 2048 * h;
    kr[0] = *reinterpret_cast<const u32x4*>(p + staged_key);
    kr[1] = *reinterpret_cast<const u32x4*>(p + staged_key1);
  };
  auto read_values = [&](int place, int h) {
    const uint8_t* p = shares.of[wave].page[place] + kPageBytes + (h ? staged_value1 : staged_value);
    vr[0] = *reinterpret_cast<const u32x4*>(p);
    vr[1] = *reinterpret_cast<const u32x4*>(p + 2048);
  };
  auto take_keys = [&] {
#pragma unroll
    for (int i = 0; i < 4; ++i) kb[i] = view8(kr[i / 2][i % 2 * 2], kr[i / 2][i % 2 * 2 + 1]);
  };
  auto take_values = [&](float rest) {
#pragma unroll
    for (int i = 0; i < 4; ++i) vb[i] = view8(vr[i / 2][i % 2 * 2], vr[i / 2][i % 2 * 2 + 1], rest);
  };
  auto logits = [&](int t) {
    f32x16 x = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) x = S::mfma(kb[i], q[t][i], x);
    return x;
  };
  auto add_values = [&](int t, const u32x4 (&pr)[2]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[t][i / 2] = S::mfma(vb[i], __builtin_bit_cast(bf16x8, pr[i % 2]), o[t][i / 2]);
  };
  // (the values' scale 2^ev is in `off`, as above)
  auto weigh = [&](const f32x16& x, float cs, float off, u32x4 (&pr)[2]) {
    float one = 0.0f, other = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
      const float p = exp2_(x[e] * cs - off), r = exp2_(x[e + 1] * cs - off);
      one += p;
      other += r;
      pr[e / 8][e % 8 / 2] = pack2(p, r);
    }
    return one + other;
  };

  // The page at hand with all that may happen, but for its first `skip` units.
  auto whole = [&](int ordinal, int skip, float ks, float vs, [[maybe_unused]] int next_page) __attribute__((always_inline)) {
    const float cs = factor_of(c2, ks);
    const int ev = max(exponent_of(vs), kLeastExponent);
    const float un = __int_as_float((127 - ev) << 23);
    if constexpr (kTiles == 1) wait_for_all();
    else wait_for_all_but_eight();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      read_keys(at_hand, h);
      read_values(at_hand, h);
      if (kTiles == 1 && h == 1) fetch(next_page, 0);
      take_keys();
      bf16x8 nb[4] = {};
      if (vs < 0.0f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t nan[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int at = i % 2 * 2 + j;
            nan[j] = nan_bytes(vr[i / 2][at]);
            vr[i / 2][at] &= ~nan[j];
          }
          nb[i] = view8(nan[0] & 0x38383838u, nan[1] & 0x38383838u);  // ones
        }
      }
      take_values(rest_of(exponent_of(vs)));
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        if (h * kTiles + t < skip) continue;
        const int left = seen[t] - ordinal * kPage - 32 * h - 16 * quarter;
        f32x16 x = logits(t);
        float m = -kInf;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          x[e] = e < left ? x[e] : -kInf;
          m = fmaxf(m, x[e]);
        }
        m = S::column_max(m) * cs;
        const float to = fmaxf(m, ref[t]), f = ref[t] == -kInf || to == ref[t] ? 1.0f : exp2_(ref[t] - to);
        ref[t] = to;
#pragma unroll
        for (int i = 0; i < 2; ++i) o[t][i] *= f;
        u32x4 pr[2];
        sum[t] = sum[t] * f + weigh(x, cs, off_of(to) - (float)ev, pr) * un;
        add_values(t, pr);
        if (vs < 0.0f) {
          // 0 times NaN is NaN: values that are NaN are taken out of the product, and reach the rows that see their tokens by one of their own
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            f32x16 count = {};
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              u32x4 sees;
#pragma unroll
              for (int j = 0; j < 4; ++j) sees[j] = (8 * k + 2 * j < left ? 0x3f80u : 0u) | (8 * k + 2 * j + 1 < left ? 0x3f800000u : 0u);
              count = S::mfma(nb[2 * i + k], __builtin_bit_cast(bf16x8, sees), count);
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) o[t][i][j] = count[j] > 0.0f ? __builtin_nanf("") : o[t][i][j];
          }
        }
      }
    }
  };

  const int begin = b.part * a.chunk, end = b.part == b.used - 1 ? b.pages : (b.part + 1) * a.chunk;
  for (int from = begin + wave; from < end; from += kWaves * 64) {
    const int at = from + kWaves * lane;
    const int lane_page = at < end ? table[at] : -1;
    const bool some = lane_page >= 0 && lane_page < a.pages;
    const int64_t unit = some ? (int64_t)lane_page * a.kv_heads + b.kv : 0;
    float lane_ks = some ? a.k_scale[unit] : 0.0f, lane_vs = some ? a.v_scale[unit] : 0.0f;
    uint64_t mask = __ballot(some);
    if (!mask) continue;
    int i = __builtin_ctzll(mask), next = 0, ordinal = 0, next_page = 0;
    float ks = 0.0f, vs = 0.0f;
    fetch(__builtin_amdgcn_readlane(lane_page, i), at_hand);
    asm volatile("" : "+v"(lane_ks), "+v"(lane_vs));  // (they are there: nothing waits for them in the loop)
    auto look_at = [&] {  // page i; the next one's (behind the last: the same one's) loads begin
      ordinal = from + kWaves * i;
      ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(lane_ks), i));
      vs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(lane_vs), i));
      mask &= mask - 1;
      next = mask ? __builtin_ctzll(mask) : i;
      next_page = __builtin_amdgcn_readlane(lane_page, next);
      if constexpr (kTiles == 2) fetch(next_page, at_hand ^ 1);
    };
    auto plain = [&] { return (ordinal + 1) * kPage <= b.least && vs >= kLeastScale; };
    look_at();
    while (true) {
      bool begun = true;
#pragma unroll
      for (int t = 0; t < kTiles; ++t) begun = begun && !__any(ref[t] == -kInf);
      int skip = 0;
      bool last = false;  // no page is left
      if (begun && plain()) {
        bool done = true;  // with all units
        f32x16 xa, xb;
        u32x4 pa[2], pb[2] = {};
#pragma unroll
        for (int k = 0; k < 4; ++k) vb[k] = bf16x8{};
        vr[0] = vr[1] = u32x4{};
        if constexpr (kTiles == 1) wait_for_all();
        else wait_for_all_but_eight();
        read_keys(at_hand, 0);
        take_keys();
        xa = logits(0);
        while (true) {
          const float cs = factor_of(c2, ks);
          const int ev = exponent_of(vs);
          const float un = __int_as_float((127 - ev) << 23);
          auto unit_of = [&](auto number, const f32x16& x, f32x16& x_next, u32x4 (&pr)[2], const u32x4 (&before)[2]) {
            constexpr int u = decltype(number)::value, t = u % kTiles;
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (kTiles == 1) {
              if (u == 1) {
                wait_for_all();
                read_values(0, 0);
              }
              read_keys(0, 1 - u);
              if (u == 0) fetch_keys(next_page, 0);
            } else {
              if (u == 0) {
                read_keys(at_hand, 1);
                read_values(at_hand, 0);
              }
              if (u == 2) {
                wait_for_all();
                read_keys(at_hand ^ 1, 0);
                read_values(at_hand, 1);
              }
            }
            if (kTiles == 1 || u % 2 == 1) take_keys();
            x_next = logits((t + 1) % kTiles);
            if (kTiles == 1 || u % 2 == 1) take_values(1.0f);
            add_values((t + 1) % kTiles, before);
            if (kTiles == 1 && u == 1) {
              read_values(0, 1);
              fetch_values(next_page, 0);
            }
            const float part = weigh(x, cs, ref[t] - (float)ev, pr) * un;
            asm volatile("" : "+v"(pr[0]), "+v"(pr[1]));  // (here, and not behind the branch: until then there would be twice as many registers)
            if (__any(part > kMaxPart)) {
              skip = u;
              done = false;
              return false;
            }
            sum[t] += part;
            return true;
          };
          if (!unit_of(std::integral_constant<int, 0>{}, xa, xb, pa, pb)) break;
          if (!unit_of(std::integral_constant<int, 1>{}, xb, xa, pb, pa)) break;
          if constexpr (kTiles == 2) {
            if (!unit_of(std::integral_constant<int, 2>{}, xa, xb, pa, pb)) break;
            if (!unit_of(std::integral_constant<int, 3>{}, xb, xa, pb, pa)) break;
          }
          last = !mask;
          if (last) break;
          i = next;
          if (kTiles == 2) at_hand ^= 1;
          look_at();
          if (!plain()) break;
        }
        if (done) {
          if (kTiles == 1) take_values(1.0f);
          add_values(kTiles - 1, pb);
        }
        if (last) break;
        if (kTiles == 1 && !done) {  // (the next page's are on their way there, or there)
          wait_for_all();
          fetch(__builtin_amdgcn_readlane(lane_page, i), 0);
        }
      }
      whole(ordinal, skip, ks, vs, next_page);
      if (!mask) break;
      i = next;
      if (kTiles == 2) at_hand ^= 1;
      look_at();
    }
    wait_for_all();  // (the last page once more)
  }

#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const float total = S::column_sum(sum[t]);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 16; j += 4)
        shares.of[wave].acc[32 * t + col][(S::channel(i, quarter, j) / 4) ^ (col % 16)] = f32x4{o[t][i][j], o[t][i][j + 1], o[t][i][j + 2], o[t][i][j + 3]};
    if (quarter == 0) {
      shares.refs[wave][32 * t + col] = ref[t];
      shares.sums[wave][32 * t + col] = total;
    }
  }
  __syncthreads();
  leave<kRows, kWaves>(a, b, threadIdx.x, shares.of[0].acc[0], sizeof(Share) / sizeof(f32x4), shares.refs[0], shares.sums[0]);
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

// Rows whose pages several workgroups shared: their parts in order, a wave to a row.  The weight of a part is worked out by a lane of its own,
// and the loads of 16 parts' values do not wait for one another or for the weights.
template <int COLS, bool CHOSEN>
__global__ __launch_bounds__(64 * kWaves) void pages_join_kernel(PagesArgs a, int blocks) {
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  Block b;
  if (!block_of<COLS, CHOSEN>(a, blockIdx.x, blocks, &b) || b.used == 1) return;
#pragma unroll 1
  for (int r = wave; r < COLS; r += kWaves) {
    const Row to = row_of(a, b, r);
    if (!to.real) break;
    const int head = to.head;
    const int64_t row = b.h.row0 + to.query;
    const int64_t at = (int64_t)head * a.rows + row, step = (int64_t)a.heads * a.rows;
    const int last = b.used - 1;
    const float* sums = a.part_sums + 2 * (at + min(lane, last) * step);
    const float m = lane <= last ? sums[0] : -kInf, x = sums[1];
    float v = 0.0f, w = 0.0f, l = 0.0f, off = 0.0f;
    for (int p0 = 0; p0 <= last; p0 += 16) {
      float value[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) value[i] = a.part[(at + min(p0 + i, last) * step) * kD + lane];
      if (p0 == 0) {
        off = off_of(over_wave(m, [](float p, float q) { return fmaxf(p, q); }));
        w = exp2_(m - off);
        l = over_wave(lane <= last ? x * w : 0.0f, [](float p, float q) { return p + q; });
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), p0 + i));
        v += p0 + i <= last ? value[i] * f : 0.0f;
      }
    }
    const_cast<uint16_t*>(a.out.p)[head * a.out.sh + row * a.out.st + lane] = (uint16_t)pack2(l == 0.0f ? 0.0f : v / l, 0.0f);
    if (lane == 0) a.lse[at] = (off + log2f(l)) * kLn2;
  }
}

struct Plan {
  long long blocks, units;  // of a sequence and key head; of all
  int parts, chunk, group, cols, waves;
  bool solo;                   // a wave to a block, four blocks to a workgroup
  bool ranked;                 // `blocks` are those of all sequences
};
constexpr long long kMostWorkgroups = (1ll << 32) / (64 * kWaves) - 1;  // threads of a launch are counted in 32 bits
long long times(long long a, long long b) { return b != 0 && a > kMostWorkgroups / b ? kMostWorkgroups + 1 : a * b; }  // as far as it matters
// Are blocks numbered over all sequences, `all` at most?  Then they are the plan's.
void number(Plan& p, const PagesArgs& a, long long all) {
  p.ranked = p.blocks > 1 && a.sequences > 1 && (a.sequences <= kRanked || by_number((double)p.blocks * a.sequences, all));
  if (p.ranked) p.blocks = a.sequences <= kRanked ? std::min(times(p.blocks, a.sequences), all) : all;
}
Plan plan_of(const PagesArgs& a) {
  Plan p{};
  const int rep = a.heads / a.kv_heads;
  const long long items = ((long long)a.longest_k + kPage - 1) / kPage;
  p.chunk = 1;
  p.group = 1;
  p.cols = 16;
  if (a.chosen) {
    if (rep <= kListRows) p.group = std::min(kListRows / rep, std::max(a.longest, 1));
    const int per = (rep + kListRows - 1) / kListRows;
    p.blocks = ((long long)a.longest + p.group - 1) / p.group * per;
    number(p, a, (((long long)a.rows + p.group - 1) / p.group + a.sequences) * per);
    p.units = times(times(p.blocks, a.kv_heads), p.ranked ? 1 : a.sequences);
    const long long entries = (long long)p.group * a.count;
    p.solo = entries <= 64 && p.units >= kSoloBlocks * entries;
    p.parts = p.solo ? 1 : (int)std::max<long long>(std::min<long long>(512 / std::max(p.units, 1ll), (a.count + kWaves - 1) / kWaves), 1);
  } else {
    const long long rows = (long long)a.longest * rep;
    auto cut = [&](int cols) {
      p.cols = cols;
      p.blocks = (rows + cols - 1) / cols;
      number(p, a, ((long long)a.rows * rep + cols - 1) / cols + a.sequences);
      p.units = times(times(p.blocks, a.kv_heads), p.ranked ? 1 : a.sequences);
    };
    long long workgroups = 1024;
    bool wide = false;
    if (rows > 32) {
      cut(64);
      const long long parts = kFull / std::max(p.units, 1ll);
      wide = p.units >= kFull || (p.units * parts * 16 >= kFull * 15 && items >= kLongPart * parts);
    }
    if (wide) workgroups = kFull;
    else cut(rows > 16 ? 32 : 16);
    const long long most = std::min<long long>(std::max<long long>(workgroups / std::max(p.units, 1ll), 1), kMostParts);
    p.chunk = (int)std::max<long long>((items + most - 1) / most, kWaves);
    if (!p.ranked && p.blocks == 1) p.chunk = (int)std::min<long long>(p.chunk, std::max<long long>(kLongest, (items + kMostParts - 1) / kMostParts));
    p.parts = (int)std::max<long long>((items + p.chunk - 1) / p.chunk, 1);
  }
  p.parts = std::min(p.parts, kMostParts);
  p.waves = kWaves;
  if (!a.chosen && p.cols == 16 && p.parts > 1 && p.units <= kManyUnits && items <= kManyPages) {
    p.waves = kManyWaves;
    p.parts = 1;
    p.chunk = (int)std::max<long long>(items, 1);
  }
  return p;
}

template <bool CHOSEN, int COLS, int WAVES = kWaves, bool SOLO = false>
hipError_t launch(PagesArgs a, const Plan& p, hipStream_t stream) {
  a.parts = p.parts;
  a.chunk = p.chunk;
  a.group = p.group;
  a.ranked = p.ranked;
  a.part_sums = a.part + (int64_t)a.parts * a.heads * a.rows * kD;
  if constexpr (COLS >= 32) pages_attend_rows_kernel<COLS / 32><<<(int)(p.units * p.parts), 64 * WAVES, 0, stream>>>(a, (int)p.blocks);
  else pages_attend_kernel<CHOSEN, WAVES, SOLO><<<SOLO ? (int)((p.units + 8 * kWaves - 1) / (8 * kWaves) * 8) : (int)(p.units * p.parts), 64 * WAVES, 0, stream>>>(a, (int)p.blocks);
  if (p.parts > 1) pages_join_kernel<COLS, CHOSEN><<<(int)p.units, 64 * kWaves, 0, stream>>>(a, (int)p.blocks);
  return hipGetLastError();
}

}  // namespace

int64_t pages_attend_workspace(const PagesArgs& a) {
  const Plan p = plan_of(a);
  return p.parts == 1 ? 0 : (int64_t)p.parts * a.heads * a.rows * (kD + 2) * (int64_t)sizeof(float);
}

bool pages_attend_fits(const PagesArgs& a) {
  const Plan p = plan_of(a);
  return p.units <= kMostWorkgroups && times(p.units, p.parts) <= kMostWorkgroups;
}

hipError_t launch_pages_attend(const PagesArgs& a, hipStream_t stream) {
  if (a.sequences == 0 || a.longest == 0) return hipSuccess;
  const Plan p = plan_of(a);
  if (p.waves == kManyWaves) return launch<false, 16, kManyWaves>(a, p, stream);
  if (a.chosen) return p.solo ? launch<true, 16, kWaves, true>(a, p, stream) : launch<true, 16>(a, p, stream);
  return p.cols == 16 ? launch<false, 16>(a, p, stream) : p.cols == 32 ? launch<false, 32>(a, p, stream) : launch<false, 64>(a, p, stream);
}

}  // namespace xsv
