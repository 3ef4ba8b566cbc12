// Attention over a paged cache in 8 bits, all pages of a sequence or the ones that are chosen for each query and key head.
//
//   S = scale * k_scale * (q . code_k) over the tokens that a row sees,  lse = log sum exp(S),  out = exp(S - lse) (code_v * v_scale)
//
// Codes become bf16 as they are (e4m3 has 4 significant bits, bf16 has 8), one instruction for two; the page's scales are powers of two,
// so that multiplying logits and probabilities by them instead rounds nothing.
#include <algorithm>
#include <type_traits>

#include "pages.h"

namespace xsv {
namespace {

constexpr int kWaves = 4;
constexpr int kCols = 16;     // rows of a block: (query, head of the key head) pairs, heads first
constexpr int kMostParts = 64;

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float off_of(float ref) { return ref == -kInf ? 0.0f : ref; }  // (nothing finite seen yet)

__device__ __forceinline__ float column_max(float x) {  // over the four lanes of a row
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float column_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// 8 codes as bf16
__device__ __forceinline__ bf16x8 view8(uint32_t a, uint32_t b) {
  const bf16x2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
  const bf16x2 r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false), s = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
  const u32x4 w = {__builtin_bit_cast(uint32_t, p), __builtin_bit_cast(uint32_t, q), __builtin_bit_cast(uint32_t, r), __builtin_bit_cast(uint32_t, s)};
  return __builtin_bit_cast(bf16x8, w);
}

// The NaN codes of a dword, as bytes 0xff.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m |= ((w >> (8 * i)) & 0x7fu) == 0x7fu ? 0xffu << (8 * i) : 0u;
  return m;
}

// A block of up to 16 rows of a key head of a sequence.
struct Block {
  Held h;
  int s, kv;
  int query, head;     // of the lane's row (behind the last: a copy of it that nobody writes)
  bool real;
  int seen;            // tokens that the lane's row sees
  int least, pages;    // tokens that all rows see; pages that any row sees one of
  int part, used;      // this workgroup of those that share the pages
  int query0, queries; // chosen pages: the queries of the block
};

// All pages: rows (query, head) 16 at a time.  Chosen pages: `group` queries with their heads, or 16 heads of a query that has more.
template <bool CHOSEN>
__device__ __forceinline__ bool block_of(const PagesArgs& a, int number, int blocks, int col, Block* b) {
  const int rep = a.heads / a.kv_heads;
  b->part = number % a.parts;
  const int unit = number / a.parts, block = unit / a.kv_heads % blocks;
  b->kv = unit % a.kv_heads;
  b->s = unit / a.kv_heads / blocks;
  b->h = held(a, b->s);
  const int per = CHOSEN && rep > kCols ? (rep + kCols - 1) / kCols : 1;  // blocks of a query
  b->query0 = CHOSEN ? block / per * a.group : 0;
  b->queries = CHOSEN ? min(a.group, b->h.n - b->query0) : b->h.n;
  const int row0 = (CHOSEN ? block % per : block) * kCols, rows = b->queries * rep;
  if (b->queries <= 0 || row0 >= rows) return false;
  const int row = min(row0 + col, rows - 1), last = min(row0 + kCols, rows) - 1;
  b->real = row0 + col < rows;
  b->query = b->query0 + row / rep;
  b->head = b->kv * rep + row % rep;
  b->seen = tokens_seen(a, b->h, b->query);
  b->least = tokens_seen(a, b->h, b->query0 + row0 / rep);
  b->pages = (tokens_seen(a, b->h, b->query0 + last / rep) + kPage - 1) / kPage;
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
  for (int q = 0; q < b.queries; ++q) {
    const int32_t* list = a.chosen + ((int64_t)(b.h.row0 + b.query0 + q) * a.kv_heads + b.kv) * a.count;
    const int end = (tokens_seen(a, b.h, b.query0 + q) + kPage - 1) / kPage;
    const uint32_t rows = rep >= kCols ? 0xffffu : ((1u << rep) - 1u) << (q * rep);
    for (int i = tid; i < a.count; i += 64 * kWaves) {
      const int j = list[i];
      if (j >= w0 && j < end && j - w0 < words) atomicOr(&l.rows[j - w0], rows);
    }
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

struct Empty {};

template <bool CHOSEN>
__global__ __launch_bounds__(64 * kWaves, CHOSEN ? 3 : 4) void pages_attend_kernel(PagesArgs a, int blocks) {
  __shared__ __align__(16) float acc[kWaves][kCols][kD + 4];
  __shared__ float refs[kWaves][kCols], sums[kWaves][kCols];
  __shared__ std::conditional_t<CHOSEN, Lists, Empty> lists;
  const int lane = threadIdx.x % 64, col = lane % 16, u = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  Block b;
  if (!block_of<CHOSEN>(a, blockIdx.x, blocks, col, &b)) return;
  const int32_t* table = a.table + (int64_t)b.s * a.width;

  bf16x8 qf[2];
  {
    const uint16_t* q = a.q.p + b.head * a.q.sh + (int64_t)(b.h.row0 + b.query) * a.q.st + 16 * u;
#pragma unroll
    for (int i = 0; i < 2; ++i) qf[i] = *reinterpret_cast<const bf16x8*>(q + 8 * i);
  }
  f32x4 o[4] = {};
  float ref = -kInf, sum = 0.0f;
  const float c2 = a.scale * kLog2e;

  // Of the pages (or entries of the list) `from`, `from` + kWaves, .. below `end`.
  auto look = [&](int from, int end, int w0) {
    Next n;
    const int at = from + kWaves * lane;
    bool some = at < end;
    n.ordinal = at;
    n.rows = 0;
    if constexpr (CHOSEN) {
      const uint32_t entry = some ? lists.found[at] : 0u;
      n.ordinal = w0 + (int)(entry & 0xffffu);
      n.rows = entry >> 16;
    }
    n.page = some ? table[n.ordinal] : -1;
    some = n.page >= 0 && n.page < a.pages;
    const int64_t unit = some ? (int64_t)n.page * a.kv_heads + b.kv : 0;
    n.ks = some ? a.k_scale[unit] : 0.0f;
    n.vs = some ? a.v_scale[unit] : 0.0f;
    n.mask = __ballot(some);
    return n;
  };
  u32x4 kr[4];
  const int key_at = (16 * (col / 4) + col % 4) * kD + 16 * u, value_at = col * kPage + 16 * u;
  auto fetch_keys = [&](int page) {
    const uint8_t* p = a.k + ((size_t)page * a.kv_heads + b.kv) * kPageBytes + key_at;
#pragma unroll
    for (int i = 0; i < 4; ++i) kr[i] = *reinterpret_cast<const u32x4*>(p + 4 * i * kD);
  };
  auto tile = [&](int page, int ordinal, uint32_t rows, float ks, float vs, int next) {
    u32x4 vr[4];
    const uint8_t* p = a.v + ((size_t)page * a.kv_heads + b.kv) * kPageBytes + value_at;
#pragma unroll
    for (int i = 0; i < 4; ++i) vr[i] = *reinterpret_cast<const u32x4*>(p + 16 * i * kPage);
    f32x4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(view8(kr[i][0], kr[i][1]), qf[0], f32x4{}, 0, 0, 0);
      x[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(view8(kr[i][2], kr[i][3]), qf[1], x[i], 0, 0, 0);
    }
    if (next >= 0) fetch_keys(next);
    const bool cut = (ordinal + 1) * kPage > b.least;         // some row does not see some of the page's tokens
    const bool mine = !CHOSEN || (rows >> col & 1);
    const int left = mine ? b.seen - ordinal * kPage - 16 * u : 0;  // of the lane's 16 tokens
    if (cut)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) x[i][j] = 4 * i + j < left ? x[i][j] : -kInf;
    float m = -kInf;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) m = fmaxf(m, x[i][j]);
    const float cs = c2 * ks;
    const float top = mine ? column_max(m) * cs : -kInf;
    if (__any(top > ref)) {
      const float to = fmaxf(top, ref), f = ref == -kInf || to == ref ? 1.0f : exp2_(ref - to);
      ref = to;
      sum *= f;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] *= f;
    }
    const float off = off_of(ref), size = fabsf(vs);
    float part = 0.0f;
    u32x4 pr[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[i][j] = exp2_(x[i][j] * cs - off);
        part += x[i][j];
        x[i][j] *= size;
      }
      pr[i / 2][i % 2 * 2] = pack2(x[i][0], x[i][1]);
      pr[i / 2][i % 2 * 2 + 1] = pack2(x[i][2], x[i][3]);
    }
    sum += mine ? part : 0.0f;
    if constexpr (CHOSEN)
#pragma unroll
      for (int i = 0; i < 8; ++i) pr[i / 4][i % 4] = mine ? pr[i / 4][i % 4] : 0u;
    if (vs < 0.0f) {
      // 0 times NaN is NaN: values that are NaN are taken out of the product, and reach the rows that see their tokens by one of their own
      u32x4 sees[2];
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) sees[k][i] = (8 * k + 2 * i < left ? 0x3f80u : 0u) | (8 * k + 2 * i + 1 < left ? 0x3f800000u : 0u);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u32x4 nan;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          nan[j] = nan_bytes(vr[i][j]);
          vr[i][j] &= ~nan[j];
          nan[j] &= 0x38383838u;  // 1
        }
        f32x4 count = {};
#pragma unroll
        for (int k = 0; k < 2; ++k)
          count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(view8(nan[2 * k], nan[2 * k + 1]), __builtin_bit_cast(bf16x8, sees[k]), count, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) o[i][j] = count[j] > 0.0f ? __builtin_nanf("") : o[i][j];
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int k = 0; k < 2; ++k)
        o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(view8(vr[i][2 * k], vr[i][2 * k + 1]), __builtin_bit_cast(bf16x8, pr[k]), o[i], 0, 0, 0);
  };
  auto over = [&](int begin, int end, int w0) {
    for (int from = begin + wave; from < end; from += kWaves * 64) {
      const Next n = look(from, end, w0);
      uint64_t mask = n.mask;
      if (!mask) continue;
      int i = __builtin_ctzll(mask), page = __builtin_amdgcn_readlane(n.page, i);
      fetch_keys(page);
      while (true) {
        mask &= mask - 1;
        const int next = mask ? __builtin_ctzll(mask) : -1, next_page = __builtin_amdgcn_readlane(n.page, max(next, 0));
        tile(page, __builtin_amdgcn_readlane(n.ordinal, i), CHOSEN ? __builtin_amdgcn_readlane(n.rows, i) : 0u,
             __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(n.ks), i)), __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(n.vs), i)),
             mask ? next_page : -1);
        if (!mask) break;
        i = next;
        page = next_page;
      }
    }
  };
  if constexpr (CHOSEN) {
    for (int w0 = 0; w0 < b.pages; w0 += kWindow) {
      const int total = list_window(a, b, w0, lists);
      over((int)((int64_t)total * b.part / b.used), (int)((int64_t)total * (b.part + 1) / b.used), w0);
      __syncthreads();
    }
  } else {
    over(b.part * a.chunk, b.part == b.used - 1 ? b.pages : (b.part + 1) * a.chunk, 0);
  }

  // The waves' results: lane (col, u) has channels 16 i + 4 u + 0..3 of row col.
  const float total = column_sum(sum);
#pragma unroll
  for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4*>(&acc[wave][col][16 * i + 4 * u]) = o[i];
  if (u == 0) {
    refs[wave][col] = ref;
    sums[wave][col] = total;
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kCols / kWaves; ++j) {
    const int r = wave * (kCols / kWaves) + j, c = lane;
    // (row r's place is what lane r has)
    if (!__builtin_amdgcn_readlane(b.real, r)) continue;
    const int head = __builtin_amdgcn_readlane(b.head, r);
    const int64_t row = b.h.row0 + __builtin_amdgcn_readlane(b.query, r);
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
    if (b.used == 1) {
      const_cast<uint16_t*>(a.out.p)[head * a.out.sh + row * a.out.st + c] = (uint16_t)pack2(l == 0.0f ? 0.0f : v / l, 0.0f);
      if (c == 0) a.lse[(int64_t)head * a.rows + row] = (off + log2f(l)) * kLn2;
    } else {
      const int64_t at = ((int64_t)b.part * a.heads + head) * a.rows + row;
      a.part[at * kD + c] = v;
      if (c < 2) a.part_sums[2 * at + c] = c ? l : top;
    }
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

// Rows whose pages several workgroups shared: their parts in order, a wave to a row.  The weight of a part is worked out by a lane of its own,
// and the loads of 16 parts' values do not wait for one another or for the weights.
template <bool CHOSEN>
__global__ __launch_bounds__(64 * kWaves) void pages_join_kernel(PagesArgs a, int blocks) {
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  Block b;
  if (!block_of<CHOSEN>(a, blockIdx.x * a.parts, blocks, lane % 16, &b) || b.used == 1) return;
#pragma unroll 1
  for (int r = wave; r < kCols; r += kWaves) {
    if (!__builtin_amdgcn_readlane(b.real, r)) break;
    const int head = __builtin_amdgcn_readlane(b.head, r);
    const int64_t row = b.h.row0 + __builtin_amdgcn_readlane(b.query, r);
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
  int parts, chunk, group;
};
constexpr long long kMostWorkgroups = (1ll << 32) / (64 * kWaves) - 1;  // threads of a launch are counted in 32 bits
long long times(long long a, long long b) { return b != 0 && a > kMostWorkgroups / b ? kMostWorkgroups + 1 : a * b; }  // as far as it matters
Plan plan_of(const PagesArgs& a) {
  Plan p;
  const int rep = a.heads / a.kv_heads;
  p.chunk = 1;
  p.group = 1;
  if (a.chosen) {
    if (rep <= kCols) p.group = std::min(kCols / rep, std::max(a.longest, 1));
    p.blocks = ((long long)a.longest + p.group - 1) / p.group * ((rep + kCols - 1) / kCols);
    p.units = times(times(p.blocks, a.kv_heads), a.sequences);
    p.parts = (int)std::max<long long>(std::min<long long>(512 / std::max(p.units, 1ll), (a.count + kWaves - 1) / kWaves), 1);
  } else {
    p.blocks = ((long long)a.longest * rep + kCols - 1) / kCols;
    p.units = times(times(p.blocks, a.kv_heads), a.sequences);
    const long long items = ((long long)a.longest_k + kPage - 1) / kPage;
    const long long most = std::min<long long>(std::max<long long>(1024 / std::max(p.units, 1ll), 1), kMostParts);
    p.chunk = (int)std::max<long long>((items + most - 1) / most, kWaves);
    p.parts = (int)std::max<long long>((items + p.chunk - 1) / p.chunk, 1);
  }
  p.parts = std::min(p.parts, kMostParts);
  return p;
}

template <bool CHOSEN>
hipError_t launch(PagesArgs a, hipStream_t stream) {
  const Plan p = plan_of(a);
  a.parts = p.parts;
  a.chunk = p.chunk;
  a.group = p.group;
  a.part_sums = a.part + (int64_t)a.parts * a.heads * a.rows * kD;
  pages_attend_kernel<CHOSEN><<<(int)(p.units * p.parts), 64 * kWaves, 0, stream>>>(a, (int)p.blocks);
  if (p.parts > 1) pages_join_kernel<CHOSEN><<<(int)p.units, 64 * kWaves, 0, stream>>>(a, (int)p.blocks);
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
  return a.chosen ? launch<true>(a, stream) : launch<false>(a, stream);
}

}  // namespace xsv
