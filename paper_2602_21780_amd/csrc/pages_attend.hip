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

// A block of 16 rows of a key head of a sequence, and the pages that it looks at.
struct Block {
  Held h;
  int head0, kv;       // the first query head of the key head
  int query, head;     // of the lane's row (behind the last: a copy of it that nobody writes)
  bool real;
  int seen;            // tokens that the lane's row sees
  int least, pages;    // tokens that all rows see; pages that any row sees one of
  int begin, end;      // the workgroup's share of the pages, or of the entries of the list
  int used;            // workgroups that have one
};

template <bool CHOSEN>
__device__ __forceinline__ bool block_of(const PagesArgs& a, int number, int blocks, int col, Block* b) {
  const int rep = a.heads / a.kv_heads;
  const int part = number % a.parts, unit = number / a.parts;
  b->kv = unit % a.kv_heads;
  const int block = unit / a.kv_heads % blocks, s = unit / a.kv_heads / blocks;
  b->h = held(a, s);
  b->head0 = b->kv * rep;
  const int per = CHOSEN ? (rep + kCols - 1) / kCols : 1;  // blocks of a query
  const int rows = CHOSEN ? rep : b->h.n * rep;            // that share their pages
  const int query0 = CHOSEN ? block / per : 0, row0 = (CHOSEN ? block % per : block) * kCols;
  if (query0 >= b->h.n || row0 >= rows) return false;
  const int row = min(row0 + col, rows - 1), last = min(row0 + kCols, rows) - 1;
  b->real = row0 + col < rows;
  b->query = query0 + row / rep;
  b->head = b->head0 + row % rep;
  b->seen = tokens_seen(a, b->h, b->query);
  b->least = tokens_seen(a, b->h, query0 + row0 / rep);
  b->pages = (tokens_seen(a, b->h, query0 + last / rep) + kPage - 1) / kPage;
  const int items = CHOSEN ? a.count : b->pages;
  b->used = min(max((items + a.chunk - 1) / a.chunk, 1), a.parts);
  if (part >= b->used) return false;
  b->begin = part * a.chunk;
  b->end = part == b->used - 1 ? items : b->begin + a.chunk;
  return true;
}

// What 64 lanes know of the next 64 pages of a wave, one a lane.
struct Next {
  int page, ordinal;
  float ks, vs;
  uint64_t mask;  // lanes that have one
};

template <bool CHOSEN>
__global__ __launch_bounds__(64 * kWaves, 2) void pages_attend_kernel(PagesArgs a, int blocks) {
  __shared__ __align__(16) float acc[kWaves][kCols][kD + 4];
  __shared__ float refs[kWaves][kCols], sums[kWaves][kCols];
  const int lane = threadIdx.x % 64, col = lane % 16, u = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  Block b;
  if (!block_of<CHOSEN>(a, blockIdx.x, blocks, col, &b)) return;
  const int s = (int)(blockIdx.x / a.parts / a.kv_heads / blocks);
  const int64_t global = b.h.row0 + b.query;
  const int32_t* table = a.table + (int64_t)s * a.width;
  const int32_t* list = CHOSEN ? a.chosen + (global * a.kv_heads + b.kv) * a.count : nullptr;

  bf16x8 qf[2];
  {
    const uint16_t* q = a.q.p + b.head * a.q.sh + global * a.q.st + 16 * u;
#pragma unroll
    for (int i = 0; i < 2; ++i) qf[i] = *reinterpret_cast<const bf16x8*>(q + 8 * i);
  }
  f32x4 o[4] = {};
  float ref = -kInf, sum = 0.0f;
  const float c2 = a.scale * kLog2e;

  auto look = [&](int from) {
    Next n;
    const int at = from + kWaves * lane;
    n.ordinal = CHOSEN ? (at < b.end ? list[at] : -1) : at;
    bool some = at < b.end && n.ordinal >= 0 && n.ordinal < b.pages;
    n.page = some ? table[n.ordinal] : -1;
    some = some && n.page >= 0 && n.page < a.pages;
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
  auto tile = [&](int page, int ordinal, float ks, float vs, int next, auto cut_) {  // cut: some row does not see some of its tokens
    constexpr bool kCut = decltype(cut_)::value;
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
    const int left = b.seen - ordinal * kPage - 16 * u;  // of the lane's 16 tokens
    float m = -kInf;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (kCut) x[i][j] = 4 * i + j < left ? x[i][j] : -kInf;
        m = fmaxf(m, x[i][j]);
      }
    const float cs = c2 * ks;
    const float top = column_max(m) * cs;
    if (__any(top > ref)) {
      const float to = fmaxf(top, ref), f = ref == -kInf || to == ref ? 1.0f : exp2_(ref - to);
      ref = to;
      sum *= f;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] *= f;
    }
    const float off = off_of(ref);
    bf16x8 pr[2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[i][j] = exp2_(x[i][j] * cs - off);
        sum += x[i][j];
        x[i][j] *= vs;
      }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x4 w = {pack2(x[2 * i][0], x[2 * i][1]), pack2(x[2 * i][2], x[2 * i][3]), pack2(x[2 * i + 1][0], x[2 * i + 1][1]),
                       pack2(x[2 * i + 1][2], x[2 * i + 1][3])};
      pr[i] = __builtin_bit_cast(bf16x8, w);
    }
    if (kCut) {
      // 0 times NaN is NaN: values that are NaN are taken out of the product, and reach the rows that see their tokens by one of their own
      u32x4 nan[4];
      uint32_t any = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          nan[i][j] = nan_bytes(vr[i][j]);
          any |= nan[i][j];
          vr[i][j] &= ~nan[i][j];
        }
      if (__any(any != 0)) {
        f32x4 count[4] = {};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          u32x4 w;
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = (8 * k + 2 * i < left ? 0x3f80u : 0u) | (8 * k + 2 * i + 1 < left ? 0x3f800000u : 0u);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            count[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(view8(nan[i][2 * k] & 0x38383838u, nan[i][2 * k + 1] & 0x38383838u),
                                                               __builtin_bit_cast(bf16x8, w), count[i], 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) o[i][j] = count[i][j] > 0.0f ? __builtin_nanf("") : o[i][j];
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int k = 0; k < 2; ++k) o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(view8(vr[i][2 * k], vr[i][2 * k + 1]), pr[k], o[i], 0, 0, 0);
  };
  for (int from = b.begin + wave; from < b.end; from += kWaves * 64) {
    const Next n = look(from);
    uint64_t mask = n.mask;
    if (!mask) continue;
    int i = __builtin_ctzll(mask), page = __builtin_amdgcn_readlane(n.page, i);
    fetch_keys(page);
    while (true) {
      mask &= mask - 1;
      const int next = mask ? __builtin_ctzll(mask) : -1, next_page = __builtin_amdgcn_readlane(n.page, max(next, 0));
      const int ordinal = __builtin_amdgcn_readlane(n.ordinal, i);
      const float ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(n.ks), i)), vs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(n.vs), i));
      if ((ordinal + 1) * kPage <= b.least) tile(page, ordinal, ks, vs, mask ? next_page : -1, std::false_type{});
      else tile(page, ordinal, ks, vs, mask ? next_page : -1, std::true_type{});
      if (!mask) break;
      i = next;
      page = next_page;
    }
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
  const int part = blockIdx.x % a.parts;
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
      const int64_t at = ((int64_t)part * a.heads + head) * a.rows + row;
      a.part[at * kD + c] = v;
      if (c < 2) a.part_sums[2 * at + c] = c ? l : top;
    }
  }
}

// Rows whose pages several workgroups shared: their parts in order, a wave to a row.
template <bool CHOSEN>
__global__ __launch_bounds__(64 * kWaves) void pages_join_kernel(PagesArgs a, int blocks) {
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  Block b;
  if (!block_of<CHOSEN>(a, blockIdx.x * a.parts, blocks, lane % 16, &b) || b.used == 1) return;
#pragma unroll 1
  for (int j = 0; j < kCols / kWaves; ++j) {
    const int r = wave * (kCols / kWaves) + j;
    if (!__builtin_amdgcn_readlane(b.real, r)) break;
    const int head = __builtin_amdgcn_readlane(b.head, r);
    const int64_t row = b.h.row0 + __builtin_amdgcn_readlane(b.query, r);
    const int64_t at = (int64_t)head * a.rows + row, step = (int64_t)a.heads * a.rows;
    float top = -kInf, l = 0.0f, v = 0.0f;
    for (int p = 0; p < b.used; ++p) top = fmaxf(top, a.part_sums[2 * (at + p * step)]);
    const float off = off_of(top);
    for (int p = 0; p < b.used; ++p) {
      const float f = exp2_(a.part_sums[2 * (at + p * step)] - off);
      l += a.part_sums[2 * (at + p * step) + 1] * f;
      v += a.part[(at + p * step) * kD + lane] * f;
    }
    const_cast<uint16_t*>(a.out.p)[head * a.out.sh + row * a.out.st + lane] = (uint16_t)pack2(l == 0.0f ? 0.0f : v / l, 0.0f);
    if (lane == 0) a.lse[at] = (off + log2f(l)) * kLn2;
  }
}

struct Plan {
  long long blocks, units;  // of a sequence and key head; of all
  int parts, chunk;
};
constexpr long long kMostWorkgroups = (1ll << 32) / (64 * kWaves) - 1;  // threads of a launch are counted in 32 bits
long long times(long long a, long long b) { return b != 0 && a > kMostWorkgroups / b ? kMostWorkgroups + 1 : a * b; }  // as far as it matters
Plan plan_of(const PagesArgs& a) {
  Plan p;
  const int rep = a.heads / a.kv_heads;
  p.blocks = a.chosen ? (long long)a.longest * ((rep + kCols - 1) / kCols) : ((long long)a.longest * rep + kCols - 1) / kCols;
  p.units = times(times(p.blocks, a.kv_heads), a.sequences);
  const long long items = a.chosen ? a.count : ((long long)a.longest_k + kPage - 1) / kPage;
  const long long most = std::min<long long>(std::max<long long>(1024 / std::max(p.units, 1ll), 1), kMostParts);
  p.chunk = (int)std::max<long long>((items + most - 1) / most, kWaves);
  p.parts = (int)std::max<long long>((items + p.chunk - 1) / p.chunk, 1);
  return p;
}

template <bool CHOSEN>
hipError_t launch(PagesArgs a, hipStream_t stream) {
  const Plan p = plan_of(a);
  a.parts = p.parts;
  a.chunk = p.chunk;
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
