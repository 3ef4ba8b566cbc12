// A paged cache in 8 bits: rows written into it and read back.
//
//   scale = 2^e, the smallest e in -100 .. 120 with 448 2^e >= max |x| over the finite elements of a page's keys (values) of one head,
//   code = e4m3(x / scale), to nearest even, at most 240 in size where e = 120 (256 2^120 is infinite); what is not finite becomes NaN
//
// e4m3 keeps four significant bits at any size down to 2^-15 of the largest, so a few channels of large keys do not cost the others
// their bits, as they would with whole numbers under one scale.  With powers of two the division is exact, and so is a later change of the
// page's scale, but for codes below 2^-6, which e4m3 holds in steps of 2^-9: a page that grows token by token is what it would be if
// written at once, but for those.  The bounds are over the codes, in halves, so that they are whole numbers up to 896, which fp16 and
// sums of their products with whole numbers in fp32 hold exactly.  A page's scale of values is negative once one of its values is NaN, so that attention has
// to look for them nowhere else.
//
// A workgroup has one page of one head: a thread 16 channels of a token on the row side, 16 bytes of a line of the page on the other; values change
// sides in LDS.  Memory bounds both: 32976 tokens of 16 heads are written in 47 us and read back in 47, 4.4 and 4.3 TB/s of what is read and written (a
// large copy: 4.9); a token each of 64 streams takes 6.3 us, the chain of offsets, table, scale, page and its way back.
#include "pages.h"

namespace xsv {
namespace {

constexpr int kThreads = 256;
constexpr int kLine = 64 + 16;  // bytes of a channel's 64 codes in LDS

// The pages that a sequence's rows are in: the one that page number `i` of the launch is, and the places in it.
struct Touched {
  Held h;
  int ordinal, page;     // of the sequence; of the pool, -1: none
  int from, to;          // places [from, to) are the rows first .. of the call
  int first;
  bool any;
};
__device__ __forceinline__ Touched touched(const PagesArgs& a, int number, int most) {
  Touched t;
  int s = number / most, i = number % most;
  if (a.ranked) {
    i = number;
    if (!numbered_block(a, [](int row) { return row / kPage; }, 2, &i, &s, &t.h)) i = 1 << 30;  // (n rows are in at most n / 64 + 2 pages)
  } else {
    t.h = held(a, s);
  }
  const int start = max(t.h.ahead, 0), end = min(t.h.ahead + t.h.n, a.width * kPage);  // (rows in front of the first token or behind the table have no place)
  t.ordinal = start / kPage + i;
  const int p0 = min(t.ordinal, a.width) * kPage;  // (of a page behind the table: the end, where no row is; it holds at most 2^30 tokens)
  t.from = max(start - p0, 0);
  t.to = min(end - p0, kPage);
  t.any = end > start && t.from < t.to;
  t.first = t.h.row0 + p0 + t.from - t.h.ahead;
  t.page = t.any ? a.table[(int64_t)s * a.width + t.ordinal] : -1;
  t.any = t.any && t.page >= 0 && t.page < a.pages;
  return t;
}

// e of the largest |x|, given by its bits
__device__ __forceinline__ int exponent_of(uint32_t largest) {
  // |x| = m 2^p, m in [1, 2): 448 = 1.75 2^8
  const int p = (int)(largest >> 23) - 127 + ((largest & 0x7fffffu) > 0x600000u);
  return min(max(p - 8, -100), 120);
}
__device__ __forceinline__ float power(int e) { return __int_as_float((e + 127) << 23); }
__device__ __forceinline__ int power_of(float scale) { return (int)((__float_as_uint(scale) >> 23) & 0xff) - 127; }

// four numbers of at most 448, or NaN, as codes
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}
__device__ __forceinline__ uint32_t rescaled(uint32_t w, float f) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  return codes4(a[0] * f, a[1] * f, b[0] * f, b[1] * f);
}
__device__ __forceinline__ bool has_nan(uint32_t w) { return (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0; }  // 0x7f and 0xff are NaN
__device__ __forceinline__ float number_or_nan(float x, float y) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u ? __builtin_nanf("") : y; }  // y where x is finite
// The largest code under a scale: with 2^120 one that stands for a number that fp32 and bf16 hold.
__device__ __forceinline__ float top_of(int e) { return e == 120 ? 240.0f : 448.0f; }

// the bytes of a dword that stand for places `at` .. at + 3 and lie in [from, to)
__device__ __forceinline__ uint32_t within(int at, int from, int to) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m |= at + i >= from && at + i < to ? 0xffu << (8 * i) : 0u;
  return m;
}

using u16x2 = __attribute__((ext_vector_type(2))) uint16_t;
struct Row16 {  // 16 channels of a token
  u32x4 r[2];
  __device__ __forceinline__ void load(const uint16_t* p) {
    r[0] = *reinterpret_cast<const u32x4*>(p);
    r[1] = *reinterpret_cast<const u32x4*>(p + 8);
  }
  // of |x|, bits of fp32; `all`: also of what is not finite
  __device__ __forceinline__ uint32_t largest(bool all) const {
    u16x2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      u16x2 x = __builtin_bit_cast(u16x2, r[i / 4][i % 4] & 0x7fff7fffu);
      if (!all) x = u16x2{(uint16_t)(x[0] < 0x7f80 ? x[0] : 0), (uint16_t)(x[1] < 0x7f80 ? x[1] : 0)};
      m = __builtin_elementwise_max(m, x);
    }
    return (uint32_t)max(m[0], m[1]) << 16;
  }
  // `ordinary`: all finite, and no code above `top`
  __device__ __forceinline__ u32x4 codes(float f, bool ordinary, float top) const {
    u32x4 c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t a = r[i / 2][i % 2 * 2], b = r[i / 2][i % 2 * 2 + 1];
      float x[4] = {bf16_low(a), bf16_high(a), bf16_low(b), bf16_high(b)};
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = ordinary ? x[j] * f : number_or_nan(x[j], fminf(fmaxf(x[j] * f, -top), top));
      c[i] = codes4(x[0], x[1], x[2], x[3]);
    }
    return c;
  }
};

__global__ __launch_bounds__(kThreads) void pages_write_kernel(PagesArgs a, int most) {
  __shared__ __align__(16) uint8_t lines[2][kD][kLine];  // the codes of keys and values by channel
  __shared__ uint32_t top[2][kThreads / 64];
  __shared__ int none[kThreads / 64];  // a wave's values are not all numbers
  const int tid = threadIdx.x, number = blockIdx.x;
  const int head = number % a.kv_heads;
  const Touched t = touched(a, number / a.kv_heads, most);
  if (!t.any) return;
  const size_t unit = (size_t)t.page * a.kv_heads + head;
  const int token = tid / 4, ch0 = tid % 4 * 16;    // the row side, and keys in the page
  const bool is_new = token >= t.from && token < t.to, is_old = token < t.from;
  Row16 k{}, v{};
  u32x4 old_k{}, old_v{};  // of this thread's 16 bytes of the page: channels ch0 .. of its token; places ch0 .. of channel `token`
  uint8_t* to_k = a.k + unit * kPageBytes + tid * 16;
  uint8_t* to_v = a.v + unit * kPageBytes + tid * 16;
  if (is_new) {
    const int64_t row = t.first + token - t.from;
    k.load(a.keys.p + head * a.keys.sh + row * a.keys.st + ch0);
    v.load(a.values.p + head * a.values.sh + row * a.values.st + ch0);
  }
  float scale_k = 0.0f, scale_v = 0.0f;  // that the page has (exponents below those of any: none)
  if (t.from > 0) {
    scale_k = a.k_scale[unit];
    scale_v = a.v_scale[unit];
    if (is_old) old_k = *reinterpret_cast<const u32x4*>(to_k);
    old_v = *reinterpret_cast<const u32x4*>(to_v);
  }
  // (rows that are not all finite, or among the largest, are rare and take a way of their own)
  uint32_t mk = k.largest(true), mv = v.largest(true);
  const bool finite = !__any(max(mk, mv) >= 0x7f800000u);
  if (!finite) {
    mk = k.largest(false);
    mv = v.largest(false);
  }
  mk = wave_largest(mk);
  mv = wave_largest(mv);
  if (tid % 64 == 0) {
    top[0][tid / 64] = mk;
    top[1][tid / 64] = mv;
  }
  __syncthreads();
  int e[2], grown[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    uint32_t m = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) m = max(m, top[x][w]);
    const int e_old = t.from > 0 ? power_of(x ? scale_v : scale_k) : -100;
    e[x] = max(exponent_of(m), e_old);
    grown[x] = t.from > 0 ? e[x] - e_old : 0;
  }
  const float fk = power(-e[0]), fv = power(-e[1]);
  u32x4 ck, cv;
  bool nan = false;
  if (finite && max(e[0], e[1]) < 120) {
    ck = k.codes(fk, true, 0.0f);
    cv = v.codes(fv, true, 0.0f);
  } else {
    ck = k.codes(fk, false, top_of(e[0]));
    cv = v.codes(fv, false, top_of(e[1]));
    nan = __any(has_nan(cv[0]) || has_nan(cv[1]) || has_nan(cv[2]) || has_nan(cv[3]));
  }
  if (tid % 64 == 0) none[tid / 64] = nan;
  if (is_old) {
    ck = old_k;
    if (grown[0] > 0)
#pragma unroll
      for (int j = 0; j < 4; ++j) ck[j] = rescaled(old_k[j], power(max(-grown[0], -126)));
  }
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    lines[0][ch0 + j][token] = (uint8_t)(ck[j / 4] >> (8 * (j % 4)));
    lines[1][ch0 + j][token] = (uint8_t)(cv[j / 4] >> (8 * (j % 4)));
  }
  if (is_new || (is_old && grown[0] > 0) || t.from == 0) *reinterpret_cast<u32x4*>(to_k) = ck;  // (behind the rows of a page begun: zeros)
  __syncthreads();
  // values: this thread's places ch0 .. of channel `token`
  const int channel = token, place = ch0;
  u32x4 nv = *reinterpret_cast<const u32x4*>(&lines[1][channel][place]);
  if (t.from > 0) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t fresh = within(place + 4 * j, t.from, t.to), before = grown[1] > 0 ? within(place + 4 * j, 0, t.from) : 0u;
      const uint32_t was = before ? rescaled(old_v[j], power(max(-grown[1], -126))) : 0u;
      nv[j] = (nv[j] & fresh) | (was & before) | (old_v[j] & ~(fresh | before));
    }
  }
  if (t.from == 0 || (place + 16 > t.from && place < t.to) || (grown[1] > 0 && place < t.from)) *reinterpret_cast<u32x4*>(to_v) = nv;
  if (tid == 0) {
    bool negative = scale_v < 0.0f;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) negative |= none[w] != 0;
    a.k_scale[unit] = power(e[0]);
    a.v_scale[unit] = negative ? -power(e[1]) : power(e[1]);
  }
  if (!a.bounds) return;
  const u32x4 line = *reinterpret_cast<const u32x4*>(&lines[0][channel][place]);
  float hi = -kInf, lo = kInf;
  const bool full = t.to == kPage;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f32x2 x = __builtin_amdgcn_cvt_pk_f32_fp8(line[j], false), y = __builtin_amdgcn_cvt_pk_f32_fp8(line[j], true);
    const float four[4] = {x[0], x[1], y[0], y[1]};
#pragma unroll
    for (int b = 0; b < 4; ++b) {  // (the larger of a number and NaN is the number)
      const bool here = full || place + 4 * j + b < t.to;
      hi = fmaxf(hi, here ? four[b] : -kInf);
      lo = fminf(lo, here ? four[b] : kInf);
    }
  }
#pragma unroll
  for (int d = 1; d < 4; d *= 2) {
    hi = fmaxf(hi, __shfl_xor(hi, d));
    lo = fminf(lo, __shfl_xor(lo, d));
  }
  if (hi < lo) hi = lo = 0.0f;  // nothing but NaN
  _Float16* bounds = reinterpret_cast<_Float16*>(a.bounds) + unit * 2 * kD;
  if (place == 0) bounds[channel] = (_Float16)ceilf(2.0f * hi);
  if (place == 16) bounds[kD + channel] = (_Float16)floorf(2.0f * lo);
}

__global__ __launch_bounds__(kThreads) void pages_read_kernel(PagesArgs a, int most) {
  __shared__ __align__(16) uint8_t lines[kD][kLine];
  const int tid = threadIdx.x, number = blockIdx.x;
  const int head = number % a.kv_heads;
  const Touched t = touched(a, number / a.kv_heads, most);
  if (!t.any) return;
  const size_t unit = (size_t)t.page * a.kv_heads + head;
  const u32x4 ck = *reinterpret_cast<const u32x4*>(a.k + unit * kPageBytes + tid * 16);
  *reinterpret_cast<u32x4*>(&lines[tid / 4][tid % 4 * 16]) = *reinterpret_cast<const u32x4*>(a.v + unit * kPageBytes + tid * 16);
  const float ks = a.k_scale[unit], vs = fabsf(a.v_scale[unit]);
  __syncthreads();
  const int token = tid / 4, ch0 = tid % 4 * 16;
  if (token < t.from || token >= t.to) return;
  const int64_t row = t.first + token - t.from;
  uint16_t* k = const_cast<uint16_t*>(a.keys.p) + head * a.keys.sh + row * a.keys.st + ch0;
  uint16_t* v = const_cast<uint16_t*>(a.values.p) + head * a.values.sh + row * a.values.st + ch0;
  u32x4 rk[2], rv[2];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t w = 0;
#pragma unroll
    for (int b = 0; b < 4; ++b) w |= (uint32_t)lines[ch0 + 4 * j + b][token] << (8 * b);
    f32x2 x = __builtin_amdgcn_cvt_pk_f32_fp8(ck[j], false), y = __builtin_amdgcn_cvt_pk_f32_fp8(ck[j], true);
    rk[j / 2][j % 2 * 2] = pack2(x[0] * ks, x[1] * ks);
    rk[j / 2][j % 2 * 2 + 1] = pack2(y[0] * ks, y[1] * ks);
    x = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
    y = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    rv[j / 2][j % 2 * 2] = pack2(x[0] * vs, x[1] * vs);
    rv[j / 2][j % 2 * 2 + 1] = pack2(y[0] * vs, y[1] * vs);
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    *reinterpret_cast<u32x4*>(k + 8 * j) = rk[j];
    *reinterpret_cast<u32x4*>(v + 8 * j) = rv[j];
  }
}

struct Plan {
  int most;          // pages that a sequence's rows can be in
  long long blocks;  // of a head: pages of all sequences
  bool ranked;       // numbered over them
};
Plan plan_of(const PagesArgs& a) {
  Plan p;
  p.most = (int)(((long long)a.longest + kPage - 2) / kPage + 1);
  const long long each = (long long)p.most * a.sequences, all = a.rows / kPage + 2ll * a.sequences;
  p.ranked = a.sequences > 1 && by_number((double)each, all);
  p.blocks = p.ranked ? all : each;
  return p;
}

}  // namespace

bool pages_move_fits(const PagesArgs& a) { return plan_of(a).blocks <= ((1ll << 32) / kThreads - 1) / a.kv_heads; }

hipError_t launch_pages_write(PagesArgs a, hipStream_t stream) {
  if (a.sequences == 0 || a.longest == 0 || a.pages == 0) return hipSuccess;
  const Plan p = plan_of(a);
  a.ranked = p.ranked;
  pages_write_kernel<<<(int)(p.blocks * a.kv_heads), kThreads, 0, stream>>>(a, p.most);
  return hipGetLastError();
}

hipError_t launch_pages_read(PagesArgs a, hipStream_t stream) {
  if (a.sequences == 0 || a.longest == 0 || a.pages == 0) return hipSuccess;
  const Plan p = plan_of(a);
  a.ranked = p.ranked;
  pages_read_kernel<<<(int)(p.blocks * a.kv_heads), kThreads, 0, stream>>>(a, p.most);
  return hipGetLastError();
}

}  // namespace xsv
