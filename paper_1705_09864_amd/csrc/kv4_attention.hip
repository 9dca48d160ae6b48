// Attention of new tokens over the paged cache of 4 bits (kv4_cache.hip):
//   o = sum_t p_t v_t / sum_t p_t,  p_t = exp(scale * q . k_t),  k_t = a_t (levels of t) + b_t, v_t = c_t (levels of t) + d_t,
// over the tokens t that a row sees.  One pass over the cache with the running maximum m of the scores and the running sum, both in 32 bits.
// Products are S^T = K Q^T and O^T = V^T P^T on the matrix cores (16 x 16 x 32, bf16), 16 rows of queries (tokens x heads that share a head of the
// cache) at a time.  Levels go in as 16 + level, which bf16 holds exactly and one shift and one v_and_or_b32 make of two of them (the four
// bits are the highest of the mantissa of 16.0), so that with Q the sum of a row's queries
//   q . k_t = a_t (q . (16 + levels)) + (b_t - 16 a_t) Q,  o = sum_t (p_t c_t) (16 + levels) + sum_t p_t (d_t - 16 c_t),
// where the second sum of either is a number of the token or of the row.  A lane's scores of S^T are those of its own column of P^T in the order of
// tokens in which the cache holds values, so weights never leave their lane.
// Queries go in as parts of 8 bits each that together are all of them: one of bf16, two of f16, three of f32.  Weights p_t c_t go in as two parts, the upper
// cut off and the lower rounded to nearest, 17 bits (16 + level is up to nine times as large as a value's share of its token's range, and sums of 16 are taken off again:
// weights of 8 bits alone would cost results of 8 bits two of theirs, and a lower part cut off too would leave a bias that grows with
// the tokens).  So a result is off by about 2^-17 of sum p_t (31 c_t + |d_t|) / sum p_t, however small it is itself, and then rounded.  For f32 results in three parts, and the
// levels less 8.  bf16 has fp32's range: nothing is held relative to a row's largest weight.
//
// Bound by the cache's bytes: a wave goes over pages of its own (8.5 KB at 128 values a head) with its queries, running maxima, sums and results in
// registers, and requests the next page's keys as soon as this one's are used up, its values as soon as these are.  Where rows x heads are few, a sequence's
// pages are split over workgroups too, and joined by the last of them (kv_join.h).  64 sequences of 8192 tokens stream at 5.3 TB/s; 131072 tokens of one,
// 8 heads of the cache of 128: 35.2 us, 4.1 TB/s (vector ALU 52 % of the time, matrix cores 15 %; the rest are the first pages and the join); 64 of 0 to 4096: 44.2 us,
// 3.2 TB/s, as long as the longest takes; 100 tokens of 8 heads of 64: 6.3 us, a launch and five trips to memory.
#include "bmx_internal.h"
#include "few_bits.h"
#include "kv_join.h"

#include <algorithm>

namespace bmx {
namespace {

using f32x16 = float __attribute__((ext_vector_type(16)));
template <bool F16>
__device__ inline f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ inline f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// What a level is more than its operand.
template <int TYPE>
constexpr float kZero = TYPE == BMX_F32 ? 8.0f : -16.0f;
// The bits of 16.0 in both halves, in a register: beside a literal v_and_or_b32 takes no other, and would fall into two instructions.
template <int TYPE>
__device__ inline uint32_t sixteen() {
  uint32_t x = TYPE == BMX_F16 ? 0x4C004C00 : 0x41804180;
  asm volatile("" : "+v"(x));
  return x;
}
// The levels in fields I and I + 4 of a dword, as operands: f16 or bf16 by the type.
template <int TYPE, int I>
__device__ inline uint32_t two_levels(uint32_t w, uint32_t sixteens) {
  constexpr int shift = 4 * I - (TYPE == BMX_F16 ? 6 : 3);  // onto the mantissa's highest four bits
  constexpr uint32_t m = TYPE == BMX_F16 ? 0x03C003C0 : 0x00780078;
  uint32_t x;
  if constexpr (shift < 0) x = ((w << -shift) & m) | sixteens;
  else x = ((w >> shift) & m) | sixteens;
  if constexpr (TYPE == BMX_F32) x = upper_halves(__builtin_bit_cast(float, x << 16) - 24.0f, __builtin_bit_cast(float, x & 0xffff0000u) - 24.0f);
  return x;
}

// Two values rounded to bf16, by the one instruction.
__device__ inline uint32_t two_bf16(float a, float b) {
  using f32x2 = float __attribute__((ext_vector_type(2)));
  using bf16x2 = __bf16 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}
// Two values as PARTS pairs of bf16: the bits of all but the last are cut off.
template <int PARTS>
__device__ inline void pair(float a, float b, uint32_t (&part)[PARTS]) {
#pragma unroll
  for (int p = 0; p < PARTS; ++p) {
    if (p + 1 < PARTS) {
      part[p] = upper_halves(a, b);
      a = lower_part(a), b = lower_part(b);
    } else {
      part[p] = two_bf16(a, b);
    }
  }
}
// The larger of x and that of the lane 16, and 32, away.
__device__ inline float max_16(float x) {
  const auto two = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  const uint32_t a = two[0], b = two[1];
  return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}
__device__ inline float max_32(float x) {
  const auto two = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  const uint32_t a = two[0], b = two[1];
  return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}
// Values changed in a branch, which stays one by it: the compiler would make selections of it, for all pages.
template <class V>
__device__ inline void apart(V& v) { asm volatile("" : "+v"(v)); }
__device__ inline float or_zero(float x) { return x == -INFINITY ? 0.0f : x; }

// By so much (of a logarithm of 2) a row's scores may pass the one that its weights are relative to, before they are taken relative to a larger one: weights have
// fp32's range, and a row's results would otherwise be multiplied anew on every other page.
// (2048 new tokens of 4096 347 us without it, 323 with.)
constexpr float kGrowth = 8.0f;

struct Args {
  const void* q;
  int64_t q_row, q_head;
  JoinTo to;
  int rows, max_new, window, prompt_splits;
  Deal deal;         // of the pages of tiles of 16 rows; no extra parts: a tile's are all one workgroup's
  int units, tiles;  // (for the deal) tiles of all sequences and of one
  int few;  // sequences of more rows than this are the other kernel's
  bool causal, aligned;
  float scale;
};

constexpr int kCounters = 16384;  // of the workspace's head
constexpr int kLeastPages = 16;  // of a split of many rows (8: level)
// Tiles of 128 rows for the kernel for many: where fewer are level goes by lengths that only the device knows (us in tiles of 16 rows, of 128, 32 heads on 8 of 128 bf16:
// 256 new tokens of 768 15.8, 29.9, of 4352 50, 53, of 16640 164, 127; 512 of 512 19.6, 22.0, of 4608 96, 74, of 16896 317, 225; 16 sequences of 64 new of 512 41, 24).
constexpr int kLeastTiles = 128;
constexpr int64_t kPlaces = 512, kMostPlaces = 2048;
constexpr int64_t kMostTiles = 65535;  // of 16 rows: a launch's second dimension

// The 16 rows from r0 on of a sequence: what any, and what every one of them sees, positions [low, high).
struct Seen {
  int low_any, high_any, low_all, high_all;
  __device__ Seen(const Args& a, const KvSpan& s, int r0) {
    const int tok0 = r0 / a.to.share, tok1 = min((r0 + 15) / a.to.share, s.count - 1);
    high_any = a.causal ? min(s.first + tok1 + 1, s.length) : s.length, high_all = a.causal ? min(s.first + tok0 + 1, s.length) : s.length;
    low_any = a.window ? max(max(s.first + tok0, 0) - a.window + 1, 0) : 0, low_all = a.window ? max(max(s.first + tok1, 0) - a.window + 1, 0) : 0;
  }
  __device__ int pages() const { return max(kv_pages_to(high_any) - low_any / kPage, 0); }
};

// Rows from r0 on that are this kernel's.
__device__ inline bool has_rows(const Args& a, const KvSpan& s, int r0) { return r0 < s.count * a.to.share && s.count * a.to.share <= a.few; }

template <int TYPE, int DC, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void kv4_attention_kernel(bmx_kv4_cache c, Args a) {
  constexpr int QP = TYPE == BMX_F32 ? 3 : TYPE == BMX_F16 ? 2 : 1, PP = TYPE == BMX_F32 ? 3 : 2;
  constexpr int ROW = DC * 32, BYTES = DC * 16, LINE = ROW + 4, LEVEL = TYPE == BMX_F32 ? BMX_F32 : BMX_BF16;
  // (the queries' three parts and a page beside them leave no registers: 16 tokens after the other, scales of values when they are needed)
  constexpr bool TIGHT = TYPE == BMX_F32 && DC > 4;
  __shared__ JoinLds<ROW, WAVES> lds;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), g = lane / 16;
  const int head = blockIdx.x % c.heads, share = a.to.share;
  Part part = {0, 0, 1, 0, kAllPages, {}};
  int seq = blockIdx.z, r0 = blockIdx.y * 16;
  if (a.deal.extra > 0) {
    part = part_of(blockIdx.x / c.heads, a.units, a.deal, [&](int n) {
      const KvSpan s = kv_span(c, n / a.tiles, a.rows, a.max_new);
      const int r0 = n % a.tiles * 16;
      return UnitPages{has_rows(a, s, r0) ? Seen(a, s, r0).pages() : -1, s};
    });
    if (part.unit < 0) return;
    seq = part.unit / a.tiles, r0 = part.unit % a.tiles * 16;
  } else {
    part.span = kv_span(c, seq, a.rows, a.max_new);
    if (!has_rows(a, part.span, r0)) return;
  }
  const KvSpan s = part.span;
  const Seen seen(a, s, r0);
  const int low_all = seen.low_all, high_all = seen.high_all;
  // this workgroup's pages
  const int pages = min(seen.pages() - part.split * part.per, part.per), begin = seen.low_any / kPage + part.split * part.per;
  const int count = max(pages - wave + WAVES - 1, 0) / WAVES;  // (of this wave, WAVES apart)

  const int64_t page_bytes = (int64_t)c.heads * 2 * kPage * BYTES;
  int ids = -1, next = 0;  // the numbers of 64 pages, a lane each; the place of the next page
  int page, at;            // the page on its way, and its place
  uint32_t k[4][DC];       // of a token, its values from 8 DC g on
  u32x4 v[DC], key_pairs[4], value_pairs[4];
  // the next of this wave's pages that is there, and its keys
  const auto load_keys = [&] {
    page = -1;
    for (; next < count; ++next) {
      if (next % 64 == 0) ids = next + lane < count ? kv_page(c, seq, begin + wave + (next + lane) * WAVES) : -1;
      page = __builtin_amdgcn_readlane(ids, next % 64);
      if (page >= 0) break;
    }
    at = next++;
    const int none = page >= 0 ? 0 : kNowhere;
    const Rsrc r = buffer(c.pages + max(page, 0) * page_bytes + (int64_t)head * 2 * kPage * BYTES, kPage * BYTES);
    const int mine = lane % 16 * BYTES + g * DC * 4 + none;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
#pragma unroll
      for (int i = 0; i < DC; i += 4) {
        if (DC - i >= 4) {
          const u32x4 x = load16(r, mine + i * 4, u * 16 * BYTES);
#pragma unroll
          for (int j = 0; j < 4; ++j) k[u][i + j < DC ? i + j : 0] = x[j];
        } else {
#pragma unroll
          for (int j = i; j < DC; ++j) k[u][j] = load4(r, mine + j * 4, u * 16 * BYTES);
        }
      }
    }
    const Rsrc rs = buffer(c.scales + ((int64_t)max(page, 0) * c.heads + head) * 4 * kPage, 4 * kPage);
#pragma unroll
    for (int u = 0; u < 4; ++u) key_pairs[u] = load16(rs, g * 16 + none, u * 64);
  };
  const auto load_value_pairs = [&] {
    const Rsrc rs = buffer(c.scales + (((int64_t)max(page, 0) * c.heads + head) * 2 + 1) * 2 * kPage, 4 * kPage);
#pragma unroll
    for (int u = 0; u < 4; ++u) value_pairs[u] = load16(rs, g * 16 + (page >= 0 ? 0 : kNowhere), u * 64);
  };
  const auto load_values = [&] {
    const int none = page >= 0 ? 0 : kNowhere;
    const Rsrc r = buffer(c.pages + max(page, 0) * page_bytes + (int64_t)(head * 2 + 1) * kPage * BYTES, kPage * BYTES);
#pragma unroll
    for (int i = 0; i < DC; ++i) v[i] = load16(r, lane * 16 + none, i * 1024);
    if (!TIGHT) load_value_pairs();
  };
  load_keys();
  load_values();

  // this lane's row of queries, with the scale's sign
  const int r = r0 + lane % 16, token = min(r / share, s.count - 1), pos = s.first + token;
  const int high = a.causal ? min(pos + 1, s.length) : s.length, low = a.window ? max(max(pos, 0) - a.window + 1, 0) : 0;
  const float factor = fmaxf(fabsf(a.scale) * 1.4426950408889634f, 0x1p-126f);  // (0 times the score of a token that is not seen would be none)
  u32x4 q[QP][DC];
  float all = 0.0f;  // the row's sum
  {
    const int64_t base = (s.row0 + token) * a.q_row + (head * share + r % share) * a.q_head;
    const float sign = a.scale < 0.0f ? -1.0f : 1.0f;
#pragma unroll
    for (int i = 0; i < DC; ++i) {
      const int d = 8 * (DC * g + i);
      float x[8];
      load_eight<TYPE>(a.q, base + d, c.dim - d, a.aligned, x);
#pragma unroll
      for (int j = 0; j < 4; ++j) {  // (in the order of a dword's fields)
        uint32_t part[QP];
        pair<QP>(sign * x[j], sign * x[4 + j], part);
        all += sign * x[j] + sign * x[4 + j];
#pragma unroll
        for (int p = 0; p < QP; ++p) q[p][i][j] = part[p];
      }
    }
    all += __shfl_xor(all, 16);
    all += __shfl_xor(all, 32);
  }

  const uint32_t sixteens = sixteen<LEVEL>();
  // what the products of 16 + level begin with, so that they end as those of the levels
  const float begin_at = TYPE == BMX_F32 ? 0.0f : -16.0f * all;
  const f32x4 z0 = {begin_at, begin_at, begin_at, begin_at};
  // held: the score, times log2 e, that the row's weights are relative to; rest: sum of p_t (d_t + kZero c_t), over this lane's tokens
  float held = -INFINITY, l = 0.0f, rest = 0.0f;
  f32x4 o[DC][2] = {};  // of each 32 values, the even ones and the odd ones
  while (page >= 0) {
    const int t0 = (begin + wave + at * WAVES) * kPage;
    const bool whole = __builtin_amdgcn_readfirstlane(kv_all_in(t0, kPage, low_all, high_all));
    float p[4][4];
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      f32x4 z = z0;
#pragma unroll
      for (int i = 0; i < DC; ++i) {
        const uint32_t w = k[u][i];
        const u32x4 x = {two_levels<LEVEL, 0>(w, sixteens), two_levels<LEVEL, 1>(w, sixteens), two_levels<LEVEL, 2>(w, sixteens), two_levels<LEVEL, 3>(w, sixteens)};
#pragma unroll
        for (int part = 0; part < QP; ++part) z = mfma(x, q[part][i], z);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w = key_pairs[u][i];
        const float ks = bf16_float(w), ko = __builtin_bit_cast(float, w & 0xffff0000u);
        p[u][i] = z[i] * ks + all * (TYPE == BMX_F32 ? ko + 8.0f * ks : ko);
      }
      if (TIGHT) __builtin_amdgcn_sched_barrier(0);
    }
    if (TIGHT) load_value_pairs();
    load_keys();
    if (!whole) {
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = t0 + 16 * u + 4 * g + i;
          const bool sees = t < high && t >= low;
          p[u][i] = sees ? p[u][i] : -INFINITY;
          value_pairs[u][i] = sees ? value_pairs[u][i] : 0;  // (those of a token that nobody has written may be anything)
        }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        apart(value_pairs[u]);
#pragma unroll
        for (int i = 0; i < 4; ++i) apart(p[u][i]);
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, p[u][i]);
    top = max_32(max_16(top));
    const float at_top = top * factor;
    if (__any(at_top > held + kGrowth)) {  // (a row's first page, and few others)
      const bool mine = at_top > held + kGrowth;
      const float shrink = mine ? __builtin_amdgcn_exp2f(held - at_top) : 1.0f;
      held = mine ? at_top : held;
      l *= shrink, rest *= shrink;
#pragma unroll
      for (int i = 0; i < DC; ++i) o[i][0] *= shrink, o[i][1] *= shrink;
    }
    const float held_at = or_zero(held);
    u32x4 w[PP][2];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      float x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t y = value_pairs[u][i];
        const float vs = bf16_float(y), vo = __builtin_bit_cast(float, y & 0xffff0000u) + kZero<TYPE> * vs;
        const float e = __builtin_amdgcn_exp2f(p[u][i] * factor - held_at);
        l += e;
        rest += e * vo;
        x[i] = e * vs;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {  // (a dword of values has tokens 0 and 2 in one operand, 1 and 3 in the next)
        uint32_t part[PP];
        pair<PP>(x[i], x[i + 2], part);
#pragma unroll
        for (int n = 0; n < PP; ++n) w[n][u / 2][u % 2 * 2 + i] = part[n];
      }
      if (TIGHT) __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < DC; ++i)
#pragma unroll
      for (int odd = 0; odd < 2; ++odd)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t y0 = v[i][2 * h], y1 = v[i][2 * h + 1];
          const u32x4 x = odd ? u32x4{two_levels<LEVEL, 1>(y0, sixteens), two_levels<LEVEL, 3>(y0, sixteens), two_levels<LEVEL, 1>(y1, sixteens), two_levels<LEVEL, 3>(y1, sixteens)}
                              : u32x4{two_levels<LEVEL, 0>(y0, sixteens), two_levels<LEVEL, 2>(y0, sixteens), two_levels<LEVEL, 0>(y1, sixteens), two_levels<LEVEL, 2>(y1, sixteens)};
#pragma unroll
          for (int part = 0; part < PP; ++part) o[i][odd] = mfma(x, w[part][h], o[i][odd]);
        }
    load_values();
  }

  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  rest += __shfl_xor(rest, 16);
  rest += __shfl_xor(rest, 32);
  if (g == 0) lds.red_m[wave][lane] = held, lds.red_l[wave][lane] = l;
#pragma unroll
  for (int i = 0; i < DC; ++i)
#pragma unroll
    for (int j = 0; j < 4; j += 2)
      *reinterpret_cast<f32x4*>(&lds.red[(wave * 16 + lane % 16) * LINE + i * 32 + 8 * g + 2 * j]) =
          f32x4{o[i][0][j] + rest, o[i][1][j] + rest, o[i][0][j + 1] + rest, o[i][1][j + 1] + rest};
  __syncthreads();
  join_rows<TYPE, ROW, WAVES>(lds, a.to, c.dim, s.row0, head, r0, min(s.count * share - r0, 16), (int64_t)part.unit * c.heads + head,
                              (int64_t)head * (a.units + a.deal.extra) + part.first, part.split, part.used);
}

// Many rows: 128 of one head of the cache per workgroup, 32 a wave, over all pages that any of them sees.  A page's levels come into LDS once for
// the four waves, as 16-bit floats in the order of the 32 x 32 x 16 products' operands, its scales and offsets as floats (a wave brings in a quarter of it, a page ahead, and
// converts it on its way), and a lane has one row's scores of 16 of 32 tokens, which again are those of its own column of P^T.  Rows of V^T are a block's 16
// even values, then its odd ones.
// SPLIT: tiles of rows fewer than the chip holds workgroups at once, whose pages are split and joined as above (32 heads on 8 of 128 bf16: 512 new tokens of 4608 74 us,
// unsplit 148, of 16896 225, 522; 1024 of 5120 138, 164; 4 sequences of 128 new of 4224 70, 135).
// GROUPS: two take turns, 256 rows a workgroup: while the four waves of one make products, those of the other, on the same SIMDs, make weights, with a barrier
// wherever they change over.  So products of a page come a turn behind its weights, beside the next page's scores; the first group brings in keys, the second values.
//
// Bound by issue: two sequences of 2048 new tokens of 4096, 32 heads on 8 of 128 bf16, 282 us in two groups, 730 TFLOP/s by the formula's products (a third of those
// made are the weights' lower parts), 319 in one.  Vector ALU 66 % of the time, matrix cores 56 % (63 and 48 in one group), two waves a SIMD; the products alone take
// 221 us, the weights alone 200.  Two tiles of 32 rows a wave, one wave a SIMD: 464.
template <int TYPE, int DC, bool SPLIT, int GROUPS>
__global__ __launch_bounds__(GROUPS * 256, DC <= 4 ? 2 : 1) void kv4_prompt_kernel(bmx_kv4_cache c, Args a) {
  static_assert(TYPE != BMX_F32 && !(SPLIT && GROUPS > 1) && (GROUPS == 1 || DC <= 4), "");
  constexpr int BYTES = DC * 16, NS = DC * 2, KN = (DC + 3) / 4;  // NS: steps of 16 values; KN: what a wave brings in of keys, and of values, by 64 lanes
  constexpr int ROWS = GROUPS * 128, SLOTS = GROUPS + 1;
  __shared__ u32x4 keys[2][NS * 128], values[SLOTS][NS * 128];
  __shared__ f32x4 of_token[SLOTS][4][16];  // [slot][keys' scales and offsets, values'][token / 4]
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), h = lane / 32, group = wave / 4, part = wave % 4;
  const int head = SPLIT ? blockIdx.x % c.heads : blockIdx.x, split = SPLIT ? blockIdx.x / c.heads : 0, seq = blockIdx.z;
  const KvSpan s = kv_span(c, seq, a.rows, a.max_new);
  const int share = a.to.share, rows = s.count * share;
  const int r0 = ((rows + ROWS - 1) / ROWS - 1 - (int)blockIdx.y) * ROWS;  // (the last rows, which see most, first)
  if (r0 < 0 || rows <= a.few) return;
  const auto first_seen = [&](int token) { return a.window ? max(max(s.first + token, 0) - a.window + 1, 0) : 0; };
  const auto end_seen = [&](int token) { return a.causal ? min(s.first + token + 1, s.length) : s.length; };
  const auto token_of = [&](int r) { return min(r, rows - 1) / share; };
  // what any row of the workgroup sees; what any, and every row of this wave does; what this lane's row does
  const int low_group = first_seen(token_of(r0)), high_group = end_seen(token_of(r0 + ROWS - 1));
  const int r_wave = r0 + wave * 32, r = r_wave + lane % 32, token = token_of(r);
  const int low_any = first_seen(token_of(r_wave)), low_all = first_seen(token_of(r_wave + 31));
  const int high_all = end_seen(token_of(r_wave)), high_any = r_wave < rows ? end_seen(token_of(r_wave + 31)) : 0;
  const int low = first_seen(token), high = end_seen(token);

  const int64_t page_bytes = (int64_t)c.heads * 2 * kPage * BYTES;
  const float factor = a.scale * 1.4426950408889634f;
  const uint32_t sixteens = sixteen<TYPE>(), sixteens_v = sixteen<BMX_BF16>();
  u32x4 in[KN][GROUPS == 1 ? 3 : 2];  // keys, and behind them values; of two groups the first brings in the keys, the second the values
  constexpr int V0 = GROUPS == 1;
  uint32_t pair_in[2] = {};  // wave 0: a token's scale and offset, of keys and of values
  int begin = low_group / kPage, last = kv_pages_to(high_group), used = 1;
  if constexpr (SPLIT) {  // this split's pages: as many for the rows that see few as for those that see most, which then are in fewer splits
    const int pages = max(last - begin, 0), most_pages = kv_pages_to(s.length) - first_seen(token_of((rows - 1) / 128 * 128)) / kPage;
    const int per = max((max(most_pages, pages) + a.prompt_splits - 1) / a.prompt_splits, kLeastPages);
    used = max((pages + per - 1) / per, 1);
    if (split >= used) return;
    last = begin + min(pages, (split + 1) * per);
    begin += split * per;
  }
  const int none = c.num_pages > 0 ? 0 : kNowhere;
  [[maybe_unused]] int ids = -1;  // of two groups: 64 pages' numbers, a lane each
  // the first page from `pg` on that is there, on its way into registers
  const auto fetch = [&](int pg) {
    int page = -1;
    for (; pg < last; ++pg) {
      if constexpr (GROUPS == 1) {
        page = kv_page(c, seq, pg);
      } else {
        if ((pg - begin) % 64 == 0) ids = pg + lane < last ? kv_page(c, seq, pg + lane) : -1;
        page = __builtin_amdgcn_readlane(ids, (pg - begin) % 64);
      }
      if (page >= 0) break;
    }
    // (behind the last page: page 0 once more, which nobody uses)
    const Rsrc r = buffer(c.pages + max(page, 0) * page_bytes + (int64_t)head * 2 * kPage * BYTES, 2 * kPage * BYTES);
    const Rsrc rs = buffer(c.scales + ((int64_t)max(page, 0) * c.heads + head) * 4 * kPage, 8 * kPage);
    if (wave == 0) pair_in[0] = load4(rs, lane * 4 + none, 0), pair_in[1] = load4(rs, lane * 4 + none, 4 * kPage);
#pragma unroll
    for (int n = 0; n < KN; ++n) {
      const int i = min(lane / 16 + 4 * n, DC - 1), block = min(part + 4 * n, DC - 1);
      if (GROUPS == 1 || group == 0) in[n][0] = load16(r, lane % 16 * BYTES + i * 16 + none, part * 16 * BYTES);
      if (GROUPS == 1 || group == 1)
#pragma unroll
        for (int g = 0; g < 2; ++g) in[n][V0 + g] = load16(r, lane / 16 % 2 * 256 + lane % 16 * 16 + none, kPage * BYTES + block * 1024 + g * 512);
    }
    return pg;
  };
  const auto convert = [&](int buf, int slot, int pg) {
    // keys: 32 values of token 16 part + lane % 16; values: of a block a pair's even ones or its odd ones, every other four tokens
    if (GROUPS == 1 || group == 0) {
#pragma unroll
      for (int n = 0; n < KN; ++n) {
        const int i = lane / 16 + 4 * n;
        if (i < DC) {
          u32x4* to = &keys[buf][(part / 2 * NS + 2 * i) * 64 + part % 2 * 16 + lane % 16];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t w = in[n][0][j];
            to[j / 2 * 64 + j % 2 * 32] = u32x4{two_levels<TYPE, 0>(w, sixteens), two_levels<TYPE, 1>(w, sixteens), two_levels<TYPE, 2>(w, sixteens), two_levels<TYPE, 3>(w, sixteens)};
          }
        }
      }
    }
    if (GROUPS == 1 || group == 1) {
#pragma unroll
      for (int n = 0; n < KN; ++n) {
        if (part + 4 * n >= DC) break;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint32_t x = in[n][V0][u] >> (h * 4), y = in[n][V0 + 1][u] >> (h * 4);
          values[slot][(u * DC + part + 4 * n) * 64 + lane / 16 % 2 * 32 + h * 16 + lane % 16] =
              u32x4{two_levels<BMX_BF16, 0>(x, sixteens_v), two_levels<BMX_BF16, 2>(x, sixteens_v), two_levels<BMX_BF16, 0>(y, sixteens_v), two_levels<BMX_BF16, 2>(y, sixteens_v)};
        }
      }
    }
    if (wave == 0) {
      // Those of tokens that nobody has written may be anything, and count as 0.  One that is no finite number, of a value, is left to the score: a weight of 0
      // times it would spoil the rows that do not see the token too.
      float scale[2], offset[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t x = pg * kPage + lane < s.length ? pair_in[i] : 0;
        scale[i] = bf16_float(x), offset[i] = __builtin_bit_cast(float, x & 0xffff0000u);
      }
      const bool none = !(fabsf(scale[1]) < INFINITY && fabsf(offset[1]) < INFINITY);
      float* to = reinterpret_cast<float*>(of_token[slot]) + lane;
      to[0] = scale[0] * factor;
      to[64] = none ? NAN : offset[0] - 16.0f * scale[0];
      to[128] = none ? 0.0f : scale[1];
      to[192] = none ? 0.0f : offset[1] - 16.0f * scale[1];
    }
  };
  int pg = fetch(begin);

  u32x4 q[NS];
  float all = 0.0f;
  {
    const int64_t base = (s.row0 + token) * a.q_row + (head * share + min(r, rows - 1) % share) * a.q_head;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const int d = 16 * i + 8 * h;
      float x[8];
      load_eight<TYPE>(a.q, base + d, c.dim - d, a.aligned, x);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        q[i][j] = TYPE == BMX_F16 ? f16_bits(x[j]) | f16_bits(x[4 + j]) << 16 : upper_halves(x[j], x[4 + j]);
        all += x[j] + x[4 + j];
      }
    }
    all += __shfl_xor(all, 32);
    all *= factor;
  }
  if (pg < last) convert(0, 0, pg);
  // (what LDS holds does not come into registers all at once: there are not as many, and they would spill; where the compiler keeps to them by itself, 347 us without, 356 with)
  const auto fence = [](bool here) {
    if ((DC == 3 || DC > 4 || (DC == 4 && (SPLIT || TYPE == BMX_F16))) && here) __builtin_amdgcn_sched_barrier(0);
  };
  // held: the score that the row's weights are relative to; limit: from where on over it a score becomes the one
  float held = 0.0f, limit = -INFINITY, l = 0.0f, rest = 0.0f;
  f32x16 o[DC] = {}, z[2];
  u32x4 w[2][4];  // [part][16 tokens]
  const auto scores = [&](int buf) {
    z[0] = z[1] = f32x16{};
#pragma unroll
    for (int i = 0; i < NS; ++i) {
#pragma unroll
      for (int t = 0; t < 2; ++t) z[t] = mfma32<TYPE == BMX_F16>(keys[buf][(t * NS + i) * 64 + lane], q[i], z[t]);
      fence(i % 4 == 3);
    }
  };
  // scales and offsets of four tokens, KEEP times: of two groups they are on their way while those before are used
  constexpr int KEEP = 4;
  [[maybe_unused]] f32x4 ks[KEEP][2];
  const auto key_scales = [&](int slot, int j) {
#pragma unroll
    for (int i = 0; i < 2; ++i) ks[j % KEEP][i] = of_token[slot][i][j * 2 + h];
  };
  const auto weights = [&](int slot, int t0) {
    [[maybe_unused]] f32x4 vs[KEEP][2];
    const auto value_scales = [&](int u) {
#pragma unroll
      for (int i = 0; i < 2; ++i) vs[u % KEEP][i] = of_token[slot][2 + i][u * 2 + h];
    };
    const bool whole = __builtin_amdgcn_readfirstlane(kv_all_in(t0, kPage, low_all, high_all));
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int at = t * 4 + j;
        if (GROUPS == 1) key_scales(slot, at);
        else if (at + KEEP - 1 < 8) key_scales(slot, at + KEEP - 1);
        else value_scales(at + KEEP - 9);
        const f32x4 scale = ks[at % KEEP][0], offset = ks[at % KEEP][1];
#pragma unroll
        for (int i = 0; i < 4; ++i) z[t][4 * j + i] = z[t][4 * j + i] * scale[i] + (all * offset[i] - held);
        fence(j % 2);
        if (GROUPS == 2) __builtin_amdgcn_sched_barrier(0);
      }
    if (!whole) {
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const int t = t0 + i / 4 * 8 + 4 * h + i % 4;
        z[i / 16][i % 16] = t < high && t >= low ? z[i / 16][i % 16] : -INFINITY;
      }
      apart(z[0]), apart(z[1]);
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) top = fmaxf(top, z[i / 16][i % 16]);
    top = max_32(top);
    if (__any(top > limit)) {  // (a row's first page, and few others)
      const bool mine = top > limit;
      const float up = mine ? top : 0.0f, shrink = limit == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(-up);
      held += up, limit = mine ? kGrowth : limit;
      l *= shrink, rest *= shrink;
#pragma unroll
      for (int t = 0; t < 2; ++t) z[t] -= up;
#pragma unroll
      for (int n = 0; n < DC; ++n) o[n] *= shrink;
    }
    float sum = 0.0f, more = 0.0f;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (GROUPS == 1) value_scales(u);
      else if (u + KEEP - 1 < 8) value_scales(u + KEEP - 1);
      const f32x4 scale = vs[u % KEEP][0], offset = vs[u % KEEP][1];
      float x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float e = __builtin_amdgcn_exp2f(z[u / 4][u % 4 * 4 + i]);
        sum += e;
        more += e * offset[i];
        x[i] = e * scale[i];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t parts[2];
        pair<2>(x[i], x[i + 2], parts);
        w[0][u / 2][u % 2 * 2 + i] = parts[0], w[1][u / 2][u % 2 * 2 + i] = parts[1];
      }
      fence(u % 2);
      if (GROUPS == 2) __builtin_amdgcn_sched_barrier(0);
    }
    l += sum, rest += more;
  };
  const auto products = [&](int slot) {
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int n0 = 0; n0 < DC; n0 += 4) {
        u32x4 x[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) x[n] = n0 + n < DC ? values[slot][(u * DC + n0 + n) * 64 + lane] : u32x4{};
#pragma unroll
        for (int p = 0; p < 2; ++p)  // (no product waits for the one before)
#pragma unroll
          for (int n = 0; n < 4 && n0 + n < DC; ++n) o[n0 + n] = mfma32<false>(x[n], w[p][u], o[n0 + n]);
        fence(true);
      }
  };
  const auto sees = [&](int pg) { return pg * kPage < high_any && pg * kPage + kPage - 1 >= low_any; };
  if constexpr (GROUPS == 1) {
    __syncthreads();
    for (int buf = 0; pg < last; buf ^= 1) {
      const int next = fetch(pg + 1);
      if (sees(pg)) {
        scores(buf);
        weights(buf, pg * kPage);
        products(buf);
      }
      if (next < last) convert(buf ^ 1, buf ^ 1, next);
      pg = next;
      __syncthreads();
    }
  } else {
    // The second group is a phase behind the first, and both pass as many barriers.  Keys of the page after this one go where those of the page before were, in the first
    // group's phase, which the second has read in the phase before; values, in the second's, where those of two pages before were, and scales, in the first's, likewise.
    // What is brought in behind the last page is read by nobody.
    const auto phase = [&] {
      __builtin_amdgcn_sched_barrier(0);
      __syncthreads();
      __builtin_amdgcn_sched_barrier(0);
    };
    // Products of the page before, then scores of this one, in eight parts: each part's operands are on their way two parts before it.
    const auto both = [&](int before, int buf, int slot, const auto& other) {
      u32x4 x[3][DC];
      const auto load = [&](int b) {
#pragma unroll
        for (int n = 0; n < DC; ++n) {
          const int e = (b - 4) * DC + n;
          x[b % 3][n] = b < 4 ? values[before][(b * DC + n) * 64 + lane] : keys[buf][(e % 2 * NS + e / 2) * 64 + lane];
        }
      };
      load(0);
      load(1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        if (b < 6) load(b + 2);
        if (b >= 5) key_scales(slot, b - 5);
        if (b < 4) {
#pragma unroll
          for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int n = 0; n < DC; ++n) o[n] = mfma32<false>(x[b % 3][n], w[p][b], o[n]);
        } else {
          if (b == 4) z[0] = z[1] = f32x16{};
#pragma unroll
          for (int n = 0; n < DC; ++n) {
            const int e = (b - 4) * DC + n;
            z[e % 2] = mfma32<TYPE == BMX_F16>(x[b % 3][n], q[e / 2], z[e % 2]);
          }
        }
        if (b == 1) other();
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    int next = fetch(pg + 1), before = 0, slot = 0, buf = 0;
#pragma unroll
    for (int u = 0; u < 8; ++u) w[u / 4][u % 4] = u32x4{};  // (before the first page: nothing of that page's own values, which are finite)
    phase();
    if (group == 1) phase();
    for (; pg < last; buf ^= 1) {
      const int after = slot == SLOTS - 1 ? 0 : slot + 1, t0 = pg * kPage;
      const auto other = [&] {
        convert(buf ^ 1, after, next);
        pg = next;
        next = fetch(next + 1);
      };
      __builtin_amdgcn_s_setprio(1);  // (ahead of the other group's weights: 273.6 us, 276.5 without)
      both(before, buf, slot, other);
      __builtin_amdgcn_s_setprio(0);
      phase();
      weights(slot, t0);
      phase();
      before = slot, slot = after;
    }
    products(before);
    if (group == 0) phase();
  }
  l += __shfl_xor(l, 32);
  rest += __shfl_xor(rest, 32);
  if (SPLIT && used > 1) {  // the parts: each lane's numbers at the same place in all of them
    const int64_t unit = ((int64_t)seq * gridDim.y + r0 / 128) * c.heads + head;
    constexpr int PART = 64 * (DC * 16 + 2);
    float* at = a.to.parts + (unit * a.prompt_splits * 4 + wave) * PART + lane * 2;
    if (r_wave < rows) {
      float* to = at + (int64_t)split * 4 * PART;
#pragma unroll
      for (int n = 0; n < DC; ++n)
#pragma unroll
        for (int i = 0; i < 8; ++i) put(to + (n * 8 + i) * 128, o[n][2 * i] + rest, o[n][2 * i + 1] + rest);
      put(to + DC * 1024, limit == -INFINITY ? limit : held, l);
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wave's numbers are there
    __shared__ uint32_t place;
    __syncthreads();
    if (threadIdx.x == 0) place = __hip_atomic_fetch_add(a.to.arrived + unit, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (place != (uint32_t)used - 1) return;
    if (threadIdx.x == 0) __hip_atomic_store(a.to.arrived + unit, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (r_wave >= rows) return;
    float m = -INFINITY;
    l = 0.0f, rest = 0.0f;
    for (int p = 0; p < used; ++p) {
      const float* from = at + (int64_t)p * 4 * PART;
      const u32x2 x = get(from + DC * 1024);
      constexpr int N = DC <= 4 ? DC : 2;
      const uint32_t x0 = x[0], x1 = x[1];
      const float m_part = __builtin_bit_cast(float, x0), m_new = fmaxf(m, m_part), m_at = or_zero(m_new);
      const float f = __builtin_amdgcn_exp2f(m - m_at), f_part = __builtin_amdgcn_exp2f(m_part - m_at);
      l = l * f + __builtin_bit_cast(float, x1) * f_part;
      m = m_new, held = m_at;
#pragma unroll
      for (int n0 = 0; n0 < DC; n0 += N) {
        u32x2 y[N * 8];  // (every read at once: each is a trip to memory)
#pragma unroll
        for (int i = 0; i < N * 8; ++i)
          if (n0 * 8 + i < DC * 8) y[i] = get(from + (n0 * 8 + i) * 128);
#pragma unroll
        for (int n = n0; n < n0 + N && n < DC; ++n)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint32_t v = y[(n - n0) * 8 + i / 2][i % 2];
            o[n][i] = (p == 0 ? 0.0f : o[n][i] * f) + __builtin_bit_cast(float, v) * f_part;
          }
      }
    }
  }
  if (r >= rows) return;
  int right = 8 * h, mine = r;
  asm("" : "+v"(right), "+v"(mine));  // (places are counted anew: kept from where the queries were read, they would be registers through the whole loop)
  const int64_t to = s.row0 + mine / share;
  const int to_head = head * share + mine % share;
  const int64_t at = to * a.to.out_row + to_head * a.to.out_head;
  const float share_of = 1.0f / l;  // (a row that sees nothing is zeros)
#pragma unroll
  for (int n = 0; n < DC; ++n)
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const int d = n * 32 + i * 4 + right;  // eight values from here on
      float x[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[2 * j] = l == 0.0f ? 0.0f : (o[n][i + j] + rest) * share_of;
        x[2 * j + 1] = l == 0.0f ? 0.0f : (o[n][8 + i + j] + rest) * share_of;
      }
      if (d + 8 <= c.dim) {
        Run<TYPE, 8> y;
#pragma unroll
        for (int j = 0; j < 8; j += 2) y.set2(j, x[j], x[j + 1]);
        y.store(a.to.out, at + d, 8);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (d + j < c.dim) store_one<TYPE>(a.to.out, at + d + j, x[j]);
      }
    }
  if (a.to.lse && h == 0)
    a.to.lse[to * a.to.q_heads + to_head] = l == 0.0f ? -INFINITY : (held + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// What a call needs: tiles of rows, parts of their pages, and bytes of the workspace.
struct Plan {
  int64_t units, tiles, prompt_tiles;  // prompt_tiles: of 128 rows, 0 where they are too few to fill the chip
  int part_rows, few, prompt_splits;
  Deal deal;
  bool deep;  // workgroups of eight waves
  size_t bytes;
};
// How the pages of so many tiles are dealt out.  Up to 64 workgroups: over one a CU.  From there on, where lengths differ, 384, half of what the chip holds, with which
// a part takes about as long as all bytes do; but not those that are no longer than others by less than a join takes.  Tiles that fill the chip are split where they
// are far longer than the others only.  (Heads of 128 bf16, 8 of the cache, us with 256, 384, 512 workgroups: 16 sequences of up to 16000 tokens 51, 42, 45, unsplit 60; 48 of
// up to 8000 71, 55, 64, unsplit 79; 32 of 2000 each 19.8, 19.7, 23.7; 16 of 4000 each, four new tokens 25, 28, 25; 64 of up to 4096 44.5, 45.7, 48.6, unsplit 44.)
Deal deal_of(int64_t units, int64_t heads, int64_t table_width) {
  if (units == 0 || units > kMostUnits || units * heads > kMostPlaces || table_width <= kWholePages || units * table_width >= 1 << 30) return {0, 0, 0};
  const int64_t fill = units * heads, most = std::min<int64_t>(units * ceil_div(table_width, kLeastPart), kMostSplits) - 1;
  const auto extra = [&](int64_t places) { return (int)std::min(ceil_div(places, heads) - 1, most); };
  const Deal d = {extra(fill > 64 && fill < kPlaces ? 384 : 256), extra(256), fill < 256 ? 4 : 14};
  return d.even > 0 ? d : Deal{0, 0, 0};
}
Plan plan(int64_t sequences, int64_t table_width, int64_t heads, int64_t q_heads, int64_t dim, int64_t max_new, int type) {
  Plan p;
  int64_t rows = max_new * (q_heads / heads);
  p.few = 0x7fffffff;
  p.prompt_tiles = 0;
  if (type != BMX_F32 && ceil_div(rows, 128) * heads * sequences >= kLeastTiles && rows > 64) {
    p.prompt_tiles = ceil_div(rows, 128);
    p.few = 64;
    rows = 64;
  }
  const size_t line = (kv4_row_bytes((int)dim) * 2 + 4) * 4;
  p.tiles = ceil_div(rows, 16);
  p.units = sequences * p.tiles;
  p.part_rows = (int)std::min<int64_t>(rows, 16);
  p.deal = deal_of(p.units, heads, table_width);
  p.deep = p.deal.extra > 0 && p.units == 1 && table_width >= 16 * (p.deal.extra + 1);
  p.bytes = p.deal.extra == 0 ? 0 : kCounters * 4 + (size_t)(p.units + p.deal.extra) * heads * p.part_rows * line;
  p.prompt_splits = 1;
  if (p.prompt_tiles) {
    const int64_t units = p.prompt_tiles * heads * sequences;
    // as many workgroups as the chip holds at once, two a CU up to 128 values and one beyond, of 16 pages each at least
    p.prompt_splits = (int)std::max<int64_t>(std::min<int64_t>((dim <= 128 ? 512 : 256) / units, table_width / kLeastPages), 1);
    if (p.prompt_splits > 1) p.bytes = std::max(p.bytes, kCounters * 4 + (size_t)units * p.prompt_splits * 128 * line);
  }
  return p;
}

// Whether prompts go to workgroups of two groups, one a CU, whose first reads nobody covers: where they have many pages, are alike and fill the rounds of the chip's
// CUs.  (us in one group, in two, 32 heads on 8 of 128 bf16, sequences x new tokens of all: 2 x 1024 of 2048 103, 90, of 1536 78, 69; 4 x 1024 of 4096 359, 332, of 2048 169,
// 165, of 1536 120, 123; 16 x 512 of 512 93, 106; 4 x 1024 of 1024 75, 84; 3 x 700 of 2700, a round of 256 and one of 8, 171, 181; 2 x 1600 of 4096 284, 257; 2 x 2048 of 2048 118,
// 109, but one of these alone, in one round with the short ones, 78, 83; a window of 512 69, 73; 6 ragged ones 124, 129.)  The host knows the table's width alone, and these tables
// are as wide as their sequences are long: with wider ones short prompts go to two groups too (4 x 1024 of 1024 82 us, 75 in one; 16 x 512 of 512 101, 87).
bool two_groups(const bmx_kv4_cache& c, const Args& a, const Plan& p) {
  if (p.prompt_splits > 1 || (c.starts && c.sequences > 1)) return false;
  const int64_t tiles = ceil_div(p.prompt_tiles, 2) * c.heads * c.sequences, rounds = ceil_div(tiles, 256);
  const int64_t most = a.window ? std::min(c.table_width, a.window / kPage + 2) : c.table_width, mean = a.window || !a.causal ? most : most - a.max_new / (2 * kPage);
  return 4 * tiles >= 3 * 256 * rounds && mean >= 16 && (rounds > 1 || 3 * mean >= 2 * most);
}

template <int TYPE, int DC>
void launch(const bmx_kv4_cache& c, const Args& a, const Plan& p, hipStream_t s) {
  // (rows of sequences as long as each other are all many or all few)
  if (!p.prompt_tiles || (c.starts && c.sequences > 1)) {
    const dim3 grid = p.deal.extra ? dim3((uint32_t)(c.heads * (p.units + p.deal.extra))) : dim3(c.heads, (uint32_t)p.tiles, c.sequences);
    int waves = 4;
    auto kern = kv4_attention_kernel<TYPE, DC, 4>;
    if constexpr (DC <= 4)  // (beyond 128 values eight waves' registers do not fit)
      if (p.deep) kern = kv4_attention_kernel<TYPE, DC, 8>, waves = 8;
    launch_kernel(kern, grid, dim3(waves * 64), 0, s, c, a);
    note_kernel("kv4_attention_kernel<%d,%d,%d> grid %ux%ux%u block %d", TYPE, DC, waves, grid.x, grid.y, grid.z, waves * 64);
  }
  if constexpr (TYPE != BMX_F32) {
    if (p.prompt_tiles) {
      int groups = 1;
      auto kern = p.prompt_splits > 1 ? kv4_prompt_kernel<TYPE, DC, true, 1> : kv4_prompt_kernel<TYPE, DC, false, 1>;
      if constexpr (DC <= 4)
        if (two_groups(c, a, p)) kern = kv4_prompt_kernel<TYPE, DC, false, 2>, groups = 2;
      const dim3 grid(c.heads * p.prompt_splits, (uint32_t)ceil_div(p.prompt_tiles, groups), c.sequences);
      Args b = a;
      if (!c.starts || c.sequences == 1) b.few = 0;
      launch_kernel(kern, grid, dim3(256 * groups), 0, s, c, b);
      note_kernel("kv4_prompt_kernel<%d,%d,%d,%d> grid %ux%ux%u block %d", TYPE, DC, p.prompt_splits > 1, groups, grid.x, grid.y, grid.z, 256 * groups);
    }
  }
}
template <int TYPE>
void launch_typed(const bmx_kv4_cache& c, const Args& a, const Plan& p, hipStream_t s) {
  const int dc = kv4_row_bytes(c.dim) / 16;
  const auto f = dc == 1 ? launch<TYPE, 1> : dc == 2 ? launch<TYPE, 2> : dc == 3 ? launch<TYPE, 3> : dc == 4 ? launch<TYPE, 4>
               : dc == 5 ? launch<TYPE, 5> : dc == 6 ? launch<TYPE, 6> : dc == 7 ? launch<TYPE, 7> : launch<TYPE, 8>;
  f(c, a, p, s);
}

__global__ void clear_kernel(uint32_t* p) { p[blockIdx.x * 256 + threadIdx.x] = 0; }

}  // namespace

size_t kv4_attention_workspace(int64_t sequences, int64_t table_width, int64_t heads, int64_t q_heads, int64_t dim, int64_t max_new) {
  // The largest of the calls' bytes.  Of 16 rows a part: that of any number of tiles, of which each sequence has as many.
  const int64_t each = sequences * heads, rows = max_new > 0 ? std::min(max_new * (q_heads / heads), kMostTiles * 16) : kMostTiles * 16;
  const size_t line = (kv4_row_bytes((int)dim) * 2 + 4) * 4;
  size_t most = 0;
  if (each == 0) return 0;
  for (int64_t tiles = 1; tiles <= std::min(ceil_div(rows, 16), (int64_t)kMostUnits); ++tiles) {
    const int64_t extra = deal_of(sequences * tiles, heads, table_width).extra;
    if (extra > 0) most = std::max<size_t>(most, (sequences * tiles + extra) * heads * std::min<int64_t>(rows, 16) * line);
  }
  const int64_t places = dim <= 128 ? 512 : 256, tiles = each * std::min(ceil_div(rows, 128), places / 2 / each);
  if (rows > 64 && tiles >= kLeastTiles && table_width / kLeastPages > 1)
    most = std::max<size_t>(most, std::min(places, tiles * (table_width / kLeastPages)) * 128 * line);
  return most ? kCounters * 4 + most : 0;
}

size_t kv4_attention_workspace_of_call(int64_t sequences, int64_t table_width, int64_t heads, int64_t q_heads, int64_t dim, int64_t max_new) {
  // (whatever the type)
  return std::max(plan(sequences, table_width, heads, q_heads, dim, max_new, BMX_F32).bytes,
                  plan(sequences, table_width, heads, q_heads, dim, max_new, BMX_F16).bytes);
}

hipError_t launch_kv4_attention(const bmx_kv4_cache& c, const void* q, int type, int64_t q_row, int64_t q_head, int q_heads, int rows,
                                int max_new, float scale, bool causal, int window, void* out, int64_t out_row, int64_t out_head, float* lse,
                                void* workspace, bool fresh, hipStream_t s) {
  const int64_t size = type_bytes(type);
  const bool aligned = (uintptr_t)q % 16 == 0 && q_row * size % 16 == 0 && q_head * size % 16 == 0;
  const Plan p = plan(c.sequences, c.table_width, c.heads, q_heads, c.dim, max_new, type);
  uint32_t* arrived = static_cast<uint32_t*>(workspace);
  const Args a = {q, q_row, q_head, {out, out_row, out_head, lse, reinterpret_cast<float*>(arrived + kCounters), arrived, q_heads, q_heads / c.heads, p.part_rows},
                  rows, max_new, window, p.prompt_splits, p.deal, p.deal.extra ? (int)p.units : 0, (int)p.tiles, p.few, causal, aligned, scale};
  const int64_t counters = std::max(p.deal.extra ? p.units * c.heads : 0, p.prompt_splits > 1 ? p.prompt_tiles * c.heads * c.sequences : 0);
  if (fresh && counters) launch_kernel(clear_kernel, dim3((uint32_t)ceil_div(counters, 256)), dim3(256), 0, s, arrived);
  const auto f = type == BMX_F32 ? launch_typed<BMX_F32> : type == BMX_F16 ? launch_typed<BMX_F16> : launch_typed<BMX_BF16>;
  f(c, a, p, s);
  return launch_error();
}

}  // namespace bmx
