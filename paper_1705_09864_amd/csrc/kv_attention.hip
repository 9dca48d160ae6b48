// Attention of new tokens over the paged cache of 8 bits (kv_cache.hip):
//   o = sum_t p_t v_t / sum_t p_t,  p_t = exp(scale * q . k_t),  k_t = a_b * (levels of t), v_t = c_b * (levels of t),
// over the tokens t that a row sees, b their block.  One pass over the cache with the running maximum m of the scores and the running
// sum, both in 32 bits.  Products are S^T = K Q^T and O^T = V^T P^T on the matrix cores (16 x 16 x 32), 16 rows of queries (tokens x heads that share
// a head of the cache) at a time: levels are whole numbers that 16-bit floats hold exactly, and the scales come to the scores and weights behind
// and before the products.  A lane's scores of S^T are those of its own column of P^T, in the order of tokens in which the cache
// holds values, so the weights never leave their lane.
// For 16-bit results the products are f16's:
//   q goes in with its row's largest value brought to [128, 256) by a power of two (exact but for values 2^-21 below the row's largest);
//   p goes in as p * c_b / W * 2^14 with W the row's own largest |p c_b| so far: at most 2^14, and with all of f16's 11 bits down to 2^-28 of that.
//   So neither tokens that the row does not see nor values without weight say how well the others are held.  W is kept as its logarithm, `lead`,
//   relative to the running maximum.  11 bits beside results of 11 or 8: error against 64 bits, f16, 5 rows over a window of 1000 2.4e-4, with weights in 32 bits 2.1e-4;
//   bf16, all cases, 1.7e-3 with either.
// For f32 results they are bf16's, q and p * c_b in three parts of 8 bits each, which together are all of them whatever the range; levels
// are exact in bf16 too.
//
// Bound by the cache's bytes: a wave goes over pages of its own (16 KB at 128 values a head) with its queries, running maxima, sums and
// results in registers, and requests the next page's keys as soon as this one's are used up, its values as soon as these are.  A workgroup's
// four waves join their parts through LDS.  Where rows x heads are few, a sequence's pages are split over workgroups too: each leaves
// its rows' sums in the workspace, and the last of them to arrive (a counter there, back at 0 behind the call) joins them, in their order, so
// the result does not depend on which that was.
//   Measured (bf16, 32 heads on 8 of 128 values): one token over 131072, 268 MB: 57 us, 4.7 TB/s (a large copy moves 4.8); one token each
// over 64 sequences of up to 4096, 269 MB: 60 us; over 4096: 10.7 us, of which the join takes 3.  Two pages on their way a wave, or eight
// waves: no faster where bytes bound it, and 1 us slower on short sequences, where the conversions' instructions do (2 us a page with two
// waves on a SIMD, 1 with one).
#include "bmx_internal.h"
#include "few_bits.h"

#include <algorithm>

namespace bmx {
namespace {


// Four levels of a dword as pairs of 16-bit floats.
template <bool F16>
__device__ inline u32x2 four_levels(uint32_t w) {
  if constexpr (F16) {  // q + 128 in the low bits of 1024, less 1152
    w ^= 0x80808080u;
    const f16x2 off = {(_Float16)-1152.0f, (_Float16)-1152.0f};
    const f16x2 a = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) + off;
    const f16x2 b = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) + off;
    return u32x2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
  } else {  // (a whole number below 256 has nothing in the lower half of an f32)
    const float a = (float)(int8_t)w, b = (float)(int8_t)(w >> 8), c = (float)(int8_t)(w >> 16), d = (float)((int32_t)w >> 24);
    return u32x2{upper_halves(a, b), upper_halves(c, d)};
  }
}
template <bool F16>
__device__ inline u32x4 eight_levels(uint32_t a, uint32_t b) {
  const u32x2 x = four_levels<F16>(a), y = four_levels<F16>(b);
  return u32x4{x[0], x[1], y[0], y[1]};
}
template <bool F16>
__device__ inline f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
using f32x16 = float __attribute__((ext_vector_type(16)));
__device__ inline f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// Two values as one pair of f16, or as three pairs of bf16.  The parts' bits are cut off, not rounded: the compiler folds a product into one
// use of a conversion and not into another, and what is left would then belong to another part than the one in use.
template <int PARTS>
__device__ inline void pair(float a, float b, uint32_t (&part)[PARTS]) {
  if constexpr (PARTS == 1) {
    part[0] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
  } else {
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      part[p] = upper_halves(a, b);
      a = lower_part(a), b = lower_part(b);
    }
  }
}

// Numbers that workgroups of other XCDs read, each with an L2 of its own: written through and read past it (relaxed atomics of the device's
// scope, eight bytes each), so nobody has to write back or throw away a whole L2, as a fence of that scope does: with __threadfence()
// around plain accesses, 64 sequences in two splits ran for 325 us, 110 in one.
__device__ inline void put(float* p, float a, float b) {
  const uint64_t x = __builtin_bit_cast(uint32_t, a) | (uint64_t)__builtin_bit_cast(uint32_t, b) << 32;
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline u32x2 get(const float* p) {
  return __builtin_bit_cast(u32x2, __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
__device__ inline f32x4 get4(const float* p) {
  const u32x2 a = get(p), b = get(p + 2);
  return __builtin_bit_cast(f32x4, u32x4{a[0], a[1], b[0], b[1]});
}

// A value's scale times what a row's weights are multiplied with.  Bounded, as a weight of 0 has to bring 0 where the row's other weights times scales
// are far below this scale; NaN stays.
__device__ inline float bounded(float x) { return fabsf(x) > 0x1.fffffep127f ? copysignf(0x1.fffffep127f, x) : x; }
// A rounded product as it is, at the place where it is used: the barrier keeps it from becoming one operation with the difference from the maximum, which is
// of rounded products (of scores beyond 2^24 that difference need not be below 0 then, and 2 to its power not below 1).
__device__ inline float rounded(float z) {
  asm("" : "+v"(z));
  return z;
}
__device__ inline float or_zero(float x) { return x == -INFINITY ? 0.0f : x; }
constexpr float kLargeScore = 0x1p20f;  // scores from here on lose too much beside a scale's logarithm: its sums are taken relative to the maximum
constexpr float kLeastLead = -100.0f;  // (so that its power stays a number: a row whose weights times scales are all below 2^-100 is held to that)

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

struct Args {
  const void* q;
  int64_t q_row, q_head;
  void* out;
  int64_t out_row, out_head;
  float* lse;
  float* parts;      // [sequence, tile of rows, head][split][part_rows][ROW + 4]: the rows' results, maximum and sum (of many rows: as their lanes hold them)
  uint32_t* arrived; // [sequence, tile of rows, head]
  int q_heads, share, rows, max_new, window, splits, part_rows, prompt_splits;
  int few;  // sequences of more rows than this are the other kernel's
  bool causal, aligned;
  float scale;
};

constexpr int kWaves = 4;
constexpr int kCounters = 16384;  // of the workspace's head; what needs more than these has rows enough not to be split
constexpr int kMostSplits = 128;
constexpr int kLeastPages = 16;   // of a split of many rows
// Tiles of 128 rows for the kernel for many.  With fewer the two are level by lengths, which only the device knows: 256 new tokens (64 tiles, 32 heads on 8 of
// 128) over 512 13 us in 16 rows and 27 in 128, over 4096 49 and 49, over 16384 173 and 118; 128 new ones over 4096 32 and 49, over 65536 396 and 220.
constexpr int kLeastTiles = 128;
constexpr int64_t kMostTiles = 65535;  // of 16 rows: a launch's second dimension

template <int TYPE, int DC>
__global__ __launch_bounds__(kWaves * 64) void kv_attention_kernel(bmx_kv_cache c, Args a) {
  constexpr int PARTS = TYPE == BMX_F32 ? 3 : 1, ROW = DC * 32, DT = DC * 2, WIDE = DC / 2;
  constexpr bool F16 = PARTS == 1;
  constexpr int LINE = ROW + 4;
  __shared__ float red[kWaves * 16 * LINE], red_m[kWaves][16], red_l[kWaves][16], factor_of[kMostSplits][16], sum_of[kMostSplits][16];
  __shared__ uint32_t place;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), g = lane / 16;
  const int head = blockIdx.x % c.heads, split = blockIdx.x / c.heads, seq = blockIdx.z;
  const KvSpan s = kv_span(c, seq, a.rows, a.max_new);
  const int r0 = blockIdx.y * 16;
  if (r0 >= s.count * a.share || s.count * a.share > a.few) return;
  // what any, and what every one of the 16 rows sees: positions [low, high)
  const int tok0 = r0 / a.share, tok1 = min((r0 + 15) / a.share, s.count - 1);
  const int high_any = a.causal ? min(s.first + tok1 + 1, s.length) : s.length, high_all = a.causal ? min(s.first + tok0 + 1, s.length) : s.length;
  const int low_any = a.window ? max(max(s.first + tok0, 0) - a.window + 1, 0) : 0, low_all = a.window ? max(max(s.first + tok1, 0) - a.window + 1, 0) : 0;
  // this workgroup's pages
  const int page0 = low_any / kPage, pages = max(kv_pages_to(high_any) - page0, 0);
  // (to join parts takes as long as two pages of a wave, so up to three pages each stay in one workgroup: 8 pages 7.8 us, in two 9.3;
  // 16 pages 10.6, in four 9.3)
  const int per = pages <= 3 * kWaves ? pages : max((pages + a.splits - 1) / a.splits, kWaves), used = pages > 0 ? (pages + per - 1) / per : 1;
  if (split >= used) return;
  const int begin = page0 + split * per, count = max(min(per, pages - split * per) - wave + kWaves - 1, 0) / kWaves;  // (of this wave, kWaves apart)

  const int blocks = kPage / c.block, log_block = 31 - __builtin_clz(c.block);
  const int64_t page_bytes = (int64_t)c.heads * 2 * kPage * ROW;
  int ids = -1, next = 0;  // the numbers of 64 pages, a lane each; the place of the next page
  int page, at;  // the page on its way, and its place
  u32x4 k[4][WIDE > 0 ? WIDE : 1], v[DT];
  u32x2 k_tail[4];
  float scale_of;  // lanes 0 to 3: a page's scales of keys, a unit of 16 tokens each; 4 to 7: of values
  const int scale_at = (lane / 4 % 2) * blocks + (lane % 4 * 16 >> log_block);
  // the next of this wave's pages that is there, and its keys
  const auto load_keys = [&] {
    page = -1;
    for (; next < count; ++next) {
      if (next % 64 == 0) ids = next + lane < count ? kv_page(c, seq, begin + wave + (next + lane) * kWaves) : -1;
      page = __builtin_amdgcn_readlane(ids, next % 64);
      if (page >= 0) break;
    }
    at = next++;
    const int none = page >= 0 ? 0 : kNowhere;
    const Rsrc r = buffer(c.pages + max(page, 0) * page_bytes + (int64_t)head * 2 * kPage * ROW, kPage * ROW);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
#pragma unroll
      for (int w = 0; w < WIDE; ++w) k[u][w] = load16(r, lane * 16 + none, u * 16 * ROW + w * 1024);
      if constexpr (DC % 2) k_tail[u] = load8(r, lane * 8 + none, u * 16 * ROW + WIDE * 1024);
    }
    const Rsrc rs = buffer(c.scales + ((int64_t)max(page, 0) * c.heads + head) * 2 * blocks, 8 * blocks);
    scale_of = __builtin_bit_cast(float, load4(rs, scale_at * 4 + none, 0));
  };
  const auto load_values = [&] {
    const int none = page >= 0 ? 0 : kNowhere;
    const Rsrc r = buffer(c.pages + max(page, 0) * page_bytes + (int64_t)(head * 2 + 1) * kPage * ROW, kPage * ROW);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) v[dt] = load16(r, lane * 16 + none, dt * 1024);
  };
  load_keys();
  load_values();

  // this lane's row of queries
  const int r = r0 + lane % 16, token = min(r / a.share, s.count - 1), pos = s.first + token;
  const int high = a.causal ? min(pos + 1, s.length) : s.length, low = a.window ? max(max(pos, 0) - a.window + 1, 0) : 0;
  u32x4 q[PARTS][DC];
  float factor;
  {
    const int64_t base = (s.row0 + token) * a.q_row + (head * a.share + r % a.share) * a.q_head;
    float x[DC][8], top = 0.0f;
#pragma unroll
    for (int i = 0; i < DC; ++i) {
      // step i of the products takes these values of a token: the order in which the cache holds keys
      const int d = i < 2 * WIDE ? i / 2 * 64 + 16 * g + i % 2 * 8 : WIDE * 64 + 8 * g;
      load_eight<TYPE>(a.q, base + d, c.dim - d, a.aligned, x[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(x[i][j]));
    }
    int e = 0;
    if constexpr (F16) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      if (top > 0.0f && top < INFINITY) (void)frexpf(top, &e);
      e -= 8;
    }
    factor = ldexpf(a.scale * 1.4426950408889634f, e);
#pragma unroll
    for (int i = 0; i < DC; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t part[PARTS];
        pair<PARTS>(F16 ? ldexpf(x[i][2 * j], -e) : x[i][2 * j], F16 ? ldexpf(x[i][2 * j + 1], -e) : x[i][2 * j + 1], part);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) q[p][i][j] = part[p];
      }
  }

  float m = -INFINITY, l = 0.0f, lead = kLeastLead;
  f32x4 o[DT] = {};
  while (page >= 0) {
    const int t0 = (begin + wave + at * kWaves) * kPage;
    float p[4][4], key_scale[4], value_scale[4], value_log[4], tops[4];
    const float log_of = F16 ? __builtin_amdgcn_logf(fabsf(scale_of)) : 0.0f;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      key_scale[u] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, scale_of), u));
      value_scale[u] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, scale_of), 4 + u));
      if constexpr (F16) value_log[u] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, log_of), 4 + u));
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      f32x4 z = {};
#pragma unroll
      for (int w = 0; w < WIDE; ++w) {
        const u32x4 k0 = eight_levels<F16>(k[u][w][0], k[u][w][1]), k1 = eight_levels<F16>(k[u][w][2], k[u][w][3]);
#pragma unroll
        for (int part = 0; part < PARTS; ++part) z = mfma<F16>(k1, q[part][2 * w + 1], mfma<F16>(k0, q[part][2 * w], z));
      }
      if constexpr (DC % 2) {
        const u32x4 k0 = eight_levels<F16>(k_tail[u][0], k_tail[u][1]);
#pragma unroll
        for (int part = 0; part < PARTS; ++part) z = mfma<F16>(k0, q[part][DC - 1], z);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) p[u][i] = z[i];
    }
    load_keys();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float f = factor * key_scale[u];
#pragma unroll
      for (int i = 0; i < 4; ++i) p[u][i] *= f;
      tops[u] = fmaxf(fmaxf(fmaxf(p[u][0], p[u][1]), p[u][2]), p[u][3]);
    }
    if (!kv_all_in(t0, kPage, low_all, high_all)) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int t = t0 + 16 * u;
        if (t >= high || t + 15 < low) value_scale[u] = 0.0f;  // (a block that the row does not see, or that nobody has written, has any scale)
#pragma unroll
        for (int i = 0; i < 4; ++i) p[u][i] = t + 4 * g + i < high && t + 4 * g + i >= low ? p[u][i] : -INFINITY;
        tops[u] = fmaxf(fmaxf(fmaxf(p[u][0], p[u][1]), p[u][2]), p[u][3]);
      }
    }
    float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])), ahead = -INFINITY;
#pragma unroll
    for (int u = 0; u < 4; ++u) ahead = F16 ? fmaxf(ahead, tops[u] + value_log[u]) : 0.0f;
    top = max_32(max_16(top));
    if constexpr (F16) ahead = max_32(max_16(ahead));
    const float m_new = fmaxf(m, top), m_at = or_zero(m_new), shrink = __builtin_amdgcn_exp2f(m - m_at);
    float sum = 0.0f, shrink_o = shrink, unit = 1.0f;
    if constexpr (F16) {
      const float before = lead + (m - m_at);
      ahead -= m_at;
      if (__any(fabsf(m_at) >= kLargeScore)) {
        ahead = -INFINITY;
#pragma unroll
        for (int u = 0; u < 4; ++u) ahead = fmaxf(ahead, tops[u] - m_at + value_log[u]);
        ahead = max_32(max_16(ahead));
      }
      lead = fmaxf(fmaxf(before, ahead), kLeastLead);
      shrink_o = __builtin_amdgcn_exp2f(before - lead);
      unit = __builtin_amdgcn_exp2f(-lead);
    }
    m = m_new;
    u32x4 w[PARTS][2];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float f = F16 ? bounded(value_scale[u] * unit * 0x1p14f) : value_scale[u];
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        const float e0 = __builtin_amdgcn_exp2f(rounded(p[u][i]) - m_at), e1 = __builtin_amdgcn_exp2f(rounded(p[u][i + 1]) - m_at);
        sum += e0 + e1;
        uint32_t part[PARTS];
        pair<PARTS>(e0 * f, e1 * f, part);
#pragma unroll
        for (int k = 0; k < PARTS; ++k) w[k][u / 2][u % 2 * 2 + i / 2] = part[k];
      }
    }
    l = l * shrink + sum;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const u32x4 v0 = eight_levels<F16>(v[dt][0], v[dt][1]), v1 = eight_levels<F16>(v[dt][2], v[dt][3]);
      o[dt] *= shrink_o;
#pragma unroll
      for (int part = 0; part < PARTS; ++part) o[dt] = mfma<F16>(v1, w[part][1], mfma<F16>(v0, w[part][0], o[dt]));
    }
    load_values();
  }

  // the four waves' parts
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (g == 0) red_m[wave][lane] = m, red_l[wave][lane] = l;
  const float unit_of = __builtin_amdgcn_exp2f(lead) * 0x1p-14f;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
    *reinterpret_cast<f32x4*>(&red[(wave * 16 + lane % 16) * LINE + dt * 16 + 4 * g]) = F16 ? o[dt] * unit_of : o[dt];
  __syncthreads();
  const int rows = min(s.count * a.share - r0, 16), quads = rows * (ROW / 4);
  const int64_t unit = ((int64_t)seq * gridDim.y + blockIdx.y) * c.heads + head;
  float* parts = a.parts + unit * a.splits * a.part_rows * LINE;
  const auto store = [&](int i, int d, f32x4 x, float top, float sum) {
    const int64_t t = s.row0 + (r0 + i) / a.share;
    const int h = head * a.share + (r0 + i) % a.share;
#pragma unroll
    for (int j = 0; j < 4; ++j)  // (a row that sees nothing is zeros)
      if (d + j < c.dim) store_one<TYPE>(a.out, t * a.out_row + h * a.out_head + d + j, sum == 0.0f ? 0.0f : x[j] / sum);
    if (a.lse && d == 0) a.lse[t * a.q_heads + h] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
  };
  for (int e = threadIdx.x; e < quads; e += kWaves * 64) {
    const int i = e / (ROW / 4), d = e % (ROW / 4) * 4;
    float top = -INFINITY, sum = 0.0f;
    f32x4 x = {};
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, red_m[w][i]);
    const float m_at = top == -INFINITY ? 0.0f : top;
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(red_m[w][i] - m_at);
      sum += f * red_l[w][i];
      x += f * *reinterpret_cast<const f32x4*>(&red[(w * 16 + i) * LINE + d]);
    }
    if (used == 1) {
      store(i, d, x, m_at, sum);
    } else {
      float* line = parts + ((int64_t)split * a.part_rows + i) * LINE;
      put(line + d, x[0], x[1]), put(line + d + 2, x[2], x[3]);
      if (d == 0) put(line + ROW, top, sum);
    }
  }
  if (used == 1) return;

  // the workgroups' parts: the last to arrive joins them
  __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wave's numbers are there
  __syncthreads();
  if (threadIdx.x == 0) place = __hip_atomic_fetch_add(a.arrived + unit, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (place != (uint32_t)used - 1) return;
  if (threadIdx.x == 0) __hip_atomic_store(a.arrived + unit, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  // (every read of a step at once: each is a trip to memory)
  for (int e = threadIdx.x; e < used * 16; e += kWaves * 64) {
    const int p = e / 16, i = e % 16;
    if (i >= rows) continue;
    const float* line = parts + ((int64_t)p * a.part_rows + i) * LINE;
    const u32x2 x = get(line + ROW);
    const uint32_t top = x[0], sum = x[1];
    factor_of[p][i] = __builtin_bit_cast(float, top), sum_of[p][i] = __builtin_bit_cast(float, sum);
  }
  __syncthreads();
  if (threadIdx.x < 64) {  // a row's maximum and sum, four lanes to a row, and what each part counts for
    const int i = threadIdx.x / 4, sub = threadIdx.x % 4;
    float top = -INFINITY, sum = 0.0f;
    for (int p = sub; p < used; p += 4) top = fmaxf(top, factor_of[p][i]);
    top = fmaxf(top, __shfl_xor(top, 1));
    top = fmaxf(top, __shfl_xor(top, 2));
    const float m_at = top == -INFINITY ? 0.0f : top;
    for (int p = sub; p < used; p += 4) {
      const float f = __builtin_amdgcn_exp2f(factor_of[p][i] - m_at);
      factor_of[p][i] = f;
      sum += f * sum_of[p][i];
    }
    sum += __shfl_xor(sum, 1);
    sum += __shfl_xor(sum, 2);
    if (sub == 0) red_m[0][i] = m_at, red_l[0][i] = sum;
  }
  __syncthreads();
  // the results, four values to a thread; where they are fewer than threads, the parts are dealt out too
  const int deal = max(kWaves * 64 / quads, 1);
  for (int e = threadIdx.x; e < quads * deal; e += kWaves * 64) {
    const int i = e % quads / (ROW / 4), d = e % quads % (ROW / 4) * 4;
    f32x4 x = {};
    for (int p = e / quads; p < used; p += 8 * deal) {
      f32x4 y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = get4(parts + ((int64_t)min(p + j * deal, used - 1) * a.part_rows + i) * LINE + d);
#pragma unroll
      for (int j = 0; j < 8; ++j) x += (p + j * deal < used ? factor_of[min(p + j * deal, used - 1)][i] : 0.0f) * y[j];
    }
    *reinterpret_cast<f32x4*>(&red[e * 4]) = x;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < quads; e += kWaves * 64) {
    f32x4 x = {};
    for (int p = 0; p < deal; ++p) x += *reinterpret_cast<const f32x4*>(&red[(p * quads + e) * 4]);
    const int i = e / (ROW / 4);
    store(i, e % (ROW / 4) * 4, x, red_m[0][i], red_l[0][i]);
  }
}

// Many rows: 128 of one head of the cache per workgroup, 32 a wave, over all pages that any of them sees.  A page comes into LDS once for
// the four waves, as 16-bit floats in the order of the 32 x 32 x 16 products' operands (a wave brings in a quarter of it, a page ahead, and
// converts it on its way), and a lane has one row's scores of 16 of 32 tokens, which again are those of its own column of P^T.
// Bound by the vector ALU: 64 tokens x 32 rows are 32 matrix-core products, 1024 cycles, and 32 exponentials, maxima, conversions a lane,
// 1600 cycles, and of two waves on a SIMD the one's products overlap little with the other's instructions (counters: matrix cores busy
// 29% of the time, vector ALU 50%).  2 prompts of 2048 new tokens over 4096, 32 heads on 8 of 128: 283 to 297 us by the card, 690 to 730 TFLOP/s; 16 rows a wave, each
// with pages of its own, 508.  The next page's scores computed beside this page's exponentials, which takes more registers than two
// waves have: 385.
// So where all of a page is seen and no scale of its values is far below the row's W, the scale goes into the exponent,
//   p c / W 2^14 = 2^(s + log2(c / W 2^14) - m),
// and comes out of the sum of p again once for each 16 tokens.
// SPLIT: tiles of rows fewer than the chip holds workgroups at once, whose pages are split and joined as above (a kernel of its own: the
// splits' arithmetic in the one kernel cost it 1%).  512 new tokens over 4096: 70 us, 120 unsplit; the join is some 15 us of that.
// Eight waves to a page, which halves the conversions, fill the chip less evenly: 272 us where 289 was, but 163 where 122, 713 where 677.
template <int TYPE, int DC, bool SPLIT>
__global__ __launch_bounds__(256, DC <= 4 ? 2 : 1) void kv_prompt_kernel(bmx_kv_cache c, Args a) {
  static_assert(TYPE != BMX_F32, "");
  constexpr int ROW = DC * 32, WIDE = DC / 2, NS = DC * 2, VN = (DC + 3) / 4;  // NS: steps of 16 values; VN: 32-value tiles of V a wave brings in
  __shared__ u32x4 lds[2][2][NS * 128];                          // [buffer][keys, values]
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), h = lane / 32;
  const int head = SPLIT ? blockIdx.x % c.heads : blockIdx.x, split = SPLIT ? blockIdx.x / c.heads : 0, seq = blockIdx.z;
  const KvSpan s = kv_span(c, seq, a.rows, a.max_new);
  const int rows = s.count * a.share;
  const int r0 = ((rows + 127) / 128 - 1 - (int)blockIdx.y) * 128;  // (the last rows, which see most, first)
  if (r0 < 0 || rows <= a.few) return;
  const auto first_seen = [&](int token) { return a.window ? max(max(s.first + token, 0) - a.window + 1, 0) : 0; };
  const auto end_seen = [&](int token) { return a.causal ? min(s.first + token + 1, s.length) : s.length; };
  const auto token_of = [&](int r) { return min(r, rows - 1) / a.share; };
  // what any row of the workgroup sees; what any, and every row of this wave does; what this lane's row does
  const int low_group = first_seen(token_of(r0)), high_group = end_seen(token_of(r0 + 127));
  const int r_wave = r0 + wave * 32, r = r_wave + lane % 32, token = token_of(r);
  const int low_any = first_seen(token_of(r_wave)), low_all = first_seen(token_of(r_wave + 31));
  const int high_all = end_seen(token_of(r_wave)), high_any = r_wave < rows ? end_seen(token_of(r_wave + 31)) : 0;
  const int low = first_seen(token), high = end_seen(token);

  const int blocks = kPage / c.block, log_block = 31 - __builtin_clz(c.block);
  const int64_t page_bytes = (int64_t)c.heads * 2 * kPage * ROW;
  u32x4 kr[WIDE > 0 ? WIDE : 1], vr[VN][2];
  u32x2 kt;
  float scale_in = 0.0f;  // lanes 0 to 3: the coming page's scales of keys; 4 to 7: of values
  const int scale_at = (lane / 4 % 2) * blocks + (lane % 4 * 16 >> log_block);
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
  // the first page from `pg` on that is there, on its way into registers
  const auto fetch = [&](int pg) {
    int page = -1;
    for (; pg < last; ++pg) {
      page = kv_page(c, seq, pg);
      if (page >= 0) break;
    }
    // (behind the last page: page 0 once more, which nobody uses; a branch here cost 5% at 256 values a head)
    const Rsrc rk = buffer(c.pages + max(page, 0) * page_bytes + (int64_t)head * 2 * kPage * ROW, 2 * kPage * ROW);
    const Rsrc rs = buffer(c.scales + ((int64_t)max(page, 0) * c.heads + head) * 2 * blocks, 8 * blocks);
    scale_in = __builtin_bit_cast(float, load4(rs, scale_at * 4 + none, 0));
#pragma unroll
    for (int w = 0; w < WIDE; ++w) kr[w] = load16(rk, lane * 16 + none, wave * 16 * ROW + w * 1024);
    if constexpr (DC % 2) kt = load8(rk, lane * 8 + none, wave * 16 * ROW + WIDE * 1024);
#pragma unroll
    for (int n = 0; n < VN; ++n) {
      const int q = min(wave + 4 * n, DC - 1);
#pragma unroll
      for (int g = 0; g < 2; ++g) vr[n][g] = load16(rk, (lane % 32 / 16) * 1024 + h * 256 + lane % 16 * 16 + none, kPage * ROW + q * 2048 + g * 512);
    }
    return pg;
  };
  const auto convert = [&](int buf) {
    // keys: unit `wave`, lane = (16 values, token); values: lane = (column, every other four tokens)
    u32x4* to = &lds[buf][0][wave / 2 * NS * 64 + wave % 2 * 16 + lane % 16];
#pragma unroll
    for (int w = 0; w < WIDE; ++w) {
      to[(4 * w + lane / 16) * 64] = eight_levels<true>(kr[w][0], kr[w][1]);
      to[(4 * w + lane / 16) * 64 + 32] = eight_levels<true>(kr[w][2], kr[w][3]);
    }
    if constexpr (DC % 2) to[(4 * WIDE + lane / 32) * 64 + lane / 16 % 2 * 32] = eight_levels<true>(kt[0], kt[1]);
#pragma unroll
    for (int n = 0; n < VN; ++n) {
      if (wave + 4 * n >= DC) break;
#pragma unroll
      for (int u = 0; u < 4; ++u) lds[buf][1][(u * DC + wave + 4 * n) * 64 + lane] = eight_levels<true>(vr[n][0][u], vr[n][1][u]);
    }
  };
  int pg = fetch(begin);

  u32x4 q[NS];
  float factor;
  {
    const int64_t base = (s.row0 + token) * a.q_row + (head * a.share + min(r, rows - 1) % a.share) * a.q_head;
    float x[NS][8], top = 0.0f;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const int d = 16 * i + 8 * h;
      load_eight<TYPE>(a.q, base + d, c.dim - d, a.aligned, x[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(x[i][j]));
    }
    top = fmaxf(top, __shfl_xor(top, 32));
    int e = 0;
    if (top > 0.0f && top < INFINITY) (void)frexpf(top, &e);
    e -= 8;
    factor = ldexpf(fabsf(a.scale) * 1.4426950408889634f, e);  // (its sign goes to q, so that the largest score is the largest product)
    const float sign = a.scale < 0.0f ? -1.0f : 1.0f;
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t part[1];
        pair<1>(ldexpf(sign * x[i][2 * j], -e), ldexpf(sign * x[i][2 * j + 1], -e), part);
        q[i][j] = part[0];
      }
  }
  if (pg < last) convert(0);
  float scale_of = scale_in;
  __syncthreads();

  float m = -INFINITY, l = 0.0f, lead = kLeastLead;
  f32x16 o[DC] = {};
  for (int buf = 0; pg < last; buf ^= 1) {
    const int next = fetch(pg + 1), t0 = pg * kPage;
    if (t0 < high_any && t0 + kPage - 1 >= low_any) {
      f32x16 z[2] = {};
#pragma unroll
      for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t) z[t] = mfma32(lds[buf][0][(t * NS + i) * 64 + lane], q[i], z[t]);
      float key_scale[4], value_log[4], tops[4];
      const float log_of = __builtin_amdgcn_logf(fabsf(scale_of));
      const auto of_lane = [](float x, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane)); };
#pragma unroll
      for (int u = 0; u < 4; ++u) key_scale[u] = factor * of_lane(scale_of, u), value_log[u] = of_lane(log_of, 4 + u);
      // (every lane has one of the eight scales)
      const bool full = __builtin_amdgcn_readfirstlane(kv_all_in(t0, kPage, low_all, high_all) && __all(scale_of >= 0x1p-100f));
      if (full) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          float t = z[u / 2][u % 2 * 8];
#pragma unroll
          for (int i = 1; i < 8; ++i) t = fmaxf(t, z[u / 2][u % 2 * 8 + i]);
          tops[u] = t * key_scale[u];
        }
      } else {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          tops[u] = -INFINITY;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int t = t0 + 16 * u + i / 4 * 8 + 4 * h + i % 4;
            const float x = t < high && t >= low ? z[u / 2][u % 2 * 8 + i] * key_scale[u] : -INFINITY;
            z[u / 2][u % 2 * 8 + i] = x;
            tops[u] = fmaxf(tops[u], x);
          }
        }
      }
      float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])), ahead = -INFINITY;
#pragma unroll
      for (int u = 0; u < 4; ++u) ahead = fmaxf(ahead, tops[u] + value_log[u]);
      top = max_32(top), ahead = max_32(ahead);
      const float m_new = fmaxf(m, top), m_at = or_zero(m_new), shrink = __builtin_amdgcn_exp2f(m - m_at);
      const float before = lead + (m - m_at);
      const bool large = __any(fabsf(m_at) >= kLargeScore);
      ahead -= m_at;
      if (large) {
        ahead = -INFINITY;
#pragma unroll
        for (int u = 0; u < 4; ++u) ahead = fmaxf(ahead, tops[u] - m_at + value_log[u]);
        ahead = max_32(ahead);
      }
      lead = fmaxf(fmaxf(before, ahead), kLeastLead);
      const float shrink_o = __builtin_amdgcn_exp2f(before - lead);
      m = m_new;
      l *= shrink;
      u32x4 w[4];
      const float least = fminf(fminf(value_log[0], value_log[1]), fminf(value_log[2], value_log[3]));
      if (full && !large && __all(least - lead >= -64.0f)) {
        const float out_of = __builtin_amdgcn_rcpf(scale_of);
        float all = 0.0f;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float at = value_log[u] - lead + 14.0f - m_at;
          float sum = 0.0f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float y0 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[u / 2][u % 2 * 8 + 2 * i], key_scale[u], at));
            const float y1 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[u / 2][u % 2 * 8 + 2 * i + 1], key_scale[u], at));
            sum += y0 + y1;
            uint32_t part[1];
            pair<1>(y0, y1, part);
            w[u][i] = part[0];
          }
          all += sum * of_lane(out_of, 4 + u);
        }
        l += all * __builtin_amdgcn_exp2f(lead - 14.0f);
      } else {
        const float unit = __builtin_amdgcn_exp2f(-lead);
        if (full) {
#pragma unroll
          for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) z[u / 2][u % 2 * 8 + i] *= key_scale[u];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          // (a block that the row does not see, or that nobody has written, has any scale)
          const bool sees = full || (t0 + 16 * u < high && t0 + 16 * u + 15 >= low);
          const float f = sees ? bounded(of_lane(scale_of, 4 + u) * unit * 0x1p14f) : 0.0f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float e0 = __builtin_amdgcn_exp2f(rounded(z[u / 2][u % 2 * 8 + 2 * i]) - m_at);
            const float e1 = __builtin_amdgcn_exp2f(rounded(z[u / 2][u % 2 * 8 + 2 * i + 1]) - m_at);
            l += e0 + e1;
            uint32_t part[1];
            pair<1>(e0 * f, e1 * f, part);
            w[u][i] = part[0];
          }
        }
      }
      if (__any(shrink_o != 1.0f)) {  // (most pages hold no new maximum)
#pragma unroll
        for (int n = 0; n < DC; ++n) o[n] *= shrink_o;
      }
#pragma unroll
      for (int n = 0; n < DC; ++n)
#pragma unroll
        for (int u = 0; u < 4; ++u) o[n] = mfma32(lds[buf][1][(u * DC + n) * 64 + lane], w[u], o[n]);
    }
    if (next < last) convert(buf ^ 1);
    scale_of = scale_in;
    pg = next;
    __syncthreads();
  }
  l += __shfl_xor(l, 32);
  float unit_of = __builtin_amdgcn_exp2f(lead) * 0x1p-14f;
  if (SPLIT && used > 1) {  // the parts: each lane's numbers at the same place in all of them
    const int64_t unit = ((int64_t)seq * ((a.max_new * a.share + 127) / 128) + r0 / 128) * c.heads + head;
    constexpr int PART = 64 * (DC * 16 + 2);
    float* at = a.parts + (unit * a.prompt_splits * 4 + wave) * PART + lane * 2;
    if (r_wave < rows) {
      float* to = at + (int64_t)split * 4 * PART;
#pragma unroll
      for (int n = 0; n < DC; ++n)
#pragma unroll
        for (int i = 0; i < 8; ++i) put(to + (n * 8 + i) * 128, o[n][2 * i] * unit_of, o[n][2 * i + 1] * unit_of);
      put(to + DC * 1024, m, l);
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wave's numbers are there
    __shared__ uint32_t place;
    __syncthreads();
    if (threadIdx.x == 0) place = __hip_atomic_fetch_add(a.arrived + unit, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (place != (uint32_t)used - 1) return;
    if (threadIdx.x == 0) __hip_atomic_store(a.arrived + unit, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (r_wave >= rows) return;
    m = -INFINITY, l = 0.0f, unit_of = 1.0f;
    for (int p = 0; p < used; ++p) {
      const float* from = at + (int64_t)p * 4 * PART;
      const u32x2 x = get(from + DC * 1024);
      u32x2 y[DC * 8];  // (every read at once: each is a trip to memory)
#pragma unroll
      for (int i = 0; i < DC * 8; ++i) y[i] = get(from + i * 128);
      const uint32_t x0 = x[0], x1 = x[1];
      const float m_part = __builtin_bit_cast(float, x0), m_new = fmaxf(m, m_part), m_at = m_new == -INFINITY ? 0.0f : m_new;
      const float f = __builtin_amdgcn_exp2f(m - m_at), f_part = __builtin_amdgcn_exp2f(m_part - m_at);
      l = l * f + __builtin_bit_cast(float, x1) * f_part;
      m = m_new;
#pragma unroll
      for (int n = 0; n < DC; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t v = y[n * 8 + i / 2][i % 2];
          o[n][i] = (p == 0 ? 0.0f : o[n][i] * f) + __builtin_bit_cast(float, v) * f_part;
        }
    }
  }
  if (r >= rows) return;
  const int64_t at = (s.row0 + token) * a.out_row + (head * a.share + r % a.share) * a.out_head;
  // (a row that sees nothing is zeros)
  const float share_of = l == 0.0f ? 0.0f : unit_of / l;
#pragma unroll
  for (int n = 0; n < DC; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int d = n * 32 + i / 4 * 8 + 4 * h + i % 4;
      if (d < c.dim) store_one<TYPE>(a.out, at + d, l == 0.0f ? 0.0f : o[n][i] * share_of);
    }
  if (a.lse && h == 0)
    a.lse[(s.row0 + token) * a.q_heads + head * a.share + r % a.share] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// What a call needs: tiles of rows, splits, and bytes of the workspace.
struct Plan {
  int64_t units, tiles, prompt_tiles;  // prompt_tiles: of 128 rows, 0 where they are too few to fill the chip
  int splits, part_rows, few, prompt_splits;
  size_t bytes;
};
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
  p.tiles = ceil_div(rows, 16);
  p.units = sequences * heads * p.tiles;
  p.part_rows = (int)std::min<int64_t>(rows, 16);
  // One workgroup for each of the chip's 256 CUs, but four pages of the longest sequence for each at least.  One token over 131072 with 256, 512,
  // 1024 workgroups: 57, 60, 67 us; over 16384: 17, 23, 23.
  p.splits = (int)std::max<int64_t>(std::min({ceil_div(256, std::max<int64_t>(p.units, 1)), ceil_div(table_width, 4), (int64_t)kMostSplits}), 1);
  if (p.units > kCounters) p.splits = 1;
  p.bytes = p.splits == 1 ? 0 : kCounters * 4 + (size_t)p.units * p.splits * p.part_rows * (kv_row_bytes((int)dim) + 4) * 4;
  p.prompt_splits = 1;
  if (p.prompt_tiles) {
    const int64_t units = p.prompt_tiles * heads * sequences;
    // As many workgroups as the chip holds at once, two a CU up to 128 values and one beyond, of 16 pages each at least (a join is four pages' time).
    // 512 new tokens, 32 heads on 8 of 128, over 4096 with 128, 256, 512 workgroups: 122, 72, 68 us; over 2048: 67, 46, 50.
    p.prompt_splits = (int)std::max<int64_t>(std::min<int64_t>((dim <= 128 ? 512 : 256) / units, table_width / kLeastPages), 1);
    if (p.prompt_splits > 1) p.bytes = std::max(p.bytes, kCounters * 4 + (size_t)units * p.prompt_splits * 128 * (kv_row_bytes((int)dim) + 4) * 4);
  }
  return p;
}

template <int TYPE, int DC>
void launch(const bmx_kv_cache& c, const Args& a, const Plan& p, hipStream_t s) {
  // (rows of sequences as long as each other are all many or all few)
  if (!p.prompt_tiles || (c.starts && c.sequences > 1)) {
    const dim3 grid(c.heads * a.splits, (uint32_t)p.tiles, c.sequences);
    launch_kernel(kv_attention_kernel<TYPE, DC>, grid, dim3(kWaves * 64), 0, s, c, a);
    note_kernel("kv_attention_kernel<%d,%d> grid %ux%ux%u block %d", TYPE, DC, grid.x, grid.y, grid.z, kWaves * 64);
  }
  if constexpr (TYPE != BMX_F32) {
    if (p.prompt_tiles) {
      const dim3 grid(c.heads * a.prompt_splits, (uint32_t)p.prompt_tiles, c.sequences);
      Args b = a;
      if (!c.starts || c.sequences == 1) b.few = 0;
      launch_kernel(a.prompt_splits > 1 ? kv_prompt_kernel<TYPE, DC, true> : kv_prompt_kernel<TYPE, DC, false>, grid, dim3(256), 0, s, c, b);
      note_kernel("kv_prompt_kernel<%d,%d,%d> grid %ux%ux%u block 256", TYPE, DC, a.prompt_splits > 1, grid.x, grid.y, grid.z);
    }
  }
}
template <int TYPE>
void launch_typed(const bmx_kv_cache& c, const Args& a, const Plan& p, hipStream_t s) {
  const int dc = kv_row_bytes(c.dim) / 32;
  const auto f = dc == 1 ? launch<TYPE, 1> : dc == 2 ? launch<TYPE, 2> : dc == 3 ? launch<TYPE, 3> : dc == 4 ? launch<TYPE, 4>
               : dc == 5 ? launch<TYPE, 5> : dc == 6 ? launch<TYPE, 6> : dc == 7 ? launch<TYPE, 7> : launch<TYPE, 8>;
  f(c, a, p, s);
}

__global__ void clear_kernel(uint32_t* p) { p[blockIdx.x * 256 + threadIdx.x] = 0; }

}  // namespace

size_t kv_attention_workspace(int64_t sequences, int64_t table_width, int64_t heads, int64_t q_heads, int64_t dim, int64_t max_new) {
  // The largest of the calls' bytes, which first grow with the rows and then, where rows fill the chip without splits, fall.  In closed form: of
  // `each` units a tile, and splits that bring t tiles to 256 workgroups, each * t * splits <= 255 + each * t while that is worth a split.
  const int64_t each = sequences * heads, rows = max_new > 0 ? std::min(max_new * (q_heads / heads), kMostTiles * 16) : kMostTiles * 16;
  const size_t line = (kv_row_bytes((int)dim) + 4) * 4;
  size_t most = 0;
  if (each == 0) return 0;
  const int64_t units = each * std::min(ceil_div(rows, 16), 255 / each), splits = std::min<int64_t>(ceil_div(table_width, 4), kMostSplits);
  if (units > 0 && splits > 1) most = std::min(units * splits, units + 255) * std::min<int64_t>(rows, 16) * line;
  const int64_t places = dim <= 128 ? 512 : 256, tiles = each * std::min(ceil_div(rows, 128), places / 2 / each);
  if (rows > 64 && tiles >= kLeastTiles && table_width / kLeastPages > 1)
    most = std::max<size_t>(most, std::min(places, tiles * (table_width / kLeastPages)) * 128 * line);
  return most ? kCounters * 4 + most : 0;
}

size_t kv_attention_workspace_of_call(int64_t sequences, int64_t table_width, int64_t heads, int64_t q_heads, int64_t dim, int64_t max_new) {
  // (whatever the type)
  return std::max(plan(sequences, table_width, heads, q_heads, dim, max_new, BMX_F32).bytes,
                  plan(sequences, table_width, heads, q_heads, dim, max_new, BMX_F16).bytes);
}

hipError_t launch_kv_attention(const bmx_kv_cache& c, const void* q, int type, int64_t q_row, int64_t q_head, int q_heads, int rows,
                               int max_new, float scale, bool causal, int window, void* out, int64_t out_row, int64_t out_head, float* lse,
                               void* workspace, bool fresh, hipStream_t s) {
  const int64_t size = type_bytes(type);
  const bool aligned = (uintptr_t)q % 16 == 0 && q_row * size % 16 == 0 && q_head * size % 16 == 0;
  const Plan p = plan(c.sequences, c.table_width, c.heads, q_heads, c.dim, max_new, type);
  uint32_t* arrived = static_cast<uint32_t*>(workspace);
  const Args a = {q, q_row, q_head, out, out_row, out_head, lse, reinterpret_cast<float*>(arrived + kCounters), arrived, q_heads,
                  q_heads / c.heads, rows, max_new, window, p.splits, p.part_rows, p.prompt_splits, p.few, causal, aligned, scale};
  const int64_t counters = std::max(p.splits > 1 ? p.units : 0, p.prompt_splits > 1 ? p.prompt_tiles * c.heads * c.sequences : 0);
  if (fresh && counters) launch_kernel(clear_kernel, dim3((uint32_t)ceil_div(counters, 256)), dim3(256), 0, s, arrived);
  const auto f = type == BMX_F32 ? launch_typed<BMX_F32> : type == BMX_F16 ? launch_typed<BMX_F16> : launch_typed<BMX_BF16>;
  f(c, a, p, s);
  return launch_error();
}

}  // namespace bmx
