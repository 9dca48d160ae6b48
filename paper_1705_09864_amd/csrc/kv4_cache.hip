// The paged cache of 4 bits: new keys and values quantised as they are written, and read back.
// A token's head has a scale s and an offset o, both bf16, for its key and for its value: with low and high the least and the largest of its values
//   o = low, s = (high - o) / 15, each rounded to bf16;  q = round((x - o) / s), 0 <= q <= 15;  x is read as q s + o.
// Levels are chosen against the rounded pair, by fp32 quotients.  No token's levels depend on another's, so none is ever written again, and a byte
// belongs to one token.
//
// Bound by the bytes of rows and levels: 13364 tokens of 8 heads of 128 f16 written in 20.2 us (69 MB, 3.4 TB/s: rows, then a token's least and largest, a barrier for
// the values' order, then levels), read in 16.1 (4.3 TB/s).  A few tokens by latency: 64 in 2.9 us, 4007 read in 8.5 to 10 (21 MB).
#include "bmx_internal.h"
#include "few_bits.h"

namespace bmx {
namespace {

constexpr float kMost = 0x1.fffffep127f, kMostBf16 = 0x1.fep127f;
__device__ inline float least(float a, float x) { return fabsf(x) <= kMost ? fminf(a, x) : a; }  // (passes over what is not finite)
__device__ inline float largest(float a, float x) { return fabsf(x) <= kMost ? fmaxf(a, x) : a; }
// The scale and the offset as they are held, in one dword.
__device__ inline uint32_t pair_of(float low, float high) {
  if (low > high) low = high = 0.0f;  // (nothing is finite)
  const float o = fminf(fmaxf(bf16_float(bf16_bits(low)), -kMostBf16), kMostBf16);
  return bf16_bits(fmaxf(fminf(high - o, kMost), 0.0f) / 15.0f) | bf16_bits(o) << 16;
}
__device__ inline float scale_of(uint32_t p) { return bf16_float(p & 0xffff); }
__device__ inline float offset_of(uint32_t p) { return __builtin_bit_cast(float, p & 0xffff0000u); }
// (the instruction itself: it makes 0 of a NaN and of what is below 0, of which C++ has no conversion)
__device__ inline uint32_t to_uint(float x) {
  uint32_t i;
  asm("v_cvt_u32_f32 %0, %1" : "=v"(i) : "v"(x));
  return i;
}
// The level of x, r = 1 / s, or 0 where s is 0: the quotient's nearest whole number n, and with what is left of it the quotient again, n + (x - o - n s) / s, in which
// a quotient halfway between two levels is just that (the remainder is exact, r off by half a bit at most), so that it goes to the even one as in a division.
// Infinities: n stays 16, and what is left is infinite.
__device__ inline uint32_t level(float x, float s, float o, float r) {
  const float d = x - o, n = rintf(fminf(d * r, 16.0f));
  return min(to_uint(rintf(__builtin_fmaf(__builtin_fmaf(-n, s, d), r, n))), 15u);
}
__device__ inline float inverse(float s) { return s >= 0x1p-126f ? 1.0f / s : 0.0f; }
// The same in the low bits, for values and differences that are finite: whole numbers are the last bits of numbers from 2^23 on, where a sum rounds to them as rint
// does.  (The second quotient is rounded beside n first: beside 2^23 it would show which way r is off, and no two levels would be halfway between.)
__device__ inline uint32_t quick_level(float x, float s, float o, float r) {
  const float d = x - o, n = __builtin_fmaf(d, r, 0x1p23f) - 0x1p23f;
  const float t = __builtin_fmaf(__builtin_fmaf(-n, s, d), r, n);
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_fmed3f(t + 0x1p23f, 0x1p23f, 0x1p23f + 15.0f));
}
__device__ inline float value_of(uint32_t q, uint32_t p) { return __builtin_fmaf((float)q, scale_of(p), offset_of(p)); }

// The new tokens of one page, [t0, t1).
struct Page {
  uint8_t* body;
  uint32_t* pairs;
  int64_t base;  // of the page's token 0 among the rows' values
  int t0, t1, page;
};
// `floor`: positions below 0 count as pages too (rows that are read as zeros).
template <bool FLOOR>
__device__ inline bool page_of(const bmx_kv4_cache& c, int rows, int max_new, int span, int64_t row_stride, int64_t head_stride, Page* p) {
  const int seq = blockIdx.x / span, head = blockIdx.y / 2, which = blockIdx.y % 2;
  const KvSpan s = kv_span(c, seq, rows, max_new);
  if (s.count == 0) return false;
  const int low = FLOOR ? s.first : max(s.first, 0), high = FLOOR ? s.first + s.count : s.length;
  int pg;
  if (!kv_page_at(low, high, blockIdx.x % span, &pg, &p->t0, &p->t1)) return false;
  p->page = pg < 0 || pg >= c.table_width ? -1 : kv_page(c, seq, pg);
  if (!FLOOR && p->page < 0) return false;
  const int64_t unit = ((int64_t)max(p->page, 0) * c.heads + head) * 2 + which;
  p->body = c.pages + unit * kPage * kv4_row_bytes(c.dim);
  p->pairs = reinterpret_cast<uint32_t*>(c.scales) + unit * kPage;
  p->base = (s.row0 + (int64_t)pg * kPage - s.first) * row_stride + head * head_stride;
  return true;
}

// CHUNKS: chunks of 16 values of a token, a power of two: lanes side by side have a token's.
template <int TYPE, int CHUNKS>
__global__ __launch_bounds__(256) void kv4_write_kernel(bmx_kv4_cache c, const void* k, const void* v, int64_t k_row, int64_t k_head,
                                                        int64_t v_row, int64_t v_head, int rows, int max_new, int span) {
  constexpr int ITEMS = CHUNKS / 4 > 1 ? CHUNKS / 4 : 1, LINE = CHUNKS * 8 + 4;
  __shared__ __attribute__((aligned(8))) uint8_t bytes[kPage * LINE];  // of values: a token's, one behind the other
  const int which = blockIdx.y % 2, row = kv4_row_bytes(c.dim);
  const int64_t x_row = which ? v_row : k_row;
  Page p;
  if (!page_of<false>(c, rows, max_new, span, x_row, which ? v_head : k_head, &p)) return;
  const void* x = which ? v : k;
  Run<TYPE, 16> r[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int e = threadIdx.x + 256 * i, t = e / CHUNKS, d = e % CHUNKS * 16;
    if (t >= p.t0 && t < p.t1 && d < c.dim) r[i].load(x, p.base + t * x_row + d, c.dim - d);
  }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int e = threadIdx.x + 256 * i, t = e / CHUNKS, d = e % CHUNKS * 16, left = c.dim - d;
    const bool there = t >= p.t0 && t < p.t1 && d < c.dim;
    float low = INFINITY, high = -INFINITY;
    bool odd = false;  // values that are infinite
    if (there) {
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float y = left >= 16 || j < left ? r[i].get(j) : NAN;  // (both pass over it)
        low = fminf(low, y), high = fmaxf(high, y);
      }
      odd = low == -INFINITY || high == INFINITY;
      if (odd) {
        low = INFINITY, high = -INFINITY;
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (left >= 16 || j < left) low = least(low, r[i].get(j)), high = largest(high, r[i].get(j));
      }
    }
#pragma unroll
    for (int o = 1; o < CHUNKS; o *= 2) low = fminf(low, __shfl_xor(low, o)), high = fmaxf(high, __shfl_xor(high, o));
    if (!there) continue;
    const uint32_t pair = pair_of(low, high);
    if (d == 0) p.pairs[t] = pair;
    const float s = scale_of(pair), o = offset_of(pair), of_s = inverse(s);
    uint32_t w[2] = {};
    if (odd || high - low > 0x1p126f) {
#pragma unroll
      for (int j = 0; j < 16; ++j) w[j / 8] |= level(r[i].get(j), s, o, of_s) << (4 * (j % 8));
    } else {
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        uint32_t b[4];  // two levels in the low byte
#pragma unroll
        for (int j = 0; j < 4; ++j)
          b[j] = quick_level(r[i].get(8 * n + 2 * j), s, o, of_s) | quick_level(r[i].get(8 * n + 2 * j + 1), s, o, of_s) << 4;
        w[n] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u), __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), 0x05040100u);
      }
    }
    if (left < 16) {
#pragma unroll
      for (int j = 0; j < 16; ++j) w[j / 8] &= j < left ? 0xffffffffu : ~(15u << (4 * (j % 8)));
    }
    if (which == 0) {
      *reinterpret_cast<u32x2*>(p.body + kv4_key_at(row, t, d)) = u32x2{w[0], w[1]};
    } else {
      uint32_t* to = reinterpret_cast<uint32_t*>(bytes + t * LINE + d / 2);
      to[0] = w[0], to[1] = w[1];
    }
  }
  if (which == 0) return;
  __syncthreads();
  // values: 16 bytes of the page are two columns of 16 tokens
  for (int e = threadIdx.x; e < row * 4; e += 256) {
    const int d = e / 64 * 32 + e % 16 * 2, g = e / 16 % 4;  // tokens 16 u + 4 g + i
    if (d >= c.dim) continue;
    uint8_t* at = p.body + e * 16;
    u32x4 w;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint8_t* b = bytes + (16 * u + 4 * g) * LINE + d / 2;
      w[u] = b[0] | (uint32_t)b[LINE] << 8 | (uint32_t)b[2 * LINE] << 16 | (uint32_t)b[3 * LINE] << 24;
    }
    if (p.t0 == 0 && p.t1 == kPage) {
      *reinterpret_cast<u32x4*>(at) = w;
      continue;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int t = 16 * u + 4 * g;
      if (t >= p.t0 && t + 4 <= p.t1) {
        reinterpret_cast<uint32_t*>(at)[u] = w[u];
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (t + i >= p.t0 && t + i < p.t1) at[u * 4 + i] = (uint8_t)(w[u] >> (8 * i));
      }
    }
  }
}

// A few tokens: a wave for each and head, keys or values; a lane has values 2 lane and 2 lane + 1, and those 128 behind them.
template <int TYPE>
__global__ __launch_bounds__(256) void kv4_append_kernel(bmx_kv4_cache c, const void* k, const void* v, int64_t k_row, int64_t k_head,
                                                         int64_t v_row, int64_t v_head, int rows, int max_new) {
  const int lane = threadIdx.x % 64, unit = blockIdx.y * 4 + threadIdx.x / 64, head = unit / 2, which = unit % 2;
  if (head >= c.heads) return;
  const KvSpan s = kv_span(c, blockIdx.x / max_new, rows, max_new);
  const int j = blockIdx.x % max_new, pos = s.first + j;
  if (j >= s.count || pos < 0 || pos >= s.length) return;
  const void* x = which ? v : k;
  const int64_t from = (s.row0 + j) * (which ? v_row : k_row) + head * (which ? v_head : k_head);
  float y[2][2], low = INFINITY, high = -INFINITY;
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int d = 128 * n + 2 * lane + i;
      y[n][i] = 0.0f;
      if (d < c.dim) {
        y[n][i] = load_one<TYPE>(x, from + d);
        low = least(low, y[n][i]), high = largest(high, y[n][i]);
      }
    }
  const int page = kv_page(c, blockIdx.x / max_new, pos >> kLogPage), t = pos & (kPage - 1);
  if (page < 0) return;
  for (int o = 1; o < 64; o *= 2) low = fminf(low, __shfl_xor(low, o)), high = fmaxf(high, __shfl_xor(high, o));
  const uint32_t pair = pair_of(low, high);
  const int64_t at = ((int64_t)page * c.heads + head) * 2 + which;
  const int row = kv4_row_bytes(c.dim);
  uint8_t* body = c.pages + at * kPage * row;
  if (lane == 0) reinterpret_cast<uint32_t*>(c.scales)[at * kPage + t] = pair;
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int d = 128 * n + 2 * lane;
    if (d >= c.dim) continue;
    const float sc = scale_of(pair), o = offset_of(pair), r = inverse(sc);
    const uint32_t q = level(y[n][0], sc, o, r) | (d + 1 < c.dim ? level(y[n][1], sc, o, r) : 0) << 4;
    body[which ? kv4_value_at(t, d) : kv4_key_at(row, t, d)] = (uint8_t)q;
  }
}

template <int TYPE, int CHUNKS>
__global__ __launch_bounds__(256) void kv4_read_kernel(bmx_kv4_cache c, void* k, void* v, int64_t k_row, int64_t k_head, int64_t v_row,
                                                       int64_t v_head, int rows, int max_new, int span) {
  constexpr int ITEMS = CHUNKS / 4 > 1 ? CHUNKS / 4 : 1, PAIRS = CHUNKS > 8 ? 2 : 1;
  const int which = blockIdx.y % 2, lane = threadIdx.x % 64, wave = threadIdx.x / 64, row = kv4_row_bytes(c.dim);
  const int64_t x_row = which ? v_row : k_row;
  Page p;
  if (!page_of<true>(c, rows, max_new, span, x_row, which ? v_head : k_head, &p)) return;
  const bool there = p.page >= 0;  // (rows of tokens that are not are zeros)
  if (which == 0) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int e = threadIdx.x + 256 * i, t = e / CHUNKS, d = e % CHUNKS * 16;
      if (t < p.t0 || t >= p.t1 || d >= c.dim) continue;
      u32x2 q = {};
      uint32_t pair = 0;
      if (there) {
        q = *reinterpret_cast<const u32x2*>(p.body + kv4_key_at(row, t, d));
        pair = p.pairs[t];
      }
      Run<TYPE, 16> x;
#pragma unroll
      for (int j = 0; j < 16; j += 2) {
        const uint32_t w = q[j / 8] >> (4 * (j % 8));
        x.set2(j, value_of(w & 15, pair), value_of(w >> 4 & 15, pair));
      }
      x.store(k, p.base + t * x_row + d, c.dim - d);
    }
  } else {
    // tokens 16 u + 4 wave + i, columns d and d + 1
    u32x4 pairs[4] = {}, q[PAIRS] = {};
    if (there) {
#pragma unroll
      for (int u = 0; u < 4; ++u) pairs[u] = *reinterpret_cast<const u32x4*>(p.pairs + 16 * u + 4 * wave);
#pragma unroll
      for (int n = 0; n < PAIRS; ++n) {
        const int d = (lane + 64 * n) * 2;
        if (d < c.dim) q[n] = *reinterpret_cast<const u32x4*>(p.body + d / 32 * 1024 + wave * 256 + d % 32 / 2 * 16);
      }
    }
#pragma unroll
    for (int n = 0; n < PAIRS; ++n) {
      const int d = (lane + 64 * n) * 2;
      if (d >= c.dim) continue;
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int t = j / 4 * 16 + 4 * wave + j % 4;
        const uint32_t b = q[n][j / 4] >> (8 * (j % 4)), pair = pairs[j / 4][j % 4];
        Run<TYPE, 2> x;
        x.set2(0, value_of(b & 15, pair), value_of(b >> 4 & 15, pair));
        if (t >= p.t0 && t < p.t1) x.store(v, p.base + t * x_row + d, c.dim - d);
      }
    }
  }
}

template <int TYPE>
auto pick_write(int dim) {
  return dim <= 32 ? kv4_write_kernel<TYPE, 2> : dim <= 64 ? kv4_write_kernel<TYPE, 4> : dim <= 128 ? kv4_write_kernel<TYPE, 8> : kv4_write_kernel<TYPE, 16>;
}
template <int TYPE>
auto pick_read(int dim) {
  return dim <= 32 ? kv4_read_kernel<TYPE, 2> : dim <= 64 ? kv4_read_kernel<TYPE, 4> : dim <= 128 ? kv4_read_kernel<TYPE, 8> : kv4_read_kernel<TYPE, 16>;
}

}  // namespace

hipError_t launch_kv4_write(const bmx_kv4_cache& c, const void* k, const void* v, int type, int64_t k_row, int64_t k_head, int64_t v_row,
                            int64_t v_head, int rows, int max_new, hipStream_t s) {
  // (us of a call and a read of one token, a wave a token, pages whole: 64 sequences of 2 new tokens 7.1, 11.0, 8 9.9, 11.5, 16 13.5, 12.0, 32 19.5, 13.1; 8 of 8 6.1, 6.8,
  // 16 6.3, 6.8, 64 8.6, 7.4)
  if (max_new <= 8) {
    const dim3 grid((uint32_t)(c.sequences * max_new), (c.heads * 2 + 3) / 4);
    const auto kern = type == BMX_F32 ? kv4_append_kernel<BMX_F32> : type == BMX_F16 ? kv4_append_kernel<BMX_F16> : kv4_append_kernel<BMX_BF16>;
    launch_kernel(kern, grid, dim3(256), 0, s, c, k, v, k_row, k_head, v_row, v_head, rows, max_new);
    note_kernel("kv4_append_kernel<%d> grid %ux%u block 256", type, grid.x, grid.y);
    return launch_error();
  }
  const int span = (int)kv_pages_of(max_new);
  const dim3 grid((uint32_t)(c.sequences * (int64_t)span), c.heads * 2);
  const auto kern = type == BMX_F32 ? pick_write<BMX_F32>(c.dim) : type == BMX_F16 ? pick_write<BMX_F16>(c.dim) : pick_write<BMX_BF16>(c.dim);
  launch_kernel(kern, grid, dim3(256), 0, s, c, k, v, k_row, k_head, v_row, v_head, rows, max_new, span);
  note_kernel("kv4_write_kernel<%d> grid %ux%u block 256", type, grid.x, grid.y);
  return launch_error();
}

hipError_t launch_kv4_read(const bmx_kv4_cache& c, void* k, void* v, int type, int64_t k_row, int64_t k_head, int64_t v_row, int64_t v_head,
                           int rows, int max_new, hipStream_t s) {
  const int span = (int)kv_pages_of(max_new);
  const dim3 grid((uint32_t)(c.sequences * (int64_t)span), c.heads * 2);
  const auto kern = type == BMX_F32 ? pick_read<BMX_F32>(c.dim) : type == BMX_F16 ? pick_read<BMX_F16>(c.dim) : pick_read<BMX_BF16>(c.dim);
  launch_kernel(kern, grid, dim3(256), 0, s, c, k, v, k_row, k_head, v_row, v_head, rows, max_new, span);
  note_kernel("kv4_read_kernel<%d> grid %ux%u block 256", type, grid.x, grid.y);
  return launch_error();
}

}  // namespace bmx
