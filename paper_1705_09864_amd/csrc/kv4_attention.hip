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
// the tokens); for f32 results in three, and the levels less 8.  bf16 has fp32's range: nothing is held relative to a row's largest weight.
//
// Bound by the cache's bytes: a wave goes over pages of its own (8.5 KB at 128 values a head) with its queries, running maxima, sums and results in
// registers, and requests the next page's keys as soon as this one's are used up, its values as soon as these are.  Where rows x heads are few, a sequence's
// pages are split over workgroups too, and joined by the last of them (kv_join.h).
#include "bmx_internal.h"
#include "few_bits.h"
#include "kv_join.h"

#include <algorithm>

namespace bmx {
namespace {

__device__ inline f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// What a level is more than its operand.
template <int TYPE>
constexpr float kZero = TYPE == BMX_F32 ? 8.0f : -16.0f;
// The bits of 16.0 in both halves, in a register: beside a literal v_and_or_b32 takes no other, and would fall into two instructions.
__device__ inline uint32_t sixteen() {
  uint32_t x = 0x41804180;
  asm volatile("" : "+v"(x));
  return x;
}
// The levels in fields I and I + 4 of a dword, as operands.
template <int TYPE, int I>
__device__ inline uint32_t two_levels(uint32_t w, uint32_t sixteens) {
  constexpr int shift = 4 * I - 3;  // onto the mantissa's highest four bits
  uint32_t x;
  if constexpr (shift < 0) x = ((w << -shift) & 0x00780078) | sixteens;
  else x = ((w >> shift) & 0x00780078) | sixteens;
  if constexpr (TYPE == BMX_F32) x = upper_halves(__builtin_bit_cast(float, x << 16) - 24.0f, __builtin_bit_cast(float, x & 0xffff0000u) - 24.0f);
  return x;
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
      part[p] = bf16_bits(a) | bf16_bits(b) << 16;
    }
  }
}
__device__ inline float or_zero(float x) { return x == -INFINITY ? 0.0f : x; }

struct Args {
  const void* q;
  int64_t q_row, q_head;
  JoinTo to;
  int rows, max_new, window;
  bool causal, aligned;
  float scale;
};

constexpr int kWaves = kJoinWaves;
constexpr int kCounters = 16384;  // of the workspace's head; what needs more than these has rows enough not to be split
constexpr int64_t kMostTiles = 65535;  // of 16 rows: a launch's second dimension

template <int TYPE, int DC>
__global__ __launch_bounds__(kWaves * 64) void kv4_attention_kernel(bmx_kv4_cache c, Args a) {
  constexpr int QP = TYPE == BMX_F32 ? 3 : TYPE == BMX_F16 ? 2 : 1, PP = TYPE == BMX_F32 ? 3 : 2;
  constexpr int ROW = DC * 32, BYTES = DC * 16, LINE = ROW + 4;
  __shared__ JoinLds<ROW> lds;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), g = lane / 16;
  const int head = blockIdx.x % c.heads, split = blockIdx.x / c.heads, seq = blockIdx.z;
  const KvSpan s = kv_span(c, seq, a.rows, a.max_new);
  const int r0 = blockIdx.y * 16, share = a.to.share;
  if (r0 >= s.count * share) return;
  // what any, and what every one of the 16 rows sees: positions [low, high)
  const int tok0 = r0 / share, tok1 = min((r0 + 15) / share, s.count - 1);
  const int high_any = a.causal ? min(s.first + tok1 + 1, s.length) : s.length, high_all = a.causal ? min(s.first + tok0 + 1, s.length) : s.length;
  const int low_any = a.window ? max(max(s.first + tok0, 0) - a.window + 1, 0) : 0, low_all = a.window ? max(max(s.first + tok1, 0) - a.window + 1, 0) : 0;
  // this workgroup's pages
  const int page0 = low_any / kPage, pages = max(kv_pages_to(high_any) - page0, 0);
  const int per = pages <= 3 * kWaves ? pages : max((pages + a.to.splits - 1) / a.to.splits, kWaves), used = pages > 0 ? (pages + per - 1) / per : 1;
  if (split >= used) return;
  const int begin = page0 + split * per, count = max(min(per, pages - split * per) - wave + kWaves - 1, 0) / kWaves;  // (of this wave, kWaves apart)

  const int64_t page_bytes = (int64_t)c.heads * 2 * kPage * BYTES;
  int ids = -1, next = 0;  // the numbers of 64 pages, a lane each; the place of the next page
  int page, at;            // the page on its way, and its place
  uint32_t k[4][DC];       // of a token, its values from 8 DC g on
  u32x4 v[DC], key_pairs[4], value_pairs[4];
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
  const auto load_values = [&] {
    const int none = page >= 0 ? 0 : kNowhere;
    const Rsrc r = buffer(c.pages + max(page, 0) * page_bytes + (int64_t)(head * 2 + 1) * kPage * BYTES, kPage * BYTES);
#pragma unroll
    for (int i = 0; i < DC; ++i) v[i] = load16(r, lane * 16 + none, i * 1024);
    const Rsrc rs = buffer(c.scales + (((int64_t)max(page, 0) * c.heads + head) * 2 + 1) * 2 * kPage, 4 * kPage);
#pragma unroll
    for (int u = 0; u < 4; ++u) value_pairs[u] = load16(rs, g * 16 + none, u * 64);
  };
  load_keys();
  load_values();

  // this lane's row of queries
  const int r = r0 + lane % 16, token = min(r / share, s.count - 1), pos = s.first + token;
  const int high = a.causal ? min(pos + 1, s.length) : s.length, low = a.window ? max(max(pos, 0) - a.window + 1, 0) : 0;
  const float factor = a.scale * 1.4426950408889634f;
  u32x4 q[QP][DC];
  float all = 0.0f;  // the row's sum, times the factor
  {
    const int64_t base = (s.row0 + token) * a.q_row + (head * share + r % share) * a.q_head;
#pragma unroll
    for (int i = 0; i < DC; ++i) {
      const int d = 8 * (DC * g + i);
      float x[8];
      load_eight<TYPE>(a.q, base + d, c.dim - d, a.aligned, x);
#pragma unroll
      for (int j = 0; j < 4; ++j) {  // (in the order of a dword's fields)
        uint32_t part[QP];
        pair<QP>(x[j], x[4 + j], part);
        all += x[j] + x[4 + j];
#pragma unroll
        for (int p = 0; p < QP; ++p) q[p][i][j] = part[p];
      }
    }
    all += __shfl_xor(all, 16);
    all += __shfl_xor(all, 32);
    all *= factor;
  }

  const uint32_t sixteens = sixteen();
  float m = -INFINITY, l = 0.0f, rest = 0.0f;  // rest: sum of p_t (d_t + kZero c_t), over this lane's tokens
  f32x4 o[DC][2] = {};  // of each 32 values, the even ones and the odd ones
  while (page >= 0) {
    const int t0 = (begin + wave + at * kWaves) * kPage;
    const bool whole = kv_all_in(t0, kPage, low_all, high_all);
    float p[4][4];
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      f32x4 z = {};
#pragma unroll
      for (int i = 0; i < DC; ++i) {
        const uint32_t w = k[u][i];
        const u32x4 x = {two_levels<TYPE, 0>(w, sixteens), two_levels<TYPE, 1>(w, sixteens), two_levels<TYPE, 2>(w, sixteens), two_levels<TYPE, 3>(w, sixteens)};
#pragma unroll
        for (int part = 0; part < QP; ++part) z = mfma(x, q[part][i], z);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w = key_pairs[u][i];
        const float ks = bf16_float(w), ko = __builtin_bit_cast(float, w & 0xffff0000u) + kZero<TYPE> * ks;
        p[u][i] = z[i] * (factor * ks) + all * ko;
      }
    }
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
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, p[u][i]);
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float m_new = fmaxf(m, top), m_at = or_zero(m_new), shrink = __builtin_amdgcn_exp2f(m - m_at);
    m = m_new;
    float sum = 0.0f, more = 0.0f;
    u32x4 w[PP][2];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      float x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t y = value_pairs[u][i];
        const float vs = bf16_float(y), vo = __builtin_bit_cast(float, y & 0xffff0000u) + kZero<TYPE> * vs;
        const float e = __builtin_amdgcn_exp2f(p[u][i] - m_at);
        sum += e;
        more += e * vo;
        x[i] = e * vs;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {  // (a dword of values has tokens 0 and 2 in one operand, 1 and 3 in the next)
        uint32_t part[PP];
        pair<PP>(x[i], x[i + 2], part);
#pragma unroll
        for (int n = 0; n < PP; ++n) w[n][u / 2][u % 2 * 2 + i] = part[n];
      }
    }
    l = l * shrink + sum;
    rest = rest * shrink + more;
#pragma unroll
    for (int i = 0; i < DC; ++i) {
#pragma unroll
      for (int odd = 0; odd < 2; ++odd) {
        o[i][odd] *= shrink;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t y0 = v[i][2 * h], y1 = v[i][2 * h + 1];
          const u32x4 x = odd ? u32x4{two_levels<TYPE, 1>(y0, sixteens), two_levels<TYPE, 3>(y0, sixteens), two_levels<TYPE, 1>(y1, sixteens), two_levels<TYPE, 3>(y1, sixteens)}
                              : u32x4{two_levels<TYPE, 0>(y0, sixteens), two_levels<TYPE, 2>(y0, sixteens), two_levels<TYPE, 0>(y1, sixteens), two_levels<TYPE, 2>(y1, sixteens)};
#pragma unroll
          for (int part = 0; part < PP; ++part) o[i][odd] = mfma(x, w[part][h], o[i][odd]);
        }
      }
    }
    load_values();
  }

  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  rest += __shfl_xor(rest, 16);
  rest += __shfl_xor(rest, 32);
  if (g == 0) lds.red_m[wave][lane] = m, lds.red_l[wave][lane] = l;
#pragma unroll
  for (int i = 0; i < DC; ++i)
#pragma unroll
    for (int j = 0; j < 4; j += 2)
      *reinterpret_cast<f32x4*>(&lds.red[(wave * 16 + lane % 16) * LINE + i * 32 + 8 * g + 2 * j]) =
          f32x4{o[i][0][j] + rest, o[i][1][j] + rest, o[i][0][j + 1] + rest, o[i][1][j + 1] + rest};
  __syncthreads();
  const int64_t unit = ((int64_t)seq * gridDim.y + blockIdx.y) * c.heads + head;
  join_rows<TYPE, ROW>(lds, a.to, c.dim, s.row0, head, r0, min(s.count * share - r0, 16), unit, split, used);
}

// What a call needs: tiles of rows, splits, and bytes of the workspace.
struct Plan {
  int64_t units, tiles;
  int splits, part_rows;
  size_t bytes;
};
Plan plan(int64_t sequences, int64_t table_width, int64_t heads, int64_t q_heads, int64_t dim, int64_t max_new) {
  Plan p;
  const int64_t rows = max_new * (q_heads / heads);
  p.tiles = ceil_div(rows, 16);
  p.units = sequences * heads * p.tiles;
  p.part_rows = (int)std::min<int64_t>(rows, 16);
  // one workgroup for each of the chip's 256 CUs, but four pages of the longest sequence for each at least
  p.splits = (int)std::max<int64_t>(std::min({ceil_div(256, std::max<int64_t>(p.units, 1)), ceil_div(table_width, 4), (int64_t)kMostSplits}), 1);
  if (p.units > kCounters) p.splits = 1;
  p.bytes = p.splits == 1 ? 0 : kCounters * 4 + (size_t)p.units * p.splits * p.part_rows * (kv4_row_bytes((int)dim) * 2 + 4) * 4;
  return p;
}

template <int TYPE, int DC>
void launch(const bmx_kv4_cache& c, const Args& a, const Plan& p, hipStream_t s) {
  const dim3 grid(c.heads * p.splits, (uint32_t)p.tiles, c.sequences);
  launch_kernel(kv4_attention_kernel<TYPE, DC>, grid, dim3(kWaves * 64), 0, s, c, a);
  note_kernel("kv4_attention_kernel<%d,%d> grid %ux%ux%u block %d", TYPE, DC, grid.x, grid.y, grid.z, kWaves * 64);
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
  // The largest of the calls' bytes, which first grow with the rows and then, where rows fill the chip without splits, fall.  In closed form: of
  // `each` units a tile, and splits that bring t tiles to 256 workgroups, each * t * splits <= 255 + each * t while that is worth a split.
  const int64_t each = sequences * heads, rows = max_new > 0 ? std::min(max_new * (q_heads / heads), kMostTiles * 16) : kMostTiles * 16;
  if (each == 0) return 0;
  const int64_t units = each * std::min(ceil_div(rows, 16), 255 / each), splits = std::min<int64_t>(ceil_div(table_width, 4), kMostSplits);
  if (units == 0 || splits <= 1) return 0;
  return kCounters * 4 + std::min(units * splits, units + 255) * std::min<int64_t>(rows, 16) * (kv4_row_bytes((int)dim) * 2 + 4) * 4;
}

size_t kv4_attention_workspace_of_call(int64_t sequences, int64_t table_width, int64_t heads, int64_t q_heads, int64_t dim, int64_t max_new) {
  return plan(sequences, table_width, heads, q_heads, dim, max_new).bytes;
}

hipError_t launch_kv4_attention(const bmx_kv4_cache& c, const void* q, int type, int64_t q_row, int64_t q_head, int q_heads, int rows,
                                int max_new, float scale, bool causal, int window, void* out, int64_t out_row, int64_t out_head, float* lse,
                                void* workspace, bool fresh, hipStream_t s) {
  const int64_t size = type_bytes(type);
  const bool aligned = (uintptr_t)q % 16 == 0 && q_row * size % 16 == 0 && q_head * size % 16 == 0;
  const Plan p = plan(c.sequences, c.table_width, c.heads, q_heads, c.dim, max_new);
  uint32_t* arrived = static_cast<uint32_t*>(workspace);
  const Args a = {q, q_row, q_head, {out, out_row, out_head, lse, reinterpret_cast<float*>(arrived + kCounters), arrived, q_heads, q_heads / c.heads, p.splits, p.part_rows},
                  rows, max_new, window, causal, aligned, scale};
  if (fresh && p.splits > 1) launch_kernel(clear_kernel, dim3((uint32_t)ceil_div(p.units, 256)), dim3(256), 0, s, arrived);
  const auto f = type == BMX_F32 ? launch_typed<BMX_F32> : type == BMX_F16 ? launch_typed<BMX_F16> : launch_typed<BMX_BF16>;
  f(c, a, p, s);
  return launch_error();
}

}  // namespace bmx
