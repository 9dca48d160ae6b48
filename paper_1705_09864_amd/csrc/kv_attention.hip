// Attention of new tokens over the paged cache of 8 bits (kv_cache.hip):
//   o = sum_t p_t v_t / sum_t p_t,  p_t = exp(scale * q . k_t),  k_t = a_b * (levels of t), v_t = c_b * (levels of t),
// over the tokens t that a row sees, b their block.  One pass over the cache with the running maximum m of the scores and the running
// sum, both in 32 bits.  Products are S^T = K Q^T and O^T = V^T P^T on the matrix cores (16 x 16 x 32), 16 rows of queries (tokens x heads that share
// a head of the cache) at a time: levels are whole numbers that 16-bit floats hold exactly, and the scales come to the scores and weights behind
// and before the products.  A lane's scores of S^T are those of its own column of P^T, in the order of tokens in which the cache
// holds values, so the weights never leave their lane.
// For 16-bit results the products are f16's:
//   q goes in with its row's largest value brought to [128, 256) by a power of two (exact but for values 2^-21 below the row's largest);
//   p goes in as p * (c_b / C) * 2^14 with C the largest c_b so far: at most 2^14, and with all of f16's 11 bits down to 2^-28 of that.
// For f32 results they are bf16's, q and p * c_b in three parts of 8 bits each, which together are all of them whatever the range; levels
// are exact in bf16 too.
#include "bmx_internal.h"
#include "few_bits.h"

namespace bmx {
namespace {

constexpr int kWaves = 4;

// The upper halves of two dwords.
__device__ inline uint32_t upper_halves(float a, float b) {
  return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x07060302u);
}
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
      a -= __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, a) & 0xffff0000u);
      b -= __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, b) & 0xffff0000u);
    }
  }
}

struct Args {
  const void* q;
  int64_t q_row, q_head;
  void* out;
  int64_t out_row, out_head;
  float* lse;
  int q_heads, share, rows, max_new, window;
  bool causal, aligned;
  float scale;
};

template <int TYPE, int DC>
__global__ __launch_bounds__(kWaves * 64) void kv_attention_kernel(bmx_kv_cache c, Args a) {
  constexpr int PARTS = TYPE == BMX_F32 ? 3 : 1, ROW = DC * 32, DT = DC * 2, WIDE = DC / 2;
  constexpr bool F16 = PARTS == 1;
  __shared__ float red_o[kWaves][16][ROW + 4], red_m[kWaves][16], red_l[kWaves][16];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), g = lane / 16;
  const int head = blockIdx.x, seq = blockIdx.z;
  const KvSpan s = kv_span(c, seq, a.rows, a.max_new);
  const int r0 = blockIdx.y * 16;
  if (r0 >= s.count * a.share) return;
  // this lane's row of queries, and what it sees: positions [low, high)
  const int r = r0 + lane % 16, token = min(r / a.share, s.count - 1), pos = s.first + token;
  const int high = a.causal ? min(pos + 1, s.length) : s.length;
  const int low = a.window ? max(pos - a.window + 1, 0) : 0;
  // what any row of the 16 sees
  const int tok0 = r0 / a.share, tok1 = min((r0 + 15) / a.share, s.count - 1);
  const int high_any = a.causal ? min(s.first + tok1 + 1, s.length) : s.length;
  const int low_any = a.window ? max(s.first + tok0 - a.window + 1, 0) : 0;

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

  const int blocks = kPage / c.block, log_block = 31 - __builtin_clz(c.block);
  float m = -INFINITY, l = 0.0f, most = 0.0f;
  f32x4 o[DT] = {};
  for (int pg = low_any / kPage + wave; pg * kPage < high_any; pg += kWaves) {
    const int page = kv_page(c, seq, pg);
    if (page < 0) continue;
    const int64_t unit = ((int64_t)page * c.heads + head) * 2;
    const int8_t* keys = c.pages + unit * kPage * ROW;
    const int8_t* values = keys + kPage * ROW;
    const float* ks = c.scales + unit * blocks;
    const float* vs = ks + blocks;
    float p[4][4], vscale[4], top = -INFINITY, most_new = most;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      f32x4 z = {};
#pragma unroll
      for (int w = 0; w < WIDE; ++w) {
        const u32x4 k = *reinterpret_cast<const u32x4*>(keys + u * 16 * ROW + w * 1024 + lane * 16);
        const u32x4 k0 = eight_levels<F16>(k[0], k[1]), k1 = eight_levels<F16>(k[2], k[3]);
#pragma unroll
        for (int part = 0; part < PARTS; ++part) z = mfma<F16>(k1, q[part][2 * w + 1], mfma<F16>(k0, q[part][2 * w], z));
      }
      if constexpr (DC % 2) {
        const u32x2 k = *reinterpret_cast<const u32x2*>(keys + u * 16 * ROW + WIDE * 1024 + lane * 8);
        const u32x4 k0 = eight_levels<F16>(k[0], k[1]);
#pragma unroll
        for (int part = 0; part < PARTS; ++part) z = mfma<F16>(k0, q[part][DC - 1], z);
      }
      const int at = pg * kPage + 16 * u, b = 16 * u >> log_block;
      const float f = factor * ks[b];
      vscale[u] = at < high_any && at + 16 > low_any ? vs[b] : 0.0f;  // (a block that nobody has written has any scale)
      most_new = fmaxf(most_new, vscale[u]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = at + 4 * g + i;
        p[u][i] = t < high && t >= low ? z[i] * f : -INFINITY;
        top = fmaxf(top, p[u][i]);
      }
    }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float m_new = fmaxf(m, top), m_at = m_new == -INFINITY ? 0.0f : m_new;
    const float shrink = __builtin_amdgcn_exp2f(m - m_at);
    float sum = 0.0f;
    // (scales below 2^-126 are those of levels that are all 0)
    const float inverse = most_new >= 0x1p-126f ? 1.0f / most_new : 0.0f, shrink_o = F16 ? shrink * (most * inverse) : shrink;
    m = m_new;
    most = most_new;
    u32x4 w[PARTS][2];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float f = F16 ? vscale[u] * inverse * 0x1p14f : vscale[u];
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        const float e0 = __builtin_amdgcn_exp2f(p[u][i] - m_at), e1 = __builtin_amdgcn_exp2f(p[u][i + 1] - m_at);
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
      const u32x4 v = *reinterpret_cast<const u32x4*>(values + dt * 1024 + lane * 16);
      const u32x4 v0 = eight_levels<F16>(v[0], v[1]), v1 = eight_levels<F16>(v[2], v[3]);
      o[dt] *= shrink_o;
#pragma unroll
      for (int part = 0; part < PARTS; ++part) o[dt] = mfma<F16>(v1, w[part][1], mfma<F16>(v0, w[part][0], o[dt]));
    }
  }

  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (g == 0) red_m[wave][lane] = m, red_l[wave][lane] = l;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 4; ++i) red_o[wave][lane % 16][dt * 16 + 4 * g + i] = F16 ? o[dt][i] * (most * 0x1p-14f) : o[dt][i];
  __syncthreads();
  for (int e = threadIdx.x; e < 16 * ROW; e += kWaves * 64) {
    const int i = e / ROW, d = e % ROW, rr = r0 + i;
    if (rr >= s.count * a.share || d >= c.dim) continue;
    float top = -INFINITY, sum = 0.0f, v = 0.0f;
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, red_m[w][i]);
    const float at = top == -INFINITY ? 0.0f : top;
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(red_m[w][i] - at);
      sum += f * red_l[w][i];
      v += f * red_o[w][i][d];
    }
    const int64_t t = s.row0 + rr / a.share;
    const int h = head * a.share + rr % a.share;
    // (a row that sees nothing is zeros)
    store_one<TYPE>(a.out, t * a.out_row + h * a.out_head + d, sum == 0.0f ? 0.0f : v / sum);
    if (a.lse && d == 0) a.lse[t * a.q_heads + h] = sum == 0.0f ? -INFINITY : (at + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
  }
}

template <int TYPE>
void launch_typed(const bmx_kv_cache& c, const Args& a, hipStream_t s) {
  const dim3 grid(c.heads, (uint32_t)ceil_div((int64_t)a.max_new * a.share, 16), c.sequences);
  const int dc = kv_row_bytes(c.dim) / 32;
  const auto kern = dc == 1 ? kv_attention_kernel<TYPE, 1> : dc == 2 ? kv_attention_kernel<TYPE, 2> : dc == 3 ? kv_attention_kernel<TYPE, 3>
                  : dc == 4 ? kv_attention_kernel<TYPE, 4> : dc == 5 ? kv_attention_kernel<TYPE, 5> : dc == 6 ? kv_attention_kernel<TYPE, 6>
                  : dc == 7 ? kv_attention_kernel<TYPE, 7> : kv_attention_kernel<TYPE, 8>;
  launch_kernel(kern, grid, dim3(kWaves * 64), 0, s, c, a);
  note_kernel("kv_attention_kernel<%d,%d> grid %ux%ux%u block %d", TYPE, dc, grid.x, grid.y, grid.z, kWaves * 64);
}

}  // namespace

hipError_t launch_kv_attention(const bmx_kv_cache& c, const void* q, int type, int64_t q_row, int64_t q_head, int q_heads, int rows,
                               int max_new, float scale, bool causal, int window, void* out, int64_t out_row, int64_t out_head, float* lse,
                               hipStream_t s) {
  const int64_t size = type_bytes(type);
  const bool aligned = (uintptr_t)q % 16 == 0 && q_row * size % 16 == 0 && q_head * size % 16 == 0;
  const Args a = {q, q_row, q_head, out, out_row, out_head, lse, q_heads, q_heads / c.heads, rows, max_new, window, causal, aligned, scale};
  const auto f = type == BMX_F32 ? launch_typed<BMX_F32> : type == BMX_F16 ? launch_typed<BMX_F16> : launch_typed<BMX_BF16>;
  f(c, a, s);
  return launch_error();
}

}  // namespace bmx
