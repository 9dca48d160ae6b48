// The paged cache of 8 bits: new keys and values quantised as they are written, and read back.
// A block of 16, 32 or 64 tokens of one head has one scale s for its keys and one for its values; a value is held as
// q = round(x / s), |q| <= 127, with s = max |x| / 127 over the block.  A block that already holds tokens keeps its scale unless a
// new value is past 127 s; then s grows and the older levels go to round(q * s_old / s).  Scales and quotients are 32-bit.
//
// Bound by the bytes of rows and levels.  A workgroup takes one page of one head, its keys or its values, in registers from the first read
// to the last write.  Keys: a lane has 16 values of a token, which lie together in the page; the lanes of a token lie side by side, so
// its row is read whole.  Values: a lane has two columns of 16 tokens, the tokens whose bytes lie together in the page, so rows are read
// and pages written in whole lines, and no value changes lanes on its way.
//   Measured: 11600 tokens of five prompts, 8 heads of 128 f16 values (71 MB in each direction): written in 26 us, read in 17 (4.2 TB/s); with
// a byte or an element a lane 111 and 70, and 35 where a lane waited for each of its reads.  One token for each of 64 sequences 5.0 us, a page's
// worth of each read back 9.5 (36.9).
#include "bmx_internal.h"
#include "few_bits.h"

namespace bmx {
namespace {

// N consecutive values, as they lie in memory at an address of an element.
template <int TYPE, int N>
struct Run {
  static constexpr int kDwords = N * (TYPE == BMX_F32 ? 4 : 2) / 4;
  struct __attribute__((packed, aligned(TYPE == BMX_F32 ? 4 : 2))) Raw {
    uint32_t w[kDwords];
  };
  uint32_t w[kDwords];

  __device__ static size_t bytes(int64_t at) { return at * (TYPE == BMX_F32 ? 4 : 2); }
  // `left` of them are there, the others are 0
  __device__ void load(const void* p, int64_t at, int left) {
    if (left >= N) {
      const Raw r = *reinterpret_cast<const Raw*>(static_cast<const char*>(p) + bytes(at));
#pragma unroll
      for (int i = 0; i < kDwords; ++i) w[i] = r.w[i];
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if constexpr (TYPE == BMX_F32) {
          w[j] = j < left ? static_cast<const uint32_t*>(p)[at + j] : 0;
        } else {
          const uint32_t h = j < left ? static_cast<const uint16_t*>(p)[at + j] : 0;
          w[j / 2] = j % 2 ? w[j / 2] | h << 16 : h;
        }
      }
    }
  }
  __device__ void store(void* p, int64_t at, int left) const {
    if (left >= N) {
      Raw r;
#pragma unroll
      for (int i = 0; i < kDwords; ++i) r.w[i] = w[i];
      *reinterpret_cast<Raw*>(static_cast<char*>(p) + bytes(at)) = r;
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if (j >= left) continue;
        if constexpr (TYPE == BMX_F32) static_cast<uint32_t*>(p)[at + j] = w[j];
        else static_cast<uint16_t*>(p)[at + j] = (uint16_t)(w[j / 2] >> (16 * (j % 2)));
      }
    }
  }
  __device__ float get(int j) const {
    if constexpr (TYPE == BMX_F32) {
      const uint32_t x = w[j];
      return __builtin_bit_cast(float, x);
    } else {
      const uint32_t h = w[j / 2] >> (16 * (j % 2)) & 0xffff;
      return TYPE == BMX_F16 ? (float)__builtin_bit_cast(_Float16, (uint16_t)h) : bf16_float(h);
    }
  }
  __device__ void set2(int j, float a, float b) {  // values j (even) and j + 1
    if constexpr (TYPE == BMX_F32) w[j] = __builtin_bit_cast(uint32_t, a), w[j + 1] = __builtin_bit_cast(uint32_t, b);
    else if constexpr (TYPE == BMX_F16) w[j / 2] = f16_bits(a) | f16_bits(b) << 16;
    else w[j / 2] = bf16_bits(a) | bf16_bits(b) << 16;
  }
};

__device__ inline float finite(float a) { return a < INFINITY ? a : 0.0f; }  // of a size: neither infinite nor NaN

// (the instruction itself: in C++ the conversion of a NaN or of too large a number has no result)
__device__ inline int to_int(float x) {
  int i;
  asm("v_cvt_i32_f32 %0, %1" : "=v"(i) : "v"(x));
  return i;
}
// The level of x: the conversion makes 0 of a NaN and the largest numbers of infinities.
__device__ inline int level(float x, float r) { return min(max(to_int(rintf(x * r)), -127), 127); }
__device__ inline uint32_t four_bytes(int a, int b, int c, int d) {
  const uint32_t lo = __builtin_amdgcn_perm((uint32_t)b, (uint32_t)a, 0x0c0c0400u), hi = __builtin_amdgcn_perm((uint32_t)d, (uint32_t)c, 0x04000c0cu);
  return lo | hi;
}
template <int CTRL>
__device__ inline float max_lane(float x) {  // the larger of x and that of the lane which a row's permutation names
  const int other = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, false);
  return fmaxf(x, __builtin_bit_cast(float, other));
}
__device__ inline float max_of_row(float x) { return max_lane<0x140>(max_lane<0x141>(max_lane<0x4e>(max_lane<0xb1>(x)))); }  // of 16 lanes
__device__ inline float byte_of(const u32x4& b, int j) {
  const uint32_t w = b[j / 4];
  return (float)(int8_t)(w >> (8 * (j % 4)));
}

// A level's value: the 32-bit product, which the type's rounding follows.  (Without the barrier f16 would be one rounding of the exact product,
// v_fma_mixlo_f16, and a value read as f16 another than the same value read as f32 and rounded.)
__device__ inline float value_of(float level, float scale) {
  float x = level * scale;
  asm("" : "+v"(x));
  return x;
}

// A page of one head, its keys or its values, and the new tokens in it: [t0, t1).
struct Page {
  int8_t* body;
  float* scales;
  int64_t base;  // of the page's token 0 among the rows' values
  int t0, t1, log_block, page;
};
// `floor`: positions below 0 count as pages too (rows that are read as zeros).
template <bool FLOOR>
__device__ inline bool page_of(const bmx_kv_cache& c, int rows, int max_new, int span, int64_t row_stride, int64_t head_stride, Page* p) {
  const int seq = blockIdx.x / span, head = blockIdx.y / 2, which = blockIdx.y % 2;
  const KvSpan s = kv_span(c, seq, rows, max_new);
  if (s.count == 0) return false;
  const int low = FLOOR ? s.first : max(s.first, 0), high = FLOOR ? s.first + s.count : s.length;
  int pg;
  if (!kv_page_at(low, high, blockIdx.x % span, &pg, &p->t0, &p->t1)) return false;
  p->page = pg < 0 || pg >= c.table_width ? -1 : kv_page(c, seq, pg);
  if (!FLOOR && p->page < 0) return false;
  p->log_block = 31 - __builtin_clz(c.block);
  const int64_t unit = ((int64_t)max(p->page, 0) * c.heads + head) * 2 + which;
  p->body = c.pages + unit * kPage * kv_row_bytes(c.dim);
  p->scales = c.scales + unit * (kPage >> p->log_block);
  p->base = (s.row0 + (int64_t)pg * kPage - s.first) * row_stride + head * head_stride;
  return true;
}

// CHUNKS: chunks of 16 values of a token, a power of two.
template <int TYPE, int CHUNKS>
__global__ __launch_bounds__(256) void kv_write_kernel(bmx_kv_cache c, const void* k, const void* v, int64_t k_row, int64_t k_head,
                                                       int64_t v_row, int64_t v_head, int rows, int max_new, int span) {
  constexpr int ITEMS = CHUNKS > 4 ? CHUNKS / 4 : 1, PAIRS = CHUNKS > 8 ? 2 : 1;
  __shared__ uint32_t top[4];
  const int which = blockIdx.y % 2, lane = threadIdx.x % 64, wave = threadIdx.x / 64, row = kv_row_bytes(c.dim);
  const int64_t x_row = which ? v_row : k_row;
  Page p;
  if (!page_of<false>(c, rows, max_new, span, x_row, which ? v_head : k_head, &p)) return;
  if (threadIdx.x < 4) top[threadIdx.x] = 0;
  const int blocks = kPage >> p.log_block, held_block = p.t0 >> p.log_block;
  const bool held = (held_block << p.log_block) < p.t0;  // (older tokens in the first block)
  const float was = held ? p.scales[held_block] : 0.0f;
  float mine = 0.0f;  // lanes 0 to 3 of every wave: a block's new scale, and what it is multiplied with
  const auto scales = [&] {
    const int b = lane % 4;
    mine = __builtin_bit_cast(float, top[b]) * (1.0f / 127.0f);
    if (held && b == held_block) mine = fmaxf(was, mine);
    if (wave == 0 && lane < blocks && b >= held_block && b <= (p.t1 - 1) >> p.log_block) p.scales[b] = mine;
  };
  const auto scale = [&](int b) { return __shfl(mine, b); };
  const auto inverse = [&](float s) { return s >= 0x1p-126f ? 1.0f / s : 0.0f; };
  if (which == 0) {
    Run<TYPE, 16> x[ITEMS];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int e = threadIdx.x + 256 * i, t = e / CHUNKS, d = e % CHUNKS * 16;
      if (t >= p.t0 && t < p.t1 && d < c.dim) x[i].load(k, p.base + t * x_row + d, c.dim - d);
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int e = threadIdx.x + 256 * i, t = e / CHUNKS, d = e % CHUNKS * 16;
      float m = 0.0f;
      if (t >= p.t0 && t < p.t1 && d < c.dim) {
#pragma unroll
        for (int j = 0; j < 16; ++j) m = fmaxf(m, fabsf(x[i].get(j)));  // (passes over a NaN)
        if (m == INFINITY) {
          m = 0.0f;
#pragma unroll
          for (int j = 0; j < 16; ++j) m = fmaxf(m, finite(fabsf(x[i].get(j))));
        }
      }
      m = max_of_row(m);  // (a row of 16 lanes has tokens of one block)
      if (lane % 16 == 0 && t < kPage) atomicMax(&top[t >> p.log_block], __builtin_bit_cast(uint32_t, m));  // (no sign: they order as integers)
    }
    __syncthreads();
    scales();
    const float grown = held ? scale(held_block) : 0.0f, ratio = grown > was ? was / grown : 1.0f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int e = threadIdx.x + 256 * i, t = e / CHUNKS, d = e % CHUNKS * 16;
      const float r = inverse(scale(min(t >> p.log_block, 3)));
      const bool again = held && grown > was && t < p.t0 && t >> p.log_block == held_block;
      if (t >= p.t1 || d >= c.dim || !(t >= p.t0 || again)) continue;
      int8_t* at = p.body + kv_key_at(row, t, d);
      const bool tail = d / 64 * 64 + 64 > row;  // (16 values in two pieces)
      u32x4 q;
      if (t >= p.t0) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          q[j] = four_bytes(level(x[i].get(4 * j), r), level(x[i].get(4 * j + 1), r), level(x[i].get(4 * j + 2), r), level(x[i].get(4 * j + 3), r));
      } else {
        const u32x2 a = *reinterpret_cast<const u32x2*>(at), b = *reinterpret_cast<const u32x2*>(at + (tail ? 128 : 8));
        const u32x4 old = {a[0], a[1], b[0], b[1]};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          int z[4];
#pragma unroll
          for (int n = 0; n < 4; ++n) z[n] = (int)rintf(byte_of(old, 4 * j + n) * ratio);
          q[j] = four_bytes(z[0], z[1], z[2], z[3]);
        }
      }
      if (tail) {
        *reinterpret_cast<u32x2*>(at) = u32x2{q[0], q[1]};
        *reinterpret_cast<u32x2*>(at + 128) = u32x2{q[2], q[3]};
      } else {
        *reinterpret_cast<u32x4*>(at) = q;
      }
    }
  } else {
    // tokens 16 u + 4 wave + i, columns d and d + 1
    Run<TYPE, 2> x[PAIRS][16];
    __syncthreads();
    float m[4] = {};
    // (all of them on their way before the first is used: a token or column that is not there reads one that is)
#pragma unroll
    for (int n = 0; n < PAIRS; ++n)
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int t = min(max(j / 4 * 16 + 4 * wave + j % 4, p.t0), p.t1 - 1), d = min((lane + 64 * n) * 2, c.dim - 1 & ~1);
        if (c.dim % 2 == 0) x[n][j].load(v, p.base + t * x_row + d, 2);
        else x[n][j].load(v, p.base + t * x_row + d, c.dim - d);
      }
#pragma unroll
    for (int n = 0; n < PAIRS; ++n)
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int t = j / 4 * 16 + 4 * wave + j % 4;
        const bool there = t >= p.t0 && t < p.t1 && (lane + 64 * n) * 2 < c.dim;
#pragma unroll
        for (int i = 0; i < Run<TYPE, 2>::kDwords; ++i) x[n][j].w[i] = there ? x[n][j].w[i] : 0;
        m[j / 4] = fmaxf(m[j / 4], fmaxf(fabsf(x[n][j].get(0)), fabsf(x[n][j].get(1))));  // (passes over a NaN)
      }
    if (fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])) == INFINITY) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        m[u] = 0.0f;
#pragma unroll
        for (int n = 0; n < PAIRS; ++n)
#pragma unroll
          for (int j = 4 * u; j < 4 * u + 4; ++j) m[u] = fmaxf(m[u], fmaxf(finite(fabsf(x[n][j].get(0))), finite(fabsf(x[n][j].get(1)))));
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      m[u] = max_of_row(m[u]);
      if (lane % 16 == 0) atomicMax(&top[16 * u >> p.log_block], __builtin_bit_cast(uint32_t, m[u]));
    }
    __syncthreads();
    scales();
    const float grown = held ? scale(held_block) : 0.0f, ratio = grown > was ? was / grown : 1.0f;
    float r[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) r[u] = inverse(scale(16 * u >> p.log_block));
    // whether any, and whether all of this wave's tokens change
    bool any = false, every = true;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const int t = j / 4 * 16 + 4 * wave + j % 4;
      const bool change = t < p.t1 && (t >= p.t0 || (held && grown > was && t >> p.log_block == held_block));
      any |= change, every &= t < p.t1 && t >= p.t0;
    }
    if (!any) return;
#pragma unroll
    for (int n = 0; n < PAIRS; ++n) {
      const int d = (lane + 64 * n) * 2;
      if (d >= c.dim) continue;
      int8_t* at = p.body + d / 16 * 1024 + wave * 256 + d % 16 * 16;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        u32x4 old = {}, q;
        if (!every) old = *reinterpret_cast<const u32x4*>(at + 16 * e);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          int b[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            b[i] = level(x[n][4 * u + i].get(e), r[u]);
            if (!every) {
              const int t = u * 16 + 4 * wave + i;
              const float z = byte_of(old, 4 * u + i);
              const bool again = held && grown > was && t < p.t0 && t >> p.log_block == held_block;
              if (t < p.t0 || t >= p.t1) b[i] = (int)(again ? rintf(z * ratio) : z);
            }
          }
          q[u] = four_bytes(b[0], b[1], b[2], b[3]);
        }
        *reinterpret_cast<u32x4*>(at + 16 * e) = q;
      }
    }
  }
}

// A few tokens: an element a lane, and only the bytes that change are touched.
template <int TYPE>
__global__ __launch_bounds__(256) void kv_append_kernel(bmx_kv_cache c, const void* k, const void* v, int64_t k_row, int64_t k_head,
                                                        int64_t v_row, int64_t v_head, int rows, int max_new, int span) {
  __shared__ uint32_t top[4];
  const int which = blockIdx.y % 2, row = kv_row_bytes(c.dim), block = c.block;
  const void* x = which ? v : k;
  const int64_t x_row = which ? v_row : k_row;
  Page p;
  if (!page_of<false>(c, rows, max_new, span, x_row, which ? v_head : k_head, &p)) return;
  const int t0 = p.t0, t1 = p.t1;
  const int64_t base = p.base;
  int8_t* body = p.body;
  float* scales = p.scales;
  if (threadIdx.x < 4) top[threadIdx.x] = 0;
  __syncthreads();
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  for (int t = t0 + wave; t < t1; t += 4) {
    float m = 0.0f;
    for (int d = lane; d < c.dim; d += 64) {
      m = fmaxf(m, finite(fabsf(load_one<TYPE>(x, base + t * x_row + d))));
    }
    for (int o = 1; o < 64; o *= 2) m = fmaxf(m, __shfl_xor(m, o));
    if (lane == 0) atomicMax(&top[t / block], __builtin_bit_cast(uint32_t, m));  // (floats that are not negative order as integers)
  }
  __syncthreads();
  for (int b = t0 / block; b <= (t1 - 1) / block; ++b) {
    const bool held = b * block < t0;
    const float was = held ? scales[b] : 0.0f;
    const float now = fmaxf(was, __builtin_bit_cast(float, top[b]) * (1.0f / 127.0f));
    if (held && now > was) {
      const float ratio = was / now;
      for (int i = threadIdx.x; i < (t0 - b * block) * c.dim; i += 256) {
        const int t = b * block + i / c.dim, d = i % c.dim, at = which ? kv_value_at(t, d) : kv_key_at(row, t, d);
        body[at] = (int8_t)rintf((float)body[at] * ratio);
      }
    }
    const float r = now >= 0x1p-126f ? 1.0f / now : 0.0f;
    const int from = max(t0, b * block), to = min(t1, (b + 1) * block);
    for (int i = threadIdx.x; i < (to - from) * c.dim; i += 256) {
      const int t = from + i / c.dim, d = i % c.dim, at = which ? kv_value_at(t, d) : kv_key_at(row, t, d);
      body[at] = (int8_t)level(load_one<TYPE>(x, base + t * x_row + d), r);
    }
    __syncthreads();  // (every thread has read the old scale)
    if (threadIdx.x == 0) scales[b] = now;
  }
}

template <int TYPE, int CHUNKS>
__global__ __launch_bounds__(256) void kv_read_kernel(bmx_kv_cache c, void* k, void* v, int64_t k_row, int64_t k_head, int64_t v_row,
                                                      int64_t v_head, int rows, int max_new, int span) {
  constexpr int ITEMS = CHUNKS > 4 ? CHUNKS / 4 : 1, PAIRS = CHUNKS > 8 ? 2 : 1;
  const int which = blockIdx.y % 2, lane = threadIdx.x % 64, wave = threadIdx.x / 64, row = kv_row_bytes(c.dim);
  const int64_t x_row = which ? v_row : k_row;
  Page p;
  if (!page_of<true>(c, rows, max_new, span, x_row, which ? v_head : k_head, &p)) return;
  const bool there = p.page >= 0;  // (rows of tokens that are not are zeros)
  if (which == 0) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int e = threadIdx.x + 256 * i, t = e / CHUNKS, d = e % CHUNKS * 16;
      if (t < p.t0 || t >= p.t1 || d >= c.dim) continue;
      u32x4 q = {};
      float s = 0.0f;
      if (there) {
        const int8_t* at = p.body + kv_key_at(row, t, d);
        if (d / 64 * 64 + 64 > row) {
          const u32x2 a = *reinterpret_cast<const u32x2*>(at), b = *reinterpret_cast<const u32x2*>(at + 128);
          q = u32x4{a[0], a[1], b[0], b[1]};
        } else {
          q = *reinterpret_cast<const u32x4*>(at);
        }
        s = p.scales[t >> p.log_block];
      }
      Run<TYPE, 16> x;
#pragma unroll
      for (int j = 0; j < 16; j += 2) x.set2(j, value_of(byte_of(q, j), s), value_of(byte_of(q, j + 1), s));
      x.store(k, p.base + t * x_row + d, c.dim - d);
    }
  } else {
    float s[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) s[u] = there ? p.scales[16 * u >> p.log_block] : 0.0f;
#pragma unroll
    for (int n = 0; n < PAIRS; ++n) {
      const int d = (lane + 64 * n) * 2;
      if (d >= c.dim) continue;
      u32x4 q[2] = {};
      if (there) {
        const int8_t* at = p.body + d / 16 * 1024 + wave * 256 + d % 16 * 16;
        q[0] = *reinterpret_cast<const u32x4*>(at), q[1] = *reinterpret_cast<const u32x4*>(at + 16);
      }
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int t = j / 4 * 16 + 4 * wave + j % 4;
        Run<TYPE, 2> x;
        x.set2(0, value_of(byte_of(q[0], j), s[j / 4]), value_of(byte_of(q[1], j), s[j / 4]));
        if (t >= p.t0 && t < p.t1) x.store(v, p.base + t * x_row + d, c.dim - d);
      }
    }
  }
}

template <int TYPE>
auto pick_write(int dim) {
  return dim <= 32 ? kv_write_kernel<TYPE, 2> : dim <= 64 ? kv_write_kernel<TYPE, 4> : dim <= 128 ? kv_write_kernel<TYPE, 8> : kv_write_kernel<TYPE, 16>;
}
template <int TYPE>
auto pick_read(int dim) {
  return dim <= 32 ? kv_read_kernel<TYPE, 2> : dim <= 64 ? kv_read_kernel<TYPE, 4> : dim <= 128 ? kv_read_kernel<TYPE, 8> : kv_read_kernel<TYPE, 16>;
}

}  // namespace

hipError_t launch_kv_write(const bmx_kv_cache& c, const void* k, const void* v, int type, int64_t k_row, int64_t k_head, int64_t v_row,
                           int64_t v_head, int rows, int max_new, hipStream_t s) {
  const int span = (int)kv_pages_of(max_new);
  const dim3 grid((uint32_t)(c.sequences * (int64_t)span), c.heads * 2);
  // (64 sequences, 8 heads of 128 bf16: 1 token each 4.9 us, and by pages 9.5; 8 tokens 15.5 and 18.4 with a read of one behind them; 16 tokens 20.1, 19.3)
  if (max_new <= 8) {
    const auto kern = type == BMX_F32 ? kv_append_kernel<BMX_F32> : type == BMX_F16 ? kv_append_kernel<BMX_F16> : kv_append_kernel<BMX_BF16>;
    launch_kernel(kern, grid, dim3(256), 0, s, c, k, v, k_row, k_head, v_row, v_head, rows, max_new, span);
    note_kernel("kv_append_kernel<%d> grid %ux%u block 256", type, grid.x, grid.y);
    return launch_error();
  }
  const auto kern = type == BMX_F32 ? pick_write<BMX_F32>(c.dim) : type == BMX_F16 ? pick_write<BMX_F16>(c.dim) : pick_write<BMX_BF16>(c.dim);
  launch_kernel(kern, grid, dim3(256), 0, s, c, k, v, k_row, k_head, v_row, v_head, rows, max_new, span);
  note_kernel("kv_write_kernel<%d> grid %ux%u block 256", type, grid.x, grid.y);
  return launch_error();
}

hipError_t launch_kv_read(const bmx_kv_cache& c, void* k, void* v, int type, int64_t k_row, int64_t k_head, int64_t v_row, int64_t v_head,
                          int rows, int max_new, hipStream_t s) {
  const int span = (int)kv_pages_of(max_new);
  const dim3 grid((uint32_t)(c.sequences * (int64_t)span), c.heads * 2);
  const auto kern = type == BMX_F32 ? pick_read<BMX_F32>(c.dim) : type == BMX_F16 ? pick_read<BMX_F16>(c.dim) : pick_read<BMX_BF16>(c.dim);
  launch_kernel(kern, grid, dim3(256), 0, s, c, k, v, k_row, k_head, v_row, v_head, rows, max_new, span);
  note_kernel("kv_read_kernel<%d> grid %ux%u block 256", type, grid.x, grid.y);
  return launch_error();
}

}  // namespace bmx
