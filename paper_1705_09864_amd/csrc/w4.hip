// Products with 4-bit weights: w[n][k] = s * q + b, a scale s and an offset b for each group of 32, 64 or 128 values of a row,
//   y[m][n] = sum_k x[m][k] w[n][k] = sum_g ( s_g * sum_{k in g} q x + b_g * sum_{k in g} x ).
// The levels go to the matrix cores as 16 + q, which a 16-bit float holds exactly and one shift and one v_and_or_b32 make of two
// nibbles (the four bits are the highest of the mantissa of 16.0), so that with S = sum over g of x (a product with ones)
//   y += s_g * ((16 + q) . x) + (b_g - 16 s_g) * S,
// both sums in 32 bits.  x stays what it is: bf16 and f16 have matrix-core products of their own, and an f32 value goes in as
// three bf16 parts (24 bits together), against q - 8.
#include "bmx_internal.h"
#include "few_bits.h"
#include "k_steps.h"

#include <algorithm>

namespace bmx {
namespace {

// The bits of 16.0 in both halves, in a register: beside a literal v_and_or_b32 takes no other, and would fall into two instructions.
template <bool F16>
__device__ inline uint32_t sixteen() {
  uint32_t x = F16 ? 0x4C004C00 : 0x41804180;
  asm volatile("" : "+v"(x));
  return x;
}
// A lane's eight levels of a step, as 16 + q: field p of either half onto the mantissa's highest four bits.  For f32 results as q - 8, which
// costs two instructions a value more and keeps the sums small beside their result (error of 1 x 256 x 512 against 64 bits 7.6e-7, so 0.9e-7).
template <int TYPE>
constexpr float kZero = TYPE == BMX_F32 ? 8.0f : -16.0f;  // what q is more than the operand
template <int TYPE>
__device__ inline u32x4 levels(uint32_t w, uint32_t one) {
  constexpr uint32_t m = TYPE == BMX_F16 ? 0x03C003C0 : 0x00780078;
  if constexpr (TYPE == BMX_F16) return u32x4{((w << 6) & m) | one, ((w << 2) & m) | one, ((w >> 2) & m) | one, ((w >> 6) & m) | one};
  u32x4 x = {((w << 3) & m) | one, ((w >> 1) & m) | one, ((w >> 5) & m) | one, ((w >> 9) & m) | one};
  if constexpr (TYPE == BMX_F32) {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = upper_halves(__builtin_bit_cast(float, x[j] << 16) - 24.0f, __builtin_bit_cast(float, x[j] & 0xffff0000u) - 24.0f);
  }
  return x;
}

template <bool F16>
__device__ inline f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Eight values of x as they lie in memory, and as matrix-core operands: themselves, or three bf16 parts of f32 values, 8 bits each, cut off
// and not rounded (together they are the value).
template <int TYPE>
struct Eight {
  static constexpr int kParts = TYPE == BMX_F32 ? 3 : 1;
  u32x4 raw[TYPE == BMX_F32 ? 2 : 1];

  // (unaligned: the address is one of an element)
  __device__ void load(const void* x, int64_t at) {
    struct __attribute__((packed, aligned(TYPE == BMX_F32 ? 4 : 2))) Raw {
      u32x4 v[TYPE == BMX_F32 ? 2 : 1];
    };
    const Raw r = *reinterpret_cast<const Raw*>(static_cast<const char*>(x) + at * (TYPE == BMX_F32 ? 4 : 2));
#pragma unroll
    for (int i = 0; i < (TYPE == BMX_F32 ? 2 : 1); ++i) raw[i] = r.v[i];
  }
  // `left` values are there, the others are 0.
  __device__ void load(const void* x, int64_t at, int left) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (TYPE == BMX_F32) {
        raw[j / 4][j % 4] = j < left ? static_cast<const uint32_t*>(x)[at + j] : 0;
      } else {
        const uint32_t h = j < left ? static_cast<const uint16_t*>(x)[at + j] : 0;
        raw[0][j / 2] = j % 2 ? raw[0][j / 2] | h << 16 : h;
      }
    }
  }
  // 16-bit types: values k to k + 7 of a row of K >= 8 values that begins at `row`, those from K on 0, by one load.  Where the row ends inside, it
  // is of the row's last eight values, and they move down.
  __device__ void load_within(const uint16_t* x, int64_t row, int k, int K) {
    static_assert(TYPE != BMX_F32, "");
    load(x, row + min(k, K - 8));
    const int over = min(max(k + 8 - K, 0), 8);
    u32x4 v = raw[0];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __builtin_amdgcn_alignbit(j < 3 ? v[j < 3 ? j + 1 : 3] : 0, v[j], 16 * (over & 1));
#pragma unroll
    for (int by = 1; by <= 4; by *= 2)
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = over / 2 & by ? (j + by < 4 ? v[j + by < 4 ? j + by : 3] : 0) : v[j];
    raw[0] = v;
  }
  __device__ void parts(u32x4 (&part)[kParts]) const {
    if constexpr (TYPE != BMX_F32) {
      part[0] = raw[0];
    } else {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t bits = raw[j / 4][j % 4];
        v[j] = __builtin_bit_cast(float, bits);
      }
#pragma unroll
      for (int p = 0; p < kParts; ++p) {
#pragma unroll
        for (int j = 0; j < 4; ++j) part[p][j] = upper_halves(v[2 * j], v[2 * j + 1]);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = lower_part(v[j]);
      }
    }
  }
};

// One result by its definition, value by value.  The kernels' sums are inf - inf where x holds an infinity, and infinite where 31 x is beyond fp32
// and x w is not; what they find not to be finite comes from here.  (A NaN in x ends it.  Rare, and slow: an infinity in every row of 64 x 4096 x 4096
// bf16 1.3 ms, of 256 rows 5.0; without any the test of the results does not show.)
template <int TYPE, int GROUP>
__device__ inline float by_value(const void* x, int64_t ldx, const u32x4* tiles, const uint32_t* scales, int K, int m, int n) {
  const int64_t tile0 = (int64_t)(n / 16) * ((K + 127) / 128);
  float v = 0.0f;
#pragma unroll 1
  for (int k = 0; k < K && v == v; k += 8) {
    const int64_t tile = tile0 + k / 128;
    uint32_t w = reinterpret_cast<const uint32_t*>(tiles)[(tile * 64 + n % 16 + k % 32 / 8 * 16) * 4 + k % 128 / 32];
    const uint32_t sb = scales[(tile * (128 / GROUP) + k % 128 / GROUP) * 16 + n % 16];
    const float s = bf16_float(sb & 0xffff), b = __builtin_bit_cast(float, sb & 0xffff0000u);
#pragma unroll 1
    for (int j = 0; j < 8 && k + j < K; ++j) {
      const float q = (float)(w >> (j % 2 ? 16 + 2 * (j - 1) : 2 * j) & 15);
      v = __builtin_fmaf(load_one<TYPE>(x, m * ldx + k + j), s * q + b, v);
    }
  }
  return v;
}
__device__ inline bool finite(float v) { return fabsf(v) < INFINITY; }

constexpr int kMostWaves = 8;

// 16 outputs x 16 MT rows per workgroup, K dealt out to its waves in steps of 128 (1 KB of weights, 16 bytes a lane).  Each wave has DEPTH
// steps on their way: a step's registers are loaded for the step DEPTH further on as soon as they are used up.
template <int TYPE, int MT, int GROUP>
__global__ __launch_bounds__(kMostWaves * 64) void w4_rows_kernel(const void* x, int64_t ldx, const u32x4* tiles, const uint32_t* scales,
                                                                  const float* bias, int M, int N, int K, void* out, int64_t ldo) {
  constexpr bool F16 = TYPE == BMX_F16;
  constexpr int PARTS = Eight<TYPE>::kParts, PER = 128 / GROUP, STEPS = GROUP / 32, DEPTH = MT == 1 && TYPE != BMX_F32 ? 4 : 2;
  constexpr uint32_t one = F16 ? 0x3C003C00 : 0x3F803F80;
  __shared__ f32x4 red[kMostWaves][MT][64];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = blockDim.x / 64;
  const int g = lane / 16, nt = blockIdx.x, m0 = blockIdx.y * 16 * MT, full = K / 128, all = (K + 127) / 128;
  const u32x4 ones = {one, one, one, one};
  int64_t row[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) row[i] = (int64_t)min(m0 + 16 * i + lane % 16, M - 1) * ldx + 8 * g;  // (rows past the last: not stored)
  const Rsrc tile_rows = buffer(tiles + (int64_t)nt * all * 64, full * 1024), scale_rows = buffer(scales + (int64_t)nt * all * PER * 16, all * PER * 64);
  f32x4 acc[MT] = {};
  const uint32_t sixteens = sixteen<F16>();
  u32x4 w[DEPTH], sb[DEPTH][PER];
  Eight<TYPE> xs[DEPTH][MT][4];
  const auto load = [&](int d, int kt) {
    w[d] = load16(tile_rows, lane * 16, kt * 1024);
#pragma unroll
    for (int gi = 0; gi < PER; ++gi) sb[d][gi] = load16(scale_rows, g * 16, (kt * PER + gi) * 64);
  };
  const auto load_x = [&](int d, int kt, int i, int step) { xs[d][i][step].load(x, row[i] + kt * 128 + 32 * step); };
  // a step's products; next: the step to load in its place
  const auto multiply = [&](int d, int groups, int next) {
#pragma unroll
    for (int gi = 0; gi < PER; ++gi) {
      if (gi >= groups) break;  // (whatever scales lie behind the last group)
      f32x4 dot[MT] = {}, sum[MT] = {};
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        const int step = gi * STEPS + st;
        const u32x4 a = levels<TYPE>(w[d][step], sixteens);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          u32x4 b[PARTS];
          xs[d][i][step].parts(b);
#pragma unroll
          for (int p = 0; p < PARTS; ++p) {
            dot[i] = mfma<F16>(a, b[p], dot[i]);
            sum[i] = mfma<F16>(ones, b[p], sum[i]);
          }
          if (next >= 0) load_x(d, next, i, step);
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float s = bf16_float(sb[d][gi][j]), o = __builtin_bit_cast(float, sb[d][gi][j] & 0xffff0000) + kZero<TYPE> * s;
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[i][j] += s * dot[i][j] + o * sum[i][j];
      }
    }
    if (next >= 0) load(d, next);
  };
  if (wave < full) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      const int kt = k_step(wave, waves, d, full);
      load(d, kt);
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int step = 0; step < 4; ++step) load_x(d, kt, i, step);
    }
    for (int kt = wave; kt < full;) {
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        if (kt < full) multiply(d, PER, k_step(kt, waves, DEPTH, full));
        kt += waves;
      }
    }
  }
  if (full < all && wave == full % waves) {  // the last step, of fewer than 128 values
    w[0] = tiles[((int64_t)nt * all + full) * 64 + lane];
#pragma unroll
    for (int gi = 0; gi < PER; ++gi) sb[0][gi] = load16(scale_rows, g * 16, (full * PER + gi) * 64);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int step = 0; step < 4; ++step) xs[0][i][step].load(x, row[i] + full * 128 + 32 * step, K - (full * 128 + 32 * step + 8 * g));
    multiply(0, (K - full * 128 + GROUP - 1) / GROUP, -1);
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) red[wave][i][lane] = acc[i];
  __syncthreads();
  for (int e = threadIdx.x; e < 256 * MT; e += blockDim.x) {
    const int m = e / 16, n = e % 16;
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < kMostWaves; ++w) v += w < waves ? red[w][m / 16][m % 16 + 16 * (n / 4)][n % 4] : 0.0f;
    if (m0 + m < M && nt * 16 + n < N) {
      if (!finite(v)) v = by_value<TYPE, GROUP>(x, ldx, tiles, scales, K, m0 + m, nt * 16 + n);
      if (bias) v += bias[nt * 16 + n];
      store_one<TYPE>(out, (int64_t)(m0 + m) * ldo + nt * 16 + n, v);
    }
  }
}

template <int TYPE, int MT>
void launch_rows(const void* x, int64_t ldx, const void* tiles, const void* scales, int group, const float* bias, int M, int N, int K,
                 void* out, int64_t ldo, hipStream_t s) {
  // Four waves; eight where a CU has one workgroup, each wave many steps and x few rows.  us with four and eight, 4096 columns: bf16, one row, K = 9216 8.0, 7.7,
  // 8192 7.3, 7.1, 6144 6.3, 6.4, 4096 4.6, 5.0; four rows of 9216 9.2, 9.5, eight 10.5, 11.4.  f32, one row 4096 10.0, 8.7, 9216 19.2, 15.8; eight rows 10.2,
  // 9.8 and 20.3, 17.2; of K = 1024 5.2, 5.6; twelve rows of 4096 11.9, 12.6.
  const dim3 grid((N + 15) / 16, (M + 16 * MT - 1) / (16 * MT));
  const bool deep = TYPE == BMX_F32 ? M <= 8 && K >= 4096 : M <= 2 && K >= 8192;
  const dim3 block(64 * std::min(grid.x * grid.y <= 256 && deep ? 8 : 4, (K + 127) / 128));
  auto* t = static_cast<const u32x4*>(tiles);
  auto* sc = static_cast<const uint32_t*>(scales);
  const auto kern = group == 32 ? w4_rows_kernel<TYPE, MT, 32> : group == 64 ? w4_rows_kernel<TYPE, MT, 64> : w4_rows_kernel<TYPE, MT, 128>;
  launch_kernel(kern, grid, block, 0, s, x, ldx, t, sc, bias, M, N, K, out, ldo);
  note_kernel("w4_rows_kernel<%d,%d,%d> grid %dx%d block %d", TYPE, MT, group, (int)grid.x, (int)grid.y, (int)block.x);
}

// 16-bit types, 9 to 64 rows: as w4_rows_kernel, but a wave brings its steps of x into LDS of its own, a step ahead, and takes the operands from
// there.  (A lane's operand is 16 bytes of a row, and lanes side by side have rows below each other: read from memory so, 16 rows lie
// on the same banks of the L1, and 64 rows of 4096 took 13 of 18 us to come.)
template <int TYPE, int MT, int GROUP>
__global__ __launch_bounds__(1024 / MT) void w4_few_kernel(const uint16_t* x, int64_t ldx, bool async, const u32x4* tiles, const uint32_t* scales,
                                                           const float* bias, int M, int N, int K, void* out, int64_t ldo) {
  constexpr bool F16 = TYPE == BMX_F16;
  constexpr int PER = 128 / GROUP, STEPS = GROUP / 32, WAVES = 16 / MT, MINE = 4 * MT;
  constexpr uint32_t one = F16 ? 0x3C003C00 : 0x3F803F80;
  __shared__ u32x4 mem[WAVES][2][MT * 256];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), g = lane / 16;
  const int nt = blockIdx.x, m0 = blockIdx.y * 16 * MT, all = (K + 127) / 128;
  const u32x4 ones = {one, one, one, one};
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)mem[wave];
  // chunk c of a row's 16 chunks of eight values lies in place c ^ (row % 16)
  uint32_t from[MINE];
#pragma unroll
  for (int i = 0; i < MINE; ++i) from[i] = (uint32_t)((min(m0 + 4 * i + g, M - 1) - m0) * ldx + ((lane % 16) ^ ((4 * i + g) % 16)) * 8) * 2;
  const char* base = reinterpret_cast<const char*>(x + m0 * ldx);
  u32x4 w, sb[PER];
  const auto load = [&](int kt, int buf) {
    if (async && (kt + 1) * 128 <= K) {
#pragma unroll
      for (int i = 0; i < MINE; ++i) {
        const uint32_t to = lds + (buf * MT * 256 + i * 64) * 16;
        const char* b = base + kt * 256;
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(from[i]), "s"(b) : "memory");
      }
    } else {  // rows on odd elements, and the last step of fewer than 128 values: eight loads on their way at a time
      int id = lane;
      asm volatile("" : "+v"(id));  // (its addresses are made here, not ahead of the loop for every launch)
      const auto row = [&](int i) { return (int64_t)min(m0 + 4 * i + id / 16, M - 1) * ldx; };
      const auto chunk = [&](int i) { return kt * 128 + ((id % 16) ^ ((4 * i + id / 16) % 16)) * 8; };
#pragma unroll 1
      for (int i0 = 0; i0 < MINE; i0 += 8) {
        Eight<TYPE> in[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (K >= 8) in[i].load_within(x, row(i0 + i), chunk(i0 + i), K);
          else in[i].load(x, row(i0 + i) + chunk(i0 + i), K - chunk(i0 + i));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) mem[wave][buf][(i0 + i) * 64 + lane] = in[i].raw[0];
      }
    }
    const int64_t tile = (int64_t)nt * all + kt;
    w = tiles[tile * 64 + lane];
#pragma unroll
    for (int gi = 0; gi < PER; ++gi) sb[gi] = *reinterpret_cast<const u32x4*>(scales + (tile * PER + gi) * 16 + 4 * g);
  };
  f32x4 acc[MT] = {};
  const uint32_t sixteens = sixteen<F16>();
  if (wave < all) load(wave, 0);
  for (int kt = wave, buf = 0; kt < all; kt += WAVES, buf ^= 1) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const u32x4 wv = w;
    u32x4 sv[PER];
#pragma unroll
    for (int gi = 0; gi < PER; ++gi) sv[gi] = sb[gi];
    if (kt + WAVES < all) load(kt + WAVES, buf ^ 1);
#pragma unroll
    for (int gi = 0; gi < PER; ++gi) {
      if (kt * 128 + gi * GROUP >= K) break;  // (whatever scales lie behind the last group)
      f32x4 dot[MT] = {}, sum[MT] = {};
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        const int step = gi * STEPS + st;
        const u32x4 a = levels<TYPE>(wv[step], sixteens);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          const u32x4 b = mem[wave][buf][(16 * i + lane % 16) * 16 + ((4 * step + g) ^ (lane % 16))];
          dot[i] = mfma<F16>(a, b, dot[i]);
          sum[i] = mfma<F16>(ones, b, sum[i]);
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float s = bf16_float(sv[gi][j]), o = __builtin_bit_cast(float, sv[gi][j] & 0xffff0000) + kZero<TYPE> * s;
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[i][j] += s * dot[i][j] + o * sum[i][j];
      }
    }
  }
  __syncthreads();
  f32x4* red = reinterpret_cast<f32x4*>(mem);
#pragma unroll
  for (int i = 0; i < MT; ++i) red[(wave * MT + i) * 64 + lane] = acc[i];
  __syncthreads();
  for (int e = threadIdx.x; e < 256 * MT; e += 64 * WAVES) {
    const int m = e / 16, n = e % 16;
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += red[(w * MT + m / 16) * 64 + m % 16 + 16 * (n / 4)][n % 4];
    if (m0 + m < M && nt * 16 + n < N) {
      if (!finite(v)) v = by_value<TYPE, GROUP>(x, ldx, tiles, scales, K, m0 + m, nt * 16 + n);
      if (bias) v += bias[nt * 16 + n];
      store_one<TYPE>(out, (int64_t)(m0 + m) * ldo + nt * 16 + n, v);
    }
  }
}

template <int TYPE, int MT>
void launch_few(const void* x, int64_t ldx, const void* tiles, const void* scales, int group, const float* bias, int M, int N, int K,
                void* out, int64_t ldo, hipStream_t s) {
  const dim3 grid((N + 15) / 16, (M + 16 * MT - 1) / (16 * MT)), block(1024 / MT);
  const bool async = (uintptr_t)x % 4 == 0 && (M == 1 || ldx % 2 == 0);
  const auto kern = group == 32 ? w4_few_kernel<TYPE, MT, 32> : group == 64 ? w4_few_kernel<TYPE, MT, 64> : w4_few_kernel<TYPE, MT, 128>;
  launch_kernel(kern, grid, block, 0, s, static_cast<const uint16_t*>(x), ldx, async, static_cast<const u32x4*>(tiles),
                static_cast<const uint32_t*>(scales), bias, M, N, K, out, ldo);
  note_kernel("w4_few_kernel<%d,%d,%d> grid %dx%d block %d", TYPE, MT, group, (int)grid.x, (int)grid.y, (int)block.x);
}

// ---- many rows ----

using f32x16 = float __attribute__((ext_vector_type(16)));
template <bool F16>
__device__ inline f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <int CTRL>
__device__ inline float add_lane(float x) {  // x plus that of the lane which a row's permutation names
  const int other = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, false);
  return x + __builtin_bit_cast(float, other);
}

// f32: 64 x 128 of y per workgroup of 2 x 2 waves, 32 x 64 each.  x passes through registers, a step of 64 values ahead, into LDS in its three
// parts; the sums over groups, which the offsets take, are made on that way.
template <int GROUP>
__global__ __launch_bounds__(256) void w4_f32_kernel(const void* x, int64_t ldx, const u32x4* tiles, const uint32_t* scales,
                                                      const float* bias, int M, int N, int K, void* out, int64_t ldo) {
  constexpr int PARTS = 3, RB = 1, CB = 2, KS = 64, CH = KS / 8, BM = 64 * RB;  // values, and chunks of eight of them, of a step
  constexpr int G = GROUP < KS ? GROUP : KS, PER = KS / G, PER_TILE = 128 / GROUP, MINE = BM * CH / 256;
  __shared__ u32x4 xs[2][PARTS][BM * CH];
  __shared__ float sums[2][PER][BM];
  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64), h = lane / 32, wm = wave / 2, wn = wave % 2;
  const int all = (K + 127) / 128, steps = (K + KS - 1) / KS;
  // Tiles in bands of eight tiles of rows, dealt out so that an XCD (every eighth workgroup) has tiles side by side.
  const int mt = (M + BM - 1) / BM, ntl = (N + 64 * CB - 1) / (64 * CB), total = mt * ntl, eighth = (total + 7) / 8;
  const int id = blockIdx.x % 8 * eighth + blockIdx.x / 8;
  if (id >= total || (int)(blockIdx.x / 8) >= eighth) return;
  const int band = id / (8 * ntl), in_band = id - band * 8 * ntl, high = min(8, mt - band * 8);
  const int m0 = (band * 8 + in_band % high) * BM, n0 = in_band / high * 64 * CB;

  int64_t row[MINE];
#pragma unroll
  for (int i = 0; i < MINE; ++i) row[i] = (int64_t)min(m0 + (tid + 256 * i) / CH, M - 1) * ldx + tid % CH * 8;
  int64_t tile[CB];
  int col[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) {
    col[c] = n0 + (wn * CB + c) * 32 + lane % 32;
    tile[c] = (int64_t)min(col[c] / 16, (N - 1) / 16) * all;
  }
  Eight<BMX_F32> in[MINE];
  constexpr int WIDE = KS / 32;  // dwords of weights a lane has of a step, twice
  uint32_t w[CB][2][WIDE], sb[CB][PER];
  const auto load = [&](int t) {
    const int k0 = t * KS;
    if (k0 + KS <= K) {
#pragma unroll
      for (int i = 0; i < MINE; ++i) in[i].load(x, row[i] + k0);
    } else {
#pragma unroll
      for (int i = 0; i < MINE; ++i) in[i].load(x, row[i] + k0, K - k0 - tid % CH * 8);
    }
  };
  const auto load_weights = [&](int t) {
    const int kt = t * KS / 128;
#pragma unroll
    for (int c = 0; c < CB; ++c) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const u32x2 v = reinterpret_cast<const u32x2*>(tiles + (tile[c] + kt) * 64 + lane % 16 + 16 * (2 * half + h))[t % 2];
        w[c][half][0] = v[0], w[c][half][1] = v[1];
      }
#pragma unroll
      for (int gi = 0; gi < PER; ++gi) {
        const int k = t * KS + gi * G;  // (a group behind the last has any scale)
        sb[c][gi] = k < K ? scales[((tile[c] + kt) * PER_TILE + k % 128 / GROUP) * 16 + lane % 16] : 0;
      }
    }
  };
  const auto store = [&](int buf) {
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
      const int r = (tid + 256 * i) / CH, c = tid % CH;
      u32x4 part[PARTS];
      in[i].parts(part);
#pragma unroll
      for (int p = 0; p < PARTS; ++p) xs[buf][p][r * CH + (c ^ (r / 2 % 8))] = part[p];
      float s = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t bits = in[i].raw[j / 4][j % 4];
        s += __builtin_bit_cast(float, bits);
      }
      s = add_lane<0xb1>(s);  // (the four lanes of 32 values, and the eight of 64)
      s = add_lane<0x4e>(s);
      if constexpr (G >= 64) s = add_lane<0x141>(s);
      if (c % (G / 8) == 0) sums[buf][c / (G / 8)][r] = s;
    }
  };
  f32x16 acc[RB][CB] = {};
  const uint32_t sixteens = sixteen<false>();
  load(0);
  load_weights(0);
  store(0);
  __syncthreads();
  for (int t = 0; t < steps; ++t) {
    const int buf = t % 2;
    uint32_t v[CB][2][WIDE], sv[CB][PER];
#pragma unroll
    for (int c = 0; c < CB; ++c) {
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int j = 0; j < WIDE; ++j) v[c][half][j] = w[c][half][j];
#pragma unroll
      for (int gi = 0; gi < PER; ++gi) sv[c][gi] = sb[c][gi];
    }
    if (t + 1 < steps) load(t + 1), load_weights(t + 1);
#pragma unroll
    for (int gi = 0; gi < PER; ++gi) {
      f32x16 dot[RB][CB] = {};
#pragma unroll
      for (int si = 0; si < G / 16; ++si) {
        const int s = gi * (G / 16) + si;
        u32x4 b[CB];
#pragma unroll
        for (int c = 0; c < CB; ++c) b[c] = levels<BMX_F32>(v[c][s % 2][s / 2], sixteens);
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          const int rr = (wm * RB + r) * 32 + lane % 32, at = rr * CH + ((2 * s + h) ^ (rr / 2 % 8));
#pragma unroll
          for (int p = 0; p < PARTS; ++p) {
            const u32x4 a = xs[buf][p][at];
#pragma unroll
            for (int c = 0; c < CB; ++c) dot[r][c] = mfma32<false>(a, b[c], dot[r][c]);
          }
        }
      }
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        f32x4 sum[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = *reinterpret_cast<const f32x4*>(&sums[buf][gi][(wm * RB + r) * 32 + 8 * i + 4 * h]);
#pragma unroll
        for (int c = 0; c < CB; ++c) {
          const float sc = bf16_float(sv[c][gi]), o = __builtin_bit_cast(float, sv[c][gi] & 0xffff0000u) + kZero<BMX_F32> * sc;
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[r][c][i] += sc * dot[r][c][i] + o * sum[i / 4][i % 4];
        }
      }
    }
    if (t + 1 < steps) store(1 - buf);
    __syncthreads();
  }
  bool good = true;
#pragma unroll
  for (int c = 0; c < CB; ++c) {
    if (col[c] >= N) continue;
    const float add = bias ? bias[col[c]] : 0.0f;
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int m = m0 + (wm * RB + r) * 32 + 8 * (i / 4) + 4 * h + i % 4;
        if (m < M) store_one<BMX_F32>(out, (int64_t)m * ldo + col[c], acc[r][c][i] + add);
        good &= finite(acc[r][c][i]);
      }
  }
  if (good) return;
#pragma unroll 1
  for (int e = 0; e < CB * RB * 16; ++e) {  // (from this lane's own stores, so that no register waits for it)
    const int n = n0 + (wn * CB + e / (RB * 16)) * 32 + lane % 32, m = m0 + (wm * RB + e / 16 % RB) * 32 + e % 16 / 4 * 8 + 4 * h + e % 4;
    if (m >= M || n >= N || finite(load_one<BMX_F32>(out, (int64_t)m * ldo + n))) continue;
    store_one<BMX_F32>(out, (int64_t)m * ldo + n, by_value<BMX_F32, GROUP>(x, ldx, tiles, scales, K, m, n) + (bias ? bias[n] : 0.0f));
  }
}

// 16-bit types: 64 RB x 64 CB of y per workgroup of 2 x 2 waves, 32 RB x 32 CB each.  x comes into LDS without passing registers, a step ahead.  Sums
// over the groups of x, which the offsets take, are products with ones on the matrix cores: one for each other at 64 x 64, one for four at 128 x 128, where of a
// wave's two 32-row blocks each column of waves makes its own, and they meet through LDS a step later.  With SPLIT the workgroup has as many sets of four waves, which take turns at K's steps and join at the end.
template <int TYPE, int RB, int CB, int GROUP, int SPLIT>
__global__ __launch_bounds__(256 * SPLIT, SPLIT == 1 ? 2 : SPLIT) void w4_deep_kernel(const uint16_t* x, int64_t ldx, bool async, const u32x4* tiles,
                                                                 const uint32_t* scales, const float* bias, int M, int N, int K,
                                                                 void* out, int64_t ldo) {
  static_assert(TYPE != BMX_F32, "");
  constexpr bool F16 = TYPE == BMX_F16, SHARE = RB == 2;
  constexpr int BM = 64 * RB, MINE = BM / 16, PER = 128 / GROUP, STEPS = GROUP / 16;
  static_assert(!SHARE || (PER == 1 && SPLIT == 1), "");
  constexpr uint32_t one = F16 ? 0x3C003C00 : 0x3F803F80;
  constexpr int kX = BM * 16;  // of a step, in 16 bytes
  __shared__ u32x4 mem[SPLIT * 2 * kX];
  __shared__ float sums[SHARE ? 2 : 1][SHARE ? BM : 4];
  const int set = __builtin_amdgcn_readfirstlane(threadIdx.x / 256), tid = threadIdx.x % 256;
  const int lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64), h = lane / 32, wm = wave / 2, wn = wave % 2;
  const int all = (K + 127) / 128;
  // Tiles in bands of eight tiles of rows, dealt out so that an XCD (every eighth workgroup) has tiles side by side.
  const int mt = (M + BM - 1) / BM, ntl = (N + 64 * CB - 1) / (64 * CB), total = mt * ntl, eighth = (total + 7) / 8;
  const int id = blockIdx.x % 8 * eighth + blockIdx.x / 8;
  if (id >= total || (int)(blockIdx.x / 8) >= eighth) return;
  const int band = id / (8 * ntl), in_band = id - band * 8 * ntl, high = min(8, mt - band * 8);
  const int m0 = (band * 8 + in_band % high) * BM, n0 = in_band / high * 64 * CB;

  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)mem;
  const auto at_x = [&](int buf) { return (set * 2 + buf) * kX; };
  // A row's 16 chunks of eight values lie in 16 places, chunk c in place c ^ (row % 16), so that 16 rows' chunks of one number lie on all banks.
  const int chunk = tid % 16 ^ tid / 16;
  uint32_t from[MINE];
#pragma unroll
  for (int i = 0; i < MINE; ++i) from[i] = (uint32_t)((min(m0 + tid / 16 + 16 * i, M - 1) - m0) * ldx + chunk * 8) * 2;
  const char* base = reinterpret_cast<const char*>(x + m0 * ldx);
  int64_t tile[CB];
  int col[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) {
    col[c] = n0 + (wn * CB + c) * 32 + lane % 32;
    tile[c] = (int64_t)min(col[c] / 16, (N - 1) / 16) * all;
  }
  const auto stage = [&](int t, int buf) {
    if (async && (t + 1) * 128 <= K) {
#pragma unroll
      for (int i = 0; i < MINE; ++i) {
        const uint32_t to = lds + (at_x(buf) + i * 256 + wave * 64) * 16;
        const char* b = base + t * 256;
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(from[i]), "s"(b) : "memory");
      }
    } else {  // rows on odd elements, and the last step of fewer than 128 values: four loads on their way at a time
      int id = tid;
      asm volatile("" : "+v"(id));  // (its addresses are made here, not ahead of the loop for every launch)
      const int k = t * 128 + (id % 16 ^ id / 16) * 8;
#pragma unroll 1
      for (int i0 = 0; i0 < MINE; i0 += 4) {
        Eight<TYPE> in[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int64_t row = (int64_t)min(m0 + id / 16 + 16 * (i0 + i), M - 1) * ldx;
          if (K >= 8) in[i].load_within(x, row, k, K);
          else in[i].load(x, row + k, K - k);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) mem[at_x(buf) + (i0 + i) * 256 + tid] = in[i].raw[0];
      }
    }
  };
  u32x4 w[CB][2];
  uint32_t sb[CB][PER];
  const auto load_weights = [&](int t) {
#pragma unroll
    for (int c = 0; c < CB; ++c) {
#pragma unroll
      for (int half = 0; half < 2; ++half) w[c][half] = tiles[(tile[c] + t) * 64 + lane % 16 + 16 * (2 * half + h)];
#pragma unroll
      for (int gi = 0; gi < PER; ++gi)  // (a group behind the last has any scale)
        sb[c][gi] = t * 128 + gi * GROUP < K ? scales[((tile[c] + t) * PER + gi) * 16 + lane % 16] : 0;
    }
  };
  f32x16 acc[RB][CB] = {};
  const uint32_t sixteens = sixteen<F16>();
  float o_before[CB] = {};
  const auto offsets = [&](int buf) {  // the step before's sums times its offsets
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 sum = *reinterpret_cast<const f32x4*>(&sums[buf][(wm * RB + r) * 32 + 8 * i + 4 * h]);
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[r][c][4 * i + j] += o_before[c] * sum[j];
      }
  };
  if (set < all) {
    load_weights(set);
    stage(set, 0);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  for (int i = 0; i * SPLIT < all; ++i) {
    const int t = i * SPLIT + set, buf = i % 2;
    if (SPLIT == 1 || t < all) {
      u32x4 v[CB][2];
      uint32_t sv[CB][PER];
#pragma unroll
      for (int c = 0; c < CB; ++c) {
        v[c][0] = w[c][0], v[c][1] = w[c][1];
#pragma unroll
        for (int gi = 0; gi < PER; ++gi) sv[c][gi] = sb[c][gi];
      }
      if (t + SPLIT < all) {
        stage(t + SPLIT, 1 - buf);
        load_weights(t + SPLIT);
      }
      if constexpr (SHARE)
        if (t > 0) offsets((t - 1) % 2);
#pragma unroll
      for (int gi = 0; gi < PER; ++gi) {
        if constexpr (PER > 1) __builtin_amdgcn_sched_barrier(0);  // (registers: one group's products at a time)
        f32x16 dot[RB][CB] = {}, sum = {};
#pragma unroll
        for (int si = 0; si < STEPS; ++si) {
          const int s = gi * STEPS + si;
          u32x4 b[CB];
#pragma unroll
          for (int c = 0; c < CB; ++c) b[c] = levels<TYPE>(v[c][s % 2][s / 2], sixteens);
          u32x4 xr[RB];
#pragma unroll
          for (int r = 0; r < RB; ++r) {
            const int rr = (wm * RB + r) * 32 + lane % 32;
            xr[r] = mem[at_x(buf) + rr * 16 + ((2 * s + h) ^ rr % 16)];
#pragma unroll
            for (int c = 0; c < CB; ++c) dot[r][c] = mfma32<F16>(xr[r], b[c], dot[r][c]);
          }
          sum = mfma32<F16>(SHARE && wn == 1 ? xr[RB - 1] : xr[0], u32x4{one, one, one, one}, sum);
        }
#pragma unroll
        for (int c = 0; c < CB; ++c) {
          const float sc = bf16_float(sv[c][gi] & 0xffff), o = __builtin_bit_cast(float, sv[c][gi] & 0xffff0000u) + kZero<TYPE> * sc;
#pragma unroll
          for (int r = 0; r < RB; ++r)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[r][c][i] += SHARE ? sc * dot[r][c][i] : sc * dot[r][c][i] + o * sum[i];
          o_before[c] = o;
        }
        if constexpr (SHARE) {
          if (lane % 32 == 0)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *reinterpret_cast<f32x4*>(&sums[t % 2][(wm * RB + wn) * 32 + 8 * i + 4 * h]) = f32x4{sum[4 * i], sum[4 * i + 1], sum[4 * i + 2], sum[4 * i + 3]};
        }
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the next step has come
    __syncthreads();
  }
  if constexpr (SHARE) offsets((all - 1) % 2);
  if constexpr (SPLIT > 1) {  // the other sets' parts, in their order
    float* part = reinterpret_cast<float*>(mem);
    if (set > 0) {
#pragma unroll
      for (int i = 0; i < 16; ++i) part[(((set - 1) * 4 + wave) * 16 + i) * 64 + lane] = acc[0][0][i];
    }
    __syncthreads();
    if (set > 0) return;
#pragma unroll
    for (int p = 0; p < SPLIT - 1; ++p)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[0][0][i] += part[((p * 4 + wave) * 16 + i) * 64 + lane];
  }
  bool good = true;
#pragma unroll
  for (int c = 0; c < CB; ++c) {
    if (col[c] >= N) continue;
    const float add = bias ? bias[col[c]] : 0.0f;
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int m = m0 + (wm * RB + r) * 32 + 8 * (i / 4) + 4 * h + i % 4;
        if (m < M) store_one<TYPE>(out, (int64_t)m * ldo + col[c], acc[r][c][i] + add);
        good &= finite(acc[r][c][i]);
      }
  }
  if (good) return;
#pragma unroll 1
  for (int e = 0; e < CB * RB * 16; ++e) {  // (from this lane's own stores, so that no register waits for it)
    const int n = n0 + (wn * CB + e / (RB * 16)) * 32 + lane % 32, m = m0 + (wm * RB + e / 16 % RB) * 32 + e % 16 / 4 * 8 + 4 * h + e % 4;
    if (m >= M || n >= N || finite(load_one<TYPE>(out, (int64_t)m * ldo + n))) continue;
    store_one<TYPE>(out, (int64_t)m * ldo + n, by_value<TYPE, GROUP>(x, ldx, tiles, scales, K, m, n) + (bias ? bias[n] : 0.0f));
  }
}

template <int TYPE, int RB, int CB, int SPLIT>
void launch_deep(const void* x, int64_t ldx, const void* tiles, const void* scales, int group, const float* bias, int M, int N, int K,
                 void* out, int64_t ldo, hipStream_t s) {
  const int64_t total = ceil_div(M, 64 * RB) * ceil_div(N, 64 * CB);
  const dim3 grid((uint32_t)(ceil_div(total, 8) * 8));
  auto* t = static_cast<const u32x4*>(tiles);
  auto* sc = static_cast<const uint32_t*>(scales);
  const bool async = (uintptr_t)x % 4 == 0 && (M == 1 || ldx % 2 == 0);
  const auto pick = [&] {
    if constexpr (RB * CB == 1) {
      if (group == 32) return w4_deep_kernel<TYPE, RB, CB, 32, SPLIT>;
      if (group == 64) return w4_deep_kernel<TYPE, RB, CB, 64, SPLIT>;
    }
    return w4_deep_kernel<TYPE, RB, CB, 128, SPLIT>;
  };
  launch_kernel(pick(), grid, dim3(256 * SPLIT), 0, s, static_cast<const uint16_t*>(x), ldx, async, t, sc, bias, M, N, K, out, ldo);
  note_kernel("w4_deep_kernel<%d,%d,%d,%d,%d> grid %d block %d", TYPE, RB, CB, group, SPLIT, (int)grid.x, 256 * SPLIT);
}

// Few rows: 16 columns a workgroup, a stream of weights.  More: tiles of 64 x 64, or of 128 x 128 where they fill the chip.
// 16-bit types, us of the kernel of few rows, through LDS, in tiles.  K = 4096, 4096 columns: 16 rows 8.1, 5.7, 17; 32 rows 12.1, 6.7, 18; 64 rows 21,
// 11.6, 18.5.  Up to 32 rows LDS is ahead for more columns too where rows are whole (steps of 128, on whole dwords): 32 rows of 6144 21.0, 11.0,
// 18.4; 9216 30.0, 15.8, 18.7; 12288 30.1, 16.6, 19.2; 16384 39, 21.4, 20.4; of K = 1024 13.7, 7.6, 8.8 at 9216; where they are not it is behind from
// 6145 on: K = 1028, 9216 columns, 17 rows 9.5, 11.5, 8.9, 16 rows 8.6, 11.2, 8.8; on odd elements (K = 1023) 25, 11.9, 10.4 and 31, 12.2, 11.1.  33 to 64 rows
// come through LDS while a CU has one workgroup of them: 64 rows of 4096 and of 4112 columns, K = 1024, 10.3, 6.1, 9.2 and 13.8, 9.9, 9.2; K = 8192 35.7,
// 18.8, 31.0 and 51.6, 32.4, 31.3; and not on odd elements (K = 4095: 67, 60, 31; K = 513: 23, 12.4, 9.9).
// Tiles in four, two, one set: 256 rows 20, 22, 28; 512 rows 37, 35, 36; 2048 rows 145, 127, 120, and 90 in tiles of 128 x 128.
// f32: the tiles' time is 6 us and 0.0255 for each of K while the chip holds them at once, that of few rows 0.0165 us and 1.43e-5 of K for each of its workgroups (of 32
// rows): level at 1780 (K + 235) / (K + 1150) of them.  4096 columns, few rows and tiles: K = 512, 96 rows 19.6, 19.1, 160 rows 30.5, 19.3; K = 2048, 160 rows
// 58.8, 58.6; K = 4096, 160 rows 95, 110, 192 rows 114, 110; K = 8192, 192 rows 200, 215; 2048 rows of K = 4096 1150, 294.
template <int TYPE>
void launch_typed(const void* x, int64_t ldx, const void* tiles, const void* scales, int group, const float* bias, int M, int N, int K,
                  void* out, int64_t ldo, hipStream_t s) {
  const bool dwords = (uintptr_t)x % 4 == 0 && (M == 1 || ldx % 2 == 0);  // (rows on whole dwords)
  const int64_t small = ceil_div(M, 64) * ceil_div(N, 64), large = ceil_div(M, 128) * ceil_div(N, 128);
  if constexpr (TYPE == BMX_F32) {
    if (M > 32 && ceil_div(M, 32) * ceil_div(N, 16) * (K + 1150) > 1780 * (int64_t)(K + 235)) {
      const dim3 grid((uint32_t)(ceil_div(ceil_div(M, 64) * ceil_div(N, 128), 8) * 8));
      const auto kern = group == 32 ? w4_f32_kernel<32> : group == 64 ? w4_f32_kernel<64> : w4_f32_kernel<128>;
      launch_kernel(kern, grid, dim3(256), 0, s, x, ldx, static_cast<const u32x4*>(tiles), static_cast<const uint32_t*>(scales), bias, M, N, K, out, ldo);
      note_kernel("w4_f32_kernel<%d> grid %d block 256", group, (int)grid.x);
      return;
    }
  } else if (M > 8 && (M <= 32 ? N <= 6144 || (N <= 12288 && K % 128 == 0 && dwords) : M <= 64 && N <= 4096 && dwords) && ldx < (1 << 24)) {
    const auto f = M <= 32 ? launch_few<TYPE, 2> : launch_few<TYPE, 4>;
    f(x, ldx, tiles, scales, group, bias, M, N, K, out, ldo, s);
    return;
  } else if (M > 8 && (M > 32 || (N > 6144 && (M > 16 || !dwords))) && ldx < (1 << 24)) {  // (offsets within a tile's rows in 32 bits)
    const auto f = group == 128 && large >= 256 ? launch_deep<TYPE, 2, 2, 1> : small <= 256 ? launch_deep<TYPE, 1, 1, 4>
                 : small <= 512 ? launch_deep<TYPE, 1, 1, 2> : launch_deep<TYPE, 1, 1, 1>;
    f(x, ldx, tiles, scales, group, bias, M, N, K, out, ldo, s);
    return;
  }
  const auto f = M <= 16 ? launch_rows<TYPE, 1> : launch_rows<TYPE, 2>;
  f(x, ldx, tiles, scales, group, bias, M, N, K, out, ldo, s);
}

// A bf16 that is no infinity: the quantiser's scales and offsets stay finite.
__device__ inline uint32_t finite_bf16(float x) {
  const uint32_t h = bf16_bits(x);
  return (h & 0x7fff) == 0x7f80 ? h - 1 : h;
}

// One wave per tile of 16 outputs x 128 values, in the lanes' own order.  A group's values lie in the four lanes of an output.
template <int GROUP>
__global__ __launch_bounds__(64) void w4_quantize_kernel(const float* w, int64_t ldw, int N, int K, u32x4* tiles, uint32_t* scales) {
  constexpr int PER = 128 / GROUP, STEPS = GROUP / 32;
  const int lane = threadIdx.x, g = lane / 16, kt_all = (K + 127) / 128;
  const int64_t tile = blockIdx.x;
  const int nt = (int)(tile / kt_all), kt = (int)(tile % kt_all), n = nt * 16 + lane % 16;
  const float* row = w + (int64_t)min(n, N - 1) * ldw;
  u32x4 packed;
#pragma unroll
  for (int gi = 0; gi < PER; ++gi) {
    float v[STEPS][8], lo = INFINITY, hi = -INFINITY;
#pragma unroll
    for (int st = 0; st < STEPS; ++st)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int k = kt * 128 + (gi * STEPS + st) * 32 + 8 * g + j;
        const bool there = n < N && k < K;
        v[st][j] = there ? row[k] : NAN;
        if (fabsf(v[st][j]) < INFINITY) lo = fminf(lo, v[st][j]), hi = fmaxf(hi, v[st][j]);
      }
#pragma unroll
    for (int m = 16; m <= 32; m *= 2) lo = fminf(lo, __shfl_xor(lo, m)), hi = fmaxf(hi, __shfl_xor(hi, m));
    if (!(lo <= hi)) lo = hi = 0.0f;  // no finite value
    const uint32_t sb = finite_bf16(hi / 15.0f - lo / 15.0f), ob = finite_bf16(lo);
    const float s = bf16_float(sb), o = bf16_float(ob), r = s >= 0x1p-126f ? 1.0f / s : 0.0f;
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      uint32_t d = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // (a difference beyond the largest float is a level beyond the last; NaN is level 0)
        const float z = (v[st][j] - o) * r;
        const uint32_t q = (uint32_t)fminf(fmaxf(rintf(z), 0.0f), 15.0f);
        d |= q << (4 * (j % 2 ? 4 + j / 2 : j / 2));
      }
      packed[gi * STEPS + st] = d;
    }
    if (g == 0) scales[(tile * PER + gi) * 16 + lane] = sb | ob << 16;
  }
  tiles[tile * 64 + lane] = packed;
}

template <int GROUP>
__global__ __launch_bounds__(64) void w4_dequantize_kernel(const u32x4* tiles, const uint32_t* scales, int N, int K, float* w, int64_t ldw) {
  constexpr int PER = 128 / GROUP, STEPS = GROUP / 32;
  const int lane = threadIdx.x, g = lane / 16, kt_all = (K + 127) / 128;
  const int64_t tile = blockIdx.x;
  const int nt = (int)(tile / kt_all), kt = (int)(tile % kt_all), n = nt * 16 + lane % 16;
  if (n >= N) return;
  const u32x4 packed = tiles[tile * 64 + lane];
#pragma unroll
  for (int step = 0; step < 4; ++step) {
    const uint32_t sb = scales[(tile * PER + step / STEPS) * 16 + lane % 16];
    const float s = bf16_float(sb), o = __builtin_bit_cast(float, sb & 0xffff0000);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int k = kt * 128 + step * 32 + 8 * g + j;
      const float q = (float)(packed[step] >> (4 * (j % 2 ? 4 + j / 2 : j / 2)) & 15);
      if (k < K) w[(int64_t)n * ldw + k] = s * q + o;
    }
  }
}

}  // namespace

hipError_t launch_w4_fc(const void* x, int type, int64_t ldx, const void* tiles, const void* scales, int group, const float* bias, int M,
                        int N, int K, void* out, int64_t ldo, hipStream_t s) {
  const auto f = type == BMX_F32 ? launch_typed<BMX_F32> : type == BMX_F16 ? launch_typed<BMX_F16> : launch_typed<BMX_BF16>;
  f(x, ldx, tiles, scales, group, bias, M, N, K, out, ldo, s);
  return launch_error();
}

hipError_t launch_w4_quantize(const float* w, int64_t ldw, int N, int K, int group, void* tiles, void* scales, hipStream_t s) {
  const dim3 grid((uint32_t)(ceil_div(N, 16) * ceil_div(K, 128)));
  const auto kern = group == 32 ? w4_quantize_kernel<32> : group == 64 ? w4_quantize_kernel<64> : w4_quantize_kernel<128>;
  launch_kernel(kern, grid, dim3(64), 0, s, w, ldw, N, K, static_cast<u32x4*>(tiles), static_cast<uint32_t*>(scales));
  note_kernel("w4_quantize_kernel<%d> grid %u block 64", group, grid.x);
  return launch_error();
}

hipError_t launch_w4_dequantize(const void* tiles, const void* scales, int N, int K, int group, float* w, int64_t ldw, hipStream_t s) {
  const dim3 grid((uint32_t)(ceil_div(N, 16) * ceil_div(K, 128)));
  const auto kern = group == 32 ? w4_dequantize_kernel<32> : group == 64 ? w4_dequantize_kernel<64> : w4_dequantize_kernel<128>;
  launch_kernel(kern, grid, dim3(64), 0, s, static_cast<const u32x4*>(tiles), static_cast<const uint32_t*>(scales), N, K, w, ldw);
  note_kernel("w4_dequantize_kernel<%d> grid %u block 64", group, grid.x);
  return launch_error();
}

}  // namespace bmx
