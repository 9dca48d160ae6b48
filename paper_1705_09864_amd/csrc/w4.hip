// Products with 4-bit weights: w[n][k] = s * q + b, a scale s and an offset b for each group of 32, 64 or 128 values of a row,
//   y[m][n] = sum_k x[m][k] w[n][k] = sum_g ( s_g * sum_{k in g} q x + b_g * sum_{k in g} x ).
// The levels go to the matrix cores as 16 + q, which a 16-bit float holds exactly and one shift and one v_and_or_b32 make of two
// nibbles (the four bits are the highest of the mantissa of 16.0), so that with S = sum over g of x (a product with ones)
//   y += s_g * ((16 + q) . x) + (b_g - 16 s_g) * S,
// both sums in 32 bits.  x stays what it is: bf16 and f16 have matrix-core products of their own, and an f32 value goes in as
// three bf16 parts (24 bits together).
#include "bmx_internal.h"
#include "few_bits.h"

namespace bmx {
namespace {

constexpr int kWaves = 8;

// The 32 levels of a lane's 16 bytes at step `step` (eight of them), as 16 + q.
template <bool F16>
__device__ inline u32x4 levels(uint32_t w) {
  // (field p of the low half and of the high half, onto the mantissa's highest four bits)
  if constexpr (F16) {
    constexpr uint32_t m = 0x03C003C0, one = 0x4C004C00;
    return u32x4{((w << 6) & m) | one, ((w << 2) & m) | one, ((w >> 2) & m) | one, ((w >> 6) & m) | one};
  } else {
    constexpr uint32_t m = 0x00780078, one = 0x41804180;
    return u32x4{((w << 3) & m) | one, ((w >> 1) & m) | one, ((w >> 5) & m) | one, ((w >> 9) & m) | one};
  }
}

template <bool F16>
__device__ inline f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Eight values of x as matrix-core operands: one, or three bf16 parts of f32 values.
template <int TYPE>
__device__ inline void operand(const void* x, int64_t at, int left, bool aligned, u32x4 (&part)[TYPE == BMX_F32 ? 3 : 1]) {
  if constexpr (TYPE != BMX_F32) {
    if (left >= 8 && aligned) {
      part[0] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(x) + at);
    } else {
      uint32_t h[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) h[j] = j < left ? static_cast<const uint16_t*>(x)[at + j] : 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) part[0][j] = h[2 * j] | h[2 * j + 1] << 16;
    }
  } else {
    float v[8];
    load_eight<TYPE>(x, at, left, aligned, v);
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      uint32_t h[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        h[j] = bf16_bits(v[j]);
        v[j] -= bf16_float(h[j]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) part[p][j] = h[2 * j] | h[2 * j + 1] << 16;
    }
  }
}

// 16 outputs x 16 MT rows per workgroup, K dealt out to its waves in steps of 128 (1 KB of weights, 16 bytes a lane).
template <int TYPE, int MT, int GROUP>
__global__ __launch_bounds__(kWaves * 64) void w4_rows_kernel(const void* x, int64_t ldx, bool aligned, const u32x4* tiles,
                                                              const uint32_t* scales, const float* bias, int M, int N, int K,
                                                              void* out, int64_t ldo) {
  constexpr bool F16 = TYPE == BMX_F16;
  constexpr int PARTS = TYPE == BMX_F32 ? 3 : 1, PER = 128 / GROUP, STEPS = GROUP / 32;
  constexpr uint32_t one = F16 ? 0x3C003C00 : 0x3F803F80;
  __shared__ f32x4 red[kWaves][MT][64];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = blockDim.x / 64;
  const int g = lane / 16, nt = blockIdx.x, m0 = blockIdx.y * 16 * MT, kt_all = (K + 127) / 128;
  const u32x4 ones = {one, one, one, one};
  int64_t row[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) row[i] = (int64_t)min(m0 + 16 * i + lane % 16, M - 1) * ldx;  // (rows past the last: not stored)
  f32x4 acc[MT] = {};
  for (int kt = wave; kt < kt_all; kt += waves) {
    const int64_t tile = (int64_t)nt * kt_all + kt;
    const u32x4 w = tiles[tile * 64 + lane];
#pragma unroll
    for (int gi = 0; gi < PER; ++gi) {
      if (kt * 128 + gi * GROUP >= K) break;  // (whatever scales lie there)
      const u32x4 sb = *reinterpret_cast<const u32x4*>(scales + (tile * PER + gi) * 16 + 4 * g);
      f32x4 dot[MT] = {}, sum[MT] = {};
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        const int step = gi * STEPS + st, k = kt * 128 + 32 * step + 8 * g;
        const u32x4 a = levels<F16>(w[step]);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          u32x4 b[PARTS];
          operand<TYPE>(x, row[i] + k, K - k, aligned, b);
#pragma unroll
          for (int p = 0; p < PARTS; ++p) {
            dot[i] = mfma<F16>(a, b[p], dot[i]);
            sum[i] = mfma<F16>(ones, b[p], sum[i]);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float s = bf16_float(sb[j]), o = __builtin_bit_cast(float, sb[j] & 0xffff0000) - 16.0f * s;
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[i][j] += s * dot[i][j] + o * sum[i][j];
      }
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) red[wave][i][lane] = acc[i];
  __syncthreads();
  for (int e = threadIdx.x; e < 256 * MT; e += blockDim.x) {
    const int m = e / 16, n = e % 16;
    float v = 0.0f;
    for (int w = 0; w < waves; ++w) v += red[w][m / 16][m % 16 + 16 * (n / 4)][n % 4];
    if (m0 + m < M && nt * 16 + n < N) {
      if (bias) v += bias[nt * 16 + n];
      store_one<TYPE>(out, (int64_t)(m0 + m) * ldo + nt * 16 + n, v);
    }
  }
}

template <int TYPE, int MT>
void launch_rows(const void* x, int64_t ldx, bool aligned, const void* tiles, const void* scales, int group, const float* bias, int M,
                 int N, int K, void* out, int64_t ldo, hipStream_t s) {
  const dim3 grid((N + 15) / 16, (M + 16 * MT - 1) / (16 * MT)), block(64 * min(kWaves, (K + 127) / 128));
  auto* t = static_cast<const u32x4*>(tiles);
  auto* sc = static_cast<const uint32_t*>(scales);
  const auto kern = group == 32 ? w4_rows_kernel<TYPE, MT, 32> : group == 64 ? w4_rows_kernel<TYPE, MT, 64> : w4_rows_kernel<TYPE, MT, 128>;
  launch_kernel(kern, grid, block, 0, s, x, ldx, aligned, t, sc, bias, M, N, K, out, ldo);
  note_kernel("w4_rows_kernel<%d,%d,%d> grid %dx%d block %d", TYPE, MT, group, (int)grid.x, (int)grid.y, (int)block.x);
}

template <int TYPE>
void launch_typed(const void* x, int64_t ldx, const void* tiles, const void* scales, int group, const float* bias, int M, int N, int K,
                  void* out, int64_t ldo, hipStream_t s) {
  const bool aligned = (uintptr_t)x % 16 == 0 && (M == 1 || ldx * type_bytes(TYPE) % 16 == 0);
  const auto f = M <= 16 ? launch_rows<TYPE, 1> : M <= 32 ? launch_rows<TYPE, 2> : launch_rows<TYPE, 4>;
  f(x, ldx, aligned, tiles, scales, group, bias, M, N, K, out, ldo, s);
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
