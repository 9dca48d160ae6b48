// The end of an attention over a cache of pages: 16 rows of queries whose waves went over pages of their own, joined through LDS, and the
// workgroups that share a sequence's pages, joined by the last of them to arrive, in their order, so the result does not depend on which that was.
#pragma once
#include "few_bits.h"

namespace bmx {

// Numbers that workgroups of other XCDs read, each with an L2 of its own: written through and read past it (relaxed atomics of the device's
// scope, eight bytes each), so nobody has to write back or throw away a whole L2, as a fence of that scope does.
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

constexpr int kJoinWaves = 4;      // of a workgroup
constexpr int kMostSplits = 128;   // workgroups that share a sequence's pages

struct JoinTo {
  void* out;
  int64_t out_row, out_head;
  float* lse;
  float* parts;       // [unit][split][part_rows][ROW + 4]: the rows' results, maximum and sum
  uint32_t* arrived;  // [unit], zeros between the calls
  int q_heads, share, splits, part_rows;
};

template <int ROW>
struct JoinLds {
  static constexpr int LINE = ROW + 4;
  float red[kJoinWaves * 16 * LINE], red_m[kJoinWaves][16], red_l[kJoinWaves][16], factor_of[kMostSplits][16], sum_of[kMostSplits][16];
  uint32_t place;
};

// red, red_m (of scores times log2 e) and red_l are filled and the workgroup is past a barrier.  Rows r0 to r0 + rows of a head of the cache; token0: the row of
// queries that the sequence's first is; unit: number of these rows among all that are joined; used: workgroups that have a part of them, this one the split-th.
template <int TYPE, int ROW>
__device__ inline void join_rows(JoinLds<ROW>& s, const JoinTo& to, int dim, int64_t token0, int head, int r0, int rows, int64_t unit, int split, int used) {
  constexpr int LINE = ROW + 4, kWaves = kJoinWaves;
  const int quads = rows * (ROW / 4);
  float* parts = to.parts + unit * to.splits * to.part_rows * LINE;
  const auto store = [&](int i, int d, f32x4 x, float top, float sum) {
    const int64_t t = token0 + (r0 + i) / to.share;
    const int h = head * to.share + (r0 + i) % to.share;
#pragma unroll
    for (int j = 0; j < 4; ++j)  // (a row that sees nothing is zeros)
      if (d + j < dim) store_one<TYPE>(to.out, t * to.out_row + h * to.out_head + d + j, sum == 0.0f ? 0.0f : x[j] / sum);
    if (to.lse && d == 0) to.lse[t * to.q_heads + h] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
  };
  for (int e = threadIdx.x; e < quads; e += kWaves * 64) {
    const int i = e / (ROW / 4), d = e % (ROW / 4) * 4;
    float top = -INFINITY, sum = 0.0f;
    f32x4 x = {};
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s.red_m[w][i]);
    const float m_at = top == -INFINITY ? 0.0f : top;
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(s.red_m[w][i] - m_at);
      sum += f * s.red_l[w][i];
      x += f * *reinterpret_cast<const f32x4*>(&s.red[(w * 16 + i) * LINE + d]);
    }
    if (used == 1) {
      store(i, d, x, m_at, sum);
    } else {
      float* line = parts + ((int64_t)split * to.part_rows + i) * LINE;
      put(line + d, x[0], x[1]), put(line + d + 2, x[2], x[3]);
      if (d == 0) put(line + ROW, top, sum);
    }
  }
  if (used == 1) return;

  // the workgroups' parts: the last to arrive joins them
  __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wave's numbers are there
  __syncthreads();
  if (threadIdx.x == 0) s.place = __hip_atomic_fetch_add(to.arrived + unit, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (s.place != (uint32_t)used - 1) return;
  if (threadIdx.x == 0) __hip_atomic_store(to.arrived + unit, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  // (every read of a step at once: each is a trip to memory)
  for (int e = threadIdx.x; e < used * 16; e += kWaves * 64) {
    const int p = e / 16, i = e % 16;
    if (i >= rows) continue;
    const float* line = parts + ((int64_t)p * to.part_rows + i) * LINE;
    const u32x2 x = get(line + ROW);
    const uint32_t top = x[0], sum = x[1];
    s.factor_of[p][i] = __builtin_bit_cast(float, top), s.sum_of[p][i] = __builtin_bit_cast(float, sum);
  }
  __syncthreads();
  if (threadIdx.x < 64) {  // a row's maximum and sum, four lanes to a row, and what each part counts for
    const int i = threadIdx.x / 4, sub = threadIdx.x % 4;
    float top = -INFINITY, sum = 0.0f;
    for (int p = sub; p < used; p += 4) top = fmaxf(top, s.factor_of[p][i]);
    top = fmaxf(top, __shfl_xor(top, 1));
    top = fmaxf(top, __shfl_xor(top, 2));
    const float m_at = top == -INFINITY ? 0.0f : top;
    for (int p = sub; p < used; p += 4) {
      const float f = __builtin_amdgcn_exp2f(s.factor_of[p][i] - m_at);
      s.factor_of[p][i] = f;
      sum += f * s.sum_of[p][i];
    }
    sum += __shfl_xor(sum, 1);
    sum += __shfl_xor(sum, 2);
    if (sub == 0) s.red_m[0][i] = m_at, s.red_l[0][i] = sum;
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
      for (int j = 0; j < 8; ++j) y[j] = get4(parts + ((int64_t)min(p + j * deal, used - 1) * to.part_rows + i) * LINE + d);
#pragma unroll
      for (int j = 0; j < 8; ++j) x += (p + j * deal < used ? s.factor_of[min(p + j * deal, used - 1)][i] : 0.0f) * y[j];
    }
    *reinterpret_cast<f32x4*>(&s.red[e * 4]) = x;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < quads; e += kWaves * 64) {
    f32x4 x = {};
    for (int p = 0; p < deal; ++p) x += *reinterpret_cast<const f32x4*>(&s.red[(p * quads + e) * 4]);
    const int i = e / (ROW / 4);
    store(i, e % (ROW / 4) * 4, x, s.red_m[0][i], s.red_l[0][i]);
  }
}

}  // namespace bmx
