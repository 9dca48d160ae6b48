// An attention over a cache of pages, 16 rows of queries a workgroup: which pages are whose, and the end, where the waves, which went over pages of
// their own, are joined through LDS, and the workgroups that share rows by the last of them to arrive, in their order, so the result does not depend on which that was.
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
// (16 bytes of a buffer in the same way: the bit for the device's scope alone)
constexpr int kDevice = 16;
__device__ inline f32x4 get4(Rsrc r, int at) { return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, kDevice)); }
__device__ inline void put4(Rsrc r, int at, f32x4 x) { __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), r, at, 0, kDevice); }

// Sums over the lanes up to each.
__device__ inline int sums_to(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // a row of 16: 1, 2, 4, 8 to the left
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // a row's last into the next
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // the second row's into the two behind it
  return x;
}

// Units of 16 rows are dealt out to workgroups by pages: each unit's pages fall into parts of about as many, so that a long sequence among short ones is
// not read by one workgroup.  Every wave finds its workgroup's part by itself.
struct Part {
  int unit, split, used, first;  // the unit's part `split` of `used`; first: the number of its first part among all; unit < 0: none
  int per;                       // pages of a part
  KvSpan span;                   // of the unit's sequence
};
struct UnitPages {
  int pages;  // below 0 where it has no rows, fewer than 2^30
  KvSpan span;
};
constexpr int kAllPages = 0x7fffffff, kMostUnits = 256;
constexpr int kWholePages = 12, kLeastPart = 4;  // (pages that a single unit keeps in one part, and that any part has at least; 6 or 8: level)
// How they are dealt out: parts beyond one for each unit, the most there are (1 or more) and those aimed at where the units are of about a size; pages that a unit's only
// part may have more than others'.
struct Deal {
  int extra, even, slack;
};
// pages_of(n): the n-th unit's pages.
template <class F>
__device__ inline Part part_of(int slot, int units, const Deal& deal, F pages_of) {
  const int lane = threadIdx.x % 64;
  if (units == 1) {
    const UnitPages u = pages_of(0);
    const int pages = u.pages, per = max((pages + deal.extra) / (deal.extra + 1), pages <= kWholePages ? pages : kLeastPart), used = pages > 0 ? (pages + per - 1) / per : 1;
    return {pages >= 0 && slot < used ? 0 : -1, slot, used, 0, used == 1 ? kAllPages : per, u.span};
  }
  // 64 units at a time, a lane each (rolled up: the code of a launch comes from memory too)
  UnitPages u = {-1, {}};
  const auto load = [&](int base) {
    u.pages = -1;
    if (base + lane < units) u = pages_of(base + lane);
  };
  int all = 0, longest = 0;
#pragma unroll 1
  for (int base = 0; base < units; base += 64) {
    load(base);
    longest = max(longest, u.pages);
    all += __builtin_amdgcn_readlane(sums_to(max(u.pages, 0)), 63);
  }
  const int extra = __any((float)longest * units > 1.25f * all) ? deal.extra : deal.even, per = max((all + extra - 1) / extra, kLeastPart);
  int first = 0;
#pragma unroll 1
  for (int base = 0; base < units; base += 64) {
    if (units > 64) load(base);
    const int parts = u.pages < 0 ? 0 : u.pages <= per + deal.slack ? 1 : (u.pages - 1) / per + 1;
    const int to = first + sums_to(parts);
    const uint64_t has = __ballot(slot < to);
    if (has) {
      const int who = __builtin_ctzll(has);
      const auto of_lane = [&](int x) { return __builtin_amdgcn_readlane(x, who); };
      const int used = of_lane(parts), from = of_lane(to) - used;
      return {base + who, slot - from, used, from, used == 1 ? kAllPages : per,
              {of_lane(u.span.row0), of_lane(u.span.count), of_lane(u.span.first), of_lane(u.span.length)}};
    }
    first = __builtin_amdgcn_readlane(to, 63);
  }
  return {-1, 0, 0, 0, 0, {}};
}

constexpr int kMostSplits = 128;  // workgroups that share rows

struct JoinTo {
  void* out;
  int64_t out_row, out_head;
  float* lse;
  float* parts;       // [part][part_rows][ROW + 4]: the rows' results, maximum and sum
  uint32_t* arrived;  // [unit], zeros between the calls
  int q_heads, share, part_rows;
};

template <int ROW, int WAVES>
struct JoinLds {
  static constexpr int LINE = ROW + 4;
  float red[WAVES * 16 * LINE], red_m[WAVES][16], red_l[WAVES][16], factor_of[kMostSplits][16], sum_of[kMostSplits][16];
  uint32_t place;
};

// red, red_m (of scores times log2 e) and red_l are filled and the workgroup is past a barrier.  Rows r0 to r0 + rows of a head of the cache; token0: the row of
// queries that the sequence's first is; unit, first_part: numbers of these rows and of their first part among all; used: workgroups that have a part of them,
// this one the split-th.
template <int TYPE, int ROW, int WAVES>
__device__ inline void join_rows(JoinLds<ROW, WAVES>& s, const JoinTo& to, int dim, int64_t token0, int head, int r0, int rows, int64_t unit, int64_t first_part,
                                 int split, int used) {
  constexpr int LINE = ROW + 4, THREADS = WAVES * 64;
  const int quads = rows * (ROW / 4), part_bytes = to.part_rows * LINE * 4;
  const Rsrc parts = buffer(to.parts + first_part * to.part_rows * LINE, used * part_bytes);
  const auto store = [&](int i, int d, f32x4 x, float top, float sum) {
    const int64_t t = token0 + (r0 + i) / to.share;
    const int h = head * to.share + (r0 + i) % to.share;
#pragma unroll
    for (int j = 0; j < 4; ++j)  // (a row that sees nothing is zeros)
      if (d + j < dim) store_one<TYPE>(to.out, t * to.out_row + h * to.out_head + d + j, sum == 0.0f ? 0.0f : x[j] / sum);
    if (to.lse && d == 0) to.lse[t * to.q_heads + h] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
  };
  for (int e = threadIdx.x; e < quads; e += THREADS) {
    const int i = e / (ROW / 4), d = e % (ROW / 4) * 4;
    float top = -INFINITY, sum = 0.0f;
    f32x4 x = {};
    for (int w = 0; w < WAVES; ++w) top = fmaxf(top, s.red_m[w][i]);
    const float m_at = top == -INFINITY ? 0.0f : top;
    for (int w = 0; w < WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f(s.red_m[w][i] - m_at);
      sum += f * s.red_l[w][i];
      x += f * *reinterpret_cast<const f32x4*>(&s.red[(w * 16 + i) * LINE + d]);
    }
    if (used == 1) {
      store(i, d, x, m_at, sum);
    } else {
      const int line = split * part_bytes + i * LINE * 4;
      put4(parts, line + d * 4, x);
      if (d == 0) put4(parts, line + ROW * 4, f32x4{top, sum, 0.0f, 0.0f});
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
  // The results, four values to a thread; where they are fewer than threads, the parts are dealt out too.  Every read is a trip to memory, and they are made
  // together: the first parts' values with the maxima and sums that say what they count for.
  constexpr int BATCH = 8;
  const int deal = max(THREADS / quads, 1), turns = (quads * deal + THREADS - 1) / THREADS;
  f32x4 y[BATCH];
  const auto fetch = [&](int e, int p) {
    const int i = e % quads / (ROW / 4), d = e % quads % (ROW / 4) * 4;
#pragma unroll
    for (int j = 0; j < BATCH; ++j) y[j] = get4(parts, min(p + j * deal, used - 1) * part_bytes + (i * LINE + d) * 4);
  };
  f32x4 tops[(kMostSplits * 16 + THREADS - 1) / THREADS];
#pragma unroll
  for (int n = 0; n < (kMostSplits * 16 + THREADS - 1) / THREADS; ++n) {
    const int e = threadIdx.x + n * THREADS, p = e / 16, i = e % 16;
    if (n * THREADS < used * 16) tops[n] = get4(parts, min(p, used - 1) * part_bytes + (min(i, rows - 1) * LINE + ROW) * 4);
  }
  fetch(threadIdx.x, (int)threadIdx.x / quads);
#pragma unroll
  for (int n = 0; n < (kMostSplits * 16 + THREADS - 1) / THREADS; ++n) {
    const int e = threadIdx.x + n * THREADS, p = e / 16, i = e % 16;
    if (p < used) s.factor_of[p][i] = tops[n][0], s.sum_of[p][i] = tops[n][1];
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
  for (int n = 0; n < turns; ++n) {
    const int e = threadIdx.x + n * THREADS;
    if (e >= quads * deal) break;
    const int i = e % quads / (ROW / 4);
    f32x4 x = {};
    for (int p = e / quads; p < used; p += BATCH * deal) {
      if (n || p != e / quads) fetch(e, p);
#pragma unroll
      for (int j = 0; j < BATCH; ++j) x += (p + j * deal < used ? s.factor_of[min(p + j * deal, used - 1)][i] : 0.0f) * y[j];
    }
    *reinterpret_cast<f32x4*>(&s.red[e * 4]) = x;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < quads; e += THREADS) {
    f32x4 x = {};
    for (int p = 0; p < deal; ++p) x += *reinterpret_cast<const f32x4*>(&s.red[(p * quads + e) * 4]);
    const int i = e / (ROW / 4);
    store(i, e % (ROW / 4) * 4, x, s.red_m[0][i], s.red_l[0][i]);
  }
}

}  // namespace bmx
