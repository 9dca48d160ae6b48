// Heads rotated by their tokens' positions: values a and b of a pair j of a token at position p become
//   a' = f (a cos t - b sin t), b' = f (b cos t + a sin t),  t = p freq_j,
// pairs of neighbours, or of a value and the one half of the rotated part behind it.
// The angle is taken in 64 bits as a part of a turn, p (freq_j / 2 pi) less the nearest whole number, and then less the nearest quarter: in 32 bits a position of 10^6
// would leave 4 digits of it.  Sine and cosine of what is left, |t| <= pi / 4, are series in 64 bits too, which end far below fp32's last bit with a^11 and a^10, and are
// rounded to fp32 once, times the factor: 1501 tokens of f32 are 2.9e-8 from 64 bits, where angles rounded to fp32 ahead of the quarters, and the factor, left 5.3e-8, in the same
// time (4.5 us; an angle is made once a token for all its heads).
//
// Bound by the heads' bytes, in and out once.  A workgroup takes ROWS tokens: a thread makes an angle's sine and cosine, which all heads of the token
// share, into LDS, while its first values are on their way; then 16 bytes of each side of the pairs a step.  8192 tokens of 40 heads of 128 bf16:
// 27.7 us, 168 MB at 6.1 TB/s (half of it is still in the last caches).  64 tokens: 2.7 us, a launch and two trips to memory.  1501 of 12 heads of 80 f32, pairs
// of neighbours: 5.0 us, 2.3 TB/s.  4000 of 20 heads of 98 bf16, which 16 bytes do not divide:
// 9.2 us, 3.4 TB/s.
#include "bmx_internal.h"
#include "few_bits.h"

#include <algorithm>
#include <type_traits>

namespace bmx {
namespace {

struct Args {
  const void* x;
  int64_t x_row, x_head;
  void* out;
  int64_t out_row, out_head;
  const int32_t* positions;
  const double* freq;
  int heads, dim, half;  // half: pairs
  int rows;
  double cos_by, sin_by;
  bool copy;  // values behind the rotated part go to another place
};

// Sine and cosine of t turns, |t| <= 1/2.
__device__ inline void turn(double t, double* s, double* c) {
  const double n = rint(4.0 * t), a = (t - 0.25 * n) * 6.283185307179586477, b = a * a;
  const double si = a + a * b * (-1.0 / 6 + b * (1.0 / 120 + b * (-1.0 / 5040 + b * (1.0 / 362880 + b * (-1.0 / 39916800)))));
  const double co = 1.0 + b * (-0.5 + b * (1.0 / 24 + b * (-1.0 / 720 + b * (1.0 / 40320 + b * (-1.0 / 3628800)))));
  const int q = (int)n;  // -2 to 2
  const double u = q & 1 ? co : si, v = q & 1 ? si : co;
  *s = q & 2 ? -u : u;
  *c = (q + 1) & 2 ? -v : v;
}

// A pair's values, f: cosine and sine.  Fused by hand, and kept from the compiler's products that round to 16 bits at once: whatever step makes a value makes the same bits.
__device__ inline float one(float r) {
  asm("" : "+v"(r));
  return r;
}
__device__ inline float first(float x, float y, float2 f) { return one(fmaf(x, f.x, -(y * f.y))); }
__device__ inline float second(float x, float y, float2 f) { return one(fmaf(y, f.x, x * f.y)); }

// A value, as Run has several.
template <int TYPE>
struct Single {
  float v;
  __device__ void load(const void* p, int64_t at, int) { v = load_one<TYPE>(p, at); }
  __device__ float get(int) const { return v; }
};

// Steps of N values that do not divide a head's: the last one begins earlier, and makes some values a second time, or, where those are overwritten in place, is a shorter one.
enum Last { kWhole, kEarlier, kShorter };
// PAIR: neighbours.  N: values of a step on each side (halves) or in all (neighbours).
template <int TYPE, bool PAIR, int N, Last LAST>
__global__ __launch_bounds__(256) void rotary_kernel(Args a, int rows_each, int head_groups) {
  constexpr int PAIRS = PAIR ? N / 2 : N;
  extern __shared__ float2 table[];  // [row][pair]
  const int row0 = blockIdx.x / head_groups * rows_each, rows = min(rows_each, a.rows - row0), group = blockIdx.x % head_groups;
  const int head0 = (int)((int64_t)group * a.heads / head_groups), heads = (int)((int64_t)(group + 1) * a.heads / head_groups) - head0;
  const int steps = LAST == kWhole ? a.half / PAIRS : (a.half + PAIRS - 1) / PAIRS, items = rows * heads * steps;
  using V = std::conditional_t<N == 1, Single<TYPE>, Run<TYPE, N == 1 ? 2 : N>>;
  const auto place = [&](int e, int* row, int* j, int* head) {
    *j = e % steps * PAIRS;
    if (LAST == kEarlier) *j = min(*j, a.half - PAIRS);
    *head = e / steps % heads + head0;
    *row = e / steps / heads;
  };
  const auto left = [&](int j) { return LAST != kShorter ? N : PAIR ? 2 * (a.half - j) : a.half - j; };
  const auto load = [&](int e, V* u, V* w) {
    int row, j, head;
    place(e, &row, &j, &head);
    const int64_t at = (int64_t)(row0 + row) * a.x_row + head * a.x_head + (PAIR ? 2 * j : j);
    u->load(a.x, at, left(j));
    if constexpr (!PAIR) w->load(a.x, at + a.half, left(j));
  };
  V u, w;
  if ((int)threadIdx.x < items) load(threadIdx.x, &u, &w);
  for (int e = threadIdx.x; e < rows * a.half; e += 256) {
    const double t = (double)a.positions[row0 + e / a.half] * (a.freq[e % a.half] * 0.15915494309189533577);
    double s, c;
    turn(t - rint(t), &s, &c);
    table[e] = float2{(float)(c * a.cos_by), (float)(s * a.sin_by)};
  }
  __syncthreads();
  for (int e = threadIdx.x; e < items; e += 256) {
    if (e != (int)threadIdx.x) load(e, &u, &w);
    int row, j, head;
    place(e, &row, &j, &head);
    const int64_t at = (int64_t)(row0 + row) * a.out_row + head * a.out_head + (PAIR ? 2 * j : j);
    const float2* f = table + row * a.half + j;
    [[maybe_unused]] V p, q;
    if constexpr (PAIR) {
#pragma unroll
      for (int i = 0; i < N; i += 2) {
        const float x = u.get(i), y = u.get(i + 1);
        p.set2(i, first(x, y, f[i / 2]), second(x, y, f[i / 2]));
      }
      p.store(a.out, at, left(j));
    } else if constexpr (N == 1) {
      const float x = u.get(0), y = w.get(0);
      store_one<TYPE>(a.out, at, first(x, y, f[0]));
      store_one<TYPE>(a.out, at + a.half, second(x, y, f[0]));
    } else {
#pragma unroll
      for (int i = 0; i < N; i += 2) {
        const float x0 = u.get(i), y0 = w.get(i), x1 = u.get(i + 1), y1 = w.get(i + 1);
        p.set2(i, first(x0, y0, f[i]), first(x1, y1, f[i + 1]));
        q.set2(i, second(x0, y0, f[i]), second(x1, y1, f[i + 1]));
      }
      p.store(a.out, at, left(j));
      q.store(a.out, at + a.half, left(j));
    }
  }
  if (a.copy) {
    constexpr int M = N > 2 ? N : 1;
    const int from = 2 * a.half, each = LAST == kWhole ? (a.dim - from) / M : (a.dim - from + M - 1) / M;
    for (int e = threadIdx.x; e < rows * heads * each; e += 256) {
      const int row = row0 + e / each / heads, head = head0 + e / each % heads, at = from + e % each * M, d = LAST == kWhole || a.dim - from < M ? at : min(at, a.dim - M);
      if constexpr (M == 1) {
        store_one<TYPE>(a.out, row * a.out_row + head * a.out_head + d, load_one<TYPE>(a.x, row * a.x_row + head * a.x_head + d));
      } else {
        Run<TYPE, M> v;
        v.load(a.x, row * a.x_row + head * a.x_head + d, LAST == kWhole ? M : a.dim - d);
        v.store(a.out, row * a.out_row + head * a.out_head + d, LAST == kWhole ? M : a.dim - d);
      }
    }
  }
}

template <int TYPE, bool PAIR>
void launch(const Args& a, hipStream_t s) {
  constexpr int SIZE = TYPE == BMX_F32 ? 4 : 2, WIDE = 16 / SIZE, NARROW = PAIR ? 2 : 1;
  const auto whole = [](int64_t n) { return n % WIDE == 0; };
  const bool wide = (PAIR ? whole(2 * a.half) : whole(a.half)) && (!a.copy || whole(a.dim - 2 * a.half));
  // (us in steps of 16 bytes, of single pairs: 4000 rows of 20 heads of 98 bf16 9.2, 15.2, of 100 f16 7.8, 15.0; 8000 of 96, 50 rotated, 18.2, 31.0; with a shorter last step
  // 10.7, 10.9 and 25.6, but 64 rows of 40 heads of 98 3.5, 2.9)
  const bool fits = (PAIR ? 2 * a.half : a.half) >= WIDE, same = a.out == a.x;
  const bool ragged = !wide && fits && (!same || (int64_t)a.rows * a.heads >= 16384);
  const int n = wide || ragged ? WIDE : NARROW, pairs = PAIR ? n / 2 : n;
  const int64_t per_row = (int64_t)a.heads * ceil_div(a.half, pairs);
  // Rows of a workgroup: three steps a thread, as long as there are two workgroups a CU; heads of few rows are dealt out to several workgroups.  (us with two,
  // three, four steps: 8192 rows of 40 heads of 128 bf16 28.8, 27.6, 27.9, 9000 rows of 20 heads of 96 f16, 48 rotated, 17.7, 18.2, 20.0; with four workgroups a CU
  // 1500 rows of 12 heads of 80 f32 5.1, with two 4.6.)
  int64_t rows_each = std::max<int64_t>(std::min<int64_t>({3 * 256 / per_row, a.rows / 512, 4096 / a.half, 64}), 1);
  int64_t groups = std::max<int64_t>(std::min<int64_t>({(per_row + 255) / 256, a.heads, (1024 + a.rows - 1) / a.rows}), 1);
  if (rows_each > 1) groups = 1;
  const dim3 grid((uint32_t)(ceil_div(a.rows, rows_each) * groups));
  const auto kern = wide      ? rotary_kernel<TYPE, PAIR, WIDE, kWhole>
                    : !ragged ? rotary_kernel<TYPE, PAIR, NARROW, kWhole>
                    : same    ? rotary_kernel<TYPE, PAIR, WIDE, kShorter>
                              : rotary_kernel<TYPE, PAIR, WIDE, kEarlier>;
  launch_kernel(kern, grid, dim3(256), (rows_each * a.half + (ragged ? WIDE : 0)) * sizeof(float2), s, a, (int)rows_each, (int)groups);
  note_kernel("rotary_kernel<%d,%d,%d,%d> grid %u block 256", TYPE, PAIR, n, ragged ? (int)(same ? kShorter : kEarlier) : (int)kWhole, grid.x);
}

}  // namespace

hipError_t launch_rotary(const void* x, int type, int64_t x_row, int64_t x_head, int heads, int dim, int rows, const int32_t* positions, const double* freq,
                         int rot, bool interleaved, double factor, bool inverse, void* out, int64_t out_row, int64_t out_head, hipStream_t s) {
  const Args a = {x, x_row, x_head, out, out_row, out_head, positions, freq, heads, dim, rot / 2, rows, factor, inverse ? -factor : factor,
                  out != x && rot < dim};
  const auto f = type == BMX_F32 ? (interleaved ? launch<BMX_F32, true> : launch<BMX_F32, false>)
               : type == BMX_F16 ? (interleaved ? launch<BMX_F16, true> : launch<BMX_F16, false>)
                                 : (interleaved ? launch<BMX_BF16, true> : launch<BMX_BF16, false>);
  f(a, s);
  return launch_error();
}

}  // namespace bmx
