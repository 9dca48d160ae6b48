// The paged cache of 8 bits: new keys and values quantised as they are written, and read back.
// A block of 16, 32 or 64 tokens of one head has one scale s for its keys and one for its values; a value is held as
// q = round(x / s), |q| <= 127, with s = max |x| / 127 over the block.  A block that already holds tokens keeps its scale unless a
// new value is past 127 s; then s grows and the older levels go to round(q * s_old / s).  Scales and quotients are 32-bit.
#include "bmx_internal.h"
#include "few_bits.h"

namespace bmx {
namespace {

__device__ inline int level(float x, float r) {
  // (a NaN is level 0, an infinity the last one)
  const float z = fminf(fmaxf(rintf(x * r), -127.0f), 127.0f);
  return x != x ? 0 : fabsf(x) == INFINITY ? (x > 0 ? 127 : -127) : (int)z;
}

// One workgroup per page that new tokens of a sequence reach, head, and keys or values.
template <int TYPE>
__global__ __launch_bounds__(256) void kv_write_kernel(bmx_kv_cache c, const void* k, const void* v, int64_t k_row, int64_t k_head,
                                                       int64_t v_row, int64_t v_head, int rows, int max_new, int span) {
  __shared__ uint32_t top[4];
  const int seq = blockIdx.x / span, head = blockIdx.y / 2, which = blockIdx.y % 2;
  const KvSpan s = kv_span(c, seq, rows, max_new);
  const int first = max(s.first, 0), pg = first / kPage + blockIdx.x % span;
  if (s.count == 0 || pg * kPage >= s.length) return;
  const int page = kv_page(c, seq, pg);
  if (page < 0) return;
  const int t0 = max(first - pg * kPage, 0), t1 = min(s.length - pg * kPage, kPage);
  const int row = kv_row_bytes(c.dim), block = c.block, blocks = kPage / block;
  const int64_t unit = ((int64_t)page * c.heads + head) * 2 + which;
  int8_t* body = c.pages + unit * kPage * row;
  float* scales = c.scales + unit * blocks;
  const void* x = which ? v : k;
  const int64_t x_row = which ? v_row : k_row;
  const int64_t base = (s.row0 + (int64_t)pg * kPage - s.first) * x_row + head * (which ? v_head : k_head);  // of the page's token 0
  if (threadIdx.x < 4) top[threadIdx.x] = 0;
  __syncthreads();
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  for (int t = t0 + wave; t < t1; t += 4) {
    float m = 0.0f;
    for (int d = lane; d < c.dim; d += 64) {
      const float a = fabsf(load_one<TYPE>(x, base + t * x_row + d));
      m = a < INFINITY ? fmaxf(m, a) : m;
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

template <int TYPE>
__global__ __launch_bounds__(256) void kv_read_kernel(bmx_kv_cache c, void* k, void* v, int64_t k_row, int64_t k_head, int64_t v_row,
                                                      int64_t v_head, int rows, int max_new, int span) {
  const int seq = blockIdx.x / span, head = blockIdx.y / 2, which = blockIdx.y % 2;
  const KvSpan s = kv_span(c, seq, rows, max_new);
  // (rows of positions below 0 or past the table, or of pages that are not there, are zeros)
  const int low = s.first < 0 ? (s.first - (kPage - 1)) / kPage : s.first / kPage, pg = low + blockIdx.x % span;
  if (s.count == 0 || pg * kPage >= s.first + s.count) return;
  const int page = pg < 0 || pg >= c.table_width ? -1 : kv_page(c, seq, pg);
  const int t0 = max(s.first - pg * kPage, 0), t1 = min(s.first + s.count - pg * kPage, kPage);
  const int row = kv_row_bytes(c.dim), block = c.block;
  const int64_t unit = ((int64_t)page * c.heads + head) * 2 + which;
  const int8_t* body = c.pages + unit * kPage * row;
  const float* scales = c.scales + unit * (kPage / block);
  void* x = which ? v : k;
  const int64_t x_row = which ? v_row : k_row;
  const int64_t base = (s.row0 + (int64_t)pg * kPage - s.first) * x_row + head * (which ? v_head : k_head);
  for (int i = threadIdx.x; i < (t1 - t0) * c.dim; i += 256) {
    const int t = t0 + i / c.dim, d = i % c.dim, at = which ? kv_value_at(t, d) : kv_key_at(row, t, d);
    store_one<TYPE>(x, base + t * x_row + d, page < 0 ? 0.0f : (float)body[at] * scales[t / block]);
  }
}

}  // namespace

hipError_t launch_kv_write(const bmx_kv_cache& c, const void* k, const void* v, int type, int64_t k_row, int64_t k_head, int64_t v_row,
                           int64_t v_head, int rows, int max_new, hipStream_t s) {
  const int span = (max_new + kPage - 2) / kPage + 1;
  const dim3 grid((uint32_t)(c.sequences * (int64_t)span), c.heads * 2);
  const auto kern = type == BMX_F32 ? kv_write_kernel<BMX_F32> : type == BMX_F16 ? kv_write_kernel<BMX_F16> : kv_write_kernel<BMX_BF16>;
  launch_kernel(kern, grid, dim3(256), 0, s, c, k, v, k_row, k_head, v_row, v_head, rows, max_new, span);
  note_kernel("kv_write_kernel<%d> grid %ux%u block 256", type, grid.x, grid.y);
  return launch_error();
}

hipError_t launch_kv_read(const bmx_kv_cache& c, void* k, void* v, int type, int64_t k_row, int64_t k_head, int64_t v_row, int64_t v_head,
                          int rows, int max_new, hipStream_t s) {
  const int span = (max_new + kPage - 2) / kPage + 1;
  const dim3 grid((uint32_t)(c.sequences * (int64_t)span), c.heads * 2);
  const auto kern = type == BMX_F32 ? kv_read_kernel<BMX_F32> : type == BMX_F16 ? kv_read_kernel<BMX_F16> : kv_read_kernel<BMX_BF16>;
  launch_kernel(kern, grid, dim3(256), 0, s, c, k, v, k_row, k_head, v_row, v_head, rows, max_new, span);
  note_kernel("kv_read_kernel<%d> grid %ux%u block 256", type, grid.x, grid.y);
  return launch_error();
}

}  // namespace bmx
