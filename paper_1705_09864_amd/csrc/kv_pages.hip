// Which pages of a cache are whose, on the GPU: sequences grow by tokens or lose some, pages that they no longer reach go onto the stack of free
// ones and those that they come to reach are taken from its top, and each new row learns its position and its place in the cache.
// All of it follows from prefix sums over the sequences (pages given back, pages taken, new rows), so one workgroup does it; the rows' maps
// of long prompts are a second launch of many.  In order of the sequences, pages given back first: the result does not depend on timing.
//
// Bound by latency: a chain of the lengths, the sums, the stack and the table, each behind the one before.
#include "bmx_internal.h"
#include "few_bits.h"

#include <algorithm>

namespace bmx {
namespace {

struct Args {
  const int32_t* change;
  int32_t* table;
  int64_t table_ld;
  int32_t* lengths;
  int32_t* pool;  // free pages, status, the stack
  int32_t* starts;
  int32_t* positions;  // or null, like slots
  int64_t* slots;
  int sequences, table_width, num_pages, rows;
};

// The number of the first of n ascending numbers that is more than x, n if none is.
__device__ inline int first_above(const int32_t* p, int n, int x) {
  int low = 0, high = n;
  while (low < high) {
    const int mid = (low + high) / 2;
    if (p[mid] > x) high = mid;
    else low = mid + 1;
  }
  return low;
}

// A row that is sequence i's, `at` rows behind its first, which stands at position `first`.
__device__ inline void put_row(const Args& a, int r, int i, int pos) {
  if (a.positions) a.positions[r] = pos;
  if (a.slots) a.slots[r] = pos < 0 ? -1 : (int64_t)a.table[i * a.table_ld + (pos >> kLogPage)] * kPage + (pos & (kPage - 1));
}

constexpr int kMostInOne = 4;  // rows a thread that the kernel itself maps

// THREADS sequences at a time.  ONE: there are no more, and what a sequence needs stays in registers.
template <int THREADS, bool ONE>
__global__ __launch_bounds__(THREADS) void kv_resize_kernel(Args a) {
  constexpr int WAVES = THREADS / 64;
  __shared__ int32_t back_to[THREADS], take_to[THREADS], more_to[THREADS], pages_of[THREADS], first_of[THREADS];
  __shared__ int64_t sums[3][WAVES];
  __shared__ int first_bad;
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int free = a.pool[0];
  if (tid == 0) first_bad = 0x7fffffff;

  KvChange c = {};
  int tokens = 0;
  const auto load = [&](int i) {
    c = {};
    if (i >= a.sequences) {
      c.fits = true;
      return;
    }
    tokens = a.lengths[i];
    c = kv_change_of(tokens, a.change[i], a.table_width);
  };
  // each thread's sums up to its own numbers over the workgroup, and (in all) the workgroup's
  const auto scan = [&](int64_t (&v)[3], int64_t (&all)[3]) {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      for (int o = 1; o < 64; o *= 2) {
        const int64_t x = __shfl_up(v[k], o);
        if (lane >= o) v[k] += x;
      }
    __syncthreads();  // (the sums of the step before are read)
    if (lane == 63)
      for (int k = 0; k < 3; ++k) sums[k][wave] = v[k];
    __syncthreads();
    for (int k = 0; k < 3; ++k) {
      all[k] = 0;
      for (int w = 0; w < WAVES; ++w) {
        if (w == wave) v[k] += all[k];
        all[k] += sums[k][w];
      }
    }
  };
  const auto mine = [&](int64_t (&v)[3]) { v[0] = max(c.pages - c.pages_then, 0), v[1] = max(c.pages_then - c.pages, 0), v[2] = c.more; };

  // all pages that come back
  int64_t v[3], all[3], back = 0;
  for (int base = 0; base < a.sequences; base += THREADS) {
    load(base + tid);
    mine(v);
    scan(v, all);
    back += all[0];
  }
  // whether everything has room
  const bool pool_is_one = free >= 0 && free <= a.num_pages && free + back <= a.num_pages;
  int64_t before[3] = {};
  const int64_t room = free + back;
  for (int base = 0; base < a.sequences; base += THREADS) {
    if (!ONE) {
      load(base + tid);
      mine(v);
      scan(v, all);
    }
    if (!c.fits || before[1] + v[1] > room || before[2] + v[2] > a.rows) atomicMin(&first_bad, base + tid);
    for (int k = 1; k < 3; ++k) before[k] += all[k];
  }
  __syncthreads();
  const int bad = first_bad;
  if (bad != 0x7fffffff || !pool_is_one) {
    if (tid == 0) a.pool[1] = pool_is_one ? bad + 1 : -1;
    for (int i = tid; i <= a.sequences; i += THREADS) a.starts[i] = 0;
    if (ONE && a.rows <= kMostInOne * THREADS)
      for (int r = tid; r < a.rows; r += THREADS) put_row(a, r, 0, -1);
    return;
  }
  const int64_t taken = before[1];
  if (tid == 0) {
    a.pool[0] = (int)(room - taken);
    a.pool[1] = 0;
    a.starts[0] = 0;
  }
  int32_t* const stack = a.pool + 2;
  // pages back onto the stack, from there into the table
  for (int way = 0; way < 2; ++way) {
    int64_t at = 0, rows = 0;  // pages and rows of the sequences before these
    for (int base = 0; base < a.sequences; base += THREADS) {
      const int n = min(a.sequences - base, THREADS);
      if (!ONE) {
        load(base + tid);
        mine(v);
        scan(v, all);
      }
      if (!ONE || way == 0) {
        back_to[tid] = (int)v[0], take_to[tid] = (int)v[1], more_to[tid] = (int)(rows + v[2]), pages_of[tid] = c.pages, first_of[tid] = tokens;
        __syncthreads();
      }
      if (way == 0) {
        for (int k = tid; k < all[0]; k += THREADS) {
          const int i = first_above(back_to, n, k), from = i ? back_to[i - 1] : 0;
          stack[free + at + k] = a.table[(base + i) * a.table_ld + pages_of[i] - 1 - (k - from)];
        }
        at += all[0];
      } else {
        for (int k = tid; k < all[1]; k += THREADS) {
          const int i = first_above(take_to, n, k), from = i ? take_to[i - 1] : 0;
          a.table[(base + i) * a.table_ld + pages_of[i] + (k - from)] = stack[room - 1 - at - k];
        }
        at += all[1];
        if (base + tid < a.sequences) {
          a.lengths[base + tid] = c.tokens_then;
          a.starts[base + tid + 1] = (int)(rows + v[2]);
        }
        rows += all[2];
      }
      if (!ONE) __syncthreads();  // (the next sequences' sums come into the same memory)
    }
    __syncthreads();
  }
  if (ONE && a.rows <= kMostInOne * THREADS) {
    for (int r = tid; r < a.rows; r += THREADS) {
      const int i = first_above(more_to, a.sequences, r);
      put_row(a, r, i, i < a.sequences ? first_of[i] + r - (i ? more_to[i - 1] : 0) : -1);
    }
  }
}

__global__ __launch_bounds__(256) void kv_slots_kernel(Args a) {
  const int r = blockIdx.x * 256 + threadIdx.x;
  if (r >= a.rows) return;
  const int i = first_above(a.starts + 1, a.sequences, r);
  put_row(a, r, i, i < a.sequences ? a.lengths[i] - (a.starts[i + 1] - r) : -1);
}

template <int THREADS, bool ONE>
void launch(const Args& a, hipStream_t s) {
  launch_kernel(kv_resize_kernel<THREADS, ONE>, dim3(1), dim3(THREADS), 0, s, a);
  note_kernel("kv_resize_kernel<%d,%d> grid 1 block %d", THREADS, ONE, THREADS);
  if ((!ONE || a.rows > kMostInOne * THREADS) && a.rows > 0 && (a.positions || a.slots))
    launch_kernel(kv_slots_kernel, dim3((uint32_t)ceil_div(a.rows, 256)), dim3(256), 0, s, a);
}

}  // namespace

hipError_t launch_kv_resize(const int32_t* change, int sequences, int32_t* table, int64_t table_ld, int table_width, int32_t* lengths, int32_t* pool,
                            int num_pages, int32_t* starts, int32_t* positions, int64_t* slots, int rows, hipStream_t s) {
  const Args a = {change, table, table_ld, lengths, pool, starts, positions, slots, sequences, table_width, num_pages, rows};
  if (sequences <= 256) launch<256, true>(a, s);
  else if (sequences <= 1024) launch<1024, true>(a, s);
  else launch<1024, false>(a, s);
  return launch_error();
}

}  // namespace bmx
