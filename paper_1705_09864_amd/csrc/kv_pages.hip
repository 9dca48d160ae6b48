// Which pages of a cache are whose, on the GPU: sequences grow by tokens or lose some, pages that they no longer reach go onto the stack of free
// ones and those that they come to reach are taken from its top, and each new row learns its position and its place in the cache.
// All of it follows from prefix sums over the sequences (pages given back, pages taken, new rows), which a workgroup makes in a microsecond.  In order of the
// sequences, pages given back first: the result does not depend on timing.
//
// Bound by latency: a chain of the lengths, the sums, the stack or the table, each behind the one before, with little code, which a launch reads from memory too.
// 64 sequences, a token more for each: 3.0 to 3.5 us.  300 sequences with 300,000 new rows (3.7 MB of maps, 0.8 us of memory): 8.6 and 2.1 us, in two
// launches.
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
  int most;  // new rows that a sequence may have
  bool wide;  // positions and slots lie on 16 bytes
};

// A sequence's change, which also fits only if the calls behind this one take all its rows.
__device__ inline KvChange change_of(const Args& a, int tokens, int change) {
  KvChange c = kv_change_of(tokens, change, a.table_width);
  c.fits = c.fits && c.more <= a.most;
  return c;
}

// Sums of numbers that are not negative, 2^32 - 1 where they are more.
__device__ inline uint32_t plus(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }
template <int CTRL, int ROWS>
__device__ inline uint32_t plus_lane(uint32_t x) { return plus(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false)); }
// Those over the lanes up to each.
__device__ inline uint32_t sums_to(uint32_t x) {
  x = plus_lane<0x118, 0xf>(plus_lane<0x114, 0xf>(plus_lane<0x112, 0xf>(plus_lane<0x111, 0xf>(x))));  // a row of 16: 1, 2, 4, 8 to the left
  return plus_lane<0x143, 0xc>(plus_lane<0x142, 0xa>(x));  // a row's last into the next, the second row's into the two behind it
}

// How many of n ascending numbers are not above x.
template <class P>
__device__ inline int not_above(const P p, int n, uint32_t x) {
  int found = 0;
  for (int by = 1 << (31 - __builtin_clz(n | 1)); by; by >>= 1)
    if (found + by <= n && (uint32_t)p[found + by - 1] <= x) found += by;
  return found;
}

__device__ inline void put_row(const Args& a, int r, int pos, int page) {
  if (a.positions) a.positions[r] = pos;
  if (a.slots) a.slots[r] = pos < 0 ? -1 : (int64_t)page * kPage + (pos & (kPage - 1));
}

// Rows a thread up to which one workgroup does it all (us of a call with one, with two launches: 8 sequences with 407 new rows 3.7, 5.9, 812 4.7, 5.7, 3252 9.1, 5.9;
// 200 sequences with 800 6.2, 6.3, 1600 8.5, 6.7; 1000 with 4000 7.3, 7.6).
constexpr int kMostInOne = 4;
enum Part { kAll, kMoves, kState };

// What all kernels begin with, EACH sequences a thread at a time: the sums, and whether everything has room.
template <int THREADS, int EACH = 1>
struct Sums {
  static constexpr int WAVES = THREADS / 64, MANY = THREADS * EACH;
  uint32_t back_to[MANY], take_to[MANY], more_to[MANY];  // of pages given back, pages taken, new rows: up to each sequence
  int32_t pages_of[MANY], first_of[MANY];                // its pages and tokens before the call
  uint32_t of_wave[3][WAVES];
  int first_bad;
};

// THREADS times SEQS sequences or fewer, SEQS behind one another to a thread; what one needs stays in registers.  kAll: one workgroup does everything.  Otherwise kMoves, any number of workgroups that move pages and map rows
// between them, each on sums of its own, and behind it kState, one that brings lengths and pool up to date.
// A page that is taken comes from the stack, or, if it is given back in this call, from where the table has it: pages go both ways at once.
template <int THREADS, int SEQS, Part PART>
__global__ __launch_bounds__(THREADS) void kv_resize_kernel(Args a) {
  __shared__ Sums<THREADS, SEQS> s;
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, n = a.sequences, mine = tid * SEQS;
  const int free = a.pool[0];
  if (tid == 0) s.first_bad = 0x7fffffff;
  KvChange c[SEQS] = {};
  uint32_t v[3] = {}, all[3];  // of this thread's sequences, then of all before them
#pragma unroll
  for (int j = 0; j < SEQS; ++j) {
    c[j].fits = true;
    if (mine + j < n) {
      const int tokens = a.lengths[mine + j];
      c[j] = change_of(a, tokens, a.change[mine + j]);
      s.pages_of[mine + j] = c[j].pages, s.first_of[mine + j] = tokens;
    }
    v[0] = plus(v[0], max(c[j].pages - c[j].pages_then, 0)), v[1] = plus(v[1], max(c[j].pages_then - c[j].pages, 0)), v[2] = plus(v[2], c[j].more);
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const uint32_t to = sums_to(v[k]);
    if (lane == 63) s.of_wave[k][wave] = to;
    v[k] = __builtin_amdgcn_update_dpp(0, (int)to, 0x138, 0xf, 0xf, false);  // the lane's before this one
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const uint32_t to = sums_to(lane < Sums<THREADS>::WAVES ? s.of_wave[k][lane % Sums<THREADS>::WAVES] : 0);
    all[k] = __builtin_amdgcn_readlane(to, 63);
    if (wave > 0) v[k] = plus(v[k], __builtin_amdgcn_readlane(to, __builtin_amdgcn_readfirstlane(max(wave - 1, 0))));
  }
  const bool pool_is_one = free >= 0 && free <= a.num_pages && (int64_t)free + all[0] <= a.num_pages;
  const uint32_t room = pool_is_one ? free + all[0] : 0, rows = a.rows;
#pragma unroll
  for (int j = 0; j < SEQS; ++j) {
    v[0] = plus(v[0], max(c[j].pages - c[j].pages_then, 0)), v[1] = plus(v[1], max(c[j].pages_then - c[j].pages, 0)), v[2] = plus(v[2], c[j].more);
    s.back_to[mine + j] = v[0], s.take_to[mine + j] = v[1], s.more_to[mine + j] = v[2];
    if (!c[j].fits || v[1] > room || v[2] > rows) atomicMin(&s.first_bad, mine + j);
  }
  __syncthreads();
  const int bad = s.first_bad;
  const bool refused = bad != 0x7fffffff || !pool_is_one;
  if (PART != kMoves) {
    if (tid == 0) a.pool[1] = !pool_is_one ? -1 : refused ? bad + 1 : 0;
    if (!refused) {
      if (tid == 0) a.pool[0] = (int)(room - all[1]);
#pragma unroll
      for (int j = 0; j < SEQS; ++j)
        if (mine + j < n) a.lengths[mine + j] = c[j].tokens_then;
    }
  }
  if (PART == kState) return;
  if (blockIdx.x == 0) {
    if (tid == 0) a.starts[0] = 0;
    for (int i = tid; i < n; i += THREADS) a.starts[i + 1] = refused ? 0 : (int)s.more_to[i];
  }
  int32_t* const stack = a.pool + 2;
  // the k-th page given back: where the table has it; the k-th taken: its number
  const auto given = [&](uint32_t k) {
    const int i = not_above(s.back_to, n, k);
    return a.table + i * a.table_ld + s.pages_of[i] - 1 - (int)(k - (i ? s.back_to[i - 1] : 0));
  };
  const auto taken = [&](uint32_t k) { return room - 1 - k < (uint32_t)free ? stack[room - 1 - k] : *given(room - 1 - k - free); };
  // Pages given back, pages taken and rows are one another's equals, and a thread has one of them at a time.  EACH rows behind one another to a thread: mostly of one
  // sequence and one page.
  constexpr int EACH = PART == kAll ? 1 : 4;
  const uint64_t back = refused ? 0 : all[0], moves = back + (refused ? 0 : all[1]), items = moves + (rows + EACH - 1) / EACH;
  for (uint64_t e = blockIdx.x * THREADS + tid; e < items; e += gridDim.x * THREADS) {
    if (e < back) {
      stack[free + e] = *given((uint32_t)e);
      continue;
    }
    if (e < moves) {
      const uint32_t k = (uint32_t)(e - back);
      const int i = not_above(s.take_to, n, k);
      a.table[i * a.table_ld + s.pages_of[i] + (int)(k - (i ? s.take_to[i - 1] : 0))] = taken(k);
      continue;
    }
    const uint32_t r0 = (uint32_t)(e - moves) * EACH;
    int i = refused ? n : not_above(s.more_to, n, r0), held = -1, page = 0, pos[EACH];
    int64_t slot[EACH];
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      const uint32_t r = r0 + j;
      if (j > 0)
        while (i < n && s.more_to[i] <= r) ++i, held = -1;
      pos[j] = -1, slot[j] = -1;
      if (i < n && r < rows) {
        pos[j] = s.first_of[i] + (int)(r - (i ? s.more_to[i - 1] : 0));
        const int at = pos[j] >> kLogPage, beyond = at - s.pages_of[i];  // (a new page is not read from the table, which other threads write)
        if (at != held) page = beyond < 0 ? a.table[i * a.table_ld + at] : taken((i ? s.take_to[i - 1] : 0) + beyond);
        held = at;
        slot[j] = (int64_t)page * kPage + (pos[j] & (kPage - 1));
      }
    }
    if (EACH == 4 && a.wide && r0 + EACH <= rows) {
      struct __attribute__((aligned(16))) Four { int32_t x[4]; };
      struct __attribute__((aligned(16))) Two { int64_t x[2]; };
      if (a.positions) *reinterpret_cast<Four*>(a.positions + r0) = Four{pos[0], pos[1 % EACH], pos[2 % EACH], pos[3 % EACH]};
      if (a.slots) {
        reinterpret_cast<Two*>(a.slots + r0)[0] = Two{slot[0], slot[1 % EACH]};
        reinterpret_cast<Two*>(a.slots + r0)[1] = Two{slot[2 % EACH], slot[3 % EACH]};
      }
    } else {
#pragma unroll
      for (int j = 0; j < EACH; ++j) {
        if (r0 + j >= rows) break;
        if (a.positions) a.positions[r0 + j] = pos[j];
        if (a.slots) a.slots[r0 + j] = slot[j];
      }
    }
  }
}

// More than 4096 sequences: one workgroup over and over (3000 with a token each 23 us, 8.9 with four to a thread), the pages first all onto the stack and then from there; the rows' maps by kv_slots_kernel.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void kv_resize_many_kernel(Args a) {
  __shared__ Sums<THREADS> s;
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int free = a.pool[0];
  if (tid == 0) s.first_bad = 0x7fffffff;
  KvChange c = {};
  int tokens = 0;
  uint32_t v[3], all[3];
  const auto sum = [&](int i) {
    c = {};
    c.fits = true;
    if (i < a.sequences) {
      tokens = a.lengths[i];
      c = change_of(a, tokens, a.change[i]);
    }
    v[0] = max(c.pages - c.pages_then, 0), v[1] = max(c.pages_then - c.pages, 0), v[2] = c.more;
#pragma unroll
    for (int k = 0; k < 3; ++k) v[k] = sums_to(v[k]);
    __syncthreads();  // (what the step before left is read)
    if (lane == 63)
#pragma unroll
      for (int k = 0; k < 3; ++k) s.of_wave[k][wave] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const uint32_t to = sums_to(lane < Sums<THREADS>::WAVES ? s.of_wave[k][lane % Sums<THREADS>::WAVES] : 0);
      all[k] = __builtin_amdgcn_readlane(to, 63);
      if (wave > 0) v[k] = plus(v[k], __builtin_amdgcn_readlane(to, __builtin_amdgcn_readfirstlane(max(wave - 1, 0))));
    }
  };
  uint32_t back = 0;
  for (int base = 0; base < a.sequences; base += THREADS) {
    sum(base + tid);
    back = plus(back, all[0]);
  }
  const bool pool_is_one = free >= 0 && free <= a.num_pages && (int64_t)free + back <= a.num_pages;
  const uint32_t room = pool_is_one ? free + back : 0;
  uint32_t taken = 0, rows = 0;
  for (int base = 0; base < a.sequences; base += THREADS) {
    sum(base + tid);
    if (!c.fits || plus(taken, v[1]) > room || plus(rows, v[2]) > (uint32_t)a.rows) atomicMin(&s.first_bad, base + tid);
    taken = plus(taken, all[1]), rows = plus(rows, all[2]);
  }
  __syncthreads();
  const int bad = s.first_bad;
  if (bad != 0x7fffffff || !pool_is_one) {
    if (tid == 0) a.pool[1] = pool_is_one ? bad + 1 : -1;
    for (int i = tid; i <= a.sequences; i += THREADS) a.starts[i] = 0;
    return;
  }
  if (tid == 0) {
    a.pool[0] = (int)(room - taken);
    a.pool[1] = 0;
    a.starts[0] = 0;
  }
  int32_t* const stack = a.pool + 2;
  for (int way = 0; way < 2; ++way) {
    uint32_t at = 0, row = 0;  // pages and rows of the sequences before these
    for (int base = 0; base < a.sequences; base += THREADS) {
      const int n = min(a.sequences - base, THREADS);
      sum(base + tid);
      uint32_t* const to = s.back_to;
      to[tid] = way ? v[1] : v[0], s.pages_of[tid] = c.pages;
      __syncthreads();
      const uint32_t count = way ? all[1] : all[0];
      for (uint32_t k = tid; k < count; k += THREADS) {
        const int i = not_above(to, n, k), by = (int)(k - (i ? to[i - 1] : 0));
        int32_t* const line = a.table + (base + i) * a.table_ld + s.pages_of[i];
        if (way) line[by] = stack[room - 1 - at - k];
        else stack[free + at + k] = line[-1 - by];
      }
      at += count;
      if (way) {
        if (base + tid < a.sequences) {
          a.lengths[base + tid] = c.tokens_then;
          a.starts[base + tid + 1] = (int)(row + v[2]);
        }
        row += all[2];
      }
    }
    __syncthreads();
  }
}

__global__ __launch_bounds__(256) void kv_slots_kernel(Args a) {
  const int r = blockIdx.x * 256 + threadIdx.x;
  if (r >= a.rows) return;
  const int i = not_above(a.starts + 1, a.sequences, r);
  if (i == a.sequences) return put_row(a, r, -1, 0);
  const int pos = a.lengths[i] - (a.starts[i + 1] - r);
  put_row(a, r, pos, a.table[i * a.table_ld + (pos >> kLogPage)]);
}

// (The host knows the rows, not the pages: those given back in a call of few rows are all one workgroup's.  256 sequences of 64 pages that end 51 us, of 512 433, of 2048 1800.)
template <int THREADS, int SEQS>
void launch(const Args& a, hipStream_t s) {
  if (a.rows <= kMostInOne * THREADS) {
    launch_kernel(kv_resize_kernel<THREADS, SEQS, kAll>, dim3(1), dim3(THREADS), 0, s, a);
    note_kernel("kv_resize_kernel<%d,%d,%d> grid 1 block %d", THREADS, SEQS, (int)kAll, THREADS);
    return;
  }
  const uint32_t grid = (uint32_t)std::min<int64_t>(ceil_div(a.rows, 4 * THREADS) * 9 / 8 + 1, 512);  // (and some for pages)
  launch_kernel(kv_resize_kernel<THREADS, SEQS, kMoves>, dim3(grid), dim3(THREADS), 0, s, a);
  launch_kernel(kv_resize_kernel<THREADS, SEQS, kState>, dim3(1), dim3(THREADS), 0, s, a);
  note_kernel("kv_resize_kernel<%d,%d,%d> grid %u block %d", THREADS, SEQS, (int)kMoves, grid, THREADS);
}

}  // namespace

hipError_t launch_kv_resize(const int32_t* change, int sequences, int32_t* table, int64_t table_ld, int table_width, int32_t* lengths, int32_t* pool,
                            int num_pages, int32_t* starts, int32_t* positions, int64_t* slots, int rows, int most, hipStream_t s) {
  const Args a = {change, table, table_ld, lengths, pool, starts, positions, slots, sequences, table_width, num_pages, rows, most,
                  (uintptr_t)positions % 16 == 0 && (uintptr_t)slots % 16 == 0};
  if (sequences <= 256) {
    launch<256, 1>(a, s);
  } else if (sequences <= 1024) {
    launch<1024, 1>(a, s);
  } else if (sequences <= 4096) {
    launch<1024, 4>(a, s);
  } else {
    launch_kernel(kv_resize_many_kernel<1024>, dim3(1), dim3(1024), 0, s, a);
    note_kernel("kv_resize_many_kernel<%d> grid 1 block %d", 1024, 1024);
    if (rows > 0 && (positions || slots)) launch_kernel(kv_slots_kernel, dim3((uint32_t)ceil_div(rows, 256)), dim3(256), 0, s, a);
  }
  return launch_error();
}

}  // namespace bmx
