// Which rows, positions and pages of a cache a call reaches.  The numbers come from device memory and may be any: plain arithmetic without a
// product or sum that leaves 32 bits, on the host too, where the tests walk it.
#pragma once
#include <stdint.h>

namespace bmx {

constexpr int kPage = 64, kLogPage = 6;  // tokens of a page

struct KvSpan {
  int row0, count;  // a sequence's new rows
  int first;        // position of the first of them (negative where there are more rows than tokens)
  int length;       // its tokens, new ones included, as far as the table reaches
};
// begin, end: the sequence's rows as the caller has them; they stay inside [0, rows), the positions inside the table.
__host__ __device__ static inline KvSpan kv_span_of(int begin, int end, int tokens, int rows, int max_new, int table_width) {
  KvSpan s;
  s.row0 = begin < 0 ? 0 : begin < rows ? begin : rows;
  const int stop = end < s.row0 ? s.row0 : end < rows ? end : rows;
  s.count = stop - s.row0 < max_new ? stop - s.row0 : max_new;
  const int64_t most = (int64_t)table_width * kPage;
  const int n = tokens < 0 ? 0 : tokens;
  s.first = n - s.count;
  s.length = n < most ? n : (int)most;
  return s;
}

// The `at`-th page, of those that positions [low, high) lie in: its place in the sequence's row of the table (negative in front of position 0),
// and its tokens [t0, t1) among them; false where there is none.  Pages are compared, not positions: 64 times a page's number need not fit.
__host__ __device__ static inline bool kv_page_at(int low, int high, int at, int* page, int* t0, int* t1) {
  const int end = high >> kLogPage, rest = high & (kPage - 1);
  *page = (low >> kLogPage) + at;
  if (*page > end) return false;
  *t0 = at == 0 ? low & (kPage - 1) : 0;
  *t1 = *page == end ? rest : kPage;
  return *t0 < *t1;
}
// How many pages a sequence's new rows lie in at most.
__host__ __device__ static inline int64_t kv_pages_of(int max_new) { return ((int64_t)max_new + kPage - 2) / kPage + 1; }

// How many pages positions 0 to `end` (not it) lie in, and whether the n positions from t0 on are all in [low, high); t0 + n - 1 fits.
__host__ __device__ static inline int kv_pages_to(int end) { return end > 0 ? (end - 1) / kPage + 1 : 0; }
__host__ __device__ static inline bool kv_all_in(int t0, int n, int low, int high) { return t0 >= low && high >= n && t0 <= high - n; }

// A sequence of `tokens` tokens that is to have `change` more (or fewer): its pages now and then, and the rows that are new.  fits: neither number of
// tokens is below 0 or more than the table has room for.
struct KvChange {
  bool fits;
  int pages, pages_then, tokens_then, more;
};
__host__ __device__ static inline KvChange kv_change_of(int tokens, int change, int table_width) {
  KvChange c = {};
  const int64_t then = (int64_t)tokens + change, most = (int64_t)table_width * kPage;
  c.fits = tokens >= 0 && tokens <= most && then >= 0 && then <= most && then <= 0x7fffffff;
  if (!c.fits) return c;
  c.pages = kv_pages_to(tokens), c.pages_then = kv_pages_to((int)then), c.tokens_then = (int)then;
  c.more = change > 0 ? change : 0;
  return c;
}

}  // namespace bmx
