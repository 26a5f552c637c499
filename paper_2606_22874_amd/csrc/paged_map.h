// Where the tokens of a paged cache lie, which rows are a sequence's, and what a row
// sees: integer arithmetic alone, that a test compiles for the host.
#pragma once

#include <stdint.h>

namespace spot {
namespace paged {

constexpr int kGroupKeys = 16;      // keys whose rows lie together: pages hold a multiple of 16

__device__ __forceinline__ int least(int a, int b) { return a < b ? a : b; }
__device__ __forceinline__ int most(int a, int b) { return a > b ? a : b; }

struct Pages {
  const int32_t* table;     // [n_seq, max_pages]
  int n_pages, page_size, max_pages;
  // Tokens of a sequence: that its table has places for, and that may be there at all.
  __host__ __device__ __forceinline__ int room() const { return max_pages * page_size; }
  __host__ __device__ __forceinline__ int cap() const { return n_pages > 0 ? room() : 0; }
  // First row (of a pool of [n_pages, h_kv, page_size] rows) of the 16 keys from
  // token t (a multiple of 16, below cap()) of KV head g; -1 where the page's id
  // lies outside the pool.
  __device__ __forceinline__ int row(int s, int t, int g, int h_kv) const {
    const int p = t / page_size;
    const int id = table[(int64_t)s * max_pages + p];
    return (unsigned)id < (unsigned)n_pages ? (id * h_kv + g) * page_size + (t - p * page_size)
                                            : -1;
  }
  // The same for any t: -1 too from cap() on.  A block of 64 keys may begin below cap(), a
  // multiple of 16, and end behind it: who goes over whole blocks looks up this way.
  __host__ __device__ __forceinline__ int row_below_cap(int s, int t, int g, int h_kv) const {
    return t < cap() ? row(s, t, g, h_kv) : -1;
  }
};

// The new tokens of sequence s: rows [start, start + n) of q.  len counts the
// tokens of the cache with the new ones, so that row i has position len - n + i.
struct Seq {
  int start, n, len;
};
__device__ __forceinline__ Seq sequence(const int32_t* seq_start, const int32_t* seq_len, int s,
                                        int rows) {
  Seq q;
  q.start = least(most(seq_start[s], 0), rows);
  q.n = least(most(seq_start[s + 1], q.start), rows) - q.start;
  q.len = most(seq_len[s], 0);
  return q;
}

// What an attention call sees and how its scores are made: score x = cap *
// tanh(scale s / cap) (cap 0: scale s) - slope_h |p - t|, for the tokens t of
// [lo, hi), lo = max(first, p - window + 1), hi = max(p + 1, prefix), and those of
// [first, first + sink) before lo.
struct Rule {
  float scale, cap;
  const float* slopes;
  int window;
  const int32_t *prefix, *first;
  int sink;
};

// Visible tokens [lo, hi) of a row (lo = hi = 0 where there are none).
__device__ __forceinline__ void visible(const Rule& u, const Seq& q, int s, int i, int cap, int& lo,
                                        int& hi) {
  const int p = q.len - q.n + i;
  hi = p + 1;
  if (u.prefix) hi = most(hi, least(u.prefix[s], q.len));
  hi = least(hi, cap);
  lo = u.window > 0 && u.window <= p ? p - u.window + 1 : 0;
  if (u.first) lo = most(lo, u.first[q.start + i]);
  if (lo >= hi) lo = hi = 0;
}

// The same with sinks: also [from, end) (from = end = 0 where there are none).
__device__ __forceinline__ void visible(const Rule& u, const Seq& q, int s, int i, int cap, int& lo,
                                        int& hi, int& from, int& end) {
  const int p = q.len - q.n + i;
  hi = p + 1;
  if (u.prefix) hi = most(hi, least(u.prefix[s], q.len));
  hi = least(hi, cap);
  from = u.first ? most(u.first[q.start + i], 0) : 0;
  lo = u.window > 0 && u.window <= p ? p - u.window + 1 : 0;
  lo = most(lo, from);
  end = least(lo - from > u.sink ? from + u.sink : lo, hi);
  if (from >= end) from = end = 0;
  if (lo >= hi) lo = hi = 0;
}

// The blocks of 64 keys that a tile of rows goes through, numbered from 0: n_sink ones
// from `sink0` on, then those from `main0` on.
struct Blocks {
  int sink0, n_sink, main0, n;
  __host__ __device__ __forceinline__ int at(int i) const {
    return i < n_sink ? sink0 + i : main0 + (i - n_sink);
  }
};
// Of rows that see tokens of [lo, hi) and [from, end), both empty where lo >= hi resp.
// from >= end.  Intervals that share a block, or lie the other way round, are one run.
__device__ __forceinline__ Blocks blocks_of(int lo, int hi, int from, int end) {
  Blocks b = {0, 0, 0, 0};
  int m0 = 0, m1 = 0;
  if (lo < hi) {
    m0 = lo / 64;
    m1 = (hi - 1) / 64 + 1;
  }
  if (from < end) {
    const int s0 = from / 64, s1 = (end - 1) / 64 + 1;
    if (lo >= hi) {
      m0 = s0;
      m1 = s1;
    } else if (s1 > m0) {
      m0 = least(m0, s0);
      m1 = most(m1, s1);
    } else {
      b.sink0 = s0;
      b.n_sink = s1 - s0;
    }
  }
  b.main0 = m0;
  b.n = b.n_sink + m1 - m0;
  return b;
}

}  // namespace paged
}  // namespace spot
