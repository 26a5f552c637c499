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
// [lo, hi), lo = max(first, p - window + 1), hi = max(p + 1, prefix).
struct Rule {
  float scale, cap;
  const float* slopes;
  int window;
  const int32_t *prefix, *first;
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

}  // namespace paged
}  // namespace spot
