// C ABI of the operators on a paged cache: argument validation, then kernel
// launches.  Nothing is enqueued unless every argument check passes.
#include <algorithm>
#include <float.h>
#include <math.h>

#include "paged_core.h"

using namespace spot;
using namespace spot::paged;

namespace {

spot_status from_hip(hipError_t e) {
  return e == hipSuccess                      ? SPOT_OK
         : e == hipErrorInvalidConfiguration ? SPOT_ERR_SHAPE     // see launchable()
                                             : SPOT_ERR_HIP;
}

bool aligned(const void* p, unsigned n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

bool valid_dtype(int dtype) { return dtype == SPOT_DTYPE_BF16 || dtype == SPOT_DTYPE_FP16; }

// A pool's sizes and those of a page table over it.
bool valid_pages(int n_pages, int page_size, int max_pages, int h_kv) {
  return n_pages >= 0 && page_size >= kGroupKeys && page_size % kGroupKeys == 0 &&
         max_pages >= 0 && h_kv >= 1 && (int64_t)max_pages * page_size <= 1 << 30 &&
         (__int128)n_pages * h_kv * page_size < (__int128)1 << 31;
}

// Whether a pool or a table that has elements is not given.
bool missing_pages(bool pools, int n_pages, const int32_t* table, int max_pages) {
  return (n_pages > 0 && !pools) || (max_pages > 0 && !table);
}

// What spot_paged_attend and spot_paged_weights share.
spot_status check_attend(int dtype, int n_pages, int page_size, int max_pages, int n_seq, int rows,
                         int h_q, int h_kv, int d, float sm_scale, float softcap, int window) {
  if (n_seq < 0 || rows < 0 || h_q < 1 || window < 0 ||
      !valid_pages(n_pages, page_size, max_pages, h_kv) || (int64_t)rows * h_q > 0x7fffffff)
    return SPOT_ERR_SHAPE;
  if (!valid_dtype(dtype) || (d != 64 && d != 128) || h_q % h_kv) return SPOT_ERR_UNSUPPORTED;
  // What the kernels multiply by: scale log2(e), cap log2(e) and scale / cap.
  if (!isfinite(sm_scale * kLog2e) || !(softcap >= 0.f) || !isfinite(softcap * kLog2e))
    return SPOT_ERR_UNSUPPORTED;
  const float ratio = softcap > 0.f ? fabsf(sm_scale / softcap) : 0.f;
  if (!isfinite(ratio) || (ratio < FLT_MIN && softcap > 0.f && sm_scale != 0.f))
    return SPOT_ERR_UNSUPPORTED;
  return SPOT_OK;
}

spot_status check_rope(int d, int rope_dim, const double* freq, float amp, int flags, int dtype) {
  if (d < 2 || d % 2 || d > 1024 || rope_dim < 0 || rope_dim % 2 || rope_dim > d ||
      rope_dim > 2 * kMaxPairs || !valid_dtype(dtype) || !isfinite(amp) ||
      (flags & ~(SPOT_ROPE_INTERLEAVED | SPOT_ROPE_INVERSE)))
    return SPOT_ERR_UNSUPPORTED;
  for (int i = 0; i < rope_dim / 2; ++i)
    if (!isfinite(freq[i])) return SPOT_ERR_UNSUPPORTED;
  return SPOT_OK;
}

// Rows (new tokens x heads of a group) of a sequence up to which it goes to the kernel of
// 16-row tiles, beyond them to that of 256.  The first reads the keys once for every 16
// rows, the second computes 256 however many there are, on fewer workgroups.  8 KV
// heads, 16 / 64 / 128 / 256 rows, us, first and second kernel: 32768 tokens 48, 70,
// 105, 169 and 64, 70, 93, 139; 4096 tokens 19, 26, 26, 32 and 30, 33, 41, 60; eight
// sequences of 4096 34, 62, 90 and 34, 57, 65.
// The lengths are on the device, so the host knows the mean of the rows and the table's
// size alone: where the mean is within 16, the first kernel takes all of them, however
// uneven (a call has one launch in a decode step), and with one sequence either one does;
// otherwise both are launched, and each passes over the other's sequences.  The bound of
// short caches is for one sequence alone: of two of 4096 tokens, 64 rows each take 31 us
// and 128 rows 44 by the general rule.
constexpr int kFewRows = 64, kFewRowsShort = 256, kShortCache = 8192;
int few_rows(int n_seq, int64_t cap) {
  return n_seq == 1 && cap <= kShortCache ? kFewRowsShort : kFewRows;
}
bool launch_many(int n_seq, int rows, int G, int64_t cap) {
  return (int64_t)rows * G > (n_seq == 1 ? few_rows(n_seq, cap) : 16 * (int64_t)n_seq);
}

// Sinks that a call has: without a window a row sees the first tokens anyway, and the call is
// the one without sinks, its kernels and bits.
int sinks(int window, int n_sink) { return window > 0 ? n_sink : 0; }

// The launches of an attention over 16-bit pages, or 8-bit ones (a.k8).
spot_status attend(AttendArgs a, int dtype, int d, void* ws, size_t ws_bytes, hipStream_t s) {
  const int G = a.h_q / a.h_kv;
  const int64_t cap = (int64_t)a.pages.max_pages * a.pages.page_size;
  const bool many = launch_many(a.n_seq, a.rows, G, cap), few = a.n_seq > 1 || !many;
  if (!ws || ws_bytes < (many ? attend_many_workspace(d) : attend_few_workspace(d)) ||
      !aligned(ws, 16))
    return SPOT_ERR_WORKSPACE;
  hipError_t e = hipSuccess;
  if (many) {
    a.from = few ? kFewRows : 0;
    a.to = 0x7fffffff;
    e = a.k8 ? launch_attend_many8(a, dtype, d, ws, s) : launch_attend_many(a, dtype, d, ws, s);
  }
  if (few && e == hipSuccess) {
    a.from = 0;
    a.to = many ? kFewRows : 0x7fffffff;
    e = a.k8 ? launch_attend_few8(a, dtype, d, ws, s) : launch_attend_few(a, dtype, d, ws, s);
  }
  return from_hip(e);
}

// Axes of the pairs: none (one position a row), or of n_axes.
spot_status check_axes(int n_axes, const uint8_t* axis, const int32_t* pos, int rows,
                       int rope_dim) {
  if (n_axes < 0 || n_axes > SPOT_ROPE_AXES) return SPOT_ERR_UNSUPPORTED;
  if (n_axes > 0) {
    if ((rope_dim > 0 && !axis) || (rows > 0 && !pos)) return SPOT_ERR_NULL;
    for (int i = 0; i < rope_dim / 2; ++i)
      if (axis[i] >= n_axes) return SPOT_ERR_UNSUPPORTED;
  }
  return SPOT_OK;
}
void set_axes(RotaryArgs& a, int n_axes, const uint8_t* axis) {
  a.n_axes = n_axes;
  if (n_axes > 0) std::copy(axis, axis + a.rope_dim / 2, a.axis);
}

const uint16_t* in16(const void* p) { return static_cast<const uint16_t*>(p); }
uint16_t* out16(void* p) { return static_cast<uint16_t*>(p); }

}  // namespace

extern "C" {

spot_status spot_rope_frequencies(int rope_dim, double rope_base, int scaling, double factor,
                                  int orig_len, double low, double high, double* freq) {
  if (!freq && rope_dim > 0) return SPOT_ERR_NULL;
  if (rope_dim < 0 || rope_dim % 2 || rope_dim > 2 * kMaxPairs || !(rope_base > 0.0) ||
      !isfinite(rope_base) || scaling < SPOT_ROPE_NONE || scaling > SPOT_ROPE_PARTS)
    return SPOT_ERR_UNSUPPORTED;
  if (scaling != SPOT_ROPE_NONE && (!(factor >= 1.0) || !isfinite(factor)))
    return SPOT_ERR_UNSUPPORTED;
  if (scaling == SPOT_ROPE_BASE && rope_dim == 2) return SPOT_ERR_UNSUPPORTED;
  if (scaling == SPOT_ROPE_PARTS && (orig_len < 1 || !isfinite(low) || !isfinite(high) || !(low < high)))
    return SPOT_ERR_UNSUPPORTED;
  double base = rope_base;
  if (scaling == SPOT_ROPE_BASE && rope_dim > 2)
    base *= pow(factor, (double)rope_dim / (rope_dim - 2));
  // the pair farthest from 1 is the last one
  if (rope_dim > 0 &&
      (!isfinite(base) || !isfinite(pow(base, -2.0 * (rope_dim / 2 - 1) / rope_dim))))
    return SPOT_ERR_UNSUPPORTED;
  for (int i = 0; i < rope_dim / 2; ++i) {
    double f = pow(base, -2.0 * i / rope_dim);
    if (scaling == SPOT_ROPE_LINEAR) f /= factor;
    if (scaling == SPOT_ROPE_PARTS) {
      const double turns = orig_len * f / 6.283185307179586;
      const double g = fmin(fmax((turns - low) / (high - low), 0.0), 1.0);
      f = g * f + (1.0 - g) * (f / factor);
    }
    freq[i] = f;
  }
  return SPOT_OK;
}

spot_status spot_rotary(const void* x, int64_t x_stride, const int32_t* pos, int rows, int heads,
                        int d, int rope_dim, const double* freq, float amp, int flags, int dtype,
                        void* out, int64_t out_stride, void* stream) {
  return spot_rotary_axes(x, x_stride, pos, 0, nullptr, rows, heads, d, rope_dim, freq, amp, flags,
                          dtype, out, out_stride, stream);
}

spot_status spot_rotary_axes(const void* x, int64_t x_stride, const int32_t* pos, int n_axes,
                             const uint8_t* axis, int rows, int heads, int d, int rope_dim,
                             const double* freq, float amp, int flags, int dtype, void* out,
                             int64_t out_stride, void* stream) {
  if ((!freq && rope_dim > 0) || (rows > 0 && (!x || !pos || !out))) return SPOT_ERR_NULL;
  if (rows < 0 || heads < 1) return SPOT_ERR_SHAPE;
  const spot_status st = check_rope(d, rope_dim, freq, amp, flags, dtype);
  if (st != SPOT_OK) return st;
  const spot_status ax = check_axes(n_axes, axis, pos, rows, rope_dim);
  if (ax != SPOT_OK) return ax;
  const int64_t row = (int64_t)heads * d;
  if (row > 1 << 24 || x_stride < row || out_stride < row || !aligned(x, 2) || !aligned(out, 2))
    return SPOT_ERR_SHAPE;
  if (rows > 1 && out == x && out_stride != x_stride) return SPOT_ERR_SHAPE;
  if (rows == 0) return SPOT_OK;
  RotaryArgs a = {};
  a.q = in16(x);
  a.q_stride = x_stride;
  a.out_stride = out_stride;
  a.pos = pos;
  a.q_out = out16(out);
  a.rows = rows;
  a.h_q = heads;
  a.h_kv = 1;
  a.d = d;
  a.rope_dim = rope_dim;
  a.amp = amp;
  a.inverse = flags & SPOT_ROPE_INVERSE;
  for (int i = 0; i < rope_dim / 2; ++i) a.freq.f[i] = freq[i];
  set_axes(a, n_axes, axis);
  return from_hip(launch_rotary(a, dtype, flags & SPOT_ROPE_INTERLEAVED,
                                static_cast<hipStream_t>(stream)));
}

spot_status spot_rotary_append(const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                               const void* v, int64_t v_stride, int dtype, const int32_t* pos,
                               const int32_t* page_table, int n_pages, int page_size,
                               int max_pages, const int32_t* seq_start, const int32_t* seq_len,
                               int n_seq, int rows, int h_q, int h_kv, int d, int rope_dim,
                               const double* freq, float amp, int flags, void* q_out,
                               void* k_pages, void* v_pages, void* stream) {
  if ((!freq && rope_dim > 0) ||
      (rows > 0 && n_seq > 0 &&
       (!q || !k || !v || !seq_start || !seq_len || !q_out ||
        missing_pages(k_pages && v_pages, n_pages, page_table, max_pages))))
    return SPOT_ERR_NULL;
  if (n_seq < 0 || rows < 0 || h_q < 1 || !valid_pages(n_pages, page_size, max_pages, h_kv) ||
      (int64_t)rows * h_q > 0x7fffffff)
    return SPOT_ERR_SHAPE;
  const spot_status st = check_rope(d, rope_dim, freq, amp, flags, dtype);
  if (st != SPOT_OK) return st;
  if ((int64_t)h_q * d > 1 << 24 || (int64_t)h_kv * d > 1 << 24 || q_stride < (int64_t)h_q * d ||
      k_stride < (int64_t)h_kv * d || v_stride < (int64_t)h_kv * d)
    return SPOT_ERR_SHAPE;
  if (rows > 0 && q_out == q && q_stride != (int64_t)h_q * d) return SPOT_ERR_SHAPE;
  for (const void* p : {q, k, v, (const void*)q_out, (const void*)k_pages, (const void*)v_pages})
    if (!aligned(p, 2)) return SPOT_ERR_SHAPE;
  if (rows == 0 || n_seq == 0) return SPOT_OK;
  RotaryArgs a = {};
  a.q = in16(q);
  a.k = in16(k);
  a.v = in16(v);
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.out_stride = (int64_t)h_q * d;
  a.pos = pos;
  a.q_out = out16(q_out);
  a.k_pages = out16(k_pages);
  a.v_pages = out16(v_pages);
  a.pages = Pages{page_table, n_pages, page_size, max_pages};
  a.seq_start = seq_start;
  a.seq_len = seq_len;
  a.n_seq = n_seq;
  a.rows = rows;
  a.h_q = h_q;
  a.h_kv = h_kv;
  a.d = d;
  a.rope_dim = rope_dim;
  a.amp = amp;
  a.inverse = flags & SPOT_ROPE_INVERSE;
  for (int i = 0; i < rope_dim / 2; ++i) a.freq.f[i] = freq[i];
  return from_hip(launch_rotary(a, dtype, flags & SPOT_ROPE_INTERLEAVED,
                                static_cast<hipStream_t>(stream)));
}

spot_status spot_rotary_append8(const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                const void* v, int64_t v_stride, int dtype, const int32_t* pos,
                                int n_axes, const uint8_t* axis, const int32_t* page_table,
                                int n_pages, int page_size, int max_pages,
                                const int32_t* seq_start, const int32_t* seq_len, int n_seq,
                                int rows, int h_q, int h_kv, int d, int rope_dim,
                                const double* freq, float amp, int flags, void* q_out,
                                void* k_pages, void* v_pages, uint8_t* k_scale, uint8_t* v_scale,
                                void* stream) {
  if ((!freq && rope_dim > 0) ||
      (rows > 0 && n_seq > 0 &&
       (!q || !k || !v || !seq_start || !seq_len || !q_out ||
        missing_pages(k_pages && v_pages && k_scale && v_scale, n_pages, page_table, max_pages))))
    return SPOT_ERR_NULL;
  if (n_seq < 0 || rows < 0 || h_q < 1 || !valid_pages(n_pages, page_size, max_pages, h_kv) ||
      (int64_t)rows * h_q > 0x7fffffff)
    return SPOT_ERR_SHAPE;
  const spot_status st = check_rope(d, rope_dim, freq, amp, flags, dtype);
  if (st != SPOT_OK) return st;
  const spot_status ax = check_axes(n_axes, axis, pos, n_seq > 0 ? rows : 0, rope_dim);
  if (ax != SPOT_OK) return ax;
  if (d != 64 && d != 128) return SPOT_ERR_UNSUPPORTED;
  if ((int64_t)h_q * d > 1 << 24 || (int64_t)h_kv * d > 1 << 24 || q_stride < (int64_t)h_q * d ||
      k_stride < (int64_t)h_kv * d || v_stride < (int64_t)h_kv * d)
    return SPOT_ERR_SHAPE;
  if (rows > 0 && q_out == q && q_stride != (int64_t)h_q * d) return SPOT_ERR_SHAPE;
  for (const void* p : {q, k, v, (const void*)q_out})
    if (!aligned(p, 2)) return SPOT_ERR_SHAPE;
  if (!aligned(k_pages, 16) || !aligned(v_pages, 16)) return SPOT_ERR_SHAPE;
  if (rows == 0 || n_seq == 0) return SPOT_OK;
  Append8Args args = {};
  RotaryArgs& a = args.r;
  a.q = in16(q);
  a.k = in16(k);
  a.v = in16(v);
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.out_stride = (int64_t)h_q * d;
  a.pos = pos;
  a.q_out = out16(q_out);
  args.k8 = static_cast<uint8_t*>(k_pages);
  args.v8 = static_cast<uint8_t*>(v_pages);
  args.k_scale = k_scale;
  args.v_scale = v_scale;
  a.pages = Pages{page_table, n_pages, page_size, max_pages};
  a.seq_start = seq_start;
  a.seq_len = seq_len;
  a.n_seq = n_seq;
  a.rows = rows;
  a.h_q = h_q;
  a.h_kv = h_kv;
  a.d = d;
  a.rope_dim = rope_dim;
  a.amp = amp;
  a.inverse = flags & SPOT_ROPE_INVERSE;
  for (int i = 0; i < rope_dim / 2; ++i) a.freq.f[i] = freq[i];
  set_axes(a, n_axes, axis);
  return from_hip(launch_append8(args, dtype, flags & SPOT_ROPE_INTERLEAVED,
                                 static_cast<hipStream_t>(stream)));
}

size_t spot_paged_workspace_bytes(int n_seq, int rows, int h_q, int h_kv, int d) {
  if (n_seq < 1 || rows < 1 || h_q < 1 || h_kv < 1 || d < 1) return 0;
  // Enough for every call of at most these sequences and rows: of as many rows the fewest
  // sequences go to the second kernel first, two before one.
  const int G = h_q / h_kv;
  const bool many = launch_many(1, rows, G, kShortCache + 1) ||
                    (n_seq > 1 && launch_many(2, rows, G, kShortCache + 1));
  return many ? attend_many_workspace(d) : attend_few_workspace(d);
}

spot_status spot_paged_attend_sinks(const void* q, int dtype, const void* k_pages,
                                    const void* v_pages, const int32_t* page_table, int n_pages,
                                    int page_size, int max_pages, const int32_t* seq_start,
                                    const int32_t* seq_len, int n_seq, int rows, int h_q, int h_kv,
                                    int d, float sm_scale, float softcap, const float* slopes,
                                    int window, int n_sink, const int32_t* prefix,
                                    const int32_t* first, void* out, float* lse, void* ws,
                                    size_t ws_bytes, void* stream) {
  if (rows > 0 && n_seq > 0 &&
      (!q || !seq_start || !seq_len || !out ||
       missing_pages(k_pages && v_pages, n_pages, page_table, max_pages)))
    return SPOT_ERR_NULL;
  const spot_status st = check_attend(dtype, n_pages, page_size, max_pages, n_seq, rows, h_q, h_kv,
                                      d, sm_scale, softcap, window);
  if (st != SPOT_OK) return st;
  if (n_sink < 0) return SPOT_ERR_SHAPE;
  if (!aligned(q, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(out, 16))
    return SPOT_ERR_SHAPE;
  if (rows == 0 || n_seq == 0) return SPOT_OK;
  AttendArgs a = {};
  a.q = in16(q);
  a.k = in16(k_pages);
  a.v = in16(v_pages);
  a.pages = Pages{page_table, n_pages, page_size, max_pages};
  a.seq_start = seq_start;
  a.seq_len = seq_len;
  a.n_seq = n_seq;
  a.rows = rows;
  a.h_q = h_q;
  a.h_kv = h_kv;
  a.rule = Rule{sm_scale, softcap, slopes, window, prefix, first, sinks(window, n_sink)};
  a.out = out16(out);
  a.lse = lse;
  return attend(a, dtype, d, ws, ws_bytes, static_cast<hipStream_t>(stream));
}

spot_status spot_paged_attend(const void* q, int dtype, const void* k_pages, const void* v_pages,
                              const int32_t* page_table, int n_pages, int page_size, int max_pages,
                              const int32_t* seq_start, const int32_t* seq_len, int n_seq, int rows,
                              int h_q, int h_kv, int d, float sm_scale, float softcap,
                              const float* slopes, int window, const int32_t* prefix,
                              const int32_t* first, void* out, float* lse, void* ws,
                              size_t ws_bytes, void* stream) {
  return spot_paged_attend_sinks(q, dtype, k_pages, v_pages, page_table, n_pages, page_size,
                                 max_pages, seq_start, seq_len, n_seq, rows, h_q, h_kv, d, sm_scale,
                                 softcap, slopes, window, 0, prefix, first, out, lse, ws, ws_bytes,
                                 stream);
}

spot_status spot_paged_attend8(const void* q, int dtype, const void* k_pages, const void* v_pages,
                               const uint8_t* k_scale, const uint8_t* v_scale,
                               const int32_t* page_table, int n_pages, int page_size, int max_pages,
                               const int32_t* seq_start, const int32_t* seq_len, int n_seq,
                               int rows, int h_q, int h_kv, int d, float sm_scale, float softcap,
                               const float* slopes, int window, int n_sink, const int32_t* prefix,
                               const int32_t* first, void* out, float* lse, void* ws,
                               size_t ws_bytes, void* stream) {
  if (rows > 0 && n_seq > 0 &&
      (!q || !seq_start || !seq_len || !out ||
       missing_pages(k_pages && v_pages && k_scale && v_scale, n_pages, page_table, max_pages)))
    return SPOT_ERR_NULL;
  const spot_status st = check_attend(dtype, n_pages, page_size, max_pages, n_seq, rows, h_q, h_kv,
                                      d, sm_scale, softcap, window);
  if (st != SPOT_OK) return st;
  if (n_sink < 0) return SPOT_ERR_SHAPE;
  if (!aligned(q, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(out, 16))
    return SPOT_ERR_SHAPE;
  if (rows == 0 || n_seq == 0) return SPOT_OK;
  AttendArgs a = {};
  a.q = in16(q);
  a.k8 = static_cast<const uint8_t*>(k_pages);
  a.v8 = static_cast<const uint8_t*>(v_pages);
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.pages = Pages{page_table, n_pages, page_size, max_pages};
  a.seq_start = seq_start;
  a.seq_len = seq_len;
  a.n_seq = n_seq;
  a.rows = rows;
  a.h_q = h_q;
  a.h_kv = h_kv;
  a.rule = Rule{sm_scale, softcap, slopes, window, prefix, first, sinks(window, n_sink)};
  a.out = out16(out);
  a.lse = lse;
  return attend(a, dtype, d, ws, ws_bytes, static_cast<hipStream_t>(stream));
}

spot_status spot_paged_weights(const void* q, const float* lse, int dtype, const void* k_pages,
                               const int32_t* page_table, int n_pages, int page_size,
                               int max_pages, const int32_t* seq_start, const int32_t* seq_len,
                               int n_seq, int rows, int h_q, int h_kv, int d, float sm_scale,
                               float softcap, const float* slopes, int window,
                               const int32_t* prefix, const int32_t* first, const float* acc,
                               float decay, float* acc_out, void* stream) {
  if (n_seq > 0 && (!seq_start || !seq_len || (max_pages > 0 && !acc_out) ||
                    missing_pages(k_pages, n_pages, page_table, max_pages) ||
                    (rows > 0 && (!q || !lse))))
    return SPOT_ERR_NULL;
  const spot_status st = check_attend(dtype, n_pages, page_size, max_pages, n_seq, rows, h_q, h_kv,
                                      d, sm_scale, softcap, window);
  if (st != SPOT_OK) return st;
  if (!aligned(q, 16) || !aligned(k_pages, 16)) return SPOT_ERR_SHAPE;
  if (!isfinite(decay) || n_seq > 65535) return SPOT_ERR_UNSUPPORTED;
  if (n_seq == 0) return SPOT_OK;
  WeightArgs a = {};
  a.q = in16(q);
  a.lse = lse;
  a.k = in16(k_pages);
  a.pages = Pages{page_table, n_pages, page_size, max_pages};
  a.seq_start = seq_start;
  a.seq_len = seq_len;
  a.n_seq = n_seq;
  a.rows = rows;
  a.h_q = h_q;
  a.h_kv = h_kv;
  a.rule = Rule{sm_scale, softcap, slopes, window, prefix, first, 0};
  a.acc = acc;
  a.decay = decay;
  a.acc_out = acc_out;
  return from_hip(launch_weights(a, dtype, d, static_cast<hipStream_t>(stream)));
}

spot_status spot_cache_evict(const float* acc, const void* k_pages, const void* v_pages,
                             const int32_t* page_table, int n_pages, int page_size, int max_pages,
                             const int32_t* seq_len, int n_seq, int h_kv, int d, int budget,
                             int n_sink, int n_recent, void* k_dst, void* v_dst,
                             const int32_t* dst_table, int n_dst_pages, int dst_max_pages,
                             int32_t* idx, int32_t* new_len, float* acc_out, int out_cap,
                             void* stream) {
  if (n_seq > 0 && (!seq_len || !idx || !new_len || (max_pages > 0 && !acc) ||
                    (out_cap > 0 && !acc_out) ||
                    missing_pages(k_pages && v_pages, n_pages, page_table, max_pages) ||
                    missing_pages(k_dst && v_dst, n_dst_pages, dst_table, dst_max_pages)))
    return SPOT_ERR_NULL;
  if (n_seq < 0 || !valid_pages(n_pages, page_size, max_pages, h_kv) ||
      !valid_pages(n_dst_pages, page_size, dst_max_pages, h_kv))
    return SPOT_ERR_SHAPE;
  if (budget < 1 || n_sink < 0 || n_recent < 0 || (int64_t)n_sink + n_recent > budget)
    return SPOT_ERR_RULE;
  if (d < 8 || d % 8 || d > 1024 || n_seq > 65535 || h_kv > 65535) return SPOT_ERR_UNSUPPORTED;
  if (budget > 1 << 30 || out_cap > 1 << 30) return SPOT_ERR_UNSUPPORTED;
  const int64_t kept = std::min((int64_t)budget, (int64_t)max_pages * page_size);   // at most
  if (kept > (int64_t)dst_max_pages * page_size || kept > out_cap) return SPOT_ERR_SHAPE;
  if (!aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(k_dst, 16) || !aligned(v_dst, 16))
    return SPOT_ERR_SHAPE;
  if (n_seq == 0) return SPOT_OK;
  if ((acc && acc_out == acc) || new_len == seq_len) return SPOT_ERR_SHAPE;
  EvictArgs a = {};
  a.acc = acc;
  a.k = in16(k_pages);
  a.v = in16(v_pages);
  a.pages = Pages{page_table, n_pages, page_size, max_pages};
  a.seq_len = seq_len;
  a.n_seq = n_seq;
  a.h_kv = h_kv;
  a.d = d;
  a.budget = budget;
  a.n_sink = n_sink;
  a.n_recent = n_recent;
  a.k_dst = out16(k_dst);
  a.v_dst = out16(v_dst);
  a.dst = Pages{dst_table, n_dst_pages, page_size, dst_max_pages};
  a.idx = idx;
  a.new_len = new_len;
  a.acc_out = acc_out;
  a.out_cap = out_cap;
  return from_hip(launch_evict(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
