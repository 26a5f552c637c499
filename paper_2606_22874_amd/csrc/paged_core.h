// Shared by the operators on a paged cache (gfx950): element types, the rows of
// a chunk and what they see, the scores' cap and distance bias, page look-up, and
// the division of the attention's work among workgroups.
//
// A sequence's new tokens and the G query heads that share a KV head form the
// rows of one matrix: row j is token j / G, head j % G of the group, so a tile of
// rows reads each key once for all its heads, whatever G is.
#pragma once

#include "spot_internal.h"

#include "paged_map.h"

namespace spot {
namespace paged {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Element types.  c + A B of 16x16 tiles: lane l holds 8 (mfma32) or 4 (mfma16)
// consecutive k of row l%16 of A (column l%16 of B) from k = 8(l/16) or 4(l/16),
// and rows 4(l/16) ..+3 of column l%16 of c.  pack2 rounds to nearest even.
struct Bf16 {
  // Largest probability before rounding: the reference maximum itself.
  static constexpr float kShift = 0.f, kLazy = 8.f;
  static __device__ __forceinline__ f32x4 mfma32(const u32x4& a, const u32x4& b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mfma16(s16x4 a, s16x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack2(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2_t));
  }
  static __device__ __forceinline__ float lo(uint32_t x) { return bf16_lo(x); }
  static __device__ __forceinline__ float hi(uint32_t x) { return bf16_hi(x); }
  static __device__ __forceinline__ float one(uint16_t x) { return bf16_lo(x); }
  static __device__ __forceinline__ uint16_t round(float x) { return (uint16_t)pack2(x, 0.f); }
  static constexpr uint32_t kExponent = 0x7f80u;   // all ones: infinite or NaN
};
struct Fp16 {
  // FP16 has 24 bits below 1, FP32's exponentials many more: probabilities are
  // kept 2^10 times larger (the reference lies 10 below the maximum), so that
  // many small ones still count; 2^14 at most, below FP16's largest number.
  static constexpr float kShift = 10.f, kLazy = 4.f;
  static __device__ __forceinline__ f32x4 mfma32(const u32x4& a, const u32x4& b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mfma16(s16x4 a, s16x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(f16x4, a),
                                                 __builtin_bit_cast(f16x4, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack2(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, f16x2));
  }
  static __device__ __forceinline__ float lo(uint32_t x) {
    return (float)__builtin_bit_cast(f16x2, x)[0];
  }
  static __device__ __forceinline__ float hi(uint32_t x) {
    return (float)__builtin_bit_cast(f16x2, x)[1];
  }
  static __device__ __forceinline__ float one(uint16_t x) { return lo(x); }
  static __device__ __forceinline__ uint16_t round(float x) { return (uint16_t)pack2(x, 0.f); }
  static constexpr uint32_t kExponent = 0x7c00u;
};

// The reference for the largest score of a block: kShift below it (`shifted`), in the log2
// domain.  Beyond 2^24 scores are whole numbers of more than 2, and the shift, rounded with
// them, could become 16: with kLazy's slack more than FP16 holds.  There it is left out.
constexpr float kFarScore = 16777216.f;
template <class T>
__device__ __forceinline__ float reference(float top, float shifted) {
  return T::kShift == 0.f || fabsf(top) > kFarScore ? top : shifted;
}

// Wait states between matrix instructions and the ordinary ones that read their
// results: 8 are needed (4 passes).  Where a branch lies between, the compiler (ROCm 7.2)
// counts them along one path only, and around a block that is skipped 1 to 3 were left:
// scores came back without their last product.  16 states in place, before any branch,
// make every path long enough.  The kernels that have none of this (decode, prefill,
// scores, projections) have 8 on every path as they are built; a test looks at all.
__device__ __forceinline__ void settle(f32x4& a) { asm volatile("s_nop 15" : "+v"(a)); }
__device__ __forceinline__ void settle(f32x4 (&a)[2]) {
  asm volatile("s_nop 15" : "+v"(a[0]), "+v"(a[1]));
}
__device__ __forceinline__ void settle(f32x4 (&a)[4]) {
  asm volatile("s_nop 15" : "+v"(a[0]), "+v"(a[1]), "+v"(a[2]), "+v"(a[3]));
}
__device__ __forceinline__ void settle(f32x4 (&a)[8]) {
  asm volatile("s_nop 15"
               : "+v"(a[0]), "+v"(a[1]), "+v"(a[2]), "+v"(a[3]), "+v"(a[4]), "+v"(a[5]),
                 "+v"(a[6]), "+v"(a[7]));
}

// Whether one of a pair of elements is infinite or NaN, and the pair with such
// elements zero.
template <class T>
__device__ __forceinline__ bool odd2(uint32_t x) {
  return (~x & T::kExponent) == 0u || (~x & (T::kExponent << 16)) == 0u;
}
template <class T>
__device__ __forceinline__ uint32_t clean2(uint32_t x) {
  if ((~x & T::kExponent) == 0u) x &= 0xffff0000u;
  if ((~x & (T::kExponent << 16)) == 0u) x &= 0xffffu;
  return x;
}

// tanh to 2e-7 relative: its Taylor polynomial up to 0.5 (the first dropped term is
// 9e-8 there), and beyond it e^(-2|y|), where 1 - e keeps its bits.
__device__ __forceinline__ float tanh_near(float y) {
  const float z = y * y;
  float t = fmaf(21844.f / 6081075, z, -1382.f / 155925);
  t = fmaf(t, z, 62.f / 2835);
  t = fmaf(t, z, -17.f / 315);
  t = fmaf(t, z, 2.f / 15);
  t = fmaf(t, z, -1.f / 3);
  return y * fmaf(t, z, 1.f);
}
__device__ __forceinline__ float tanh_any(float y) {
  const float a = fabsf(y), e = __builtin_amdgcn_exp2f(a * (-2.f * kLog2e));
  const float far = copysignf((1.f - e) * __builtin_amdgcn_rcpf(1.f + e), y);
  return a < 0.5f ? tanh_near(y) : far;
}

// cap tanh(y) as cap - 2 cap / (1 + e^(2 y)), of y2 = 2 y log2(e), within 4e-7 cap (exponential
// and reciprocal to one place, four roundings; 2.2e-7 measured, lse's included): for scores
// beyond those of tanh_near, half the operations of tanh_any.  A score of 16 bits'
// products is off by 1e-5 and more by itself, so caps up to kQuickCap take it (900 tokens
// over an 8-bit cache of 7500, cap 30, scores of both kinds: 259 us with tanh_any, 212).
// Of y2's factor, 2 log2(e) scale / cap: an infinite one would make NaN of a score of 0.
constexpr float kQuickCap = 64.f, kQuickMul = 1e38f;
__device__ __forceinline__ float capped(float y2, float cap) {
  return fmaf(-2.f * cap, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(y2)), cap);
}

// Scores in the log2 domain.  `ahead`: the row's position less the key's, in FP32 from
// their difference as integers (positions themselves may need more than 24 bits).
// QUICK: capped() where it is near enough, and from a block that needs it on in all of the
// wave's (hot), which saves the look at each score's size.  Which form is taken follows from
// keys that the rows see: of blocks that are not `whole` (some row does not see all of it) the
// scores include those of keys that hold anything, and such a block has tanh_near or tanh_any,
// which agree to the bit where both do.
template <bool CAP, bool BIAS, bool QUICK = false>
struct Scores {
  float mul, cap2, slope2;   // scale log2e, or scale / cap; cap log2e; slope log2e
  int p;                     // the row's position
  bool hot = false;
  __device__ __forceinline__ Scores() {}
  __device__ __forceinline__ Scores(const Rule& u, const Seq& q, int i, int head) {
    mul = CAP ? u.scale / u.cap : u.scale * kLog2e;
    cap2 = u.cap * kLog2e;
    slope2 = BIAS && u.slopes ? u.slopes[head] * kLog2e : 0.f;
    p = q.len - q.n + i;
  }
  // Four scores of a lane, `ahead` of the first.  kNear: all of the wave's lie where
  // tanh_near does (most calls have a cap well above their scores).
  enum How { kAny, kNear, kQuick };
  template <How HOW>
  __device__ __forceinline__ f32x4 scaled(f32x4 s, float ahead) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float y = s[i] * mul;
      float x = !CAP            ? y
                : HOW == kQuick ? capped(s[i] * (mul * (2.f * kLog2e)), cap2)
                                : cap2 * (HOW == kNear ? tanh_near(y) : tanh_any(y));
      if (BIAS) x = fmaf(-slope2, fabsf(ahead - (float)i), x);
      s[i] = x;
    }
    return s;
  }
  // N such quads, 16 keys from one to the next.
  template <int N>
  __device__ __forceinline__ void operator()(f32x4 (&s)[N], float ahead, bool whole = false) {
    if constexpr (CAP) {
      if (!QUICK || !hot) {
        float top = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, fabsf(s[e][i]));
        if (!__ballot(top * fabsf(mul) >= 0.5f)) {
#pragma unroll
          for (int e = 0; e < N; ++e) s[e] = scaled<kNear>(s[e], ahead - 16.f * e);
          return;
        }
        hot = QUICK & whole & (cap2 <= kQuickCap * kLog2e) & (fabsf(mul) <= kQuickMul);
      }
      if (QUICK && hot) {
#pragma unroll
        for (int e = 0; e < N; ++e) s[e] = scaled<kQuick>(s[e], ahead - 16.f * e);
        return;
      }
    }
#pragma unroll
    for (int e = 0; e < N; ++e) s[e] = scaled<kAny>(s[e], ahead - 16.f * e);
  }
  __device__ __forceinline__ float one(float s, float ahead) const {
    return scaled<kAny>(f32x4{s, s, s, s}, ahead)[0];
  }
};

// ------------------------------------------------------- division of work
// Work is counted in (row tile, KV head, 64-key block) steps.  A tile whose keys
// are more than 1/kTarget of all steps is split along the keys, so that a long
// sequence among short ones, or few rows over a long cache, still fill the
// device; the parts of a tile are joined by the last one to finish.  Every
// workgroup finds its own part from the lengths on the device, so the host needs
// none of them and a captured call stays right when they change.
constexpr int kTarget = 512;
constexpr int kMaxParts = 2 * kTarget + 64;  // parts of split tiles (each has at most twice its share)
constexpr int kMaxSplit = kTarget + 64;      // split tiles

struct Part {
  int s, tile;        // sequence (-1: no work), row tile
  int split, n_split; // part and number of parts of the tile
  int slot, counter;  // workspace slot of part 0, completion counter (n_split > 1)
  Seq q;
};

// Blocks of 64 keys that the rows of a sequence see at most (documents aside).
__device__ __forceinline__ int span_blocks(const Seq& q, int window, int sink, int cap) {
  const int hi = min(q.len, cap), p0 = q.len - q.n;
  const int lo = window > 0 && window <= p0 ? p0 - window + 1 : 0;
  const int sinks = sink > 0 ? min((sink - 1) / 64 + 1, min(lo, cap) / 64) : 0;
  return (hi > lo ? (hi + 63) / 64 - lo / 64 : 0) + sinks;
}

// The part of unit `unit` (of the parts of all tiles of TR rows, one KV head), found by
// one wave; every lane gets it.  Sequences of from < rows (new tokens x heads) <= to
// take part.  A tile has at most kMaxJoin parts: the one that joins them reads them
// all.
// ROUND 0 (many workgroups at once, bound by the keys' bytes): parts of at least 2, 4
// or 8 blocks by the number of tiles, as splitting costs a join (us, decode, 2 / 4 / 8:
// one sequence of 700 tokens, 8 tiles, 9.8 / 11.3 / 12.9; 8 of 700, 64 tiles, 13.2 /
// 12.4 / 13.6; 16 of 300, 128 tiles, 13.2 / 11.9 / 11.0), and at most twice the root of
// a tile's blocks, where blocks of a part and parts of a join add least (one sequence
// of 4000 tokens 17.8 us without that bound, 15.1 with it, 16.3 with 2.5 times the
// root; two of them 21.2 at 2.5, 16.8).
// ROUND > 0: that many workgroups run at once, each as long as its blocks; the blocks
// of a part then grow from their least number, up to four times as many, to what ends
// first: rounds of workgroups x (blocks of a part + 8, about what a part costs beside
// them), and a join, about a block for each part.
// FIT > 0: so many workgroups run at once; where the parts are a few more, those that start
// last run alone, so the blocks of a part grow to at most twice their number until all fit
// (a mixed batch's 11 single sequences of up to 24000 tokens, 8-bit cache: 82 -> 63 us).  Not
// for a 16-bit cache without sinks, whose division of work, and so whose bits, this would
// change; what it would gain there has not been measured.
constexpr int kMaxJoin = 64;
template <int TR, int ROUND, int FIT = 0>
__device__ __forceinline__ Part find_part(int unit, const int32_t* seq_start,
                                          const int32_t* seq_len, int n_seq, int rows, int G,
                                          int h_kv, int window, int sink, int cap, int from,
                                          int to) {
  const int lane = __lane_id();
  auto most_parts = [](int nb) {
    return ROUND ? kMaxJoin : min(kMaxJoin, (int)ceilf(2.f * sqrtf((float)nb)));
  };
  auto tiles_of = [&](const Seq& q) {
    const int n = q.n * G;
    return n > from && n <= to ? (int)(((unsigned)n + TR - 1) / TR) : 0;
  };
  const float share = (float)h_kv / (float)kTarget;
  auto least_blocks = [&](int tiles) {
    return ROUND ? 4 : tiles * h_kv <= 16 ? 2 : tiles * h_kv <= 96 ? 4 : 8;
  };
  Part r;
  r.s = -1;
  if (ROUND == 0 && n_seq == 1) {
    // One sequence: the same numbers without a wave's sums and scans, in scalar registers (a
    // short call waits for its instructions too: one token over 600 of an 8-bit cache 10.75 to
    // 10.2 us, over 700 of a 16-bit one 10.4 to 9.8).
    const Seq q = sequence(seq_start, seq_len, 0, rows);
    const int T = tiles_of(q), nb = span_blocks(q, window, sink, cap);
    if (T > (int)((unsigned)rows * (unsigned)G / TR) + 1) return r;
    const int per = max(least_blocks(T), (int)ceilf((float)T * (float)nb * share));
    int ns = max(1, min((nb + per - 1) / per, most_parts(nb)));
    if (FIT && ns > 1 && T * ns * h_kv > FIT)
      for (int e = 9; e <= 16; ++e) {
        const int p = (per * e + 7) / 8, n = max(1, min((nb + p - 1) / p, most_parts(nb)));
        if (T * n * h_kv <= FIT) {
          ns = n;
          break;
        }
      }
    if (unit >= T * ns) return r;
    r.s = 0;
    r.tile = T - 1 - unit / ns;
    r.split = unit % ns;
    r.n_split = ns;
    r.slot = unit - r.split;
    r.counter = unit / ns;
    r.q = q;
    return r;
  }
  // all steps
  float steps = 0.f;
  int tiles = 0;
  Seq q0 = {0, 0, 0};
  for (int base = 0; base < n_seq; base += 64) {
    Seq q = {0, 0, 0};
    if (base + lane < n_seq) q = sequence(seq_start, seq_len, base + lane, rows);
    if (base == 0) q0 = q;
    const int T = tiles_of(q);
    steps += wave_sum((float)T * (float)span_blocks(q, window, sink, cap));
    tiles += wave_sum_i(T);
  }
  // More tiles than ascending starts can give: the grid has no workgroups for them, and
  // a split tile that lacks one would leave its counter standing.
  if (tiles > (int)((unsigned)rows * (unsigned)G / TR) + n_seq) return r;
  int per = max(least_blocks(tiles), (int)ceilf(steps * share));
  if (ROUND && n_seq <= 64) {
    const int T = tiles_of(q0), nb = T ? span_blocks(q0, window, sink, cap) : 0;
    if (__ballot(nb > per)) {
      int best = 0x7fffffff, at = per;
      for (int e = 8; e <= 32; e += e < 12 ? 1 : e < 20 ? 2 : 4) {
        const int p = (per * e + 7) / 8, ns = min(max(1, (nb + p - 1) / p), kMaxJoin);
        const int units = wave_sum_i(T * ns) * h_kv;
        // the longest part of any tile
        const int most = (int)wave_max_u((uint32_t)((nb + ns - 1) / ns));
        const int cost = (units + ROUND - 1) / max(ROUND, 1) * (most + 8) +
                         (int)wave_max_u((uint32_t)ns);
        if (cost < best) {
          best = cost;
          at = p;
        }
      }
      per = at;
    }
  }
  // (parts: at most the steps' share and one more a tile)
  if (FIT && n_seq <= 64 && steps * (float)h_kv > (float)per * (float)(FIT - tiles * h_kv)) {
    const int T = tiles_of(q0), nb = T ? span_blocks(q0, window, sink, cap) : 0;
    for (int e = 8; e <= 16; ++e) {
      const int p = (per * e + 7) / 8;
      const int ns = max(1, min((nb + p - 1) / p, most_parts(nb)));
      if (wave_sum_i(T * ns) * h_kv <= FIT) {
        per = p;
        break;
      }
    }
  }
  // the sequence that holds the unit
  int unit0 = 0, slot0 = 0, cnt0 = 0;
  for (int base = 0; base < n_seq; base += 64) {
    Seq q = q0;
    if (base) {
      q = Seq{0, 0, 0};
      if (base + lane < n_seq) q = sequence(seq_start, seq_len, base + lane, rows);
    }
    const int T = tiles_of(q), nb = span_blocks(q, window, sink, cap);
    const int ns = max(1, min((nb + per - 1) / per, most_parts(nb)));
    const int units = T * ns;
    const int incl = wave_incl_scan_i(units);
    const int split_units = ns > 1 ? units : 0, split_tiles = ns > 1 ? T : 0;
    const int si = wave_incl_scan_i(split_units), ti = wave_incl_scan_i(split_tiles);
    const uint64_t hit = __ballot(unit >= unit0 + incl - units && unit < unit0 + incl);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      const int in = unit - unit0 - __builtin_amdgcn_readlane(incl - units, l);
      const int n_tiles = __builtin_amdgcn_readlane(T, l);
      r.n_split = __builtin_amdgcn_readlane(ns, l);
      r.s = base + l;
      r.tile = n_tiles - 1 - in / r.n_split;       // the longest first
      r.split = in % r.n_split;
      r.slot = slot0 + __builtin_amdgcn_readlane(si - split_units, l) + in - r.split;
      r.counter = cnt0 + __builtin_amdgcn_readlane(ti - split_tiles, l) + in / r.n_split;
      r.q.start = __builtin_amdgcn_readlane(q.start, l);
      r.q.n = __builtin_amdgcn_readlane(q.n, l);
      r.q.len = __builtin_amdgcn_readlane(q.len, l);
      return r;
    }
    unit0 += __builtin_amdgcn_readlane(incl, 63);
    slot0 += __builtin_amdgcn_readlane(si, 63);
    cnt0 += __builtin_amdgcn_readlane(ti, 63);
  }
  return r;
}

// Workspace of the attention: completion counters (zero between calls, at the same
// place for every size), then the parts' (m, l) and O.
struct Workspace {
  unsigned* counters;   // [kMaxSplit]
  float* ml;            // [kMaxParts, TR, 2]
  float* o;             // [kMaxParts, TR, d]
};
constexpr size_t kCounterBytes = SPOT_PAGED_WORKSPACE_ZEROS;
static_assert(kMaxSplit * sizeof(unsigned) <= kCounterBytes, "room for the counters");

// A launch's threads are counted in 32 bits a dimension.
inline bool launchable(int64_t groups, unsigned threads) {
  return groups < ((int64_t)1 << 32) / threads;
}

struct AttendArgs {
  const uint16_t *q, *k, *v;
  const uint8_t *k8, *v8, *k_scale, *v_scale;   // of an 8-bit cache, in place of k and v
  Pages pages;
  const int32_t *seq_start, *seq_len;
  int n_seq, rows, h_q, h_kv;
  Rule rule;
  uint16_t* out;
  float* lse;
  Workspace ws;
  int from, to;      // sequences of from < rows (new tokens x heads of a group) <= to
};
// ws as the kernel's *_workspace sizes it.
hipError_t launch_attend_few(AttendArgs a, int dtype, int d, void* ws, hipStream_t s);
size_t attend_few_workspace(int d);
hipError_t launch_attend_many(AttendArgs a, int dtype, int d, void* ws, hipStream_t s);
size_t attend_many_workspace(int d);
hipError_t launch_sinks_many(AttendArgs a, int dtype, int d, void* ws, hipStream_t s);
// The same over an 8-bit cache.
hipError_t launch_attend_few8(AttendArgs a, int dtype, int d, void* ws, hipStream_t s);
hipError_t launch_attend_many8(AttendArgs a, int dtype, int d, void* ws, hipStream_t s);
hipError_t launch_sinks_many8(AttendArgs a, int dtype, int d, void* ws, hipStream_t s);

// Workgroups of a launch over tiles of TR rows: every tile in one part, and the parts
// that kTarget shares of the work add.
template <int TR>
inline int64_t attend_grid(const AttendArgs& a) {
  const int64_t rows = (int64_t)a.rows * (a.h_q / a.h_kv);
  int64_t tiles = rows / TR + a.n_seq;
  const int64_t most = (int64_t)a.n_seq * ((a.to - 1) / TR + 1);   // of sequences up to a.to
  if (tiles > most) tiles = most;
  return (tiles + kTarget / a.h_kv + 2) * a.h_kv;
}

struct WeightArgs {
  const uint16_t* q;
  const float* lse;
  const uint16_t* k;
  Pages pages;
  const int32_t *seq_start, *seq_len;
  int n_seq, rows, h_q, h_kv;
  Rule rule;
  const float* acc;     // [n_seq, h_kv, cap] or NULL (0)
  float decay;
  float* acc_out;
};
hipError_t launch_weights(const WeightArgs& a, int dtype, int d, hipStream_t s);

struct EvictArgs {
  const float* acc;     // [n_seq, h_kv, cap]
  const uint16_t *k, *v;
  Pages pages;
  const int32_t* seq_len;
  int n_seq, h_kv, d, budget, n_sink, n_recent;
  uint16_t *k_dst, *v_dst;
  Pages dst;            // of the same page size
  int32_t *idx, *new_len;
  float* acc_out;       // [n_seq, h_kv, out_cap]
  int out_cap;
};
hipError_t launch_evict(const EvictArgs& a, hipStream_t s);

constexpr int kMaxPairs = 128;        // rotary pairs of a head
struct PairFreq {
  double f[kMaxPairs];
};
struct RotaryArgs {
  const uint16_t *q, *k, *v;
  int64_t q_stride, k_stride, v_stride, out_stride;   // elements from row to row
  const int32_t* pos;
  uint16_t *q_out, *k_pages, *v_pages;
  Pages pages;
  const int32_t *seq_start, *seq_len;                 // seq_start NULL: q alone
  int n_seq, rows, h_q, h_kv, d, rope_dim;
  float amp;
  bool inverse;
  int n_axes;              // 0: one position a row; else [rows, n_axes]
  uint8_t axis[kMaxPairs];
  PairFreq freq;
};
hipError_t launch_rotary(const RotaryArgs& a, int dtype, bool interleaved, hipStream_t s);

// The same into an 8-bit cache.
struct Append8Args {
  RotaryArgs r;            // k_pages, v_pages not used
  uint8_t *k8, *v8, *k_scale, *v_scale;
};
hipError_t launch_append8(const Append8Args& a, int dtype, bool interleaved, hipStream_t s);

}  // namespace paged
}  // namespace spot
