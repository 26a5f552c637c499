// Attention of many rows over a paged cache (gfx950): chunks and whole prompts.
//
// One workgroup of 8 waves takes one part of a tile of 256 rows (new tokens x the
// query heads that share a KV head), 32 rows a wave; blocks of 64 keys pass through
// LDS and are used by all waves.  The mathematics is that of attend_few.hip, with
// S^T = K Q^T in 16x16x32 tiles (Q^T in registers for the whole key loop), the
// softmax down the lanes' columns, and O^T += V^T P^T, P^T straight from the
// accumulators (its keys permuted like those of the transposing LDS read of V).
//
// The two waves of a SIMD share its matrix core and its vector unit, so they go through
// a block in opposite order; period t is
//   waves 0-3: P V of block t-1, K Q of block t; start the copy of V(t); softmax of
//              block t; wait for the copy
//   waves 4-7: start the copy of K(t+1); softmax of block t-1; wait for the copy;
//              P V of block t-1, K Q of block t
// with one barrier behind it: what a period writes, V(t) and K(t+1), lies in the buffers
// that the period before it read last.  (A second barrier between the halves, so that
// matrix phases and softmaxes meet exactly, costs the longer of both twice: a prompt of
// 8192 tokens, 64 heads of 64, capped, 1653 us with it and 1341 without; plain, d = 128,
// 1198 and 1071.)  A softmax goes at a higher priority than matrix instructions, which
// wait for their own results anyway (16000 tokens, d = 128: 3891 to 3815 us; d = 64,
// 8192 tokens: 963 to 811; the other way round 3848 and 945).
// The copies fly behind a softmax and are down before the wave's next matrix phase: the
// compiler orders the LDS reads of a wave with a copy in flight one by one.
// A prompt of 16000 tokens, 64 heads of 128 over 8: 3.8 .. 4.0 ms, 1.05 .. 1.1 PFLOP/s;
// the matrix cores are busy 44 % of the cycles, the vector units 50 %.  Tiles of 128 rows
// (4 waves, two workgroups a CU) read the keys twice as often: 14 % slower; a third pair
// of buffers, or touching the next blocks ahead for L2, 3 .. 5 %.
// With sinks a tile goes through two runs of blocks, numbered through (paged_map.h): a prompt
// of 12000 tokens, 32 heads of 128 over 8, window 2048 and 16 sinks, 464 .. 475 us (442
// without the sinks).  Over an 8-bit cache the tiles are widened on their way (Widen): a prompt
// of 14000, 64 heads over 8, 3.16 ms, 1.01 PFLOP/s; 512 tokens over 49152, 784 .. 797 us.
// K and V go from memory to LDS 16 bytes a lane (1 KiB a wave instruction), rows
// swizzled by 16-byte chunks against bank conflicts; each of the buffers is a
// variable of its own and the loop is unrolled by two, so that the compiler can tell
// the copies in flight from the reads.
#pragma once

#include <type_traits>

#include "cache8.h"
#include "decode_core.h"

namespace spot {
namespace paged {
namespace many {

using dec::lanes_max_xor16;
using dec::lanes_max_xor32;
using dec::lanes_sum_xor16;
using dec::lanes_sum_xor32;

constexpr int kRows = 256;         // rows of a tile
constexpr int kWaves = 8;
constexpr int kRound = 256;        // workgroups at once: one a CU
constexpr int kListBlocks = 512;   // blocks whose pages are looked up at once
typedef __attribute__((address_space(3))) void lds_void;
#define SPOT_INLINE __attribute__((always_inline))

// Physical 16-byte chunk of logical chunk c of row r.  K is read one chunk of 16 rows
// at a time, V 8 bytes of 8 rows at two neighbouring chunks.
template <int D>
__device__ __forceinline__ int swz_k(int r, int c) {
  return c ^ (r & (D / 8 - 1));
}
template <int D>
__device__ __forceinline__ int swz_v(int r, int c) {
  return D == 128 ? c ^ ((r & 7) << 1) : c ^ (((r >> 1) & 3) << 1);
}

// The lane's number, made anew where it is used: held or kept in scratch memory, what
// follows from it costs registers or waits for every copy in flight.
__device__ __forceinline__ int fresh_lane() {
  int lane;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(lane));
  return lane;
}

// Copies of a block of 64 rows by 4 waves: instruction u of wave w fills rows
// R (4u + w) .. + R, R rows of 1 KiB, all of one group of 16 keys.
template <int D, bool IS_K>
struct Copy {
  static constexpr int R = 1024 / (2 * D);       // 4 or 8 rows an instruction
  static constexpr int N = 64 / R / 4;           // instructions of a wave
  static constexpr int CH = D / 8;               // chunks of a row
  static __device__ __forceinline__ int row(int u, int wave, int lane) {
    return R * (4 * u + wave) + lane / CH;
  }
  static __device__ __forceinline__ void issue(const uint16_t* pool, const int* list,
                                               unsigned char* dst, int wave) {
    const int lane = fresh_lane();
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int r = row(u, wave, lane), pc = lane % CH;
      const int lc = IS_K ? swz_k<D>(r, pc) : swz_v<D>(r, pc);
      const int group = R * (4 * u + wave) / 16;
      const int at = __builtin_amdgcn_readfirstlane(list[group]);   // -1: a row of no use
      const uint16_t* src = pool + (int64_t)(at < 0 ? 0 : at) * D;
      const uint32_t off = (uint32_t)((r & 15) * D + lc * 8);
      __builtin_amdgcn_global_load_lds(src + off, (lds_void*)(dst + (4 * u + wave) * 1024), 16, 0,
                                       0);
    }
  }
};

// The same of an 8-bit cache, in two steps: thread i of the 4 waves loads the 16 codes of
// chunk i % CH of rows i / CH + RW u, which are on their way behind a softmax, and then
// stores them as two chunks of elements.  (By way of a place of the thread's own in LDS,
// which needs no registers meanwhile: 3 % slower, and with sinks, where some then go to
// scratch memory, still 2 %: the wait for the copy, one more read and the stores follow each
// other before the barrier.  Stored before the softmax instead of behind it: 3 % again.
// Stored in an order that keeps eight lanes off each other's banks, by selects: 1.5 %.)
template <class T, int D, bool IS_K>
struct Widen {
  static constexpr int CH = D / 16;              // 16-byte chunks of a row's codes
  static constexpr int RW = 256 / CH;            // rows of the 4 waves at once
  static constexpr int N = 64 / RW;
  static __device__ __forceinline__ int row(int u, int wave, int lane) {
    return RW * u + wave * (64 / CH) + lane / CH;
  }
  // (the rows of a wave's load lie in one group of 16 keys)
  static __device__ __forceinline__ void load(const uint8_t* pool, const int* list,
                                              u32x4 (&raw)[N], int wave) {
    const int lane = fresh_lane();
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int group = (RW * u + wave * (64 / CH)) / 16;
      const int at = __builtin_amdgcn_readfirstlane(list[group]);   // -1: a row of no use
      const uint8_t* src = pool + (int64_t)(at < 0 ? 0 : at) * D;
      const uint32_t off = (uint32_t)((row(u, wave, lane) & 15) * D + lane % CH * 16);
      raw[u] = *reinterpret_cast<const u32x4*>(src + off);
    }
  }
  static __device__ __forceinline__ float scale(const uint16_t* scales, int u, int wave) {
    const uint32_t x = scales[(RW * u + wave * (64 / CH)) / 16];
    return scale8(__builtin_amdgcn_readfirstlane(IS_K ? x & 255u : x >> 8));
  }
  static __device__ __forceinline__ void put(unsigned char* dst, int r, int c, const u32x4& x) {
    const int pc = IS_K ? swz_k<D>(r, c) : swz_v<D>(r, c);
    *reinterpret_cast<u32x4*>(dst + r * (2 * D) + (pc << 4)) = x;
  }
  static __device__ __forceinline__ void store(const u32x4 (&raw)[N], const uint16_t* scales,
                                               unsigned char* dst, int wave) {
    const int lane = fresh_lane(), c = lane % CH * 2;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int r = row(u, wave, lane);
      const float s = scale(scales, u, wave);
      const u32x4& x = raw[u];
      put(dst, r, c, wide8<T>(x[0], x[1], s, s));
      put(dst, r, c + 1, wide8<T>(x[2], x[3], s, s));
    }
  }
  // store() of rows that not every row of the tile sees: zeros for tokens that none sees
  // (unseen) or that have no page, and for infinite and NaN elements of the others, of
  // which it tells.
  template <class F>
  static __device__ __forceinline__ bool mend(const u32x4 (&raw)[N], const int* list,
                                              const uint16_t* scales, unsigned char* dst, int wave,
                                              F unseen) {
    const int lane = fresh_lane(), c = lane % CH * 2;
    bool odd = false;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int r = row(u, wave, lane);
      const float s = scale(scales, u, wave);
      const u32x4& y = raw[u];
      const bool none = (list[r >> 4] < 0) | unseen(r);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        u32x4 x = wide8<T>(y[2 * e], y[2 * e + 1], s, s);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          odd |= !none & odd2<T>(x[i]);
          x[i] = none ? 0u : clean2<T>(x[i]);
        }
        put(dst, r, c + e, x);
      }
    }
    return odd;
  }
};

__device__ __forceinline__ void wait_vm() { __builtin_amdgcn_s_waitcnt(0x0F70); }   // vmcnt(0)

// Barrier over the waves' LDS accesses.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_s_waitcnt(0xC07F);      // lgkmcnt(0)
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// What a row of the tile sees, and what its scores need: read from LDS where a block
// calls for it (registers are short).
struct RowRule {
  int lo, hi, p;
  float slope2;
};
struct SinkRule {
  int from, end;
};

template <class T, int D, bool CAP, bool BIAS, bool SINK, bool QUICK>
struct Wave {
  static constexpr int RB = D * 2, KS = D / 32, DT = D / 16;
  u32x4 qf[KS][2];            // Q^T as the B operand [dims][16 rows]
  f32x4 o[2][DT];
  f32x4 s[2][4];              // scores, then probabilities, of the current block
  u32x4 pb[2][2];             // the probabilities as the B operand
  float m_run[2], l_run[2];
  const RowRule* rows;        // the wave's 32
  const SinkRule* sinks;
  float mul, cap2;            // see Scores
  bool hot;
  int* far;                   // set where a maximum lies beyond kFarScore
  int G, r16;

  // S^T of one block; the K fragments of a step are read one step ahead.  The chunks'
  // swizzle is an exclusive or: one address and immediates give all fragments.
  __device__ __forceinline__ void qk(const unsigned char* Kt) {
    u32x4 a[2][4];
    const int lane = fresh_lane(), r16 = lane & 15, G = lane >> 4;
    const int at = r16 * RB + (swz_k<D>(r16, G) << 4);
    auto load = [&](int ks, int slot) {
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
        a[slot][kt] = *reinterpret_cast<const u32x4*>(Kt + (at ^ ks << 6) + kt * 16 * RB);
    };
    load(0, 0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int cur = ks & 1;
      if (ks + 1 < KS) load(ks + 1, cur ^ 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int qt = 0; qt < 2; ++qt)
          s[qt][kt] = T::mfma32(a[cur][kt], qf[ks][qt],
                                ks == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[qt][kt]);
    }
  }

  // O^T += V^T P^T of one block.  Lane (G, r16) of the transposing read addresses row
  // 32 ks + 4 G + r16 / 4 (and 16 below), columns 4 (r16 % 4) .. +3 of the d tile, and
  // gets column r16 of rows 4 G .. +3.
  __device__ __forceinline__ void pv(const unsigned char* Vt) {
    u32x4 a[2][DT];
    const int lane = fresh_lane(), r16 = lane & 15, G = lane >> 4;
    const int r0 = 4 * G + (r16 >> 2);
    const int at = r0 * RB + (swz_v<D>(r0, (r16 & 3) >> 1) << 4) + (r16 & 1) * 8;
    auto load = [&](int ks, int dt0) {
#pragma unroll
      for (int dt = dt0; dt < dt0 + 4; ++dt) {
        const int off = (at ^ dt << 5) + 32 * ks * RB;
        const u32x2 y0 = __builtin_bit_cast(
            u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                       (__attribute__((address_space(3))) s16x4*)(Vt + off)));
        const u32x2 y1 = __builtin_bit_cast(
            u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                       (__attribute__((address_space(3))) s16x4*)(Vt + off + 16 * RB)));
        a[ks][dt] = u32x4{y0[0], y0[1], y1[0], y1[1]};
      }
    };
    auto mma = [&](int ks, int dt0) {
#pragma unroll
      for (int dt = dt0; dt < dt0 + 4; ++dt)
#pragma unroll
        for (int qt = 0; qt < 2; ++qt) o[qt][dt] = T::mfma32(a[ks][dt], pb[qt][ks], o[qt][dt]);
    };
    if constexpr (DT == 8) {
      load(0, 0);
      load(0, 4);
      __builtin_amdgcn_sched_barrier(0);
      mma(0, 0);
      load(1, 0);
      __builtin_amdgcn_sched_barrier(0);
      mma(0, 4);
      load(1, 4);
      __builtin_amdgcn_sched_barrier(0);
      mma(1, 0);
      mma(1, 4);
    } else {
      load(0, 0);
      load(1, 0);
      __builtin_amdgcn_sched_barrier(0);
      mma(0, 0);
      mma(1, 0);
    }
  }

  // Online softmax of the scores into pb.  below, above: some row does not see the
  // first or last keys of the block; pages: bit kt says that keys 16 kt .. are there.
  // sunk: the first keys may be sinks.  EXACT: every scaled score is rounded.
  template <bool EXACT>
  __device__ __forceinline__ void softmax(int t0, bool below, bool above, bool sunk,
                                          unsigned pages) {
    asm volatile("s_nop 15"
                 : "+v"(s[0][0]), "+v"(s[0][1]), "+v"(s[0][2]), "+v"(s[0][3]), "+v"(s[1][0]),
                   "+v"(s[1][1]), "+v"(s[1][2]), "+v"(s[1][3]));   // see settle()
    // Without a cap a positive scale waits until the exponent (and the bias is taken in
    // its units): an operation less for each score.
    const bool late = !CAP && !EXACT && mul > 1e-6f;
    const float c = late ? mul : 1.f;
    if (CAP || BIAS || EXACT) {
#pragma unroll
      for (int qt = 0; qt < 2; ++qt) {
        const int lane = fresh_lane();
        Scores<CAP, BIAS, QUICK> sc;
        sc.mul = mul;
        sc.cap2 = cap2;
        sc.slope2 = 0.f;
        sc.hot = hot;
        float ahead = 0.f;
        if (BIAS) {
          const RowRule u = rows[16 * qt + (lane & 15)];
          sc.slope2 = u.slope2;
          ahead = (float)(u.p - (t0 + 4 * (lane >> 4)));
        }
        if (BIAS && late) {
          const float m = -sc.slope2 * (1.f / mul);
#pragma unroll
          for (int kt = 0; kt < 4; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              s[qt][kt][i] = fmaf(m, fabsf(ahead - (float)(16 * kt + i)), s[qt][kt][i]);
        } else {
          sc(s[qt], ahead, !(below | above | (pages != 15u)));
          if (QUICK) hot = sc.hot;
        }
      }
    }
    if (below | above | (pages != 15u)) {
#pragma unroll
      for (int qt = 0; qt < 2; ++qt) {
        const int lane = fresh_lane(), at = t0 + 4 * (lane >> 4);
        const RowRule u = rows[16 * qt + (lane & 15)];
        const int from = u.lo - at, to = u.hi - at;
        if (SINK && sunk) {
          const SinkRule e = sinks[16 * qt + (lane & 15)];
          const int s0 = e.from - at, s1 = e.end - at;
#pragma unroll
          for (int kt = 0; kt < 4; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int k = 16 * kt + i;
              const bool seen = ((k >= from) & (k < to)) | ((k >= s0) & (k < s1));
              s[qt][kt][i] = seen ? s[qt][kt][i] : -INFINITY;
            }
        } else {
          if (below) {
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                s[qt][kt][i] = 16 * kt + i < from ? -INFINITY : s[qt][kt][i];
          }
          if (above) {
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                s[qt][kt][i] = 16 * kt + i >= to ? -INFINITY : s[qt][kt][i];
          }
        }
#pragma unroll
        for (int kt = 0; kt < 4; ++kt)
          if (!(pages >> kt & 1)) s[qt][kt] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      }
    }
    if constexpr (EXACT) {               // (not one operation with the subtraction below)
#pragma unroll
      for (int qt = 0; qt < 2; ++qt)
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) asm("" : "+v"(s[qt][kt]));
    }
    float mt[2];
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
      // (a NaN may be passed over here: its probability makes l NaN)
      float mx = fmaxf(fmaxf(s[qt][0][0], s[qt][0][1]), s[qt][0][2]);
      mx = fmaxf(fmaxf(mx, s[qt][0][3]), s[qt][1][0]);
      mx = fmaxf(fmaxf(mx, s[qt][1][1]), s[qt][1][2]);
      mx = fmaxf(fmaxf(mx, s[qt][1][3]), s[qt][2][0]);
      mx = fmaxf(fmaxf(mx, s[qt][2][1]), s[qt][2][2]);
      mx = fmaxf(fmaxf(mx, s[qt][2][3]), s[qt][3][0]);
      mx = fmaxf(fmaxf(mx, s[qt][3][1]), s[qt][3][2]);
      mx = fmaxf(mx, s[qt][3][3]);
      mx = lanes_max_xor16(lanes_max_xor32(mx));
      mt[qt] = EXACT || CAP ? reference<T>(mx, mx - T::kShift) : mx * c - T::kShift;
    }
    // The reference maximum moves only when a column's grows by more than kLazy, so
    // that most blocks leave O and l as they are.
    if (__ballot(mt[0] > m_run[0] + T::kLazy || mt[1] > m_run[1] + T::kLazy)) {
      if constexpr (!CAP && !EXACT) {
        const float big = fmaxf(mt[0] == -INFINITY ? 0.f : fabsf(mt[0]),
                                mt[1] == -INFINITY ? 0.f : fabsf(mt[1]));
        if (big > kFarScore) *far = 1;
      }
#pragma unroll
      for (int qt = 0; qt < 2; ++qt) {
        const float m_new = fmaxf(m_run[qt], mt[qt]);
        const float alpha =
            __builtin_amdgcn_exp2f(m_run[qt] - (m_new == -INFINITY ? 0.f : m_new));
        m_run[qt] = m_new;
        l_run[qt] *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[qt][dt] *= alpha;
      }
    }
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
      const float mu = m_run[qt] == -INFINITY ? 0.f : m_run[qt];
      float ps[4];
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          s[qt][kt][i] = __builtin_amdgcn_exp2f(CAP ? s[qt][kt][i] - mu
                                                    : fmaf(s[qt][kt][i], c, -mu));
        ps[kt] = (s[qt][kt][0] + s[qt][kt][1]) + (s[qt][kt][2] + s[qt][kt][3]);
      }
      l_run[qt] += (ps[0] + ps[1]) + (ps[2] + ps[3]);
      // k entry 8 G + e is key 32 ks + 4 G + e for e < 4, and 16 further on from 4 on
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
        pb[qt][ks] = u32x4{T::pack2(s[qt][2 * ks][0], s[qt][2 * ks][1]),
                           T::pack2(s[qt][2 * ks][2], s[qt][2 * ks][3]),
                           T::pack2(s[qt][2 * ks + 1][0], s[qt][2 * ks + 1][1]),
                           T::pack2(s[qt][2 * ks + 1][2], s[qt][2 * ks + 1][3])};
    }
  }
};

// SINK: the rows also see the first tokens of their text, before the window.  C8: an
// 8-bit cache.
template <class T, int D, bool CAP, bool BIAS, bool SINK, bool C8>
__device__ __forceinline__ void attend_many(const AttendArgs& a) {
  typedef Wave<T, D, CAP, BIAS, SINK, SINK || C8> W;
  typedef Copy<D, true> CopyK;
  typedef Copy<D, false> CopyV;
  typedef Widen<T, D, true> WidenK;
  typedef Widen<T, D, false> WidenV;
  constexpr int kTile = 64 * D * 2, DT = D / 16;
  __shared__ __attribute__((aligned(16))) unsigned char sk0[kTile], sk1[kTile];
  __shared__ __attribute__((aligned(16))) unsigned char sv0[kTile], sv1[kTile];
  __shared__ int s_list[kListBlocks * 4];   // pool row of each 16-key group, -1 without a page
  __shared__ uint16_t s_scale[C8 ? kListBlocks * 4 : 1];   // their scales: K, and V << 8
  __shared__ int s_lim[kWaves][SINK ? 6 : 4];
  __shared__ int s_missing, s_last, s_odd, s_far;
  __shared__ float s_join[kRows][2];
  __shared__ RowRule s_rule[kRows];
  __shared__ SinkRule s_sink[SINK ? kRows : 1];
  __shared__ int s_see[4];           // the tokens that some row of the tile sees
  __shared__ Part s_part;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int G = a.h_q / a.h_kv, g = blockIdx.x % a.h_kv;
  const int cap = a.pages.cap();
  if (wave == 0) {
    const Part p = find_part<kRows, kRound>(blockIdx.x / a.h_kv, a.seq_start, a.seq_len, a.n_seq,
                                            a.rows, G, a.h_kv, a.rule.window,
                                            SINK ? a.rule.sink : 0, cap, a.from, a.to);
    if (lane == 0) {
      s_part = p;
      s_odd = s_far = 0;
    }
  }
  __syncthreads();
  const Part pt = s_part;
  if (pt.s < 0) return;

  W w;
  w.G = lane >> 4;
  w.r16 = lane & 15;
  const unsigned j0 = pt.tile * kRows;
  const int n_real = min((unsigned)kRows, (unsigned)(pt.q.n * G) - j0);
  // row of q and out of the tile's row r
  auto row_of = [&](int r) SPOT_INLINE {
    const unsigned j = j0 + r, tok = j / (unsigned)G;
    return (size_t)(pt.q.start + tok) * a.h_q + g * G + (j - tok * G);
  };
  w.rows = s_rule + wave * 32;
  w.sinks = s_sink + (SINK ? wave * 32 : 0);
  w.hot = false;
  w.far = &s_far;
  int lo[2], hi[2], from[2], end[2];
#pragma unroll
  for (int qt = 0; qt < 2; ++qt) {
    const int r = wave * 32 + qt * 16 + w.r16;
    const bool real = r < n_real;
    const unsigned j = j0 + (real ? r : 0);
    const int tok = j / (unsigned)G, head = g * G + (j - tok * G);
    lo[qt] = hi[qt] = from[qt] = end[qt] = 0;
    if (real) {
      if constexpr (SINK)
        visible(a.rule, pt.q, pt.s, tok, cap, lo[qt], hi[qt], from[qt], end[qt]);
      else
        visible(a.rule, pt.q, pt.s, tok, cap, lo[qt], hi[qt]);
    }
    const Scores<CAP, BIAS> sc(a.rule, pt.q, tok, head);
    w.mul = sc.mul;
    w.cap2 = sc.cap2;
    if (w.G == 0) s_rule[r] = RowRule{lo[qt], hi[qt], sc.p, sc.slope2};
    if (SINK && w.G == 0) s_sink[r] = SinkRule{from[qt], end[qt]};
    const uint16_t* q = a.q + row_of(real ? r : 0) * D + 8 * w.G;
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) w.qf[ks][qt] = *reinterpret_cast<const u32x4*>(q + ks * 32);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) w.o[qt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    w.m_run[qt] = -INFINITY;
    w.l_run[qt] = 0.f;
  }
  // what some row of the wave sees and what all of them do, and of the workgroup
  constexpr uint32_t kFar = 0x7fffffffu;
  uint32_t lim[4] = {kFar, 0u, 0u, kFar};
#pragma unroll
  for (int qt = 0; qt < 2; ++qt) {
    const bool any = hi[qt] > lo[qt], real = wave * 32 + qt * 16 + w.r16 < n_real;
    lim[0] = min(lim[0], any ? (uint32_t)lo[qt] : kFar);
    lim[1] = max(lim[1], (uint32_t)hi[qt]);
    lim[2] = max(lim[2], real ? (any ? (uint32_t)lo[qt] : kFar) : 0u);
    lim[3] = min(lim[3], real ? (uint32_t)hi[qt] : kFar);
  }
  const int w_lo = (int)wave_min_u(lim[0]), w_hi = (int)wave_max_u(lim[1]);
  const int all_lo = (int)wave_max_u(lim[2]), all_hi = (int)wave_min_u(lim[3]);
  if (lane == 0) {
    s_lim[wave][0] = w_lo;
    s_lim[wave][1] = w_hi;
    s_lim[wave][2] = all_lo;
    s_lim[wave][3] = all_hi;
  }
  int ws_lo = 0, ws_hi = 0;              // sinks that some row of the wave sees
  if constexpr (SINK) {
    const bool any0 = end[0] > from[0], any1 = end[1] > from[1];
    ws_lo = (int)wave_min_u(min(any0 ? (uint32_t)from[0] : kFar, any1 ? (uint32_t)from[1] : kFar));
    ws_hi = (int)wave_max_u((uint32_t)max(end[0], end[1]));
    if (lane == 0) {
      s_lim[wave][4] = ws_lo;
      s_lim[wave][5] = ws_hi;
    }
  }
  __syncthreads();
  int LO = (int)kFar, HI = 0, FLO = 0, FHI = (int)kFar;
  for (int u = 0; u < kWaves; ++u) {
    LO = min(LO, s_lim[u][0]);
    HI = max(HI, s_lim[u][1]);
    FLO = max(FLO, s_lim[u][2]);
    FHI = min(FHI, s_lim[u][3]);
  }
  LO = __builtin_amdgcn_readfirstlane(LO);
  HI = __builtin_amdgcn_readfirstlane(HI);
  FLO = __builtin_amdgcn_readfirstlane(FLO);
  FHI = __builtin_amdgcn_readfirstlane(FHI);
  int SLO = (int)kFar, SHI = 0;
  Blocks bl = {0, 0, LO < HI ? LO / 64 : 0, 0};
  bl.n = LO < HI ? (HI + 63) / 64 - bl.main0 : 0;
  if constexpr (SINK) {
    for (int u = 0; u < kWaves; ++u) {
      SLO = min(SLO, s_lim[u][4]);
      SHI = max(SHI, s_lim[u][5]);
    }
    SLO = __builtin_amdgcn_readfirstlane(SLO);
    SHI = __builtin_amdgcn_readfirstlane(SHI);
    bl = blocks_of(LO, HI, SLO, SHI);
  }
  // blocks of the part by their number among those of the tile; without sinks they are
  // numbered by their place
  const int b0 = SINK ? 0 : bl.main0, b1 = b0 + bl.n;
  auto block = [&](int i) SPOT_INLINE { return SINK ? bl.at(i) : i; };
  if (tid == 0) {                    // (read behind the barriers of the key loop)
    s_see[0] = LO;
    s_see[1] = HI;
    s_see[2] = SLO;
    s_see[3] = SHI;
  }
  const int share = (b1 - b0 + pt.n_split - 1) / pt.n_split;
  const int e0 = min(b0 + pt.split * share, b1), e1 = min(e0 + share, b1);
  const bool second = wave >= kWaves / 2;

  auto go = [&](auto exact) SPOT_INLINE {
    constexpr bool EXACT = decltype(exact)::value;
    for (int c0 = e0; c0 < e1; c0 += kListBlocks) {
      const int nb = min(kListBlocks, e1 - c0);
      __syncthreads();                   // the list and the buffers are done with
      if (tid == 0) s_missing = 0;
      __syncthreads();
      for (int i = tid; i < 4 * nb; i += 64 * kWaves) {
        const int t = SINK ? block(c0 + i / 4) * 64 + i % 4 * kGroupKeys : c0 * 64 + i * kGroupKeys;
        const int r = a.pages.row_below_cap(pt.s, t, g, a.h_kv);
        s_list[i] = r;
        if constexpr (C8) {
          const int at = max(r, 0) / kGroupKeys;
          s_scale[i] = (uint16_t)(a.k_scale[at] | a.v_scale[at] << 8);
        }
        if (r < 0) s_missing = 1;
      }
      __syncthreads();
      const bool missing = __builtin_amdgcn_readfirstlane(s_missing) != 0;
      auto pages_of = [&](int t) SPOT_INLINE -> unsigned {   // bit kt: the keys 16 kt .. are there
        if (!missing) return 15u;
        unsigned m = 0;
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) m |= s_list[4 * t + kt] >= 0 ? 1u << kt : 0u;
        return __builtin_amdgcn_readfirstlane(m);
      };
      // Blocks that some row of the workgroup sees in part only.
      auto edge = [&](int t) SPOT_INLINE {
        const int t0 = block(c0 + t) * 64;
        return t0 < FLO || t0 + 64 > FHI || pages_of(t) != 15u;
      };
      auto active = [&](int t) SPOT_INLINE {
        const int t0 = block(c0 + t) * 64;
        return (t0 < w_hi && t0 + 64 > w_lo) || (SINK && t0 < ws_hi && t0 + 64 > ws_lo);
      };
      auto vector_phase = [&](int t) SPOT_INLINE {
        const int t0 = block(c0 + t) * 64;
        const unsigned pages = pages_of(t);
        w.template softmax<EXACT>(t0, t0 < all_lo, t0 + 64 > all_hi, SINK && t0 < ws_hi, pages);
      };
      // Values that no row sees become zero (they may be infinite or NaN, and meet the
      // probability 0).  So do infinite and NaN elements of the others, which not every
      // row sees: those that see them get theirs after the loop.  Each lane looks at
      // what it copied itself.
      auto mend = [&](int t, unsigned char* v) SPOT_INLINE {
        const int t0 = block(c0 + t) * 64;
        const unsigned pages = pages_of(t);
        const int lane = fresh_lane();
#pragma unroll 1
        for (int u = 0; u < CopyV::N; ++u) {
          const int r = CopyV::row(u, wave, lane), tok = t0 + r;
          u32x4* at = reinterpret_cast<u32x4*>(v + (4 * u + wave) * 1024 + lane * 16);
          if (((tok < LO || tok >= HI) && !(SINK && tok >= SLO && tok < SHI)) ||
              !(pages >> (r >> 4) & 1)) {
            *at = u32x4{0u, 0u, 0u, 0u};
          } else {
            u32x4 x = *at;
            if (odd2<T>(x[0]) || odd2<T>(x[1]) || odd2<T>(x[2]) || odd2<T>(x[3])) {
#pragma unroll
              for (int e = 0; e < 4; ++e) x[e] = clean2<T>(x[e]);
              *at = x;
              s_odd = 1;
            }
          }
        }
      };
      auto matrix_phase = [&](int t, const unsigned char* k, const unsigned char* v) SPOT_INLINE {
        __builtin_amdgcn_s_setprio(0);
        if (t >= 1 && active(t - 1)) w.pv(v);
        if (t < nb && active(t)) w.qk(k);
        __builtin_amdgcn_s_setprio(1);      // the softmax first, where both could go on
      };
      u32x4 raw[WidenK::N];             // codes of keys or of values, by the wave
      auto unseen = [&](int t) SPOT_INLINE {
        const int t0 = block(c0 + t) * 64;
        return [=](int r) SPOT_INLINE {
          const int tok = t0 + r;
          const bool main = (tok >= s_see[0]) & (tok < s_see[1]);
          return !(SINK ? main | ((tok >= s_see[2]) & (tok < s_see[3])) : main);
        };
      };
      if (second) {
        if constexpr (C8) {
          WidenK::load(a.k8, s_list, raw, wave - kWaves / 2);
          WidenK::store(raw, s_scale, sk0, wave - kWaves / 2);
        } else {
          CopyK::issue(a.k, s_list, sk0, wave - kWaves / 2);
          wait_vm();
        }
      }
      lds_barrier();
      auto period = [&](auto parity, int t) SPOT_INLINE {
        constexpr int P = decltype(parity)::value;     // t % 2
        unsigned char* const kcur = P ? sk1 : sk0;
        unsigned char* const knext = P ? sk0 : sk1;
        unsigned char* const vcur = P ? sv1 : sv0;
        unsigned char* const vprev = P ? sv0 : sv1;
        if (!second) {
          matrix_phase(t, kcur, vprev);
          if constexpr (C8) {
            if (t < nb) WidenV::load(a.v8, s_list + 4 * t, raw, wave);
            if (t < nb && active(t)) vector_phase(t);
            if (t < nb) {
              if (edge(t)) {
                if (WidenV::mend(raw, s_list + 4 * t, s_scale + 4 * t, vcur, wave, unseen(t)))
                  s_odd = 1;
              } else {
                WidenV::store(raw, s_scale + 4 * t, vcur, wave);
              }
            }
          } else {
            if (t < nb) CopyV::issue(a.v, s_list + 4 * t, vcur, wave);
            if (t < nb && active(t)) vector_phase(t);
            wait_vm();
            if (t < nb && edge(t)) mend(t, vcur);
          }
          lds_barrier();
        } else {
          if constexpr (C8) {
            if (t + 1 < nb)
              WidenK::load(a.k8, s_list + 4 * (t + 1), raw, wave - kWaves / 2);
            if (t >= 1 && active(t - 1)) vector_phase(t - 1);
            if (t + 1 < nb) WidenK::store(raw, s_scale + 4 * (t + 1), knext, wave - kWaves / 2);
          } else {
            if (t + 1 < nb) CopyK::issue(a.k, s_list + 4 * (t + 1), knext, wave - kWaves / 2);
            if (t >= 1 && active(t - 1)) vector_phase(t - 1);
            wait_vm();
          }
          matrix_phase(t, kcur, vprev);
          lds_barrier();
        }
      };
      for (int t = 0;; t += 2) {
        period(std::integral_constant<int, 0>(), t);
        if (t + 1 > nb) break;
        period(std::integral_constant<int, 1>(), t + 1);
        if (t + 2 > nb) break;
      }
    }
  };
  go(std::false_type());
  // The exact product of a score and its scale less the maximum's, which is rounded, is off by
  // half of that one's last place: beyond 2^24 more than a probability bears.  A tile that has
  // met such scores is gone through once more, each score rounded as the maximum is.  (Of other
  // calls that takes nothing over a 16-bit cache, 1.6 % over an 8-bit one; in the one loop, by a
  // branch of its own or beside the maxima's growth, it took 1 .. 8 %.)
  if constexpr (!CAP) {
    __syncthreads();
    if (__builtin_amdgcn_readfirstlane(s_far)) {
#pragma unroll
      for (int qt = 0; qt < 2; ++qt) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) w.o[qt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        w.m_run[qt] = -INFINITY;
        w.l_run[qt] = 0.f;
      }
      go(std::true_type());
    }
  }

  // What only the end needs is read again here: held, it costs registers in the loop.
  const Part pe = s_part;
  const unsigned j1 = pe.tile * kRows;
  const int n_rows = min((unsigned)kRows, (unsigned)(pe.q.n * G) - j1);
  auto out_row = [&](int r) SPOT_INLINE {
    const unsigned j = j1 + r, tok = j / (unsigned)G;
    return (size_t)(pe.q.start + tok) * a.h_q + g * G + (j - tok * G);
  };
  // lane (G, r16) holds O^T[16 dt + 4 G + i][row r16]
  settle(w.o[0]);
  settle(w.o[1]);
  __syncthreads();
  if (s_odd) {
    // The infinite and NaN elements that mend() left out, for the rows that see their
    // tokens: p v of each, p from the row's score once more.  Rare, and slow (one near the
    // end of a 16000-token prompt makes 4 ms 14).
    // (a run of blocks by their place, or with sinks one by their number)
#pragma unroll 1
    for (int v = SINK ? e0 * 64 : max(e0 * 64, LO); v < (SINK ? e1 * 64 : min(e1 * 64, HI)); ++v) {
      const int tok = SINK ? block(v >> 6) * 64 + (v & 63) : v, t0 = tok & ~63;
      bool edge = t0 < FLO || t0 + 64 > FHI;
      for (int t = t0; t < t0 + 64; t += kGroupKeys)
        edge = edge || a.pages.row_below_cap(pe.s, t, g, a.h_kv) < 0;
      const int at = a.pages.row_below_cap(pe.s, tok & ~(kGroupKeys - 1), g, a.h_kv);
      if (!edge || at < 0) continue;
      const size_t row = ((size_t)at + (tok & (kGroupKeys - 1))) * D;
      float k_scale = 1.f, v_scale = 1.f;
      if constexpr (C8) {
        k_scale = scale8(a.k_scale[at / kGroupKeys]);
        v_scale = scale8(a.v_scale[at / kGroupKeys]);
      }
      u32x2 y[DT];
      bool odd = false;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        if constexpr (C8)
          y[dt] = wide4(T(), *reinterpret_cast<const uint32_t*>(a.v8 + row + dt * 16 + 4 * w.G),
                        v_scale);
        else
          y[dt] = *reinterpret_cast<const u32x2*>(a.v + row + dt * 16 + 4 * w.G);
        odd = odd || odd2<T>(y[dt][0]) || odd2<T>(y[dt][1]);
      }
      if (!__ballot(odd)) continue;
#pragma unroll
      for (int qt = 0; qt < 2; ++qt) {
        const RowRule u = w.rows[16 * qt + w.r16];
        bool seen = tok >= u.lo && tok < u.hi;
        if constexpr (SINK) {
          const SinkRule e = w.sinks[16 * qt + w.r16];
          seen = seen || (tok >= e.from && tok < e.end);
        }
        if (!seen) continue;
        Scores<CAP, BIAS, SINK> sc;
        sc.mul = w.mul;
        sc.cap2 = w.cap2;
        sc.slope2 = u.slope2;
        float dot = 0.f;
#pragma unroll 1
        for (int d = 0; d < D; ++d) {
          const float q = T::one(a.q[out_row(wave * 32 + qt * 16 + w.r16) * D + d]);
          if constexpr (C8)
            dot = fmaf(q, T::lo(wide4(T(), a.k8[row + d], k_scale)[0]), dot);
          else
            dot = fmaf(q, T::one(a.k[row + d]), dot);
        }
        const float p = __builtin_amdgcn_exp2f(sc.one(dot, (float)(u.p - tok)) - w.m_run[qt]);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t h = i & 1 ? y[dt][i >> 1] >> 16 : y[dt][i >> 1] & 0xffffu;
            if ((~h & T::kExponent) == 0u)
              w.o[qt][dt][i] = fmaf(p, T::one((uint16_t)h), w.o[qt][dt][i]);
          }
      }
    }
  }
  const size_t slot0 = (size_t)pe.slot * a.h_kv + (size_t)g * pe.n_split;
#pragma unroll
  for (int qt = 0; qt < 2; ++qt) {
    const float L = lanes_sum_xor16(lanes_sum_xor32(w.l_run[qt])), M = w.m_run[qt];
    const int r = wave * 32 + qt * 16 + w.r16;
    if (r >= n_rows) continue;
    if (pe.n_split > 1) {
      const size_t at = (slot0 + pe.split) * kRows + r;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        float* o = a.ws.o + at * D + dt * 16 + 4 * w.G;
        dec::store_coherent(o, make_float2(w.o[qt][dt][0], w.o[qt][dt][1]));
        dec::store_coherent(o + 2, make_float2(w.o[qt][dt][2], w.o[qt][dt][3]));
      }
      if (w.G == 0) dec::store_coherent(a.ws.ml + at * 2, make_float2(M, L));
    } else {
      const float inv = L == 0.f ? 0.f : 1.f / L;
      const size_t row = out_row(r);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        *reinterpret_cast<u32x2*>(a.out + row * D + dt * 16 + 4 * w.G) =
            u32x2{T::pack2(w.o[qt][dt][0] * inv, w.o[qt][dt][1] * inv),
                  T::pack2(w.o[qt][dt][2] * inv, w.o[qt][dt][3] * inv)};
      if (a.lse && w.G == 0)
        a.lse[row] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * kLn2;
    }
  }
  if (pe.n_split == 1) return;

  dec::wait_stores();
  __syncthreads();
  unsigned* const counter = a.ws.counters + (size_t)pe.counter * a.h_kv + g;
  if (tid == 0)
    s_last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
             (unsigned)(pe.n_split - 1);
  __syncthreads();
  if (!s_last) return;

  // the last part joins them: each row's M and 1 / L, then its output 4 dims a lane
  const int n = pe.n_split;
  const float* const ml = a.ws.ml + slot0 * kRows * 2;
  if (tid < n_rows) {
    float M = -INFINITY, L = 0.f;
    for (int u0 = 0; u0 < n; u0 += 8) {
      float2 t[8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        t[u] = dec::load_coherent(ml + ((size_t)min(u0 + u, n - 1) * kRows + tid) * 2);
      float m = M;
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (t[u].y != 0.f) m = fmaxf(m, t[u].x);
      L *= M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - m);
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (t[u].y != 0.f && u0 + u < n) L = fmaf(t[u].y, __builtin_amdgcn_exp2f(t[u].x - m), L);
      M = m;
    }
    s_join[tid][0] = M;
    s_join[tid][1] = L == 0.f ? 0.f : 1.f / L;
    if (a.lse) a.lse[out_row(tid)] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * kLn2;
  }
  __syncthreads();
  constexpr int Q = D / 4, U = 4;      // quads of a row; rows of a lane in flight
  constexpr int step = 64 * kWaves / Q;
  for (int r0 = tid / Q; r0 < n_rows; r0 += step * U) {
    const int c = tid % Q;
    f32x4 acc[U];
    float M[U], inv[U];
#pragma unroll
    for (int e = 0; e < U; ++e) {
      acc[e] = f32x4{0.f, 0.f, 0.f, 0.f};
      const int r = min(r0 + e * step, n_rows - 1);
      M[e] = s_join[r][0];
      inv[e] = s_join[r][1];
    }
    for (int u0 = 0; u0 < n; u0 += 2) {
      float2 t[2 * U], x[2 * U], y[2 * U];
#pragma unroll
      for (int h = 0; h < 2 * U; ++h) {
        const size_t at =
            (size_t)min(u0 + h / U, n - 1) * kRows + min(r0 + h % U * step, n_rows - 1);
        t[h] = dec::load_coherent(ml + at * 2);
        const float* o = a.ws.o + (slot0 * kRows + at) * D + 4 * c;
        x[h] = dec::load_coherent(o);
        y[h] = dec::load_coherent(o + 2);
      }
#pragma unroll
      for (int h = 0; h < 2 * U; ++h) {
        const int e = h % U;
        if (t[h].y == 0.f || u0 + h / U >= n) continue;
        const float wt = __builtin_amdgcn_exp2f(t[h].x - M[e]);
        acc[e][0] = fmaf(x[h].x, wt, acc[e][0]);
        acc[e][1] = fmaf(x[h].y, wt, acc[e][1]);
        acc[e][2] = fmaf(y[h].x, wt, acc[e][2]);
        acc[e][3] = fmaf(y[h].y, wt, acc[e][3]);
      }
    }
#pragma unroll
    for (int e = 0; e < U; ++e) {
      const int r = r0 + e * step;
      if (r < n_rows)
        *reinterpret_cast<u32x2*>(a.out + out_row(r) * D + 4 * c) =
            u32x2{T::pack2(acc[e][0] * inv[e], acc[e][1] * inv[e]),
                  T::pack2(acc[e][2] * inv[e], acc[e][3] * inv[e])};
    }
  }
  if (tid == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

}  // namespace many
}  // namespace paged
}  // namespace spot
