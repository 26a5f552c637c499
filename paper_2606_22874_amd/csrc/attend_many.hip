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
// K and V go from memory to LDS 16 bytes a lane (1 KiB a wave instruction), rows
// swizzled by 16-byte chunks against bank conflicts; each of the buffers is a
// variable of its own and the loop is unrolled by two, so that the compiler can tell
// the copies in flight from the reads.
#include <type_traits>

#include "decode_core.h"
#include "paged_core.h"

namespace spot {
namespace paged {
namespace {

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

template <class T, int D, bool CAP, bool BIAS>
struct Wave {
  static constexpr int RB = D * 2, KS = D / 32, DT = D / 16;
  u32x4 qf[KS][2];            // Q^T as the B operand [dims][16 rows]
  f32x4 o[2][DT];
  f32x4 s[2][4];              // scores, then probabilities, of the current block
  u32x4 pb[2][2];             // the probabilities as the B operand
  float m_run[2], l_run[2];
  const RowRule* rows;        // the wave's 32
  float mul, cap2;            // see Scores
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
  __device__ __forceinline__ void softmax(int t0, bool below, bool above, unsigned pages) {
    asm volatile("s_nop 15"
                 : "+v"(s[0][0]), "+v"(s[0][1]), "+v"(s[0][2]), "+v"(s[0][3]), "+v"(s[1][0]),
                   "+v"(s[1][1]), "+v"(s[1][2]), "+v"(s[1][3]));   // see settle()
    // Without a cap a positive scale waits until the exponent (and the bias is taken in
    // its units): an operation less for each score.
    const bool late = !CAP && mul > 1e-6f;
    const float c = late ? mul : 1.f;
    if (CAP || BIAS) {
#pragma unroll
      for (int qt = 0; qt < 2; ++qt) {
        const int lane = fresh_lane();
        Scores<CAP, BIAS> sc;
        sc.mul = mul;
        sc.cap2 = cap2;
        sc.slope2 = 0.f;
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
          sc(s[qt], ahead);
        }
      }
    }
    if (below | above | (pages != 15u)) {
#pragma unroll
      for (int qt = 0; qt < 2; ++qt) {
        const int lane = fresh_lane(), at = t0 + 4 * (lane >> 4);
        const RowRule u = rows[16 * qt + (lane & 15)];
        const int from = u.lo - at, to = u.hi - at;
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
#pragma unroll
        for (int kt = 0; kt < 4; ++kt)
          if (!(pages >> kt & 1)) s[qt][kt] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      }
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
      mt[qt] = lanes_max_xor16(lanes_max_xor32(mx)) * c - T::kShift;
    }
    // The reference maximum moves only when a column's grows by more than kLazy, so
    // that most blocks leave O and l as they are.
    if (__ballot(mt[0] > m_run[0] + T::kLazy || mt[1] > m_run[1] + T::kLazy)) {
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

template <class T, int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(64 * kWaves) void attend_many_kernel(AttendArgs a) {
  typedef Wave<T, D, CAP, BIAS> W;
  typedef Copy<D, true> CopyK;
  typedef Copy<D, false> CopyV;
  constexpr int kTile = 64 * D * 2, DT = D / 16;
  __shared__ __attribute__((aligned(16))) unsigned char sk0[kTile], sk1[kTile];
  __shared__ __attribute__((aligned(16))) unsigned char sv0[kTile], sv1[kTile];
  __shared__ int s_list[kListBlocks * 4];   // pool row of each 16-key group, -1 without a page
  __shared__ int s_lim[kWaves][4];
  __shared__ int s_missing, s_last, s_odd;
  __shared__ float s_join[kRows][2];
  __shared__ RowRule s_rule[kRows];
  __shared__ Part s_part;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int G = a.h_q / a.h_kv, g = blockIdx.x % a.h_kv;
  const int cap = a.pages.cap();
  if (wave == 0) {
    const Part p = find_part<kRows, kRound>(blockIdx.x / a.h_kv, a.seq_start, a.seq_len, a.n_seq,
                                            a.rows, G, a.h_kv, a.rule.window, cap, a.from, a.to);
    if (lane == 0) {
      s_part = p;
      s_odd = 0;
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
  int lo[2], hi[2];
#pragma unroll
  for (int qt = 0; qt < 2; ++qt) {
    const int r = wave * 32 + qt * 16 + w.r16;
    const bool real = r < n_real;
    const unsigned j = j0 + (real ? r : 0);
    const int tok = j / (unsigned)G, head = g * G + (j - tok * G);
    lo[qt] = hi[qt] = 0;
    if (real) visible(a.rule, pt.q, pt.s, tok, cap, lo[qt], hi[qt]);
    const Scores<CAP, BIAS> sc(a.rule, pt.q, tok, head);
    w.mul = sc.mul;
    w.cap2 = sc.cap2;
    if (w.G == 0) s_rule[r] = RowRule{lo[qt], hi[qt], sc.p, sc.slope2};
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
  const int b0 = LO < HI ? LO / 64 : 0, b1 = LO < HI ? (HI + 63) / 64 : 0;
  const int share = (b1 - b0 + pt.n_split - 1) / pt.n_split;
  const int e0 = min(b0 + pt.split * share, b1), e1 = min(e0 + share, b1);
  const bool second = wave >= kWaves / 2;

  for (int c0 = e0; c0 < e1; c0 += kListBlocks) {
    const int nb = min(kListBlocks, e1 - c0);
    __syncthreads();                   // the list and the buffers are done with
    if (tid == 0) s_missing = 0;
    __syncthreads();
    for (int i = tid; i < 4 * nb; i += 64 * kWaves) {
      const int t = c0 * 64 + i * kGroupKeys;
      const int r = t < cap ? a.pages.row(pt.s, t, g, a.h_kv) : -1;
      s_list[i] = r;
      if (r < 0) s_missing = 1;
    }
    __syncthreads();
    const bool missing = __builtin_amdgcn_readfirstlane(s_missing) != 0;
    auto pages_of = [&](int t) SPOT_INLINE -> unsigned {     // bit kt: the keys 16 kt .. are there
      if (!missing) return 15u;
      unsigned m = 0;
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) m |= s_list[4 * t + kt] >= 0 ? 1u << kt : 0u;
      return __builtin_amdgcn_readfirstlane(m);
    };
    // Blocks that some row of the workgroup sees in part only.
    auto edge = [&](int t) SPOT_INLINE {
      const int t0 = (c0 + t) * 64;
      return t0 < FLO || t0 + 64 > FHI || pages_of(t) != 15u;
    };
    auto active = [&](int t) SPOT_INLINE {
      const int t0 = (c0 + t) * 64;
      return t0 < w_hi && t0 + 64 > w_lo;
    };
    auto vector_phase = [&](int t) SPOT_INLINE {
      const int t0 = (c0 + t) * 64;
      const unsigned pages = pages_of(t);
      w.softmax(t0, t0 < all_lo, t0 + 64 > all_hi, pages);
    };
    // Values that no row sees become zero (they may be infinite or NaN, and meet the
    // probability 0).  So do infinite and NaN elements of the others, which not every
    // row sees: those that see them get theirs after the loop.  Each lane looks at
    // what it copied itself.
    auto mend = [&](int t, unsigned char* v) SPOT_INLINE {
      const int t0 = (c0 + t) * 64;
      const unsigned pages = pages_of(t);
      const int lane = fresh_lane();
#pragma unroll 1
      for (int u = 0; u < CopyV::N; ++u) {
        const int r = CopyV::row(u, wave, lane), tok = t0 + r;
        u32x4* at = reinterpret_cast<u32x4*>(v + (4 * u + wave) * 1024 + lane * 16);
        if (tok < LO || tok >= HI || !(pages >> (r >> 4) & 1)) {
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
    if (second) {
      CopyK::issue(a.k, s_list, sk0, wave - kWaves / 2);
      wait_vm();
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
        if (t < nb) CopyV::issue(a.v, s_list + 4 * t, vcur, wave);
        if (t < nb && active(t)) vector_phase(t);
        wait_vm();
        if (t < nb && edge(t)) mend(t, vcur);
        lds_barrier();
      } else {
        if (t + 1 < nb) CopyK::issue(a.k, s_list + 4 * (t + 1), knext, wave - kWaves / 2);
        if (t >= 1 && active(t - 1)) vector_phase(t - 1);
        wait_vm();
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

  // lane (G, r16) holds O^T[16 dt + 4 G + i][row r16]
  settle(w.o[0]);
  settle(w.o[1]);
  __syncthreads();
  if (s_odd) {
    // The infinite and NaN elements that mend() left out, for the rows that see their
    // tokens: p v of each, p from the row's score once more.  Rare, and slow (one near the
    // end of a 16000-token prompt makes 4 ms 14).
#pragma unroll 1
    for (int tok = max(e0 * 64, LO); tok < min(e1 * 64, HI); ++tok) {
      const int t0 = tok & ~63;
      bool edge = t0 < FLO || t0 + 64 > FHI;
      for (int t = t0; t < t0 + 64; t += kGroupKeys)
        edge = edge || t >= cap || a.pages.row(pt.s, t, g, a.h_kv) < 0;
      const int at = a.pages.row(pt.s, tok & ~(kGroupKeys - 1), g, a.h_kv);
      if (!edge || at < 0) continue;
      const size_t row = ((size_t)at + (tok & (kGroupKeys - 1))) * D;
      u32x2 y[DT];
      bool odd = false;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        y[dt] = *reinterpret_cast<const u32x2*>(a.v + row + dt * 16 + 4 * w.G);
        odd = odd || odd2<T>(y[dt][0]) || odd2<T>(y[dt][1]);
      }
      if (!__ballot(odd)) continue;
#pragma unroll
      for (int qt = 0; qt < 2; ++qt) {
        const RowRule u = w.rows[16 * qt + w.r16];
        if (tok < u.lo || tok >= u.hi) continue;
        Scores<CAP, BIAS> sc;
        sc.mul = w.mul;
        sc.cap2 = w.cap2;
        sc.slope2 = u.slope2;
        float dot = 0.f;
#pragma unroll 1
        for (int d = 0; d < D; ++d)
          dot = fmaf(T::one(a.q[row_of(wave * 32 + qt * 16 + w.r16) * D + d]), T::one(a.k[row + d]),
                     dot);
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
  const size_t slot0 = (size_t)pt.slot * a.h_kv + (size_t)g * pt.n_split;
#pragma unroll
  for (int qt = 0; qt < 2; ++qt) {
    const float L = lanes_sum_xor16(lanes_sum_xor32(w.l_run[qt])), M = w.m_run[qt];
    const int r = wave * 32 + qt * 16 + w.r16;
    if (r >= n_real) continue;
    if (pt.n_split > 1) {
      const size_t at = (slot0 + pt.split) * kRows + r;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        float* o = a.ws.o + at * D + dt * 16 + 4 * w.G;
        dec::store_coherent(o, make_float2(w.o[qt][dt][0], w.o[qt][dt][1]));
        dec::store_coherent(o + 2, make_float2(w.o[qt][dt][2], w.o[qt][dt][3]));
      }
      if (w.G == 0) dec::store_coherent(a.ws.ml + at * 2, make_float2(M, L));
    } else {
      const float inv = L == 0.f ? 0.f : 1.f / L;
      const size_t row = row_of(r);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        *reinterpret_cast<u32x2*>(a.out + row * D + dt * 16 + 4 * w.G) =
            u32x2{T::pack2(w.o[qt][dt][0] * inv, w.o[qt][dt][1] * inv),
                  T::pack2(w.o[qt][dt][2] * inv, w.o[qt][dt][3] * inv)};
      if (a.lse && w.G == 0)
        a.lse[row] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * kLn2;
    }
  }
  if (pt.n_split == 1) return;

  dec::wait_stores();
  __syncthreads();
  unsigned* const counter = a.ws.counters + (size_t)pt.counter * a.h_kv + g;
  if (tid == 0)
    s_last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
             (unsigned)(pt.n_split - 1);
  __syncthreads();
  if (!s_last) return;

  // the last part joins them: each row's M and 1 / L, then its output 4 dims a lane
  const int n = pt.n_split;
  const float* const ml = a.ws.ml + slot0 * kRows * 2;
  if (tid < n_real) {
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
    if (a.lse) a.lse[row_of(tid)] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * kLn2;
  }
  __syncthreads();
  constexpr int Q = D / 4, U = 4;      // quads of a row; rows of a lane in flight
  constexpr int step = 64 * kWaves / Q;
  for (int r0 = tid / Q; r0 < n_real; r0 += step * U) {
    const int c = tid % Q;
    f32x4 acc[U];
    float M[U], inv[U];
#pragma unroll
    for (int e = 0; e < U; ++e) {
      acc[e] = f32x4{0.f, 0.f, 0.f, 0.f};
      const int r = min(r0 + e * step, n_real - 1);
      M[e] = s_join[r][0];
      inv[e] = s_join[r][1];
    }
    for (int u0 = 0; u0 < n; u0 += 2) {
      float2 t[2 * U], x[2 * U], y[2 * U];
#pragma unroll
      for (int h = 0; h < 2 * U; ++h) {
        const size_t at =
            (size_t)min(u0 + h / U, n - 1) * kRows + min(r0 + h % U * step, n_real - 1);
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
      if (r < n_real)
        *reinterpret_cast<u32x2*>(a.out + row_of(r) * D + 4 * c) =
            u32x2{T::pack2(acc[e][0] * inv[e], acc[e][1] * inv[e]),
                  T::pack2(acc[e][2] * inv[e], acc[e][3] * inv[e])};
    }
  }
  if (tid == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <class T, int D>
void launch(const AttendArgs& a, dim3 grid, hipStream_t s) {
  // the plain form takes maxima before it scales: it needs a positive scale
  const bool cap = a.rule.cap > 0.f;
  const bool bias = a.rule.slopes || (!cap && !(a.rule.scale * kLog2e > 1e-6f));
  auto f = cap ? (bias ? attend_many_kernel<T, D, true, true> : attend_many_kernel<T, D, true, false>)
               : (bias ? attend_many_kernel<T, D, false, true>
                       : attend_many_kernel<T, D, false, false>);
  hipLaunchKernelGGL(f, grid, dim3(64 * kWaves), 0, s, a);
}

}  // namespace

hipError_t launch_attend_many(AttendArgs a, int dtype, int d, void* ws, hipStream_t s) {
  a.ws.counters = static_cast<unsigned*>(ws);
  a.ws.ml = reinterpret_cast<float*>(static_cast<char*>(ws) + kCounterBytes);
  a.ws.o = a.ws.ml + (size_t)kMaxParts * kRows * 2;
  const int64_t groups = attend_grid<kRows>(a);
  if (!launchable(groups, 64 * kWaves)) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)groups);
  if (dtype == SPOT_DTYPE_BF16)
    d == 128 ? launch<Bf16, 128>(a, grid, s) : launch<Bf16, 64>(a, grid, s);
  else
    d == 128 ? launch<Fp16, 128>(a, grid, s) : launch<Fp16, 64>(a, grid, s);
  return hipGetLastError();
}

size_t attend_many_workspace(int d) {
  return kCounterBytes + (size_t)kMaxParts * kRows * (2 + d) * sizeof(float);
}

}  // namespace paged
}  // namespace spot
