// Attention of few rows over a paged cache (gfx950): decode steps, a handful of
// new tokens a sequence.
//
// One workgroup of 4 waves takes one part of a tile of 16 rows (new tokens x the
// query heads that share a KV head): a run of 64-key blocks.  Wave w owns keys
// [16w, 16w + 16) of every block with its own running maximum m and sum l, and
//   S^T = K Q^T       D/32 MFMAs 16x16x32, K rows as the A operand by way of LDS
//                     (so that the loads stay coalesced), Q^T held as B;
//   x = cap, bias, mask of S^T;  p = 2^(x - m);  l += p
//   O^T += V^T P^T    D/16 MFMAs 16x16x16, P^T straight from the accumulators,
//                     V^T through the transposing LDS read.
// P is rounded to the element type (a matrix instruction has one for both operands); l is
// summed before that, in FP32.
// The four states meet in LDS; a tile split along its keys leaves (m, l, O) in the
// workspace, and the part that finishes last joins them:
//   M = max m,  L = sum l 2^(m - M),  out = sum O 2^(m - M) / L.
// The keys' bytes bound it: each is read once for all 16 rows (decode, four sequences of
// 131072 tokens, 8 KV heads of 128: 334 us, 6.4 TB/s).  On one short sequence the chain of
// lengths, pages, keys and join does: 700 tokens 9.2 us, two blocks of keys a part.
// With sinks a tile goes through two runs of blocks, numbered through (paged_map.h); its
// masks look at both.  Eight sequences of 20000 .. 60000 tokens, window 4096 and 4 sinks: 31
// us, 4.3 TB/s.
#include "attend_join.h"

namespace spot {
namespace paged {
namespace {

using namespace few;

// Physical 16-byte chunk of logical chunk c of row r: K is read 16 rows x one chunk
// at a time, V 8 bytes from each of 8 rows at two neighbouring chunks.
template <int D>
__device__ __forceinline__ int swz_k(int r, int c) {
  return c ^ (r & (D / 8 - 1));
}
template <int D>
__device__ __forceinline__ int swz_v(int r, int c) {
  return D == 128 ? c ^ ((r & 7) << 1) : c ^ (((r >> 1) & 3) << 1);
}

// SINK: the rows also see the first tokens of their text, before the window.
template <class T, int D, bool CAP, bool BIAS, bool SINK>
__device__ __forceinline__ void attend_few(const AttendArgs& a) {
  constexpr int RB = D * 2;             // bytes of a row
  constexpr int LR = 64 * 16 / RB;      // rows of a wave's load: 4 or 8
  constexpr int NL = 16 / LR;           // loads of 16 rows
  constexpr int CH = D / 8;             // 16-byte chunks of a row
  __shared__ Smem<D, 2 * 16 * D * 2> sm;   // kv: a wave's V rows, then its K rows
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r16 = lane & 15, kg = lane >> 4;
  const int G = a.h_q / a.h_kv, g = blockIdx.x % a.h_kv;
  const int cap = a.pages.cap();
  if (wave == 0) {
    const Part p = find_part<kRows, 0, SINK ? kFit<D> : 0>(
        blockIdx.x / a.h_kv, a.seq_start, a.seq_len, a.n_seq, a.rows, G, a.h_kv, a.rule.window,
        SINK ? a.rule.sink : 0, cap, a.from, a.to);
    if (lane == 0) sm.part = p;
  }
  __syncthreads();
  const Part pt = sm.part;
  if (pt.s < 0) return;

  // this lane's column: row j of the sequence's matrix
  const unsigned j = pt.tile * kRows + r16, n_rows = pt.q.n * G;
  const bool real = j < n_rows;
  const int tok = real ? j / G : 0, head = g * G + (real ? j - tok * G : 0);
  int lo = 0, hi = 0, from = 0, end = 0;
  if (real) {
    if constexpr (SINK)
      visible(a.rule, pt.q, pt.s, tok, cap, lo, hi, from, end);
    else
      visible(a.rule, pt.q, pt.s, tok, cap, lo, hi);
  }
  // (with sinks, comparisons are joined without branches: of a select behind short-circuit
  // ones and a uniform branch the compiler, ROCm 7.2, has kept the uniform part only)
  auto sees = [&](int t) { return ((t >= lo) & (t < hi)) | ((t >= from) & (t < end)); };
  Scores<CAP, BIAS, SINK> sc(a.rule, pt.q, tok, head);
  u32x4 qf[D / 32];
  const size_t qrow = (size_t)(pt.q.start + tok) * a.h_q + head;
#pragma unroll
  for (int kc = 0; kc < D / 32; ++kc) {
    qf[kc] = u32x4{0u, 0u, 0u, 0u};
    if (real) qf[kc] = *reinterpret_cast<const u32x4*>(a.q + qrow * D + 32 * kc + 8 * kg);
  }
  // what some row sees, and what all of them do
  const bool any = hi > lo;
  const int LO = (int)wave_min_u(any ? (uint32_t)lo : 0x7fffffffu);
  const int HI = (int)wave_max_u((uint32_t)hi);
  const int FLO = (int)wave_max_u(real ? (uint32_t)(any ? lo : 0x7fffffff) : 0u);
  const int FHI = (int)wave_min_u(real ? (uint32_t)hi : 0x7fffffffu);

  int SLO = 0, SHI = 0;                 // of the sinks
  Blocks bl = {0, 0, LO < HI ? LO / 64 : 0, 0};
  bl.n = LO < HI ? (HI + 63) / 64 - bl.main0 : 0;
  if constexpr (SINK) {
    SLO = (int)wave_min_u(end > from ? (uint32_t)from : 0x7fffffffu);
    SHI = (int)wave_max_u((uint32_t)end);
    bl = blocks_of(LO, HI, SLO, SHI);
  }
  // blocks of the part by their number among those of the tile; 16-bit calls without
  // sinks number them by their place
  const int b0 = SINK ? 0 : bl.main0, b1 = b0 + bl.n;
  auto block = [&](int i) { return SINK ? bl.at(i) : i; };
  const int share = (b1 - b0 + pt.n_split - 1) / pt.n_split;
  const int e0 = min(b0 + pt.split * share, b1), e1 = min(e0 + share, b1);

  unsigned char* vs = sm.kv[wave];
  unsigned char* ks = vs + 16 * RB;
  u32x4 krA[NL], vrA[NL], krB[NL], vrB[NL];
  f32x4 o[D / 16];
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_lane = 0.f;

  for (int c0 = e0; c0 < e1; c0 += kListBlocks) {
    const int nb = min(kListBlocks, e1 - c0);
    if (c0 > e0) __syncthreads();       // the list is done with
    for (int i = tid; i < 4 * nb; i += 64 * kWaves) {
      const int t = SINK ? block(c0 + i / 4) * 64 + i % 4 * kGroupKeys : c0 * 64 + i * kGroupKeys;
      sm.list[i] = a.pages.row_below_cap(pt.s, t, g, a.h_kv);
    }
    __syncthreads();
    auto row_of = [&](int n) { return __builtin_amdgcn_readfirstlane(sm.list[4 * n + wave]); };
    auto load = [&](u32x4(&kr)[NL], u32x4(&vr)[NL], int n) {
      const size_t at = (size_t)max(row_of(n), 0) * D + lane * 8;
#pragma unroll
      for (int i = 0; i < NL; ++i)
        kr[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.k + at + i * 512));
#pragma unroll
      for (int i = 0; i < NL; ++i)
        vr[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.v + at + i * 512));
    };
    // Blocks that some row sees in part: the probability 0 of a token that a row does
    // not see must not meet an infinite or NaN value that another row does see (odd).
    bool odd = false;
    auto front = [&](u32x4(&kr)[NL], u32x4(&vr)[NL], int n) -> f32x4 {
      const int t0 = block(c0 + n) * 64 + wave * 16;
      odd = false;
      // Values that no row sees never meet the zero probabilities: they may be
      // infinite or NaN.
      if (t0 < LO || t0 + 16 > HI || row_of(n) < 0) {
        const bool page = row_of(n) >= 0;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          const int t = t0 + i * LR + lane / CH;
          if constexpr (SINK) {
            const bool seen = page & (((t >= LO) & (t < HI)) | ((t >= SLO) & (t < SHI)));
#pragma unroll
            for (int e = 0; e < 4; ++e) vr[i][e] = seen ? vr[i][e] : 0u;
          } else {
            if (!page || t < LO || t >= HI) vr[i] = u32x4{0u, 0u, 0u, 0u};
          }
        }
      }
      if (t0 < FLO || t0 + 16 > FHI) {
#pragma unroll
        for (int i = 0; i < NL; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) odd = odd || odd2<T>(vr[i][e]);
        odd = __ballot(odd) != 0ull;
      }
      wave_lds_sync();  // this wave's reads of the previous rows are issued
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int r = LR * i + lane / CH, c = lane % CH;
        *reinterpret_cast<u32x4*>(ks + r * RB + (swz_k<D>(r, c) << 4)) = kr[i];
        *reinterpret_cast<u32x4*>(vs + r * RB + (swz_v<D>(r, c) << 4)) = vr[i];
      }
      wave_lds_sync();
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kc = 0; kc < D / 32; ++kc)
        s = T::mfma32(*reinterpret_cast<const u32x4*>(ks + r16 * RB +
                                                      (swz_k<D>(r16, 4 * kc + kg) << 4)),
                      qf[kc], s);
      settle(s);
      return s;
    };
    auto back = [&](int n, f32x4 s) {
      const int t0 = block(c0 + n) * 64 + wave * 16;
      f32x4 quad[1] = {s};
      const bool part = t0 < FLO || t0 + 16 > FHI || row_of(n) < 0;
      sc(quad, (float)(sc.p - (t0 + 4 * kg)), !part);
      float x[4] = {quad[0][0], quad[0][1], quad[0][2], quad[0][3]};
      if (part) {
        const bool page = row_of(n) >= 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = t0 + 4 * kg + i;
          if constexpr (SINK)
            x[i] = (page & sees(t)) ? x[i] : -INFINITY;
          else if (!page || t < lo || t >= hi)
            x[i] = -INFINITY;
        }
      }
      float mx = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
      mx = lanes_max_xor32(lanes_max_xor16(mx));
      mx = reference<T>(mx, mx - T::kShift);
      if (__ballot(mx > m_run + T::kLazy) != 0ull) {
        const float m_new = fmaxf(m_run, mx);
        const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
        l_lane *= alpha;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) o[dt] *= alpha;
        m_run = m_new;
      }
      float p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        p[i] = x[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x[i] - m_run);
      l_lane += (p[0] + p[1]) + (p[2] + p[3]);
      const s16x4 pb =
          __builtin_bit_cast(s16x4, u32x2{T::pack2(p[0], p[1]), T::pack2(p[2], p[3])});
      const int vr_row = 4 * kg + (r16 >> 2);
      const unsigned char* vrow = vs + vr_row * RB + (r16 & 1) * 8;
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) {
        const int c = 2 * dt + ((r16 & 3) >> 1);
        s16x4 f = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)(vrow + (swz_v<D>(vr_row, c) << 4)));
        if (odd) {
          const u32x2 y = __builtin_bit_cast(u32x2, f);
          f = __builtin_bit_cast(s16x4, u32x2{clean2<T>(y[0]), clean2<T>(y[1])});
        }
        o[dt] = T::mfma16(f, pb, o[dt]);
      }
      if (odd) {   // the elements left out, for the rows that see their tokens
        settle(o);
#pragma unroll 1
        for (int k = 0; k < 16; ++k) {
          const float pk = __shfl(k & 2 ? (k & 1 ? p[3] : p[2]) : (k & 1 ? p[1] : p[0]),
                                  (k >> 2) * 16 + r16);
          const bool seen = SINK ? sees(t0 + k) : t0 + k >= lo && t0 + k < hi;
          const unsigned char* row = vs + k * RB + (kg & 1) * 8;
#pragma unroll
          for (int dt = 0; dt < D / 16; ++dt) {
            const u32x2 y = *reinterpret_cast<const u32x2*>(
                row + (swz_v<D>(k, 2 * dt + (kg >> 1)) << 4));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t h = i & 1 ? y[i >> 1] >> 16 : y[i >> 1] & 0xffffu;
              if (seen && (~h & T::kExponent) == 0u)
                o[dt][i] = fmaf(pk, T::one((uint16_t)h), o[dt][i]);
            }
          }
        }
      }
    };
    // Two register stages: blocks n + 1 and n + 2 are loading while n is computed
    // (prefetches without a condition, so that each wait counts its stage only).
    int n = 0;
    if (nb >= 4) {
      load(krA, vrA, 0);
      load(krB, vrB, 1);
      for (; n + 3 < nb; n += 2) {
        f32x4 s = front(krA, vrA, n);
        load(krA, vrA, n + 2);
        back(n, s);
        s = front(krB, vrB, n + 1);
        load(krB, vrB, n + 3);
        back(n + 1, s);
      }
      f32x4 s = front(krA, vrA, n);
      if (n + 2 < nb) load(krA, vrA, n + 2);
      back(n, s);
      s = front(krB, vrB, n + 1);
      back(n + 1, s);
      if (n + 2 < nb) {
        s = front(krA, vrA, n + 2);
        back(n + 2, s);
      }
    } else {
      load(krA, vrA, 0);
      if (nb > 1) load(krB, vrB, 1);
      f32x4 s = front(krA, vrA, 0);
      if (nb > 2) load(krA, vrA, 2);
      back(0, s);
      if (nb > 1) {
        s = front(krB, vrB, 1);
        back(1, s);
      }
      if (nb > 2) {
        s = front(krA, vrA, 2);
        back(2, s);
      }
    }
  }

  finish<T, D>(sm, a, pt, g, G, n_rows, m_run, l_lane, o);
}

template <class T, int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(64 * kWaves, 2) void attend_few_kernel(AttendArgs a) {
  attend_few<T, D, CAP, BIAS, false>(a);
}
template <class T, int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(64 * kWaves, 2) void sinks_few_kernel(AttendArgs a) {
  attend_few<T, D, CAP, BIAS, true>(a);
}

template <class T, int D>
void launch(const AttendArgs& a, dim3 grid, hipStream_t s) {
  const bool cap = a.rule.cap > 0.f, bias = a.rule.slopes != nullptr;
  auto f = cap ? (bias ? attend_few_kernel<T, D, true, true> : attend_few_kernel<T, D, true, false>)
               : (bias ? attend_few_kernel<T, D, false, true>
                       : attend_few_kernel<T, D, false, false>);
  auto g = cap ? (bias ? sinks_few_kernel<T, D, true, true> : sinks_few_kernel<T, D, true, false>)
               : (bias ? sinks_few_kernel<T, D, false, true>
                       : sinks_few_kernel<T, D, false, false>);
  hipLaunchKernelGGL(a.rule.sink > 0 ? g : f, grid, dim3(64 * kWaves), 0, s, a);
}

}  // namespace

hipError_t launch_attend_few(AttendArgs a, int dtype, int d, void* ws, hipStream_t s) {
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

size_t attend_few_workspace(int d) {
  return kCounterBytes + (size_t)kMaxParts * kRows * (2 + d) * sizeof(float);
}

}  // namespace paged
}  // namespace spot
