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
// The four states meet in LDS; a tile split along its keys leaves (m, l, O) in the
// workspace, and the part that finishes last joins them:
//   M = max m,  L = sum l 2^(m - M),  out = sum O 2^(m - M) / L.
// The keys' bytes bound it: each is read once for all 16 rows (decode, four sequences of
// 131072 tokens, 8 KV heads of 128: 334 us, 6.4 TB/s).  On one short sequence the chain of
// lengths, pages, keys and join does: 700 tokens 10.4 us, two blocks of keys a part.
#include "decode_core.h"
#include "paged_core.h"

namespace spot {
namespace paged {
namespace {

using dec::lanes_max_xor16;
using dec::lanes_max_xor32;
using dec::lanes_sum_xor16;
using dec::lanes_sum_xor32;
using dec::wave_lds_sync;

constexpr int kRows = 16;          // rows of a tile
constexpr int kWaves = 4;
constexpr int kListBlocks = 512;   // blocks whose pages are looked up at once

template <int D>
struct Smem {
  struct Merge {
    float ml[kWaves][kRows][2];
    alignas(16) float o[kWaves][kRows][D];
  };
  struct Join {
    float weight[kMaxJoin][kRows];  // of part and row: 2^(m - M) / L
  };
  union {
    alignas(16) unsigned char kv[kWaves][2 * 16 * D * 2];   // a wave's V rows, then its K rows
    Merge merge;
    Join join;
  };
  int list[kListBlocks * 4];       // pool row of each 16-key group, -1 without a page
  Part part;
  int last;
};

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

template <class T, int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(64 * kWaves, 2) void attend_few_kernel(AttendArgs a) {
  constexpr int RB = D * 2;             // bytes of a row
  constexpr int LR = 64 * 16 / RB;      // rows of a wave's load: 4 or 8
  constexpr int NL = 16 / LR;           // loads of 16 rows
  constexpr int CH = D / 8;             // 16-byte chunks of a row
  constexpr int PL = D / 64;
  __shared__ Smem<D> sm;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r16 = lane & 15, kg = lane >> 4;
  const int G = a.h_q / a.h_kv, g = blockIdx.x % a.h_kv;
  const int cap = a.pages.cap();
  if (wave == 0) {
    const Part p = find_part<kRows, 0>(blockIdx.x / a.h_kv, a.seq_start, a.seq_len, a.n_seq,
                                       a.rows, G, a.h_kv, a.rule.window, cap, a.from, a.to);
    if (lane == 0) sm.part = p;
  }
  __syncthreads();
  const Part pt = sm.part;
  if (pt.s < 0) return;

  // this lane's column: row j of the sequence's matrix
  const unsigned j = pt.tile * kRows + r16, n_rows = pt.q.n * G;
  const bool real = j < n_rows;
  const int tok = real ? j / G : 0, head = g * G + (real ? j - tok * G : 0);
  int lo = 0, hi = 0;
  if (real) visible(a.rule, pt.q, pt.s, tok, cap, lo, hi);
  const Scores<CAP, BIAS> sc(a.rule, pt.q, tok, head);
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

  const int b0 = LO < HI ? LO / 64 : 0, b1 = LO < HI ? (HI + 63) / 64 : 0;
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
      const int t = c0 * 64 + i * kGroupKeys;
      sm.list[i] = t < cap ? a.pages.row(pt.s, t, g, a.h_kv) : -1;
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
      const int t0 = (c0 + n) * 64 + wave * 16;
      odd = false;
      // Values that no row sees never meet the zero probabilities: they may be
      // infinite or NaN.
      if (t0 < LO || t0 + 16 > HI || row_of(n) < 0) {
        const bool page = row_of(n) >= 0;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          const int t = t0 + i * LR + lane / CH;
          if (!page || t < LO || t >= HI) vr[i] = u32x4{0u, 0u, 0u, 0u};
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
      const int t0 = (c0 + n) * 64 + wave * 16;
      f32x4 quad[1] = {s};
      sc(quad, (float)(sc.p - (t0 + 4 * kg)));
      float x[4] = {quad[0][0], quad[0][1], quad[0][2], quad[0][3]};
      if (t0 < FLO || t0 + 16 > FHI || row_of(n) < 0) {
        const bool page = row_of(n) >= 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = t0 + 4 * kg + i;
          if (!page || t < lo || t >= hi) x[i] = -INFINITY;
        }
      }
      float mx = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) - T::kShift;
      mx = lanes_max_xor32(lanes_max_xor16(mx));
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
          const bool sees = t0 + k >= lo && t0 + k < hi;
          const unsigned char* row = vs + k * RB + (kg & 1) * 8;
#pragma unroll
          for (int dt = 0; dt < D / 16; ++dt) {
            const u32x2 y = *reinterpret_cast<const u32x2*>(
                row + (swz_v<D>(k, 2 * dt + (kg >> 1)) << 4));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t h = i & 1 ? y[i >> 1] >> 16 : y[i >> 1] & 0xffffu;
              if (sees && (~h & T::kExponent) == 0u)
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

  settle(o);
  // the four waves' states, then one row per wave and turn
  const float l_row = lanes_sum_xor32(lanes_sum_xor16(l_lane));
  __syncthreads();
  if (kg == 0) {
    sm.merge.ml[wave][r16][0] = m_run;
    sm.merge.ml[wave][r16][1] = l_row;
  }
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt)
    *reinterpret_cast<f32x4*>(&sm.merge.o[wave][r16][16 * dt + 4 * kg]) = o[dt];
  __syncthreads();
  const int n_real = min((unsigned)kRows, n_rows - pt.tile * kRows);
  auto row_of = [&](int c) __attribute__((always_inline)) {   // row of the tile in out
    const unsigned jc = pt.tile * kRows + c, tc = jc / (unsigned)G;
    return (size_t)(pt.q.start + tc) * a.h_q + g * G + (jc - tc * G);
  };
  const size_t slot0 = ((size_t)pt.slot * a.h_kv + (size_t)g * pt.n_split);
  float* const wml = a.ws.ml + (slot0 + pt.split) * kRows * 2;
  float* const wo = a.ws.o + (slot0 + pt.split) * kRows * D;
  for (int c = wave; c < n_real; c += kWaves) {
    float M = -INFINITY, L = 0.f, acc[PL] = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
      if (sm.merge.ml[w][c][1] != 0.f) M = fmaxf(M, sm.merge.ml[w][c][0]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float lw = sm.merge.ml[w][c][1];
      if (lw != 0.f) {
        const float wt = __builtin_amdgcn_exp2f(sm.merge.ml[w][c][0] - M);
        L = fmaf(lw, wt, L);
#pragma unroll
        for (int e = 0; e < PL; ++e) acc[e] = fmaf(sm.merge.o[w][c][PL * lane + e], wt, acc[e]);
      }
    }
    if (pt.n_split > 1) {
      if constexpr (PL == 2)
        dec::store_coherent(wo + c * D + 2 * lane, make_float2(acc[0], acc[1]));
      else
        __hip_atomic_store(wo + c * D + lane, acc[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (lane == 0) dec::store_coherent(wml + c * 2, make_float2(M, L));
    } else {
      const size_t row = row_of(c);
      const float inv = L == 0.f ? 0.f : 1.f / L;
      if constexpr (PL == 2)
        reinterpret_cast<uint32_t*>(a.out + row * D)[lane] = T::pack2(acc[0] * inv, acc[1] * inv);
      else
        a.out[row * D + lane] = T::round(acc[0] * inv);
      if (a.lse && lane == 0)
        a.lse[row] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * kLn2;
    }
  }
  if (pt.n_split == 1) return;

  dec::wait_stores();
  __syncthreads();
  unsigned* const counter = a.ws.counters + (size_t)pt.counter * a.h_kv + g;
  if (tid == 0)
    sm.last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
              (unsigned)(pt.n_split - 1);
  __syncthreads();
  if (!sm.last) return;
  // Row c of 16 threads: each has the (m, l) of every 16th part, then D / 16 dims.  The
  // first parts' O is on its way while the weights are made.
  constexpr int E = D / 32, U = 4;           // float pairs of a thread; parts in flight
  const int c = min(tid >> 4, n_real - 1), k = tid & 15, n = pt.n_split;
  const float* const ml = a.ws.ml + (slot0 * kRows + c) * 2;
  const float* const po = a.ws.o + (slot0 * kRows + c) * D + k * 2 * E;
  float2 v[U][E];
  auto load = [&](int u0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < E; ++e)
        v[u][e] = dec::load_coherent(po + (size_t)min(u0 + u, n - 1) * kRows * D + 2 * e);
  };
  load(0);
  constexpr int P = kMaxJoin / 16;
  float2 t[P];
  float M = -INFINITY, L = 0.f;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    t[i] = make_float2(-INFINITY, 0.f);
    if (k + 16 * i < n) t[i] = dec::load_coherent(ml + (size_t)(k + 16 * i) * kRows * 2);
  }
#pragma unroll
  for (int i = 0; i < P; ++i)
    if (t[i].y != 0.f) M = fmaxf(M, t[i].x);
  M = fmaxf(M, dpp_f<kDppQuadXor1>(M));
  M = fmaxf(M, dpp_f<kDppQuadXor2>(M));
  M = fmaxf(M, dpp_f<kDppHalfMirror>(M));
  M = fmaxf(M, dpp_f<kDppMirror>(M));
  float wt[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    wt[i] = t[i].y != 0.f ? __builtin_amdgcn_exp2f(t[i].x - M) : 0.f;
    if (t[i].y != 0.f) L = fmaf(t[i].y, wt[i], L);
  }
  L += dpp_f<kDppQuadXor1>(L);
  L += dpp_f<kDppQuadXor2>(L);
  L += dpp_f<kDppHalfMirror>(L);
  L += dpp_f<kDppMirror>(L);
  const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
  for (int i = 0; i < P; ++i)
    if (k + 16 * i < n) sm.join.weight[k + 16 * i][tid >> 4] = wt[i] * inv;
  wave_lds_sync();               // a row's threads lie in one wave
  float2 acc[E] = {};
  for (int u0 = 0; u0 < n; u0 += U) {
    if (u0) load(u0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u0 + u >= n) continue;
      const float w = sm.join.weight[u0 + u][tid >> 4];
      if (w == 0.f) continue;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        acc[e].x = fmaf(v[u][e].x, w, acc[e].x);
        acc[e].y = fmaf(v[u][e].y, w, acc[e].y);
      }
    }
  }
  if (tid >> 4 < n_real) {
    const size_t row = row_of(c);
#pragma unroll
    for (int e = 0; e < E; ++e)
      reinterpret_cast<uint32_t*>(a.out + row * D)[k * E + e] = T::pack2(acc[e].x, acc[e].y);
    if (a.lse && k == 0)
      a.lse[row] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * kLn2;
  }
  if (tid == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <class T, int D>
void launch(const AttendArgs& a, dim3 grid, hipStream_t s) {
  const bool cap = a.rule.cap > 0.f, bias = a.rule.slopes != nullptr;
  auto f = cap ? (bias ? attend_few_kernel<T, D, true, true> : attend_few_kernel<T, D, true, false>)
               : (bias ? attend_few_kernel<T, D, false, true>
                       : attend_few_kernel<T, D, false, false>);
  hipLaunchKernelGGL(f, grid, dim3(64 * kWaves), 0, s, a);
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
