// The end of the attention of few rows (gfx950): the states of a tile's waves, and of the
// parts of a tile that is split along its keys, become its rows' outputs.
#pragma once

#include "decode_core.h"
#include "paged_core.h"

namespace spot {
namespace paged {
namespace few {

using dec::lanes_max_xor16;
using dec::lanes_max_xor32;
using dec::lanes_sum_xor16;
using dec::lanes_sum_xor32;
using dec::wave_lds_sync;

constexpr int kRows = 16;          // rows of a tile
constexpr int kWaves = 4;
constexpr int kListBlocks = 512;   // blocks whose pages are looked up at once

// Workgroups that run at once, two or (D 64) three on a CU.
template <int D>
constexpr int kFit = D == 64 ? 768 : 512;

// KV: bytes of K and V rows that a wave holds.
template <int D, int KV>
struct Smem {
  struct Merge {
    float ml[kWaves][kRows][2];
    // (rows 16 bytes apart in the banks: 16 of them are written at once)
    alignas(16) float o[kWaves][kRows][D + 4];
  };
  struct Join {
    float weight[kMaxJoin][kRows];  // of part and row: 2^(m - M) / L
  };
  union {
    alignas(16) unsigned char kv[kWaves][KV];
    Merge merge;
    Join join;
  };
  int list[kListBlocks * 4];       // pool row of each 16-key group, -1 without a page
  Part part;
  int last;
};

// o: O^T of the wave's keys, lane (kg, r16) dims 16 dt + 4 kg + i of row r16; m_run the
// rows' reference maximum, l_lane the lane's share of their sums.  g: KV head, G: heads of
// its group, n_rows: rows of the sequence.
template <class T, int D, class S>
__device__ __forceinline__ void finish(S& sm, const AttendArgs& a, const Part& pt, int g, int G,
                                       unsigned n_rows, float m_run, float l_lane,
                                       f32x4 (&o)[D / 16]) {
  constexpr int PL = D / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r16 = lane & 15, kg = lane >> 4;
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

}  // namespace few
}  // namespace paged
}  // namespace spot
