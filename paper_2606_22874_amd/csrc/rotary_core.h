// The rotation of a row's heads (gfx950), shared by the rotations and the appends.
#pragma once

#include "frontend_core.h"
#include "paged_core.h"

namespace spot {
namespace paged {
namespace rot {

constexpr int kThreads = 256;

// The new token's sequence and index in it; s < 0 where the row belongs to none.
struct Row {
  int s, i;
  Seq q;
};
__device__ __forceinline__ Row find_row(const RotaryArgs& a, int row) {
  const int lane = __lane_id();
  Row r;
  r.s = -1;
  for (int base = 0; base < a.n_seq; base += 64) {
    Seq q = {0, 0, 0};
    if (base + lane < a.n_seq) q = sequence(a.seq_start, a.seq_len, base + lane, a.rows);
    const uint64_t hit = __ballot(row >= q.start && row < q.start + q.n);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      r.s = base + l;
      r.q.start = __builtin_amdgcn_readlane(q.start, l);
      r.q.n = __builtin_amdgcn_readlane(q.n, l);
      r.q.len = __builtin_amdgcn_readlane(q.len, l);
      r.i = row - r.q.start;
      return r;
    }
  }
  return r;
}

// One rotated pair.  The FP32 values stay apart from their conversion: fused with it
// (FP16 has such an instruction), results would differ in a last bit between the
// two forms of the kernel.
__device__ __forceinline__ f32x2 turn(float a, float b, float c, float s) {
  f32x2 r = {fmaf(a, c, -(b * s)), fmaf(b, c, a * s)};
  asm("" : "+v"(r[0]), "+v"(r[1]));
  return r;
}

// One row per workgroup.  VEC: 16-byte chunks (every address a multiple of 16 bytes,
// rope_dim a multiple of 16, d of 16); otherwise one pair of elements at a time.
// AXES: a pair's position is that of its axis.  QUERIES: of an append, the queries alone.
template <class T, bool VEC, bool IL, bool AXES, bool QUERIES>
__device__ __forceinline__ void rotate_row(const RotaryArgs& a, int row) {
  __shared__ float s_cos[kMaxPairs], s_sin[kMaxPairs];
  const int tid = threadIdx.x;
  const int half = a.rope_dim / 2;
  const bool append = !QUERIES && a.seq_start != nullptr;
  const int d = a.d;
  const int n_rot = a.h_q + (append ? a.h_kv : 0);
  const int n_vec = n_rot + (append ? a.h_kv : 0);
  auto input = [&](int h) {                  // of vector h: query heads, key heads, value heads
    return h < a.h_q   ? a.q + row * a.q_stride + h * d
           : h < n_rot ? a.k + row * a.k_stride + (h - a.h_q) * d
                       : a.v + row * a.v_stride + (h - n_rot) * d;
  };
  // VEC: two chunks (element offsets): the two halves of eight pairs, or neighbours
  struct Unit {
    int h, ca, cb, p0;
    bool rot;
  };
  auto unit = [&](int w) {
    const int units = d / 16, h = w / units, u = w % units;
    const bool hf = !IL && u < half / 8;
    return Unit{h, hf ? 8 * u : 16 * u, hf ? half + 8 * u : 16 * u + 8, 8 * u,
                IL ? 16 * u < a.rope_dim : hf};
  };
  // A thread's first chunks are on their way while its place and angles are found.  (Not in
  // a rotation with axes, which has no place to find: 12001 x 32 heads of 64, 21.5 us
  // against 20.5.)
  constexpr bool kAhead = VEC && (QUERIES || !AXES);
  u32x4 x = {0u, 0u, 0u, 0u}, y = x;
  auto load = [&](const Unit& t) {
    const uint16_t* in = input(t.h);
    x = *reinterpret_cast<const u32x4*>(in + t.ca);
    y = *reinterpret_cast<const u32x4*>(in + t.cb);
  };
  if (kAhead && tid < n_vec * (d / 16)) load(unit(tid));
  int pos, krow = -1;                        // krow: pool row of the slot, KV head 0
  if (QUERIES) {
    const Row r = find_row(a, row);
    if (r.s < 0) return;
    pos = AXES ? 0 : a.pos ? a.pos[row] : r.q.len - r.q.n + r.i;
  } else if (append) {
    const Row r = find_row(a, row);
    if (r.s < 0) return;
    const int slot = r.q.len - r.q.n + r.i;
    pos = a.pos ? a.pos[row] : slot;
    if (slot >= 0 && slot < a.pages.cap()) {
      krow = a.pages.row(r.s, slot & ~(kGroupKeys - 1), 0, a.h_kv);
      if (krow >= 0) krow += slot & (kGroupKeys - 1);
    }
  } else {
    pos = AXES ? 0 : a.pos[row];
  }
  if (tid < half) {
    float sn, cs;
    if (AXES) pos = a.pos[(int64_t)row * a.n_axes + a.axis[tid]];
    rope_sincos(pos, a.freq.f[tid], sn, cs);
    s_cos[tid] = cs * a.amp;
    s_sin[tid] = a.inverse ? -sn * a.amp : sn * a.amp;
  }
  __syncthreads();
  // output of vector h
  auto place = [&](int h, uint16_t*& out) {
    if (h < a.h_q) {
      out = a.q_out + row * a.out_stride + h * d;
      return true;
    }
    if (krow < 0) return false;
    const int g = h < n_rot ? h - a.h_q : h - n_rot;
    out = (h < n_rot ? a.k_pages : a.v_pages) +
          ((int64_t)krow + (int64_t)g * a.pages.page_size) * d;
    return true;
  };
  if constexpr (VEC) {
    for (int w = tid; w < n_vec * (d / 16); w += kThreads) {
      const Unit t = unit(w);
      uint16_t* out;
      if (!place(t.h, out)) continue;
      if (!kAhead || w != tid) load(t);
      const int ca = t.ca, cb = t.cb, p0 = t.p0;
      const bool rot = t.rot && t.h < n_rot;
      if (rot) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (!IL) {
            const float c0 = s_cos[p0 + 2 * e], s0 = s_sin[p0 + 2 * e];
            const float c1 = s_cos[p0 + 2 * e + 1], s1 = s_sin[p0 + 2 * e + 1];
            const f32x2 t0 = turn(T::lo(x[e]), T::lo(y[e]), c0, s0);
            const f32x2 t1 = turn(T::hi(x[e]), T::hi(y[e]), c1, s1);
            x[e] = T::pack2(t0[0], t1[0]);
            y[e] = T::pack2(t0[1], t1[1]);
          } else {
            const float c0 = s_cos[p0 + e], s0 = s_sin[p0 + e];
            const float c1 = s_cos[p0 + 4 + e], s1 = s_sin[p0 + 4 + e];
            const f32x2 t0 = turn(T::lo(x[e]), T::hi(x[e]), c0, s0);
            const f32x2 t1 = turn(T::lo(y[e]), T::hi(y[e]), c1, s1);
            x[e] = T::pack2(t0[0], t0[1]);
            y[e] = T::pack2(t1[0], t1[1]);
          }
        }
      }
      *reinterpret_cast<u32x4*>(out + ca) = x;
      *reinterpret_cast<u32x4*>(out + cb) = y;
    }
  } else {
    const int pairs = d / 2;
    for (int w = tid; w < n_vec * pairs; w += kThreads) {
      const int h = w / pairs, i = w % pairs;
      const uint16_t* in = input(h);
      uint16_t* out;
      if (!place(h, out)) continue;
      const bool pr = i < half;
      const int ia = pr && !IL ? i : 2 * i, ib = pr && !IL ? i + half : 2 * i + 1;
      const uint16_t xa = in[ia], xb = in[ib];
      if (pr && h < n_rot) {
        const f32x2 t = turn(T::one(xa), T::one(xb), s_cos[i], s_sin[i]);
        out[ia] = T::round(t[0]);
        out[ib] = T::round(t[1]);
      } else {
        out[ia] = xa;
        out[ib] = xb;
      }
    }
  }
}

}  // namespace rot
}  // namespace paged
}  // namespace spot
