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
  const int n_rot = a.h_q + (append ? a.h_kv : 0);
  const int n_vec = n_rot + (append ? a.h_kv : 0);
  const int d = a.d;
  // input and output of vector h: query heads, key heads, value heads
  auto place = [&](int h, const uint16_t*& in, uint16_t*& out) {
    if (h < a.h_q) {
      in = a.q + row * a.q_stride + h * d;
      out = a.q_out + row * a.out_stride + h * d;
      return true;
    }
    if (krow < 0) return false;
    const int g = h < n_rot ? h - a.h_q : h - n_rot;
    in = (h < n_rot ? a.k + row * a.k_stride : a.v + row * a.v_stride) + g * d;
    out = (h < n_rot ? a.k_pages : a.v_pages) + ((int64_t)krow + (int64_t)g * a.pages.page_size) * d;
    return true;
  };
  if constexpr (VEC) {
    const int units = d / 16;                // of two chunks
    for (int w = tid; w < n_vec * units; w += kThreads) {
      const int h = w / units, u = w % units;
      const uint16_t* in;
      uint16_t* out;
      if (!place(h, in, out)) continue;
      // chunks (element offsets): the two halves of eight pairs, or neighbours
      int ca, cb, p0;
      bool rot;
      if (!IL) {
        rot = u < half / 8;
        ca = rot ? 8 * u : 16 * u;
        cb = rot ? half + 8 * u : 16 * u + 8;
        p0 = 8 * u;
      } else {
        ca = 16 * u;
        cb = ca + 8;
        rot = ca < a.rope_dim;
        p0 = 8 * u;
      }
      rot = rot && h < n_rot;
      u32x4 x = *reinterpret_cast<const u32x4*>(in + ca);
      u32x4 y = *reinterpret_cast<const u32x4*>(in + cb);
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
      const uint16_t* in;
      uint16_t* out;
      if (!place(h, in, out)) continue;
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
