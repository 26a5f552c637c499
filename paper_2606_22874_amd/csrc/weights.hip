// Attention weight that each cached token received from a call's new tokens
// (gfx950): acc_out[s, g, t] = decay acc[s, g, t] + sum over the rows (new tokens x
// the heads of KV head g) of e^(x - lse), with the scores x and lse of the attention.
//
// One workgroup of 4 waves per 256 keys of a KV head, 64 keys a wave, held in
// registers as the A operand of S^T = K Q^T; the rows pass by 16 at a time as the B
// operand.  A key belongs to one wave, so there are no atomics and the order of the
// sums is fixed.
#include "decode_core.h"
#include "paged_core.h"

namespace spot {
namespace paged {
namespace {

constexpr int kKeys = 256;      // of a workgroup
constexpr int kWaves = 4;

template <class T, int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(64 * kWaves) void weights_kernel(WeightArgs a) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r16 = lane & 15, kg = lane >> 4;
  const int G = a.h_q / a.h_kv, cap = a.pages.cap();
  const int g = blockIdx.x % a.h_kv, s = blockIdx.y;
  const int t0 = (blockIdx.x / a.h_kv) * kKeys + wave * 64;
  if (t0 >= cap) return;
  const Seq q = sequence(a.seq_start, a.seq_len, s, a.rows);
  const int end = min(q.len, cap);

  float sum[4][4] = {};
  if (t0 < end && q.n > 0) {
    u32x4 kf[4][D / 32];
    bool page[4];
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) {
      const int t = t0 + 16 * kt;
      const int row = t < cap ? a.pages.row(s, t, g, a.h_kv) : -1;
      page[kt] = row >= 0;
      const uint16_t* p = a.k + ((int64_t)max(row, 0) + r16) * D + 8 * kg;
#pragma unroll
      for (int kc = 0; kc < D / 32; ++kc)
        kf[kt][kc] = *reinterpret_cast<const u32x4*>(p + 32 * kc);
    }
    // the new tokens that see some of these keys
    const int p0 = q.len - q.n;
    int i0 = max(0, t0 - p0), i1 = q.n;
    if (a.rule.prefix && a.rule.prefix[s] > t0) i0 = 0;
    if (a.rule.window > 0)
      i1 = (int)min((int64_t)i1, max((int64_t)t0 + 63 + a.rule.window - p0, (int64_t)0));
    const int64_t j1 = (int64_t)i1 * G;
    for (int64_t j0 = (int64_t)i0 * G; j0 < j1; j0 += 16) {
      const int64_t j = j0 + r16;
      const bool real = j < j1;
      const int tok = real ? (int)(j / G) : 0, head = g * G + (real ? (int)(j % G) : 0);
      const size_t row = (size_t)(q.start + tok) * a.h_q + head;
      int lo = 0, hi = 0;
      if (real) visible(a.rule, q, s, tok, cap, lo, hi);
      const float lse = real ? a.lse[row] : -INFINITY;
      const Scores<CAP, BIAS> sc(a.rule, q, tok, head);
      f32x4 x[4];
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) x[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kc = 0; kc < D / 32; ++kc) {
        const u32x4 qf =
            *reinterpret_cast<const u32x4*>(a.q + row * D + 32 * kc + 8 * kg);
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) x[kt] = T::mfma32(kf[kt][kc], qf, x[kt]);
      }
      settle(x);
      sc(x, (float)(sc.p - (t0 + 4 * kg)));
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = t0 + 16 * kt + 4 * kg + i;
          const float w = __builtin_amdgcn_exp2f(x[kt][i] - lse * kLog2e);
          sum[kt][i] += page[kt] && t >= lo && t < hi && lse != -INFINITY ? w : 0.f;
        }
    }
  }
  // the 16 columns of a key
#pragma unroll
  for (int kt = 0; kt < 4; ++kt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v = sum[kt][i];
      v += dpp_f<kDppQuadXor1>(v);
      v += dpp_f<kDppQuadXor2>(v);
      v += dpp_f<kDppHalfMirror>(v);
      v += dpp_f<kDppMirror>(v);
      sum[kt][i] = v;
    }
  if (r16 == 0) {
    const int64_t base = ((int64_t)s * a.h_kv + g) * cap;
#pragma unroll
    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = t0 + 16 * kt + 4 * kg + i;
        if (t < cap)
          a.acc_out[base + t] = a.acc ? fmaf(a.decay, a.acc[base + t], sum[kt][i]) : sum[kt][i];
      }
  }
}

template <class T, int D>
void launch(const WeightArgs& a, dim3 grid, hipStream_t s) {
  const bool cap = a.rule.cap > 0.f, bias = a.rule.slopes != nullptr;
  auto f = cap ? (bias ? weights_kernel<T, D, true, true> : weights_kernel<T, D, true, false>)
               : (bias ? weights_kernel<T, D, false, true> : weights_kernel<T, D, false, false>);
  hipLaunchKernelGGL(f, grid, dim3(64 * kWaves), 0, s, a);
}

}  // namespace

hipError_t launch_weights(const WeightArgs& a, int dtype, int d, hipStream_t s) {
  const int cap = a.pages.cap();
  if (cap == 0) return hipSuccess;
  const dim3 grid((unsigned)((cap + kKeys - 1) / kKeys) * (unsigned)a.h_kv, (unsigned)a.n_seq);
  if (dtype == SPOT_DTYPE_BF16)
    d == 128 ? launch<Bf16, 128>(a, grid, s) : launch<Bf16, 64>(a, grid, s);
  else
    d == 128 ? launch<Fp16, 128>(a, grid, s) : launch<Fp16, 64>(a, grid, s);
  return hipGetLastError();
}

}  // namespace paged
}  // namespace spot
