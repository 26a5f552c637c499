// Attention weight that each cached token received from a call's new tokens
// (gfx950): acc_out[s, g, t] = decay acc[s, g, t] + sum over the rows (new tokens x
// the heads of KV head g) of e^(x - lse), with the scores x and lse of the attention.
//
// A wave holds 32 or 128 keys of a KV head in registers as the A operand of
// S^T = K Q^T, and the rows pass by 16 at a time as the B operand, the next 16 on their
// way from memory meanwhile.  The keys come by way of LDS, so that their loads are
// coalesced.  Few rows (a decode step, bound by the keys' bytes): the 4 waves of a
// workgroup take 128 keys between them (4.9 TB/s over four sequences of 20000 .. 32768
// keys, 41 us).  Many rows (bound by exponentials and matrix instructions): they take
// the same 128 keys and a quarter of the rows each (64 tokens of 64 heads over 32768
// keys: 60 us, 574 TFLOP/s).  A key belongs to one workgroup, so there are no atomics
// and the order of the sums is fixed.
#include "decode_core.h"
#include "paged_core.h"

namespace spot {
namespace paged {
namespace {

constexpr int kWaves = 4;
constexpr int kFewKeys = 32;       // keys of a wave, few rows (four sequences of 20000 ..
                                   // 32768 keys, 41.0 us; with 64 keys, half the
                                   // workgroups on a CU, 45.7)
typedef __attribute__((address_space(3))) void lds_void;

template <class T, int D, bool CAP, bool BIAS, bool ROWS>
__global__ __launch_bounds__(64 * kWaves, 2) void weights_kernel(WeightArgs a) {
  constexpr int RB = D * 2, CH = D / 8;        // bytes and 16-byte chunks of a row
  constexpr int R = 1024 / RB;                 // rows of a copy instruction
  constexpr int NK = ROWS ? 8 : kFewKeys / 16, kKeys = 16 * NK;   // groups of 16 keys of a wave
  constexpr int kTile = kKeys * RB;
  __shared__ __attribute__((aligned(16))) unsigned char s_k[(ROWS ? 1 : kWaves) * kTile];
  __shared__ float s_sum[ROWS ? kWaves : 1][kKeys];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r16 = lane & 15, kg = lane >> 4;
  const int G = a.h_q / a.h_kv, cap = a.pages.room();
  const int g = blockIdx.x % a.h_kv, s = blockIdx.y;
  const int t0 = (ROWS ? blockIdx.x / a.h_kv : (blockIdx.x / a.h_kv) * kWaves + wave) * kKeys;
  const Seq q = sequence(a.seq_start, a.seq_len, s, a.rows);
  const int end = min(q.len, a.pages.cap());

  // lane (kg, r16) ends with the sums of keys 16 kt + 4 kg + i: it keeps those of
  // 4 (kt % 4) + i = r16, one key a lane and 64 (or 32: r16 < 8)
  constexpr int NX = NK < 4 ? NK : 4;
  const int mine_key = 16 * (r16 >> 2) + 4 * kg + (r16 & 3);
  const int64_t base = ((int64_t)s * a.h_kv + g) * cap;
  const bool mine_real = !ROWS && mine_key < kKeys && t0 + mine_key < cap;
  // what the key has already, on its way beside the keys (in place it is this lane's)
  const float had = a.acc && mine_real ? a.acc[base + t0 + mine_key] : 0.f;

  float sum[NK][4] = {};
  if (t0 < end && q.n > 0) {
    // the keys; bit kt of pages: those from 16 kt on are there
    unsigned char* const ks = s_k + (ROWS ? 0 : wave * kTile);
    unsigned pages = 0;
    int at[NK];
#pragma unroll
    for (int kt = 0; kt < NK; ++kt) {
      const int t = t0 + 16 * kt;
      at[kt] = t < cap ? a.pages.row(s, t, g, a.h_kv) : -1;
      pages |= at[kt] >= 0 ? 1u << kt : 0u;
    }
#pragma unroll
    for (int u = 0; u < kKeys / R / (ROWS ? kWaves : 1); ++u) {
      const int i = ROWS ? kWaves * u + wave : u;        // rows R i ..
      const int r = R * i + lane / CH, c = (lane % CH) ^ (r & (CH - 1));
      int from = at[0];
#pragma unroll
      for (int kt = 1; kt < NK; ++kt) from = R * i / 16 == kt ? at[kt] : from;
      const uint16_t* src = a.k + (int64_t)__builtin_amdgcn_readfirstlane(max(from, 0)) * D;
      __builtin_amdgcn_global_load_lds(src + (uint32_t)((r & 15) * D + c * 8),
                                       (lds_void*)(ks + i * 1024), 16, 0, 0);
    }
    // the new tokens that see some of these keys
    const int p0 = q.len - q.n;
    int i0 = min(max(0, t0 - p0), q.n), i1 = q.n;
    if (a.rule.prefix && a.rule.prefix[s] > t0) i0 = 0;
    if (a.rule.window > 0)
      i1 = (int)min((int64_t)i1, max((int64_t)t0 + kKeys - 1 + a.rule.window - p0, (int64_t)0));
    const int end_row = i1 * G;
    // Rows of a step: this lane's is j = i0 G + 16 (step of the wave) + r16; token and
    // head advance without a division.
    constexpr int kStride = 16 * (ROWS ? kWaves : 1);
    const int dt = kStride / G, dh = kStride % G;
    int j = i0 * G + (ROWS ? 16 * wave : 0) + r16;
    int tok = (int)((unsigned)j / (unsigned)G), hd = j - tok * G;
    struct Step {
      u32x4 q[D / 32];
      float lse;
      int lo, hi, tok, hd;
    };
    auto load = [&](Step& e) __attribute__((always_inline)) {
      const bool real = j < end_row;
      e.tok = real ? tok : i0;
      e.hd = real ? hd : 0;
      e.lo = e.hi = 0;
      if (real) visible(a.rule, q, s, e.tok, cap, e.lo, e.hi);
      const size_t row = (size_t)(q.start + min(e.tok, q.n - 1)) * a.h_q + g * G + e.hd;
      e.lse = a.lse[row] * kLog2e;
#pragma unroll
      for (int kc = 0; kc < D / 32; ++kc)
        e.q[kc] = *reinterpret_cast<const u32x4*>(a.q + row * D + 32 * kc + 8 * kg);
      j += kStride;
      tok += dt;
      hd += dh;
      if (hd >= G) {
        hd -= G;
        ++tok;
      }
    };
    const int first = i0 * G + (ROWS ? 16 * wave : 0);
    const int steps = end_row > first ? (end_row - first + kStride - 1) / kStride : 0;
    Step cur, nxt;
    if (steps > 0) load(cur);
    __builtin_amdgcn_s_waitcnt(0x0F70);        // vmcnt(0): the copies
    if (ROWS) __syncthreads();
    u32x4 kf[NK][D / 32];
#pragma unroll
    for (int kt = 0; kt < NK; ++kt)
#pragma unroll
      for (int kc = 0; kc < D / 32; ++kc)
        kf[kt][kc] = *reinterpret_cast<const u32x4*>(
            ks + (16 * kt + r16) * RB + (((4 * kc + kg) ^ (r16 & (CH - 1))) << 4));
    for (int n = 0; n < steps; ++n) {
      if (n + 1 < steps) load(nxt);
      const Scores<CAP, BIAS> sc(a.rule, q, cur.tok, g * G + cur.hd);
      const float mul = CAP || BIAS ? 1.f : sc.mul;
      const bool counts = cur.lse != -INFINITY;
      const bool part = __ballot(cur.lo > t0 || cur.hi < t0 + kKeys || !counts) != 0ull ||
                        pages != (1u << NK) - 1u;
      const int from = counts ? cur.lo - (t0 + 4 * kg) : kKeys;
      const int to = counts ? cur.hi - (t0 + 4 * kg) : 0;
#pragma unroll
      for (int k0 = 0; k0 < NK; k0 += NX) {    // 64 keys at a time
        f32x4 x[NX];
#pragma unroll
        for (int kt = 0; kt < NX; ++kt) x[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kc = 0; kc < D / 32; ++kc)
#pragma unroll
          for (int kt = 0; kt < NX; ++kt) x[kt] = T::mfma32(kf[k0 + kt][kc], cur.q[kc], x[kt]);
        settle(x);
        if (CAP || BIAS) sc(x, (float)(sc.p - (t0 + 16 * k0 + 4 * kg)));
        if (part) {
#pragma unroll
          for (int kt = 0; kt < NX; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int key = 16 * (k0 + kt) + i;
              const float w = __builtin_amdgcn_exp2f(fmaf(x[kt][i], mul, -cur.lse));
              sum[k0 + kt][i] += (pages >> (k0 + kt) & 1) && key >= from && key < to ? w : 0.f;
            }
        } else {
#pragma unroll
          for (int kt = 0; kt < NX; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              sum[k0 + kt][i] += __builtin_amdgcn_exp2f(fmaf(x[kt][i], mul, -cur.lse));
        }
      }
      cur = nxt;
    }
  }
  // the 16 columns of a key
#pragma unroll
  for (int kt = 0; kt < NK; ++kt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v = sum[kt][i];
      v += dpp_f<kDppQuadXor1>(v);
      v += dpp_f<kDppQuadXor2>(v);
      v += dpp_f<kDppHalfMirror>(v);
      v += dpp_f<kDppMirror>(v);
      sum[kt][i] = v;
    }
#pragma unroll
  for (int e = 0; e < NK / NX; ++e) {
    float mine = 0.f;
#pragma unroll
    for (int kt = 0; kt < NX; ++kt)
#pragma unroll
      for (int i = 0; i < 4; ++i) mine = r16 == 4 * kt + i ? sum[4 * e + kt][i] : mine;
    if (ROWS)
      s_sum[wave][64 * e + mine_key] = mine;
    else if (mine_real)
      a.acc_out[base + t0 + mine_key] = a.acc ? fmaf(a.decay, had, mine) : mine;
  }
  if (ROWS) {
    __syncthreads();
    if (tid < kKeys && t0 + tid < cap) {
      const float v = (s_sum[0][tid] + s_sum[1][tid]) + (s_sum[2][tid] + s_sum[3][tid]);
      const int64_t t = base + t0 + tid;
      a.acc_out[t] = a.acc ? fmaf(a.decay, a.acc[t], v) : v;
    }
  }
}

template <class T, int D, bool ROWS>
void launch(const WeightArgs& a, dim3 grid, hipStream_t s) {
  const bool cap = a.rule.cap > 0.f, bias = a.rule.slopes != nullptr;
  auto f = cap ? (bias ? weights_kernel<T, D, true, true, ROWS>
                       : weights_kernel<T, D, true, false, ROWS>)
               : (bias ? weights_kernel<T, D, false, true, ROWS>
                       : weights_kernel<T, D, false, false, ROWS>);
  hipLaunchKernelGGL(f, grid, dim3(64 * kWaves), 0, s, a);
}
template <bool ROWS>
hipError_t launch(const WeightArgs& a, int dtype, int d, hipStream_t s) {
  const int keys = ROWS ? 128 : kFewKeys * kWaves, cap = a.pages.room();
  const int64_t groups = (int64_t)((cap + keys - 1) / keys) * a.h_kv;
  if (!launchable(groups, 64 * kWaves)) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)groups, (unsigned)a.n_seq);
  if (dtype == SPOT_DTYPE_BF16)
    d == 128 ? launch<Bf16, 128, ROWS>(a, grid, s) : launch<Bf16, 64, ROWS>(a, grid, s);
  else
    d == 128 ? launch<Fp16, 128, ROWS>(a, grid, s) : launch<Fp16, 64, ROWS>(a, grid, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_weights(const WeightArgs& a, int dtype, int d, hipStream_t s) {
  if (a.pages.room() == 0) return hipSuccess;
  // By the mean of the rows (new tokens x heads of a group), as the lengths are on the
  // device.  8 KV heads, us, few / many: 32768 keys 32 rows 17 / 22, 64 rows 24 / 24, 128
  // rows 39 / 31; eight sequences of 4096 17 / 24, 25 / 26, 40 / 33; one 4.5 / 5.8,
  // 5.9 / 6.2, 8.6 / 8.0.
  const bool many = (int64_t)a.rows * (a.h_q / a.h_kv) > 64 * (int64_t)a.n_seq;
  return many ? launch<true>(a, dtype, d, s) : launch<false>(a, dtype, d, s);
}

}  // namespace paged
}  // namespace spot
