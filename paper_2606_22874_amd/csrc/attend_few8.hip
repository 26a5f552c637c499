// Attention of few rows over an 8-bit paged cache (gfx950): decode steps, a handful of new
// tokens a sequence.
//
// The division of work, the softmax and the end are those of attend_few.hip: a workgroup of
// 4 waves takes a run of 64-key blocks for a tile of 16 rows.  A wave takes every fourth
// half block of 32 keys:
//   S^T = K Q^T       K rows from memory as the A operand, without LDS: a lane's 16 codes are
//                     16 neighbouring dims, so Q's dims go to the same places (a dot
//                     product does not ask for their order), and 8 codes become the operand
//                     of one MFMA 16x16x32;
//   O^T += V^T P^T    V as codes through LDS and the transposing read of bytes, which gives
//                     a lane 8 keys of one dim: D/16 MFMAs 16x16x32, P^T straight from the
//                     scores' accumulators.
// The codes' bytes bound it (2 D + 1/8 a key and KV head): decode, four sequences of 131072
// tokens, 8 KV heads of 128, 177 us, 6.1 TB/s; 48 of up to 40000 with a window of 8192, heads
// of 64, 76 us, 4.9 TB/s.  On one short sequence the chain of lengths, pages, keys and join
// does: 600 tokens 9.6 us.
#include "attend_join.h"
#include "cache8.h"

namespace spot {
namespace paged {
namespace {

using namespace few;

constexpr int kKeys = 32;          // keys of a wave's step
typedef int i32x2 __attribute__((ext_vector_type(2)));

// Physical 16-byte chunk of logical chunk c of row r of V (D bytes): a transposing read
// takes one chunk of 8 rows, 4 kg .. + 3 and 16 more, which have to lie in all banks.
template <int D>
__device__ __forceinline__ int swz8(int r, int c) {
  return D == 128 ? c ^ (r & 3) ^ ((r >> 4 & 1) << 2) : c ^ (r >> 1 & 1) ^ ((r >> 4 & 1) << 1);
}

template <class T, int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(64 * kWaves, 2) void attend8_few_kernel(AttendArgs a) {
  constexpr int KL = D / 64;            // 16-byte loads of a lane for 16 keys
  constexpr int VL = kKeys * D / 1024;  // the same for 32 values
  constexpr int LR = 1024 / D;          // rows of such a load: 8 or 16
  constexpr int CH = D / 16;            // 16-byte chunks of a row
  __shared__ Smem<D, kKeys * D> sm;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r16 = lane & 15, kg = lane >> 4;
  const int G = a.h_q / a.h_kv, g = blockIdx.x % a.h_kv;
  const int cap = a.pages.cap();
  if (wave == 0) {
    const Part p = find_part<kRows, 0, kFit<D>>(blockIdx.x / a.h_kv, a.seq_start, a.seq_len,
                                                a.n_seq, a.rows, G, a.h_kv, a.rule.window,
                                                a.rule.sink, cap, a.from, a.to);
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
  if (real) visible(a.rule, pt.q, pt.s, tok, cap, lo, hi, from, end);
  // (comparisons joined without branches, here and where values are masked: of a select
  // behind short-circuit ones and a uniform branch the compiler, ROCm 7.2, has kept the
  // uniform part only)
  auto sees = [&](int t) { return ((t >= lo) & (t < hi)) | ((t >= from) & (t < end)); };
  Scores<CAP, BIAS, true> sc(a.rule, pt.q, tok, head);
  u32x4 qf[2 * KL];
  const size_t qrow = (size_t)(pt.q.start + tok) * a.h_q + head;
#pragma unroll
  for (int i = 0; i < 2 * KL; ++i) {
    qf[i] = u32x4{0u, 0u, 0u, 0u};
    if (real)
      qf[i] = *reinterpret_cast<const u32x4*>(a.q + qrow * D + i / 2 * 64 + 16 * kg + i % 2 * 8);
  }
  // what some row sees, and what all of them do
  const bool any = hi > lo;
  const int LO = (int)wave_min_u(any ? (uint32_t)lo : 0x7fffffffu);
  const int HI = (int)wave_max_u((uint32_t)hi);
  const int FLO = (int)wave_max_u(real ? (uint32_t)(any ? lo : 0x7fffffff) : 0u);
  const int FHI = (int)wave_min_u(real ? (uint32_t)hi : 0x7fffffffu);
  const int SLO = (int)wave_min_u(end > from ? (uint32_t)from : 0x7fffffffu);
  const int SHI = (int)wave_max_u((uint32_t)end);
  const Blocks bl = blocks_of(LO, HI, SLO, SHI);
  const int share = (bl.n + pt.n_split - 1) / pt.n_split;
  const int e0 = min(pt.split * share, bl.n), e1 = min(e0 + share, bl.n);

  unsigned char* vs = sm.kv[wave];
  struct Stage {
    u32x4 k[2][KL], v[VL];
    uint32_t scale;                     // of lane l % 4: K (0, 1), V (2, 3) of 16 keys
  } A, B;
  f32x4 o[D / 16];
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_lane = 0.f;

  for (int c0 = e0; c0 < e1; c0 += kListBlocks) {
    const int nb = min(kListBlocks, e1 - c0);
    if (c0 > e0) __syncthreads();       // the list is done with
    for (int i = tid; i < 4 * nb; i += 64 * kWaves) {
      const int t = bl.at(c0 + i / 4) * 64 + i % 4 * kGroupKeys;
      sm.list[i] = a.pages.row_below_cap(pt.s, t, g, a.h_kv);
    }
    __syncthreads();
    const int steps = (2 * nb - wave + kWaves - 1) / kWaves;    // half blocks wave, wave + 4, ..
    auto row_of = [&](int n, int u) {
      return __builtin_amdgcn_readfirstlane(sm.list[2 * (wave + kWaves * n) + u]);
    };
    auto load = [&](Stage& st, int n) {
      const int row[2] = {max(row_of(n, 0), 0), max(row_of(n, 1), 0)};
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < KL; ++i)
          st.k[u][i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(
              a.k8 + (size_t)row[u] * D +
              (KL == 1 ? r16 * D + 16 * kg
                       : (8 * i + (r16 & 7)) * D + 64 * (r16 >> 3) + 16 * kg)));
#pragma unroll
      for (int i = 0; i < VL; ++i)
        st.v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(
            a.v8 + (size_t)row[LR * i / 16] * D + (LR * i % 16) * D + lane * 16));
      const uint8_t* p = lane & 2 ? a.v_scale : a.k_scale;
      st.scale = p[(lane & 1 ? row[1] : row[0]) >> 4];
    };
    bool odd = false;
    float vsc[2];
    // Scores of a step; its values lie in LDS then, and their scales in vsc.
    auto front = [&](Stage& st, int n, f32x4(&s)[2]) {
      const int hb = wave + kWaves * n, t0 = bl.at(c0 + hb / 2) * 64 + hb % 2 * kKeys;
      float ksc[2];
      uint32_t vb[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        ksc[u] = scale8(__builtin_amdgcn_readlane(st.scale, u));
        vb[u] = __builtin_amdgcn_readlane(st.scale, 2 + u);
        vsc[u] = scale8(vb[u]);
      }
      odd = false;
      // Values that no row sees never meet the zero probabilities: they may be NaN, and
      // so may their scale.
      const bool part = t0 < FLO || t0 + kKeys > FHI || row_of(n, 0) < 0 || row_of(n, 1) < 0;
      if (part) {
#pragma unroll
        for (int i = 0; i < VL; ++i) {
          const int u = LR * i / 16, t = t0 + i * LR + lane / CH;
          const bool seen = (row_of(n, u) >= 0) &
                            (((t >= LO) & (t < HI)) | ((t >= SLO) & (t < SHI)));
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            st.v[i][e] = seen ? st.v[i][e] : 0u;
            odd |= nan4(st.v[i][e]);
          }
        }
        odd = __ballot(odd) != 0ull || far8<T>(vb[0]) || far8<T>(vb[1]);
      }
      wave_lds_sync();  // this wave's reads of the previous rows are issued
#pragma unroll
      for (int i = 0; i < VL; ++i) {
        const int r = LR * i + lane / CH, c = lane % CH;
        *reinterpret_cast<u32x4*>(vs + r * D + (swz8<D>(r, c) << 4)) = st.v[i];
      }
      wave_lds_sync();
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        s[u] = f32x4{0.f, 0.f, 0.f, 0.f};
        // D 128: a load took 8 whole rows, and of the lanes r16 and r16 ^ 8 the first gets the
        // second half of its row from the second's first load, the other way round the first
        // half (loads of 16 half rows: 179.6 against 177.1 us for four sequences of 131072).
        u32x4 k[KL];
        k[0] = st.k[u][0];
        if constexpr (KL == 2) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            constexpr int kRor8 = 0x128, kUpper = 0xc, kLower = 0x3;
            k[0][e] = __builtin_amdgcn_update_dpp(st.k[u][0][e], st.k[u][1][e], kRor8, 0xf, kUpper,
                                                  false);
            k[1][e] = __builtin_amdgcn_update_dpp(st.k[u][1][e], st.k[u][0][e], kRor8, 0xf, kLower,
                                                  false);
          }
        }
#pragma unroll
        for (int i = 0; i < 2 * KL; ++i) {
          const u32x4& x = k[i / 2];
          s[u] = T::mfma32(wide8<T>(x[i % 2 * 2], x[i % 2 * 2 + 1], ksc[u], ksc[u]), qf[i], s[u]);
        }
      }
      settle(s);
    };
    auto back = [&](int n, f32x4(&s)[2]) {
      const int hb = wave + kWaves * n, t0 = bl.at(c0 + hb / 2) * 64 + hb % 2 * kKeys;
      const bool part = t0 < FLO || t0 + kKeys > FHI || row_of(n, 0) < 0 || row_of(n, 1) < 0;
      sc(s, (float)(sc.p - (t0 + 4 * kg)), !part);
      if (part) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const bool page = row_of(n, u) >= 0;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            s[u][i] = (page & sees(t0 + 16 * u + 4 * kg + i)) ? s[u][i] : -INFINITY;
        }
      }
      float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                       fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
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
#pragma unroll
      for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          s[u][i] = s[u][i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s[u][i] - m_run);
        l_lane += (s[u][0] + s[u][1]) + (s[u][2] + s[u][3]);
      }
      // k entry 8 kg + e is key 4 kg + e for e < 4, and 12 further on from 4 on
      const u32x4 pb = {T::pack2(s[0][0], s[0][1]), T::pack2(s[0][2], s[0][3]),
                        T::pack2(s[1][0], s[1][1]), T::pack2(s[1][2], s[1][3])};
      const int row = 4 * kg + (r16 >> 1 & 3) + (r16 >> 3) * 16;
      const unsigned char* vrow = vs + row * D + (r16 & 1) * 8;
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) {
        const u32x2 y = __builtin_bit_cast(
            u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                       (__attribute__((address_space(3))) i32x2*)(vrow + (swz8<D>(row, dt) << 4))));
        u32x4 f = wide8<T>(y[0], y[1], vsc[0], vsc[1]);
        if (odd) {
#pragma unroll
          for (int e = 0; e < 4; ++e) f[e] = clean2<T>(f[e]);
        }
        o[dt] = T::mfma32(f, pb, o[dt]);
      }
      if (odd) {   // the elements left out, for the rows that see their tokens
        settle(o);
#pragma unroll 1
        for (int k = 0; k < kKeys; ++k) {
          const float lo4 = k & 2 ? (k & 1 ? s[0][3] : s[0][2]) : (k & 1 ? s[0][1] : s[0][0]);
          const float hi4 = k & 2 ? (k & 1 ? s[1][3] : s[1][2]) : (k & 1 ? s[1][1] : s[1][0]);
          const float pk = __shfl(k & 16 ? hi4 : lo4, (k >> 2 & 3) * 16 + r16);
          const bool seen = sees(t0 + k) & (row_of(n, k >> 4) >= 0);
          const float scale = k & 16 ? vsc[1] : vsc[0];
#pragma unroll
          for (int dt = 0; dt < D / 16; ++dt) {
            const u32x2 y = wide4(T(), *reinterpret_cast<const uint32_t*>(
                                           vs + k * D + (swz8<D>(k, dt) << 4) + kg * 4), scale);
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
    // Two register stages: steps n + 1 and n + 2 are loading while n is computed.
    if (steps <= 0) continue;
    f32x4 s[2];
    load(A, 0);
    if (steps > 1) load(B, 1);
    int n = 0;
    for (; n + 3 < steps; n += 2) {
      front(A, n, s);
      load(A, n + 2);
      back(n, s);
      front(B, n + 1, s);
      load(B, n + 3);
      back(n + 1, s);
    }
    front(A, n, s);
    if (n + 2 < steps) load(A, n + 2);
    back(n, s);
    if (n + 1 < steps) {
      front(B, n + 1, s);
      back(n + 1, s);
    }
    if (n + 2 < steps) {
      front(A, n + 2, s);
      back(n + 2, s);
    }
  }
  finish<T, D>(sm, a, pt, g, G, n_rows, m_run, l_lane, o);
}

template <class T, int D>
void launch(const AttendArgs& a, dim3 grid, hipStream_t s) {
  const bool cap = a.rule.cap > 0.f, bias = a.rule.slopes != nullptr;
  auto f = cap ? (bias ? attend8_few_kernel<T, D, true, true>
                       : attend8_few_kernel<T, D, true, false>)
               : (bias ? attend8_few_kernel<T, D, false, true>
                       : attend8_few_kernel<T, D, false, false>);
  hipLaunchKernelGGL(f, grid, dim3(64 * kWaves), 0, s, a);
}

}  // namespace

hipError_t launch_attend_few8(AttendArgs a, int dtype, int d, void* ws, hipStream_t s) {
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

}  // namespace paged
}  // namespace spot
