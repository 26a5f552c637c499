// Rotary positions and the append of keys and values to an 8-bit paged cache (gfx950).
//
// Keys (rotated) and values become e4m3 codes with one power of two for every 16 tokens of
// a head: the smallest for which no value of theirs exceeds the largest code, 448.  A
// rotated pair (a, b) counts as amp (|a| + |b|), which bounds both of its values at any
// angle: the scale follows from the inputs alone, whatever the rounding of sines.  (At
// most a factor of 2 sqrt 2 above what the values need, of 2^15 that the codes span at full
// precision.)  New tokens that join earlier ones of their 16 keep the scale or raise it;
// then the earlier codes are rounded again, which costs those of the smallest values bits
// and leaves the others as they were, the factor being a power of two.
//
// The queries' rows are rotated as by rotary_kernel, a workgroup each; four heads' keys, or
// values, of 16 tokens are another workgroup, one head a wave.  Every element is read and
// written once and memory bounds it; sines of a token are made once for its queries and once
// for every four KV heads.  8000 tokens of 64 + 8 + 8 heads of 128, three axes, 276 MB: 61.6
// us, 4.5 TB/s; 16 single tokens 4.9 us between calls.
#include <algorithm>

#include "cache8.h"
#include "rotary_core.h"

namespace spot {
namespace paged {
namespace {

using namespace rot;

constexpr int kHeads = 4;             // of a workgroup: one a wave
constexpr int kLeast = 27;            // least scale, 2^-100: its products are BF16 numbers
constexpr float kTop = 448.f;         // the largest code

// The largest e4m3 number times a power of two that the element type has: values beyond
// it are held back to it.
template <class T>
constexpr float kLargest = 61440.f;                               // FP16
template <>
constexpr float kLargest<Bf16> = 240.f * 1.329227995784916e36f;   // 2^120

// 16 tokens that new ones belong to.
struct Group {
  int s;                  // sequence (-1: no work)
  int t0;                 // first token
  int from, to;           // new tokens of the 16: [from, to)
  int row;                // row of the first of them
};
// Number `unit` of all sequences' groups, found by one wave.
__device__ __forceinline__ Group find_group(const RotaryArgs& a, int unit) {
  const int lane = __lane_id();
  Group r = {-1, 0, 0, 0, 0};
  int at = 0;
  for (int base = 0; base < a.n_seq; base += 64) {
    Seq q = {0, 0, 0};
    if (base + lane < a.n_seq) q = sequence(a.seq_start, a.seq_len, base + lane, a.rows);
    // tokens at negative places are not there
    const int first = max(q.len - q.n, 0);
    const int n = q.n > 0 && q.len > first
                      ? (q.len - 1) / kGroupKeys - first / kGroupKeys + 1
                      : 0;
    const int incl = wave_incl_scan_i(n);
    const uint64_t hit = __ballot(unit >= at + incl - n && unit < at + incl);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      const int in = unit - at - __builtin_amdgcn_readlane(incl - n, l);
      const int f = __builtin_amdgcn_readlane(first, l), len = __builtin_amdgcn_readlane(q.len, l);
      const int start = __builtin_amdgcn_readlane(q.start, l);
      const int p0 = len - __builtin_amdgcn_readlane(q.n, l);
      r.s = base + l;
      r.t0 = (f / kGroupKeys + in) * kGroupKeys;
      r.from = max(f - r.t0, 0);
      r.to = min(len - r.t0, kGroupKeys);
      r.row = start + (r.t0 + r.from - p0);
      return r;
    }
    at += __builtin_amdgcn_readlane(incl, 63);
  }
  return r;
}

// The byte of the smallest power of two n with x <= 448 n.
__device__ __forceinline__ int scale_byte(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x);
  // 448 = 1.75 x 2^8
  const int e = (int)(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u);
  return max(e, kLeast);
}
__device__ __forceinline__ float power(int e) {          // 2^e, at least 2^-126
  return __builtin_bit_cast(float, (uint32_t)(max(e, -126) + 127) << 23);
}

// x / 2^(byte - 127) within the codes (NaN stays).
template <class T>
__device__ __forceinline__ float fit(float x, float inv) {
  constexpr float L = kLargest<T>;
  x = x > L ? L : x;
  x = x < -L ? -L : x;
  x *= inv;
  x = x > kTop ? kTop : x;
  return x < -kTop ? -kTop : x;
}
__device__ __forceinline__ uint32_t code4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}

// A head's 16 tokens, keys (K) or values, in rounds of 64 / kLanes tokens: a lane has four
// pairs of elements of one.  A round without new tokens is passed over, so that a decode
// step's one token costs a quarter of a group's instructions (the wave's own chain of them
// is what a small append waits for).
// VEC: four neighbouring pairs, two loads of 8 bytes; otherwise every kLanes-th pair.
template <class T, int D, bool VEC, bool IL, bool K>
struct Head {
  static constexpr int kLanes = D / 8;       // of a token
  static constexpr int kTokens = 64 / kLanes, kRounds = kGroupKeys / kTokens;
  // (values alone: a reference to the arguments would put them all into scratch memory)
  uint8_t *pool, *scales;
  int64_t head_rows;                         // from KV head 0 to this one
  int64_t stride;
  float amp;
  int half, from, to, tk, part, old;
  const uint16_t* in;                        // of the first new token
  u32x2 raw[VEC ? 2 * kRounds : 1];

  __device__ __forceinline__ Head(const Append8Args& args, const Group& gr, int h) {
    const RotaryArgs& a = args.r;
    const int lane = threadIdx.x & 63;
    pool = K ? args.k8 : args.v8;
    scales = K ? args.k_scale : args.v_scale;
    head_rows = (int64_t)h * a.pages.page_size;
    amp = fabsf(a.amp);
    half = K ? a.rope_dim / 2 : 0;
    from = gr.from;
    to = gr.to;
    tk = lane / kLanes;
    part = lane % kLanes;
    stride = K ? a.k_stride : a.v_stride;
    in = (K ? a.k : a.v) + gr.row * stride + h * D;
  }
  // Four pairs from element ca and cb on: the two halves of them, or neighbours.
  struct Unit {
    int ca, cb;
    bool hf, rot;
  };
  __device__ __forceinline__ Unit unit() const {
    const bool hf = !IL && 4 * part < half;
    return Unit{hf ? 4 * part : 8 * part, hf ? half + 4 * part : 8 * part + 4, hf,
                4 * part < half};
  }
  // The elements of pair m of four, in other forms than VEC.
  struct Pair {
    int i, a, b;
    bool rot;
  };
  __device__ __forceinline__ Pair pair(int m) const {
    const int i = part + kLanes * m;
    const bool rot = i < half;
    return Pair{i, rot && !IL ? i : 2 * i, rot && !IL ? i + half : 2 * i + 1, rot};
  }
  __device__ __forceinline__ bool round_has(int r) const {       // (the same in all lanes)
    return r * kTokens < to && (r + 1) * kTokens > from;
  }
  __device__ __forceinline__ bool now(int r) const {
    const int t = r * kTokens + tk;
    return t >= from && t < to;
  }
  __device__ __forceinline__ const uint16_t* row(int r) const {
    return in + (r * kTokens + tk - from) * stride;
  }
  // The new tokens' elements, on their way.
  __device__ __forceinline__ void load() {
    if constexpr (VEC) {
      const Unit t = unit();
#pragma unroll
      for (int r = 0; r < kRounds; ++r) {
        raw[2 * r] = raw[2 * r + 1] = u32x2{0u, 0u};
        if (now(r)) {
          raw[2 * r] = *reinterpret_cast<const u32x2*>(row(r) + t.ca);
          raw[2 * r + 1] = *reinterpret_cast<const u32x2*>(row(r) + t.cb);
        }
      }
    }
  }
  // A lane's four pairs of a round.
  __device__ __forceinline__ void values(int r, float (&a)[4], float (&b)[4]) const {
    if constexpr (VEC) {
      const bool hf = unit().hf;
      const u32x2 x = raw[2 * r], y = raw[2 * r + 1];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t n = e < 2 ? x[e] : y[e - 2];
        const float fx = e & 1 ? T::hi(x[e / 2]) : T::lo(x[e / 2]);
        const float fy = e & 1 ? T::hi(y[e / 2]) : T::lo(y[e / 2]);
        const float nx = T::lo(n), ny = T::hi(n);
        a[e] = hf ? fx : nx;
        b[e] = hf ? fy : ny;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        a[e] = b[e] = 0.f;
        if (now(r)) {
          a[e] = T::one(row(r)[pair(e).a]);
          b[e] = T::one(row(r)[pair(e).b]);
        }
      }
    }
  }
  __device__ __forceinline__ int64_t slots(int krow) const {   // pool row of the 16 tokens
    return krow + head_rows;
  }
  // The scale of the earlier tokens.
  __device__ __forceinline__ void load_scale(int krow) {
    old = 0;
    if (from > 0) old = scales[slots(krow) / kGroupKeys];
  }
  __device__ __forceinline__ void store(int krow, const float* s_cos, const float* s_sin) {
    float turned = 0.f, plain = 0.f;         // largest magnitudes of finite values
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      if (!round_has(r)) continue;
      float a[4], b[4];
      values(r, a, b);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool rot = VEC ? unit().rot : pair(e).rot;
        const float x = fabsf(a[e]), y = fabsf(b[e]), z = x + y;
        turned = (rot & (z < INFINITY)) ? fmaxf(turned, z) : turned;
        plain = (!rot & (x < INFINITY)) ? fmaxf(plain, x) : plain;
        plain = (!rot & (y < INFINITY)) ? fmaxf(plain, y) : plain;
      }
    }
    const float top = wave_max(fmaxf(turned * amp, plain));
    const int64_t at = slots(krow) / kGroupKeys;
    uint8_t* const out = pool + (slots(krow) + tk) * D;
    int byte = scale_byte(top < INFINITY ? top : 3.4028235e38f);
    if (from > 0) {
      if (byte > old) {          // the earlier tokens' codes once more
        const float down = power(old - byte);
#pragma unroll 1
        for (int r = 0; r * kTokens < from; ++r) {
          if (r * kTokens + tk >= from) continue;
          u32x2* const c = reinterpret_cast<u32x2*>(out + r * kTokens * D) + part;
          u32x2 z = *c;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const f32x2 x = __builtin_amdgcn_cvt_pk_f32_fp8(z[i], false);
            const f32x2 y = __builtin_amdgcn_cvt_pk_f32_fp8(z[i], true);
            z[i] = code4(x[0] * down, x[1] * down, y[0] * down, y[1] * down);
          }
          *c = z;
        }
      } else {
        byte = old;
      }
    }
    if ((threadIdx.x & 63) == 0) scales[at] = (uint8_t)byte;
    const float inv = power(127 - byte);
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      if (!round_has(r)) continue;
      float a[4], b[4];
      values(r, a, b);
      const int t = r * kTokens + tk;
      if constexpr (K) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          // (sines of pairs that are not rotated: whatever lies there, and not used)
          const int p = VEC ? 4 * part + e : pair(e).i;
          const bool rot = VEC ? unit().rot : pair(e).rot;
          const f32x2 w = turn(a[e], b[e], s_cos[t * kPitch + p], s_sin[t * kPitch + p]);
          a[e] = rot ? w[0] : a[e];
          b[e] = rot ? w[1] : b[e];
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        a[e] = fit<T>(a[e], inv);
        b[e] = fit<T>(b[e], inv);
      }
      uint8_t* const o = out + r * kTokens * D;
      if constexpr (VEC) {
        const Unit u = unit();
        const float x1 = u.hf ? a[1] : b[0], x2 = u.hf ? a[2] : a[1], x3 = u.hf ? a[3] : b[1];
        const float y0 = u.hf ? b[0] : a[2], y1 = u.hf ? b[1] : b[2], y2 = u.hf ? b[2] : a[3];
        if (now(r)) {
          *reinterpret_cast<uint32_t*>(o + u.ca) = code4(a[0], x1, x2, x3);
          *reinterpret_cast<uint32_t*>(o + u.cb) = code4(y0, y1, y2, b[3]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t c = code4(a[e], b[e], 0.f, 0.f);
          if (now(r)) {
            o[pair(e).a] = (uint8_t)c;
            o[pair(e).b] = (uint8_t)(c >> 8);
          }
        }
      }
    }
  }
  static constexpr int kPitch = D / 2 + 4;   // rows of sines, in other banks
};

// Workgroups: `units` groups x ceil(h_kv / 4) x (keys, values), then the queries' rows.
template <class T, int D, bool VEC, bool IL, bool AXES>
__global__ __launch_bounds__(kThreads) void append8_kernel(Append8Args args, int units) {
  const RotaryArgs& a = args.r;
  const int chunks = (a.h_kv + kHeads - 1) / kHeads;
  const int64_t first = (int64_t)units * chunks * 2;
  if (blockIdx.x >= first) {
    rotate_row<T, VEC, IL, AXES, true>(a, (int)(blockIdx.x - first));
    return;
  }
  constexpr int kPitch = Head<T, D, VEC, IL, true>::kPitch;
  __shared__ __attribute__((aligned(16))) float s_cos[kGroupKeys * kPitch];
  __shared__ __attribute__((aligned(16))) float s_sin[kGroupKeys * kPitch];
  const int tid = threadIdx.x, wave = tid >> 6;
  const bool keys = blockIdx.x % 2 == 0;
  const int chunk = blockIdx.x / 2 % chunks;
  const Group gr = find_group(a, blockIdx.x / 2 / chunks);
  if (gr.s < 0 || gr.t0 >= a.pages.cap()) return;
  const int h = chunk * kHeads + wave;
  // What depends on the place in the cache, and the angles, come while the elements do.
  if (keys) {
    Head<T, D, VEC, IL, true> head(args, gr, min(h, a.h_kv - 1));
    head.load();
    const int krow = a.pages.row(gr.s, gr.t0, 0, a.h_kv);
    if (krow < 0) return;
    head.load_scale(krow);
    const int half = a.rope_dim / 2;
    for (int i = tid; i < (gr.to - gr.from) * half; i += kThreads) {
      const int tk = gr.from + i / half, p = i % half;
      const int row = gr.row + tk - gr.from;
      const int pos = AXES    ? a.pos[(int64_t)row * a.n_axes + a.axis[p]]
                      : a.pos ? a.pos[row]
                              : gr.t0 + tk;
      float sn, cs;
      rope_sincos(pos, a.freq.f[p], sn, cs);
      s_cos[tk * kPitch + p] = cs * a.amp;
      s_sin[tk * kPitch + p] = a.inverse ? -sn * a.amp : sn * a.amp;
    }
    __syncthreads();
    if (h < a.h_kv) head.store(krow, s_cos, s_sin);
  } else if (h < a.h_kv) {
    Head<T, D, VEC, IL, false> head(args, gr, h);
    head.load();
    const int krow = a.pages.row(gr.s, gr.t0, 0, a.h_kv);
    if (krow < 0) return;
    head.load_scale(krow);
    head.store(krow, s_cos, s_sin);
  }
}

template <class T, int D, bool AXES>
void launch(const Append8Args& a, int units, dim3 grid, bool vec, bool il, hipStream_t s) {
  auto f = vec ? (il ? append8_kernel<T, D, true, true, AXES>
                     : append8_kernel<T, D, true, false, AXES>)
               : (il ? append8_kernel<T, D, false, true, AXES>
                     : append8_kernel<T, D, false, false, AXES>);
  hipLaunchKernelGGL(f, grid, dim3(kThreads), 0, s, a, units);
}

}  // namespace

hipError_t launch_append8(const Append8Args& args, int dtype, bool interleaved, hipStream_t s) {
  const RotaryArgs& a = args.r;
  // groups that new tokens of ascending starts can belong to
  const int64_t units =
      std::min((int64_t)a.rows, (int64_t)a.rows / kGroupKeys + 2 * (int64_t)a.n_seq);
  const int64_t groups = units * ((a.h_kv + kHeads - 1) / kHeads) * 2 + a.rows;
  if (!launchable(groups, kThreads)) return hipErrorInvalidConfiguration;
  auto whole = [](const void* p, int64_t stride) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0;
  };
  const bool vec = a.rope_dim % 16 == 0 && whole(a.q, a.q_stride) && whole(a.q_out, a.out_stride) &&
                   whole(a.k, a.k_stride) && whole(a.v, a.v_stride);
  const dim3 grid((unsigned)groups);
  auto go = [&](auto t) {
    typedef decltype(t) T;
    if (a.n_axes > 0)
      a.d == 128 ? launch<T, 128, true>(args, (int)units, grid, vec, interleaved, s)
                 : launch<T, 64, true>(args, (int)units, grid, vec, interleaved, s);
    else
      a.d == 128 ? launch<T, 128, false>(args, (int)units, grid, vec, interleaved, s)
                 : launch<T, 64, false>(args, (int)units, grid, vec, interleaved, s);
  };
  dtype == SPOT_DTYPE_BF16 ? go(Bf16()) : go(Fp16());
  return hipGetLastError();
}

}  // namespace paged
}  // namespace spot
