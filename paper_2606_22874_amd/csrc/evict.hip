// Eviction from a paged cache by accumulated attention weight (gfx950).
//
// Per sequence and KV head the sink prefix, the recency suffix and the heaviest of
// the other tokens stay, `budget` in all.  evict_select_kernel, one workgroup per
// (sequence, KV head), finds the K-th largest weight by three radix passes over
// order-preserving keys (11, 11 and 10 bits, counted in LDS), then writes the kept
// tokens in ascending order with their weights (each wave has a run of tokens, so that
// their places follow from counts); equal weights go to the lower index.
// evict_move_kernel copies their keys and values to the new pages, 16 bytes a lane.
// The copy is bound by memory: 4 sequences of 8 heads, 4096 tokens of 128 dims each, 25 us,
// 5.4 TB/s.  The selection is bound by one compute unit's passes over a row: 22.7 us
// for 32768 weights of each of those heads, 8 for 5000.
#include "paged_core.h"

namespace spot {
namespace paged {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kAhead = 8;
constexpr int kBins = 2048;

// Order-preserving key of a weight; -0 equals 0, NaN lies below every number.
__device__ __forceinline__ uint32_t key_of(float x) {
  if (x != x) return 0u;
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Inclusive sums over the workgroup of one value per thread.
__device__ __forceinline__ int scan_block(int v, int* s_wave) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int incl = wave_incl_scan_i(v);
  __syncthreads();
  if (lane == 63) s_wave[wave] = incl;
  __syncthreads();
  int before = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) before += w < wave ? s_wave[w] : 0;
  return before + incl;
}

// A wave's tokens [from, end): each() calls f(token, key, weight, whether the token is
// below end), 64 tokens a step and in order.  HELD steps' weights are read once, into
// registers; with 0 they come from memory in each pass, kAhead steps' loads in
// flight.  us for rows of 32768 tokens, held / from memory: 22 / 31; of 5003 tokens,
// 8 held / 32 held / from memory: 8.2 / 15.9 / 11.0.
template <int HELD>
struct Tokens {
  const float* acc;
  int from, end, lane;
  uint32_t bits[HELD ? HELD : 1];
  __device__ __forceinline__ Tokens(const float* acc_, int from_, int end_)
      : acc(acc_), from(from_), end(end_), lane(threadIdx.x & 63) {
    if constexpr (HELD != 0)
#pragma unroll
      for (int e = 0; e < HELD; ++e)
        if (from + 64 * e < end) bits[e] = __float_as_uint(acc[min(from + 64 * e + lane, end - 1)]);
  }
  template <class F>
  __device__ __forceinline__ void each(const F& f) {
    if constexpr (HELD != 0) {
#pragma unroll
      for (int e = 0; e < HELD; ++e)
        if (from + 64 * e < end) {
          const float x = __uint_as_float(bits[e]);
          const int t = from + 64 * e + lane;
          f(t, key_of(x), x, t < end);
        }
    } else {
      for (int base = from; base < end; base += 64 * kAhead) {
        float x[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) x[e] = acc[min(base + 64 * e + lane, end - 1)];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
          const int t = base + 64 * e + lane;
          if (base + 64 * e < end) f(t, key_of(x[e]), x[e], t < end);
        }
      }
    }
  }
};

struct Shared {
  int hist[kBins];
  int wave[kWaves], larger[kWaves], equal[kWaves];
  uint32_t prefix;
  int need;
};

// The `want` heaviest of the tokens [f0, f1) in order, to idx and acc_out.
template <int HELD>
__device__ __forceinline__ void keep_heaviest(Shared& sm, const float* acc, int f0, int f1,
                                              int want, int32_t* idx, float* acc_out) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // each wave has a run of whole steps of 64 tokens
  const int run = ((f1 - f0 + kThreads - 1) / kThreads) * 64;
  const int from = min(f0 + wave * run, f1);
  Tokens<HELD> tokens(acc, from, min(from + run, f1));

  // the want-th largest key; `need` counts how many equal to it are kept
  uint32_t prefix = 0, mask = 0;
  int need = want;
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const int bins = pass == 2 ? kBins / 2 : kBins, per = bins / kThreads;
    for (int i = tid; i < bins; i += kThreads) sm.hist[i] = 0;
    __syncthreads();
    tokens.each([&](int, uint32_t u, float, bool in) {
      if (in && (u & mask) == prefix) atomicAdd(&sm.hist[(u >> shift) & (bins - 1)], 1);
    });
    __syncthreads();
    // bins from the top, two (or one) a thread
    int c[2] = {0, 0}, mine = 0;
    for (int e = 0; e < per; ++e) mine += c[e] = sm.hist[bins - 1 - (tid * per + e)];
    int above = scan_block(mine, sm.wave) - mine;
    for (int e = 0; e < per; ++e) {
      if (above < need && need <= above + c[e]) {
        sm.prefix = prefix | (uint32_t)(bins - 1 - (tid * per + e)) << shift;
        sm.need = need - above;
      }
      above += c[e];
    }
    __syncthreads();
    prefix = sm.prefix;
    need = sm.need;
    mask |= (uint32_t)(bins - 1) << shift;
  }
  // larger ones, and the first `need` equal ones
  int larger = 0, equal = 0;
  tokens.each([&](int, uint32_t u, float, bool in) {
    larger += __popcll(__ballot(in && u > prefix));
    equal += __popcll(__ballot(in && u == prefix));
  });
  if (lane == 0) {
    sm.larger[wave] = larger;
    sm.equal[wave] = equal;
  }
  __syncthreads();
  larger = equal = 0;                          // of the tokens before
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    larger += w < wave ? sm.larger[w] : 0;
    equal += w < wave ? sm.equal[w] : 0;
  }
  const uint64_t lower = (1ull << lane) - 1ull;
  tokens.each([&](int t, uint32_t u, float x, bool in) {
    const bool gt = in && u > prefix, eq = in && u == prefix;
    const uint64_t mg = __ballot(gt), me = __ballot(eq);
    const int e = equal + __popcll(me & lower);
    if (gt || (eq && e < need)) {
      const int j = larger + __popcll(mg & lower) + min(e, need);
      idx[j] = t;
      acc_out[j] = x;
    }
    larger += __popcll(mg);
    equal += __popcll(me);
  });
}

__global__ __launch_bounds__(kThreads) void evict_select_kernel(EvictArgs a) {
  __shared__ Shared sm;
  const int tid = threadIdx.x;
  const int g = blockIdx.x % a.h_kv, s = blockIdx.x / a.h_kv;
  const int cap = a.pages.room();
  const int len = min(max(a.seq_len[s], 0), cap);
  const int keep = min(len, a.budget);
  const float* acc = a.acc + ((int64_t)s * a.h_kv + g) * cap;
  int32_t* idx = a.idx + ((int64_t)s * a.h_kv + g) * a.budget;
  float* acc_out = a.acc_out + ((int64_t)s * a.h_kv + g) * a.out_cap;
  if (tid == 0 && g == 0) a.new_len[s] = keep;
  for (int j = keep + tid; j < a.budget; j += kThreads) idx[j] = -1;
  for (int j = keep + tid; j < a.out_cap; j += kThreads) acc_out[j] = 0.f;
  if (len <= a.budget) {
    for (int j = tid; j < len; j += kThreads) {
      idx[j] = j;
      acc_out[j] = acc[j];
    }
    return;
  }
  const int f0 = a.n_sink, f1 = len - a.n_recent;     // the tokens to choose from
  const int want = a.budget - a.n_sink - a.n_recent;
  for (int j = tid; j < a.n_sink; j += kThreads) {
    idx[j] = j;
    acc_out[j] = acc[j];
  }
  for (int j = tid; j < a.n_recent; j += kThreads) {
    idx[keep - a.n_recent + j] = f1 + j;
    acc_out[keep - a.n_recent + j] = acc[f1 + j];
  }
  if (want == 0) return;
  idx += a.n_sink;
  acc_out += a.n_sink;
  if (f1 - f0 <= 8 * kThreads)
    keep_heaviest<8>(sm, acc, f0, f1, want, idx, acc_out);
  else if (f1 - f0 <= 32 * kThreads)
    keep_heaviest<32>(sm, acc, f0, f1, want, idx, acc_out);
  else
    keep_heaviest<0>(sm, acc, f0, f1, want, idx, acc_out);
}

__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a) {
  const int chunks = a.d / 8;
  const int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int j = (int)(w / chunks), c = (int)(w % chunks);
  const int g = blockIdx.y, s = blockIdx.z;
  if (j >= a.budget) return;
  const int t = a.idx[((int64_t)s * a.h_kv + g) * a.budget + j];
  if (t < 0) return;
  const int ps = a.pages.page_size;
  const int dst = a.dst.table[(int64_t)s * a.dst.max_pages + j / ps];
  if ((unsigned)dst >= (unsigned)a.dst.n_pages) return;
  const int src = a.pages.row(s, t & ~(kGroupKeys - 1), g, a.h_kv);
  u32x4 k = {0u, 0u, 0u, 0u}, v = k;
  if (src >= 0) {
    const int64_t from = ((int64_t)src + (t & (kGroupKeys - 1))) * a.d + c * 8;
    k = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.k + from));
    v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.v + from));
  }
  const int64_t to = (((int64_t)dst * a.h_kv + g) * ps + j % ps) * a.d + c * 8;
  *reinterpret_cast<u32x4*>(a.k_dst + to) = k;
  *reinterpret_cast<u32x4*>(a.v_dst + to) = v;
}

}  // namespace

hipError_t launch_evict(const EvictArgs& a, hipStream_t s) {
  const int64_t work = (int64_t)min(a.budget, a.pages.room()) * (a.d / 8);   // most that stays
  const int64_t heads = (int64_t)a.n_seq * a.h_kv, groups = (work + 255) / 256;
  if (!launchable(heads, kThreads) || !launchable(groups, 256)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)heads), dim3(kThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || groups == 0) return e;
  hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)groups, (unsigned)a.h_kv, (unsigned)a.n_seq),
                     dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace paged
}  // namespace spot
