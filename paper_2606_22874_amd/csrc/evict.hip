// Eviction from a paged cache by accumulated attention weight (gfx950).
//
// Per sequence and KV head the sink prefix, the recency suffix and the heaviest of
// the other tokens stay, `budget` in all.  evict_select_kernel, one workgroup per
// (sequence, KV head), finds the K-th largest weight by three radix passes over
// order-preserving keys (11, 11 and 10 bits, counted in LDS), then writes the kept
// tokens in ascending order with their weights; equal weights go to the lower
// index.  evict_move_kernel copies their keys and values to the new pages, 16 bytes
// a lane.  The copy is bound by memory; the selection by the reads of one compute
// unit (four passes over a row's weights, which stay in the L2).
#include "paged_core.h"

namespace spot {
namespace paged {
namespace {

constexpr int kThreads = 1024;
constexpr int kBins = 2048;

// Order-preserving key of a weight; -0 equals 0, NaN lies below every number.
__device__ __forceinline__ uint32_t key_of(float x) {
  if (x != x) return 0u;
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Inclusive sums over the workgroup of one value per thread, and their total.
__device__ __forceinline__ int scan_block(int v, int* s_wave, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int incl = wave_incl_scan_i(v);
  __syncthreads();
  if (lane == 63) s_wave[wave] = incl;
  __syncthreads();
  int before = 0;
  total = 0;
  for (int w = 0; w < kThreads / 64; ++w) {
    const int t = s_wave[w];
    if (w < wave) before += t;
    total += t;
  }
  return before + incl;
}

__global__ __launch_bounds__(kThreads) void evict_select_kernel(EvictArgs a) {
  __shared__ int s_hist[kBins];
  __shared__ int s_wave[kThreads / 64];
  __shared__ uint32_t s_prefix;
  __shared__ int s_need;
  const int tid = threadIdx.x;
  const int g = blockIdx.x % a.h_kv, s = blockIdx.x / a.h_kv;
  const int cap = a.pages.cap();
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

  // the want-th largest key; s_need counts how many equal to it are kept
  uint32_t prefix = 0, mask = 0;
  int need = want;
  const int shifts[3] = {21, 10, 0}, bits[3] = {11, 11, 10};
  if (want > 0) {
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = shifts[pass], bins = 1 << bits[pass];
      for (int i = tid; i < bins; i += kThreads) s_hist[i] = 0;
      __syncthreads();
      for (int t = f0 + tid; t < f1; t += kThreads) {
        const uint32_t u = key_of(acc[t]);
        if ((u & mask) == prefix) atomicAdd(&s_hist[(u >> shift) & (bins - 1)], 1);
      }
      __syncthreads();
      // bins from the top, two (or one) a thread
      const int per = bins / kThreads;
      int c[2] = {0, 0}, mine = 0;
      for (int e = 0; e < per; ++e) mine += c[e] = s_hist[bins - 1 - (tid * per + e)];
      int total;
      const int incl = scan_block(mine, s_wave, total);
      int above = incl - mine;
      for (int e = 0; e < per; ++e) {
        if (above < need && need <= above + c[e]) {
          s_prefix = prefix | (uint32_t)(bins - 1 - (tid * per + e)) << shift;
          s_need = need - above;
        }
        above += c[e];
      }
      __syncthreads();
      prefix = s_prefix;
      need = s_need;
      mask |= (uint32_t)(bins - 1) << shift;
      __syncthreads();
    }
  }
  // kept tokens in order: larger ones, and the first `need` equal ones
  for (int j = tid; j < a.n_sink; j += kThreads) {
    idx[j] = j;
    acc_out[j] = acc[j];
  }
  for (int j = tid; j < a.n_recent; j += kThreads) {
    idx[keep - a.n_recent + j] = f1 + j;
    acc_out[keep - a.n_recent + j] = acc[f1 + j];
  }
  if (want == 0) return;
  int larger = 0, equal = 0;                   // among the tokens before this step
  for (int base = f0; base < f1; base += kThreads) {
    const int t = base + tid;
    const float x = t < f1 ? acc[t] : 0.f;
    const uint32_t u = key_of(x);
    const bool gt = t < f1 && u > prefix, eq = t < f1 && u == prefix;
    int total;
    const int incl = scan_block((gt ? 1 : 0) | (eq ? 1 << 16 : 0), s_wave, total);
    const int l = larger + (incl & 0xffff) - (gt ? 1 : 0);
    const int e = equal + (incl >> 16) - (eq ? 1 : 0);
    if (gt || (eq && e < need)) {
      const int j = a.n_sink + l + min(e, need);
      idx[j] = t;
      acc_out[j] = x;
    }
    larger += total & 0xffff;
    equal += total >> 16;
  }
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
  hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)a.n_seq * (unsigned)a.h_kv),
                     dim3(kThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t work = (int64_t)a.budget * (a.d / 8);
  hipLaunchKernelGGL(evict_move_kernel,
                     dim3((unsigned)((work + 255) / 256), (unsigned)a.h_kv, (unsigned)a.n_seq),
                     dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace paged
}  // namespace spot
