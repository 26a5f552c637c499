// Attention of many rows over an 8-bit paged cache (gfx950), the instances with sinks: see
// attend_many_core.h.
#include "attend_many_core.h"

namespace spot {
namespace paged {
namespace {

using namespace many;

template <class T, int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(64 * kWaves) void sinks8_many_kernel(AttendArgs a) {
  attend_many<T, D, CAP, BIAS, true, true>(a);
}

template <class T, int D>
void launch(const AttendArgs& a, dim3 grid, hipStream_t s) {
  // the plain form takes maxima before it scales: it needs a positive scale
  const bool cap = a.rule.cap > 0.f;
  const bool bias = a.rule.slopes || (!cap && !(a.rule.scale * kLog2e > 1e-6f));
  auto f = cap ? (bias ? sinks8_many_kernel<T, D, true, true>
                       : sinks8_many_kernel<T, D, true, false>)
               : (bias ? sinks8_many_kernel<T, D, false, true>
                       : sinks8_many_kernel<T, D, false, false>);
  hipLaunchKernelGGL(f, grid, dim3(64 * kWaves), 0, s, a);
}

}  // namespace

hipError_t launch_sinks_many8(AttendArgs a, int dtype, int d, void* ws, hipStream_t s) {
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
