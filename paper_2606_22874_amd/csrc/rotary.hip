// Rotary positions, and the append of rotated keys and of values to a paged cache
// (gfx950).
//
// Pair i of a head, (a, b), becomes amp (a cos - b sin, b cos + a sin) of the angle
// pos f_i: elements i and i + rope_dim / 2, or 2i and 2i + 1 (interleaved); elements
// from rope_dim on are copied.  The sines and cosines of a row are computed once
// (angle and reduction in FP64, rope_sincos) into LDS and used by all its heads.
// Every element is read and written once, so memory bounds it; a row's heads of
// q, k and v are taken two 16-byte chunks a thread, eight (d = 128) or four threads a
// head.  8000 new tokens of 64 + 8 + 8 heads of 128, 314 MB read and written: 64 us,
// 4.9 TB/s, what a copy reaches; a decode step of 8 tokens 6 us between replayed
// launches, 4.5 of them the kernel: its chain of lengths, page, sines and stores.
// With positions of several axes a pair's angle is pos[axis of the pair] f_i: three axes, 12001
// tokens of 32 heads of 64, 98 MB, 20.6 us, 4.8 TB/s.
#include "rotary_core.h"

namespace spot {
namespace paged {
namespace {

using namespace rot;

template <class T, bool VEC, bool IL>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a) {
  rotate_row<T, VEC, IL, false, false>(a, blockIdx.x);
}
// Positions of several axes.
template <class T, bool VEC, bool IL>
__global__ __launch_bounds__(kThreads) void axes_kernel(RotaryArgs a) {
  rotate_row<T, VEC, IL, true, false>(a, blockIdx.x);
}

template <class T>
void launch(const RotaryArgs& a, bool vec, bool il, hipStream_t s) {
  auto f = vec ? (il ? rotary_kernel<T, true, true> : rotary_kernel<T, true, false>)
               : (il ? rotary_kernel<T, false, true> : rotary_kernel<T, false, false>);
  auto g = vec ? (il ? axes_kernel<T, true, true> : axes_kernel<T, true, false>)
               : (il ? axes_kernel<T, false, true> : axes_kernel<T, false, false>);
  hipLaunchKernelGGL(a.n_axes > 0 ? g : f, dim3((unsigned)a.rows), dim3(kThreads), 0, s, a);
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, int dtype, bool interleaved, hipStream_t s) {
  if (!launchable(a.rows, kThreads)) return hipErrorInvalidConfiguration;
  auto whole = [](const void* p, int64_t stride) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0;
  };
  bool vec = a.d % 16 == 0 && a.rope_dim % 16 == 0 && whole(a.q, a.q_stride) &&
             whole(a.q_out, a.out_stride);
  if (a.seq_start)
    vec = vec && whole(a.k, a.k_stride) && whole(a.v, a.v_stride) && whole(a.k_pages, 0) &&
          whole(a.v_pages, 0);
  dtype == SPOT_DTYPE_BF16 ? launch<Bf16>(a, vec, interleaved, s)
                           : launch<Fp16>(a, vec, interleaved, s);
  return hipGetLastError();
}

}  // namespace paged
}  // namespace spot
