// What the block's kernels (convolution, norms) share: the sigmoid and the ordered sum of partial rows.
#pragma once
#include "m2rnn_io.hpp"
#include "m2rnn_kernels.hpp"
#include "m2rnn_mfma_common.hpp"

namespace m2rnn {
namespace {

// 1 / (1 + e^-u) on the hardware's exp2 and reciprocal (1 ulp each; e^-u = inf gives 0)
__device__ __forceinline__ float sigmoidf_(float u) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * u));
}

// Ordered sum of R partial rows of E floats.  A workgroup adds up to 32 columns with 32 walkers
// (rows wl, wl + 32, ..., four loads in flight) and the walkers in LDS.  Up to kDirectRows rows
// that is all; more are first added in groups of about kDirectRows / 4 (blockIdx.y) into rows
// of `lvl` (kSumGroups rows behind the partials).  What bounds it is the chain of dependent
// loads: 128 rows of 7360 took two launches, some 13 us, with one column per thread; 4.7 us now.
constexpr int kSumGroups = 32;
constexpr int kDirectRows = 512;

// (Out::put(e, sum of column e))
template <typename Out>
__global__ void __launch_bounds__(1024)
    ordered_sum_kernel(const float *__restrict__ part, float *__restrict__ lvl, Out out, int E, int R) {
  const int e = blockIdx.x * 32 + (threadIdx.x & 31), per = (R + gridDim.y - 1) / gridDim.y;
  const int r0 = blockIdx.y * per, r1 = r0 + per < R ? r0 + per : R;
  const float t = column_sum(part, E, e, r0, r1);
  if (threadIdx.x < 32 && e < E) {
    if (gridDim.y > 1) lvl[(size_t)blockIdx.y * E + e] = t;
    else out.put(e, t);
  }
}
template <typename Out>
hipError_t ordered_sum(const float *part, float *lvl, const Out &out, int E, int R, hipStream_t s) {
  const int bx = (E + 31) / 32;
  if (R > kDirectRows) {
    const int want = (R + kDirectRows / 4 - 1) / (kDirectRows / 4), G = want < kSumGroups ? want : kSumGroups;
    hipLaunchKernelGGL(ordered_sum_kernel<Out>, dim3(bx, G), dim3(1024), 0, s, part, lvl, out, E, R);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    part = lvl;
    R = G;
  }
  hipLaunchKernelGGL(ordered_sum_kernel<Out>, dim3(bx, 1), dim3(1024), 0, s, part, lvl, out, E, R);
  return hipGetLastError();
}

}  // namespace
}  // namespace m2rnn
