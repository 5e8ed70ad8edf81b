// Gated delta rule step by step (m2rnn_delta.hpp): a token of serving, and segments of a few steps.
//
// A workgroup owns VB columns of one state, spread over its threads as 16-byte pieces of rows.  Both
// products with the state of a step are taken from the decayed state Hd before its update,
//     y = H^T q = Hd^T q + (k.q) u,     u = beta (v - Hd^T k),
// so that a step is one pass over the registers, one sum over the rows (lanes, then waves through LDS)
// and one barrier.  In front of and behind the steps the state makes one trip through memory, which is what
// bounds a large batch; a small one is bound by the launch.
#include "m2rnn_delta.hpp"

namespace m2rnn {
namespace {

template <typename IO, int K, int VB>
struct Step {
  static constexpr int LPR = VB / 4;                                     // lanes per row piece
  static constexpr int THREADS = K * LPR < 256 ? K * LPR : 256;
  static constexpr int RS = THREADS / LPR;                               // rows side by side
  static constexpr int R = K / RS;                                       // rows per thread
  static constexpr int WAVES = (THREADS + 63) / 64;
};

template <typename IO, int K, int VB>
__global__ void __launch_bounds__(256) delta_step_kernel(DeltaArgs a) {
  using S = Step<IO, K, VB>;
  constexpr int LPR = S::LPR, R = S::R, W = S::WAVES;
  __shared__ f4_t red[2][W][2][LPR];
  __shared__ float redkq[2][W];
  const int parts = a.V / VB, unit = blockIdx.x / parts, part = blockIdx.x - unit * parts;
  const int b = unit / a.N, n = unit - b * a.N, nq = n / (a.N / a.Nqk);
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, cl = threadIdx.x % LPR, rl = threadIdx.x / LPR;
  const size_t h0 = (size_t)unit * K * a.V + part * VB + 4 * cl;
  f4_t H[R];
#pragma unroll
  for (int r = 0; r < R; ++r)
    H[r] = a.H0 ? *(const f4_t *)(a.H0 + h0 + (size_t)(rl + r * S::RS) * a.V) : f4_t{0.f, 0.f, 0.f, 0.f};
  for (int t = 0; t < a.T; ++t) {
    const size_t bt = (size_t)b * a.T + t, qe = (bt * a.Nqk + nq) * K, ve = (bt * a.N + n) * a.V + part * VB + 4 * cl;
    const float gate = __expf(a.g[bt * a.N + n]), beta = a.beta[bt * a.N + n];
    float q[R], k[R], v[4];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      q[r] = to_f32<IO>(((const IO *)a.q)[qe + rl + r * S::RS]);
      k[r] = to_f32<IO>(((const IO *)a.k)[qe + rl + r * S::RS]);
    }
    Vec4<IO>::widen(Vec4<IO>::load_raw(a.v, ve), v);
    f4_t kh = {0.f, 0.f, 0.f, 0.f}, qh = kh;
    float kq = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      H[r] *= gate;
      kh += k[r] * H[r];
      qh += q[r] * H[r];
      kq = fmaf(k[r], q[r], kq);
    }
    // over the rows of the wave; k.q likewise (every column of lanes holds all of it)
#pragma unroll
    for (int d = LPR; d < 64 && d < S::THREADS; d *= 2) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        kh[x] += __shfl_xor(kh[x], d, 64);
        qh[x] += __shfl_xor(qh[x], d, 64);
      }
      kq += __shfl_xor(kq, d, 64);
    }
    if constexpr (W > 1) {
      const int p = t & 1;
      if (lane < LPR) {
        red[p][wv][0][lane] = kh;
        red[p][wv][1][lane] = qh;
        if (lane == 0) redkq[p][wv] = kq;
      }
      __syncthreads();  // (the other parity's words are free again: every wave has read them)
      kh = red[p][0][0][cl];
      qh = red[p][0][1][cl];
      kq = redkq[p][0];
#pragma unroll
      for (int w = 1; w < W; ++w) {
        kh += red[p][w][0][cl];
        qh += red[p][w][1][cl];
        kq += redkq[p][w];
      }
    }
    f4_t u;
#pragma unroll
    for (int x = 0; x < 4; ++x) u[x] = beta * (v[x] - kh[x]);
#pragma unroll
    for (int r = 0; r < R; ++r) H[r] += k[r] * u;
    if (threadIdx.x < LPR) {
      float y[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) y[x] = fmaf(kq, u[x], qh[x]);
      Vec4<IO>::store(a.y, ve, y);
    }
  }
  if (a.HT)
#pragma unroll
    for (int r = 0; r < R; ++r) *(f4_t *)(a.HT + h0 + (size_t)(rl + r * S::RS) * a.V) = H[r];
}

// Columns of V per workgroup: 32, a cache line of a row; 64 where that still fills the chip, which reads longer
// stretches (4096 states of 128 x 128: 103.0 -> 100.5 us, 5.4 TB/s; a multiply-copy reaches 6.1).
template <typename IO, int K>
hipError_t go(const DeltaArgs &a, hipStream_t s) {
  const unsigned units = (unsigned)(a.B * a.N);
  if (a.V == 16)
    hipLaunchKernelGGL((delta_step_kernel<IO, K, 16>), dim3(units), dim3(Step<IO, K, 16>::THREADS), 0, s, a);
  else if (a.V % 64 == 0 && units * (a.V / 64) >= 512)
    hipLaunchKernelGGL((delta_step_kernel<IO, K, 64>), dim3(units * (a.V / 64)), dim3(Step<IO, K, 64>::THREADS), 0, s, a);
  else
    hipLaunchKernelGGL((delta_step_kernel<IO, K, 32>), dim3(units * (a.V / 32)), dim3(Step<IO, K, 32>::THREADS), 0, s, a);
  return hipGetLastError();
}
template <typename IO>
hipError_t pick(const DeltaArgs &a, hipStream_t s) {
  switch (a.K) {
    case 16: return go<IO, 16>(a, s);
    case 32: return go<IO, 32>(a, s);
    case 64: return go<IO, 64>(a, s);
    default: return go<IO, 128>(a, s);
  }
}

}  // namespace

// Up to how many steps a forward without checkpoints runs here rather than by chunks, which hardly depend on how many
// they are.  A step costs 0.85 us, or what the workgroups that do not fit on the chip at once make of it: about as
// much for small heads as for large ones, whose chunks cost more.  us of 6, 8, 12 and 16 steps here | by chunks:
//     bf16   32 states of 128 x 128   7.6   9.3  12.7  16.3 |  13.4        fp32     7.6   9.1  12.5  16.0 |  14.9
//          1024 of 128 x 128         30.7  36.2  46.0  57.5 |  65                  31.5  37.1  47.3  58.7 | 115
//           256 of 64 x 64            8.7  10.6  14.6  18.5 |  14.5                 8.7  10.6  14.5  18.3 |  17
//          1024 of 32 x 32           12.5  16.1  22.3  28.8 |  20                  12.6  16.2  22.6  29.2 |  18.4
//          5376 of 64 x 16           61.8  80.8 119   158   |  66                  61.9  80.8 119   158   |  65
int delta_step_most(double states, int K, int V) {
  if (K >= 32 && K * V <= 1024) return states <= 512 ? 12 : states <= 2048 ? 8 : 6;
  return K >= 32 && V >= 64 && states * K * V >= 1 << 22 ? 16 : 12;
}
hipError_t delta_step_fwd(const DeltaArgs &a, hipStream_t s) {
  return a.io == 0 ? pick<float>(a, s) : pick<__hip_bfloat16>(a, s);
}

}  // namespace m2rnn
