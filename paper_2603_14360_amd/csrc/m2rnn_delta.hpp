// Internal declarations of the gated delta rule: arguments, the layout of checkpoints and workspace, and
// device code that its kernels share.
//
// The rule, for every batch row and head on its own, with a state H of K x V:
//     Hd_t = e^{g_t} H_{t-1},   u_t = beta_t (v_t - Hd_t^T k_t),   H_t = Hd_t + k_t u_t^T,   y_t = H_t^T q_t.
// By chunks of C steps (G_i the sum of g over the chunk's steps up to i, H the state in front of the chunk,
// rows of Q, K, V, U, Y the chunk's vectors):
//     A_ij = beta_i e^{G_i - G_j} k_i.k_j  (j < i),   T = (I + A)^{-1},   P_ij = e^{G_i - G_j} q_i.k_j  (j <= i)
//     U = T diag(beta) (V - diag(e^G) K H)
//     Y = diag(e^G) Q H + P U,        H <- e^{G_C} H + K^T diag(e^{G_C - G}) U
// and back, with dH the gradient of the state behind the chunk:
//     Z = T^T (P^T dY + diag(e^{G_C - G}) K dH),   dV = diag(beta) Z
//     dH <- e^{G_C} dH + Q^T diag(e^G) dY - K^T diag(beta e^G) Z
//     S1 = (dY U^T) masked and times e^{G_i - G_j} as P,  S2 = (Z U^T) likewise, strictly lower
//     dQ = diag(e^G) dY H^T + S1 K
//     a  = -diag(e^G) Z H^T - S2 K                        what k_i gets as the one that asks, over beta_i
//     c  = diag(e^{G_C - G}) U dH^T + S1^T Q - S2^T diag(beta) K        what k_j gets as the one that is kept
//     dK = diag(beta) a + c,   dbeta_i = Z_i.v_i + k_i.a_i
//     dg_i = sum over j >= i of (q_j.dq_j + beta_j k_j.a_j - k_j.c_j)  + <H_C, dH>,  H_C the state behind
// (every exponent that appears belongs to a span of steps, so with g <= 0 no factor exceeds one).
//
// T and P depend on nothing that is carried: one launch forms them for all chunks at once; only the lines
// with H and dH run in order, and those are independent for every column block of V; the rest of the
// backward is again one launch over all chunks.
#pragma once
#include "m2rnn_io.hpp"
#include "m2rnn_kernels.hpp"
#include "m2rnn_mfma_common.hpp"

namespace m2rnn {

struct DeltaArgs {
  int B, T, N, Nqk, K, V, io;
  const void *q, *k, *v;
  const float *g, *beta, *H0;
  void *y;
  float *HT;
  char *ckpt;  // states in front of the chunks, and U; null: not wanted (forward)
  int write_y;
  // backward (own_ckpt: `ckpt` is room for the checkpoints, to be made first)
  int own_ckpt;
  const void *dy;
  const float *dHT;
  void *dq, *dk, *dv, *dg, *dbeta;
  float *dH0;
  char *ws;
};

// Sizes in bytes (multiples of 256) of the parts of the scratch and of the checkpoints of a chunked call.
struct DeltaLayout {
  int C, chunks;
  bool kept;      // gates, T and P are kept with the checkpoints
  size_t gates;   // per unit and chunk: e^G, e^{G_C - G}, and G / ln 2 as a sum of two floats, C each
  size_t mats;    // T and P of every chunk
  size_t carry;   // the states between the launches of a forward (0: there is one)
  size_t states;  // one state per chunk
  size_t rows;    // U or Z of every step
  size_t exps;    // with the checkpoints: the powers of two of states and U (0: none)
  size_t dexps;   // powers of two of the gradients (0: none)
  size_t heads;   // dq or dk of every head in fp32 (0 where no heads share q, k)
};

DeltaLayout delta_f32_layout(const DeltaArgs &a);
hipError_t delta_f32_fwd(const DeltaArgs &a, hipStream_t s);
hipError_t delta_f32_bwd(const DeltaArgs &a, hipStream_t s);

// bf16 io with K, V >= 32: chunks of 64 on the fp16 matrix instructions
bool delta_half_serves(int K, int V, int io);
DeltaLayout delta_half_layout(const DeltaArgs &a);
hipError_t delta_half_fwd(const DeltaArgs &a, hipStream_t s);
hipError_t delta_half_bwd(const DeltaArgs &a, hipStream_t s);

// The recurrence step by step, the state in registers: serving, and segments of a few steps.
// Up to how many steps that is the faster way.
int delta_step_most(double states, int K, int V);
hipError_t delta_step_fwd(const DeltaArgs &a, hipStream_t s);

constexpr float kLog2e = 1.4426950408889634f;

// 2^x on the hardware's instruction (1 ulp; results below 2^-126 are zero)
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// Running sum of g over a chunk, lane i of a wave holding step i's, over ln 2 and as hi + lo: the exponents
// of a chunk are differences of these sums, which in one float would be off by 2^-24 of the larger one.
// g = -inf (a reset) counts as -1e4, whose exponential is zero as well.
struct GateSum {
  float hi, lo;
};
__device__ __forceinline__ GateSum gate_sum(float g) {
  const int lane = threadIdx.x & 63;
  double s = g < -1e4f ? -1e4 : (double)g;
  s *= 1.4426950408889634074;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const double o = __shfl_up(s, d, 64);
    if (lane >= d) s += o;
  }
  GateSum r;
  r.hi = (float)s;
  r.lo = (float)(s - (double)r.hi);
  return r;
}

// Workgroups are dealt to the 8 XCDs in turn: the `parts` workgroups of a unit get ids that are equal
// modulo 8 and so one L2, which then serves all but the first read of q, k, T and P.
__device__ __forceinline__ bool delta_map(int units, int parts, int &unit, int &part) {
  const int xcd = blockIdx.x & 7, r = blockIdx.x >> 3;
  part = r % parts;
  unit = xcd + 8 * (r / parts);
  return unit < units;
}
inline unsigned delta_grid(int units, int parts) { return 8u * (unsigned)parts * (unsigned)((units + 7) / 8); }

}  // namespace m2rnn
