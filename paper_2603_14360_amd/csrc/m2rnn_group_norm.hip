// Group norm of a token's channels with an activation, channels last.  x [B,T,D] in G groups of L = D / G
// neighbouring channels, every token and group on its own:
//     mu = mean x (0 unless centred),  s = 1 / sqrt(mean (x - mu)^2 + eps),  xh = (x - mu) s,  n = w xh + b
//     out = n,  SiLU(n)  or  n SiLU(a)
// backward, with dn the gradient of n:
//     p = w dn,  dx = s (p - mean p [centred] - xh mean(p xh)),  da = dout n SiLU'(a)
//     dw = sum over tokens of dn xh,  db = sum over tokens of dn
// One pass over the tensors: a group's channels stay in registers between its sums and its outputs, and the
// backward takes the statistics again from the x that it reads anyway, so none are kept.
//
// Layout.  A lane holds eight neighbouring channels.  A group is P lanes, P the power of two that holds its
// L / 8 vectors (groups above 512 channels: a wave, NV vectors a lane), so that its sums are log2 P lane
// exchanges and never cross a wave.  The lanes of a token's groups lie side by side; a workgroup of 256 takes
// as many tokens as fit, or one of several slices of a wide token, and walks over the tokens in steps: a
// thread's channels stay the same, and dw, db stay in its registers until the end.
#include "m2rnn_block.hpp"

#include <algorithm>

namespace m2rnn {
namespace {

constexpr int kThreads = 256;
// most partial rows of dw, db; with one slice per token four workgroups per CU, which in bf16 all run at once (fp32: three)
constexpr int kRows = 1024;

struct NormPlan {
  int L, LV;     // channels and vectors of a group
  int slots;     // lanes of a token (P per group)
  int slices;    // workgroups side by side for one token
  int tokens;    // tokens side by side in a workgroup
};
inline NormPlan norm_plan(int D, int G, int P) {
  NormPlan p;
  p.L = D / G;
  p.LV = p.L / 8;
  p.slots = G * P;
  p.slices = (p.slots + kThreads - 1) / kThreads;
  p.tokens = p.slices > 1 ? 1 : kThreads / p.slots;
  return p;
}

template <int P>
__device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
  for (int m = 1; m < P; m *= 2) x += __shfl_xor(x, m, 64);
  return x;
}

// Where a thread stands: its token within a step, its group and first vector, and whether it has any.
template <int P>
struct Place {
  int sub, vec;
  bool on;
  size_t chan;
  __device__ __forceinline__ Place(const NormPlan &p, int G, int slice) {
    const int i = threadIdx.x;
    sub = p.slices > 1 ? 0 : i / p.slots;
    const int slot = p.slices > 1 ? slice * kThreads + i : i - sub * p.slots;
    const int g = slot / P;
    vec = slot % P;
    on = sub < p.tokens && g < G;
    chan = (size_t)(on ? g : 0) * p.L;
  }
};

// mu and s of the group whose channels a lane holds in x (absent ones: have[q] false); x becomes x - mu
template <int P, int NV>
__device__ __forceinline__ float centre_and_scale(float (&x)[NV][8], const bool (&have)[NV], int L, bool center,
                                                  float eps) {
  const float inv = 1.f / (float)L;
  if (center) {
    float m = 0.f;
#pragma unroll
    for (int q = 0; q < NV; ++q)
#pragma unroll
      for (int i = 0; i < 8; ++i) m += have[q] ? x[q][i] : 0.f;
    m = lanes_sum<P>(m) * inv;
#pragma unroll
    for (int q = 0; q < NV; ++q)
#pragma unroll
      for (int i = 0; i < 8; ++i) x[q][i] -= m;
  }
  float ss = 0.f;
#pragma unroll
  for (int q = 0; q < NV; ++q)
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = have[q] ? fmaf(x[q][i], x[q][i], ss) : ss;
  return 1.f / sqrtf(lanes_sum<P>(ss) * inv + eps);
}

template <typename IO>
__device__ __forceinline__ void load_or(const void *p, size_t e, float other, float (&x)[8]) {
  if (p) Vec8<IO>::load(p, e, x);
  else
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = other;
}

// Memory-bound: 32 768 tokens, 16 groups of 128 with a gate, bf16: 76 us, 5.3 TB/s (the next tokens' loads in flight
// beside these: 75).
template <typename IO, int P, int NV>
__global__ void __launch_bounds__(kThreads) group_norm_fwd_kernel(GroupNormArgs a, NormPlan p) {
  typedef typename Vec8<IO>::Raw Raw;
  const int slice = blockIdx.x % p.slices;
  const Place<P> at(p, a.G, slice);
  const size_t tokens = (size_t)a.B * a.T, step = (size_t)(gridDim.x / p.slices) * p.tokens;
  bool have[NV];
  size_t ch[NV];
  float w[NV][8], b[NV][8];
#pragma unroll
  for (int q = 0; q < NV; ++q) {
    have[q] = at.on && at.vec + P * q < p.LV;
    ch[q] = at.chan + 8 * (size_t)(have[q] ? at.vec + P * q : 0);  // (clamped: loads are unconditional)
    load_or<IO>(a.w, ch[q], 1.f, w[q]);
    load_or<IO>(a.b, ch[q], 0.f, b[q]);
  }
  for (size_t t0 = (size_t)(blockIdx.x / p.slices) * p.tokens; t0 < tokens; t0 += step) {
    const bool in = t0 + at.sub < tokens;
    const size_t row = (in ? t0 + at.sub : tokens - 1) * (size_t)a.D;
    Raw rx[NV], ra[NV];
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      rx[q] = Vec8<IO>::load_raw(a.x, row + ch[q]);
      if (a.a) ra[q] = Vec8<IO>::load_raw(a.a, row + ch[q]);
    }
    float x[NV][8];
#pragma unroll
    for (int q = 0; q < NV; ++q) Vec8<IO>::widen(rx[q], x[q]);
    const float s = centre_and_scale<P, NV>(x, have, p.L, a.center, a.eps);
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      float o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = fmaf(w[q][i], x[q][i] * s, b[q][i]);
      if (a.silu)
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] *= sigmoidf_(o[i]);
      if (a.a) {
        float z[8];
        Vec8<IO>::widen(ra[q], z);
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] *= z[i] * sigmoidf_(z[i]);
      }
      if (in && have[q]) Vec8<IO>::store(a.out, row + ch[q], o);
    }
  }
}

// Partial sums of dw and db: part[walker][2 D], columns d and D + d.  Memory-bound: 123 us on the forward's sizes,
// 5.5 TB/s (with the next tokens' loads in flight 158: it spills).
template <typename IO, int P, int NV>
__global__ void __launch_bounds__(kThreads) group_norm_bwd_kernel(GroupNormArgs a, NormPlan p) {
  typedef typename Vec8<IO>::Raw Raw;
  const int slice = blockIdx.x % p.slices, walker = blockIdx.x / p.slices;
  const Place<P> at(p, a.G, slice);
  const size_t tokens = (size_t)a.B * a.T, step = (size_t)(gridDim.x / p.slices) * p.tokens;
  bool have[NV];
  size_t ch[NV];
  float w[NV][8], b[NV][8], dw[NV][8], db[NV][8];
#pragma unroll
  for (int q = 0; q < NV; ++q) {
    have[q] = at.on && at.vec + P * q < p.LV;
    ch[q] = at.chan + 8 * (size_t)(have[q] ? at.vec + P * q : 0);
    load_or<IO>(a.w, ch[q], 1.f, w[q]);
    load_or<IO>(a.b, ch[q], 0.f, b[q]);
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[q][i] = db[q][i] = 0.f;
  }
  const float inv = 1.f / (float)p.L;
  for (size_t t0 = (size_t)walker * p.tokens; t0 < tokens; t0 += step) {
    const bool in = t0 + at.sub < tokens;
    const size_t row = (in ? t0 + at.sub : tokens - 1) * (size_t)a.D;
    Raw rx[NV], ra[NV], rd[NV];
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      rx[q] = Vec8<IO>::load_raw(a.x, row + ch[q]);
      rd[q] = Vec8<IO>::load_raw(a.dout, row + ch[q]);
      if (a.a) ra[q] = Vec8<IO>::load_raw(a.a, row + ch[q]);
    }
    float x[NV][8], d[NV][8];
#pragma unroll
    for (int q = 0; q < NV; ++q) Vec8<IO>::widen(rx[q], x[q]);
    const float s = centre_and_scale<P, NV>(x, have, p.L, a.center, a.eps);
    float m1 = 0.f, m2 = 0.f;
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      Vec8<IO>::widen(rd[q], d[q]);
      const bool on = in && have[q];
      float z[8], da[8];
      if (a.a) Vec8<IO>::widen(ra[q], z);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[q][i] *= s;  // xh
        const float n = fmaf(w[q][i], x[q][i], b[q][i]);
        if (a.a) {
          const float sg = sigmoidf_(z[i]);
          da[i] = d[q][i] * n * (sg * (1.f + z[i] * (1.f - sg)));
          d[q][i] *= z[i] * sg;
        } else if (a.silu) {
          const float sg = sigmoidf_(n);
          d[q][i] *= sg * (1.f + n * (1.f - sg));
        }
        if (on) {
          dw[q][i] = fmaf(d[q][i], x[q][i], dw[q][i]);
          db[q][i] += d[q][i];
        }
        d[q][i] *= w[q][i];  // p
        m1 += on ? d[q][i] : 0.f;
        m2 = on ? fmaf(d[q][i], x[q][i], m2) : m2;
      }
      if (a.a && on) Vec8<IO>::store(a.da, row + ch[q], da);
    }
    m1 = a.center ? lanes_sum<P>(m1) * inv : 0.f;
    m2 = lanes_sum<P>(m2) * inv;
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      float o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = s * (d[q][i] - m1 - x[q][i] * m2);
      if (in && have[q]) Vec8<IO>::store(a.dx, row + ch[q], o);
    }
  }
  if (!a.part) return;
  // the tokens side by side are added through LDS, vector by vector, in increasing order
  __shared__ float red[kThreads][17];
  float *part = a.part + (size_t)walker * 2 * a.D;
  for (int q = 0; q < NV; ++q) {
    if (p.tokens > 1) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        red[threadIdx.x][i] = dw[q][i];
        red[threadIdx.x][8 + i] = db[q][i];
      }
      __syncthreads();
      if (at.sub == 0)
        for (int u = 1; u < p.tokens; ++u)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            dw[q][i] += red[threadIdx.x + u * p.slots][i];
            db[q][i] += red[threadIdx.x + u * p.slots][8 + i];
          }
    }
    if (at.sub == 0 && have[q])
#pragma unroll
      for (int i = 0; i < 8; i += 4) {
        *(f4_t *)&part[ch[q] + i] = f4_t{dw[q][i], dw[q][i + 1], dw[q][i + 2], dw[q][i + 3]};
        *(f4_t *)&part[a.D + ch[q] + i] = f4_t{db[q][i], db[q][i + 1], db[q][i + 2], db[q][i + 3]};
      }
  }
}

struct NormOut {
  float *dw, *db;
  int D;
  __device__ __forceinline__ void put(int e, float s) const {
    if (e < D) {
      if (dw) dw[e] = s;
    } else if (db) {
      db[e - D] = s;
    }
  }
};

template <typename IO, int P, int NV>
hipError_t go(const GroupNormArgs &a, bool bwd, hipStream_t s) {
  const NormPlan p = norm_plan(a.D, a.G, P);
  const size_t tokens = (size_t)a.B * a.T, steps = (tokens + p.tokens - 1) / p.tokens;
  if (!bwd) {
    if (tokens == 0) return hipSuccess;
    const unsigned walkers = (unsigned)std::min<size_t>(steps, (size_t)(8192 + p.slices - 1) / p.slices);
    hipLaunchKernelGGL((group_norm_fwd_kernel<IO, P, NV>), dim3(walkers * p.slices), dim3(kThreads), 0, s, a, p);
    return hipGetLastError();
  }
  const unsigned walkers = (unsigned)std::min<size_t>(steps, (size_t)(kRows + p.slices - 1) / p.slices);
  if (tokens > 0) {
    hipLaunchKernelGGL((group_norm_bwd_kernel<IO, P, NV>), dim3(walkers * p.slices), dim3(kThreads), 0, s, a, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!a.part) return hipSuccess;
  return ordered_sum(a.part, a.part + (size_t)walkers * 2 * a.D, NormOut{a.dw, a.db, a.D}, 2 * a.D, (int)walkers, s);
}
template <typename IO>
hipError_t pick(const GroupNormArgs &a, bool bwd, hipStream_t s) {
  const int LV = a.D / a.G / 8;
  if (LV <= 1) return go<IO, 1, 1>(a, bwd, s);
  if (LV <= 2) return go<IO, 2, 1>(a, bwd, s);
  if (LV <= 4) return go<IO, 4, 1>(a, bwd, s);
  if (LV <= 8) return go<IO, 8, 1>(a, bwd, s);
  if (LV <= 16) return go<IO, 16, 1>(a, bwd, s);
  if (LV <= 32) return go<IO, 32, 1>(a, bwd, s);
  if (LV <= 64) return go<IO, 64, 1>(a, bwd, s);
  return go<IO, 64, 2>(a, bwd, s);
}

}  // namespace

int group_norm_max_group() { return 64 * 2 * 8; }
size_t group_norm_scratch_bytes(int B, int T, int D) {
  const size_t tokens = (size_t)B * T, rows = std::min<size_t>(tokens, kRows);
  return align256((rows + kSumGroups) * 2 * D * sizeof(float));
}
hipError_t group_norm_fwd(const GroupNormArgs &a, hipStream_t s) {
  return a.io == 0 ? pick<float>(a, false, s) : pick<__hip_bfloat16>(a, false, s);
}
hipError_t group_norm_bwd(const GroupNormArgs &a, hipStream_t s) {
  return a.io == 0 ? pick<float>(a, true, s) : pick<__hip_bfloat16>(a, true, s);
}

}  // namespace m2rnn
