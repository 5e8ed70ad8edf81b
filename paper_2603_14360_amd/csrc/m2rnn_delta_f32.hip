// Gated delta rule, chunks of 32 steps, everything in fp32 on the fp32 matrix instructions (16x16x4): the
// kernels of fp32 io.  The lines of the rule by chunks stand in m2rnn_delta.hpp.
//
//   delta_prep_kernel   one workgroup per chunk: gates, T and P                     -> checkpoints or workspace
//   delta_fwd_kernel    one workgroup per state and 16 columns of V, chunks in order -> y, HT, (H, U)
//   delta_bwd_kernel    the same, backwards                                          -> dv, dH0, dH and Z
//   delta_grad_kernel   one workgroup per chunk: S1, S2 and what follows             -> dq, dk, dg, dbeta
//
// Products are D = A B^T on 16 x 16 tiles with both operands' rows contiguous along the contraction: a lane
// reads four consecutive elements of row (lane % 16) at 4 (lane / 16), which are the operands of four
// instructions, and of D it holds rows 4 (lane / 16) .. + 3 of column lane % 16.  Which of two factors is A is
// free; it is chosen so that those four are neighbours where D goes next.
//
// Chunks of 32 and not 64, because q, k and their transposes of a chunk lie in LDS: 81 KB at K = 128.
//
// What bounds them is the latency of a chunk's dependent products; 16 columns a workgroup make the chains as many as
// there can be.  4 x 512 steps, 8 heads of 32 x 32, fp32: T and P 9 us, forward 24, backward 31 (1.5 and 1.9 a chunk on
// 64 workgroups), gradients 12.
#include "m2rnn_delta.hpp"

namespace m2rnn {
namespace {

constexpr int C = 32;
constexpr int VB = 16;       // columns of V per workgroup of the kernels that run in order
constexpr int LC = C + 4;    // floats per row of an LDS array with a chunk's steps side by side (16-byte rows)

__device__ __forceinline__ f4_t mma(f4_t a, f4_t b, f4_t c) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
  return c;
}
// acc += A B^T over n (a multiple of 16) elements; a, b point at the lane's row and first element
__device__ __forceinline__ f4_t mma_rows(const float *a, const float *b, int n, f4_t acc) {
#pragma unroll 4
  for (int i = 0; i < n; i += 16) acc = mma(*(const f4_t *)(a + i), *(const f4_t *)(b + i), acc);
  settle(acc);
  return acc;
}
template <typename IO>
__device__ __forceinline__ f4_t load4(const void *p, size_t e, bool ok) {
  float x[4];
  Vec4<IO>::widen(Vec4<IO>::load_raw(p, ok ? e : 0), x);
  return ok ? f4_t{x[0], x[1], x[2], x[3]} : f4_t{0.f, 0.f, 0.f, 0.f};
}
template <typename IO>
__device__ __forceinline__ void store4(void *p, size_t e, f4_t v) {
  const float x[4] = {v[0], v[1], v[2], v[3]};
  Vec4<IO>::store(p, e, x);
}

struct Ws {  // device pointers into the workspace
  float *gates, *mats, *states, *rows, *dqh, *dkh;
};

// ------------------------------------------------------------------ gates, T, P of one chunk
template <typename IO>
__global__ void __launch_bounds__(256, 2) delta_prep_kernel(DeltaArgs a, int chunks, float *__restrict__ gates,
                                                         float *__restrict__ mats) {
  __shared__ __align__(16) float A[C][C + 4];
  __shared__ float hi[C], lo[C], be[C];
  const int unit = blockIdx.x / chunks, ch = blockIdx.x - unit * chunks;
  const int b = unit / a.N, n = unit - b * a.N, nq = n / (a.N / a.Nqk);
  const int t0 = ch * C, lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float *gt = gates + (size_t)blockIdx.x * 4 * C;
  float *Tm = mats + (size_t)blockIdx.x * 2 * C * C, *Pm = Tm + C * C;
  // tile (r, c) of K K^T and of Q K^T: wave 2 r + c
  const int r = wv >> 1, c = wv & 1, l16 = lane & 15, g4 = lane >> 4;
  const size_t row = (size_t)a.Nqk * a.K, base = ((size_t)b * a.T + t0) * row + (size_t)nq * a.K + 4 * g4;
  const int ti = 16 * r + l16, tj = 16 * c + l16;
  const bool iok = t0 + ti < a.T, jok = t0 + tj < a.T;
  f4_t kk = {0.f, 0.f, 0.f, 0.f}, qk = kk;
  for (int e = 0; e < a.K; e += 16) {  // D[j][i] with A = rows j: a lane holds four j of one i
    const f4_t kj = load4<IO>(a.k, base + tj * row + e, jok);
    kk = mma(kj, load4<IO>(a.k, base + ti * row + e, iok), kk);
    qk = mma(kj, load4<IO>(a.q, base + ti * row + e, iok), qk);
  }
  settle(kk);
  settle(qk);
  if (wv == 0) {
    const bool in = lane < C && t0 + lane < a.T;
    const size_t e = ((size_t)b * a.T + (in ? t0 + lane : 0)) * a.N + n;
    const GateSum G = gate_sum(in ? a.g[e] : 0.f);
    const float ghi = __shfl(G.hi, C - 1, 64), glo = __shfl(G.lo, C - 1, 64);
    if (lane < C) {
      hi[lane] = G.hi;
      lo[lane] = G.lo;
      be[lane] = in ? a.beta[e] : 0.f;
      gt[lane] = exp2_(G.hi) * exp2_(G.lo);
      gt[C + lane] = exp2_((ghi - G.hi) + (glo - G.lo));
      gt[2 * C + lane] = G.hi;
      gt[3 * C + lane] = G.lo;
    }
  }
  __syncthreads();
  f4_t p;
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const int i = ti, j = 16 * c + 4 * g4 + x;
    const float e = exp2_((hi[i] - hi[j]) + (lo[i] - lo[j]));
    p[x] = j <= i ? e * qk[x] : 0.f;
    A[i][j] = j < i ? be[i] * e * kk[x] : 0.f;
  }
  *(f4_t *)&Pm[ti * C + 16 * c + 4 * g4] = p;
  __syncthreads();
  // (I + A)^{-1} column by column: row i is e_i less the rows above it times A's row i
  if (threadIdx.x < C) {
    float x[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
      float s[4] = {(int)threadIdx.x == i ? 1.f : 0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < i; ++j) s[j & 3] = fmaf(-A[i][j], x[j], s[j & 3]);
      x[i] = (s[0] + s[1]) + (s[2] + s[3]);
    }
#pragma unroll
    for (int i = 0; i < C; ++i) Tm[i * C + threadIdx.x] = x[i];
  }
}

// ------------------------------------------------------------------ staging
// A chunk's rows of q or k: K / 4 x C vectors of four, dealt to 256 threads along a row first.
template <typename IO, int K>
struct Rows {
  static constexpr int PER = (C * K / 4 + 255) / 256;
  f4_t x[PER];
  __device__ __forceinline__ void load(const void *p, size_t base, size_t row, int t0, int T) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = threadIdx.x + 256 * i, t = e / (K / 4), c = e - t * (K / 4);
      x[i] = load4<IO>(p, base + (size_t)(t0 + t) * row + 4 * c, t < C && t0 + t < T);
    }
  }
  __device__ __forceinline__ void pin() {  // (they have arrived here)
#pragma unroll
    for (int i = 0; i < PER; ++i) asm volatile("" : "+v"(x[i]));
  }
  // row-major [C][K + 4] and / or transposed [K][LC]
  __device__ __forceinline__ void store(float *rows, float *cols) const {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = threadIdx.x + 256 * i, t = e / (K / 4), c = e - t * (K / 4);
      if (t < C) {
        if (rows) *(f4_t *)&rows[t * (K + 4) + 4 * c] = x[i];
        if (cols)
#pragma unroll
          for (int u = 0; u < 4; ++u) cols[(4 * c + u) * LC + t] = x[i][u];
      }
    }
  }
};

constexpr int lds_fwd(int K) { return (2 * C * (K + 4) + K * LC + VB * (K + 4) + 3 * VB * LC + 2 * C * LC + 3 * C) * 4; }
constexpr int lds_bwd(int K) { return (C * (K + 4) + 2 * K * LC + VB * (K + 4) + 4 * VB * LC + 2 * C * LC + 3 * C) * 4; }

// ------------------------------------------------------------------ forward, chunks in order
template <typename IO, int K>
__global__ void __launch_bounds__(256, 2)
    delta_fwd_kernel(DeltaArgs a, int chunks, const float *__restrict__ gates, const float *__restrict__ mats,
                     float *__restrict__ states, float *__restrict__ rows_u) {
  constexpr int KT = K / 16, PW = (KT + 3) / 4;  // row tiles of the state; of a wave: wave, wave + 4
  extern __shared__ __align__(16) float lds[];
  float *qs = lds, *ks = qs + C * (K + 4), *kT = ks + C * (K + 4), *Ht = kT + K * LC, *Rt = Ht + VB * (K + 4);
  float *Ut = Rt + VB * LC, *Wt = Ut + VB * LC, *Ts = Wt + VB * LC, *Ps = Ts + C * LC, *ge = Ps + C * LC;
  float *gl = ge + C, *be = gl + C;
  int unit, vb;
  if (!delta_map(a.B * a.N, a.V / VB, unit, vb)) return;
  const int b = unit / a.N, n = unit - b * a.N, nq = n / (a.N / a.Nqk);
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g4 = lane >> 4;
  const size_t qrow = (size_t)a.Nqk * K, qbase = (size_t)b * a.T * qrow + (size_t)nq * K;
  const size_t vrow = (size_t)a.N * a.V, vbase = (size_t)b * a.T * vrow + (size_t)n * a.V + vb * VB + 4 * g4;

  f4_t H[PW];  // rows 16 tile + 4 g4 .., column vb VB + l16
#pragma unroll
  for (int p = 0; p < PW; ++p) {
    const int kt = wv + 4 * p;
#pragma unroll
    for (int x = 0; x < 4; ++x)
      H[p][x] = a.H0 && kt < KT ? a.H0[((size_t)unit * K + 16 * kt + 4 * g4 + x) * a.V + vb * VB + l16] : 0.f;
  }
  // The next chunk's inputs, in flight for a whole chunk and taken before this one's results are stored: the counter
  // that a wait for loads looks at counts stores as well, in order.
  const int tt = 16 * (wv & 1) + l16;
  Rows<IO, K> q, k;
  f4_t tm, pm, nv;
  float gv = 0.f;
  auto fetch = [&](int ch) {
    const int t0 = ch * C;
    const size_t at = (size_t)unit * chunks + ch;
    q.load(a.q, qbase, qrow, t0, a.T);
    k.load(a.k, qbase, qrow, t0, a.T);
    nv = load4<IO>(a.v, vbase + (size_t)(t0 + tt) * vrow, t0 + tt < a.T);
    tm = *(const f4_t *)(mats + at * 2 * C * C + 4 * tid);
    pm = *(const f4_t *)(mats + at * 2 * C * C + C * C + 4 * tid);
    if (tid < 2 * C) gv = gates[at * 4 * C + tid];
    else if (tid < 3 * C) gv = t0 + tid - 2 * C < a.T ? a.beta[((size_t)b * a.T + t0 + tid - 2 * C) * a.N + n] : 0.f;
  };
  auto arrived = [&]() {
    q.pin();
    k.pin();
    asm volatile("" : "+v"(tm), "+v"(pm), "+v"(nv), "+v"(gv));
  };
  if (chunks > 0) {
    fetch(0);
    arrived();
  }
  for (int ch = 0; ch < chunks; ++ch) {
    const int t0 = ch * C;
    q.store(qs, nullptr);
    k.store(ks, kT);
    *(f4_t *)&Ts[(tid >> 3) * LC + 4 * (tid & 7)] = tm;
    *(f4_t *)&Ps[(tid >> 3) * LC + 4 * (tid & 7)] = pm;
    if (tid < 3 * C) ge[tid] = gv;
#pragma unroll
    for (int p = 0; p < PW; ++p) {
      const int kt = wv + 4 * p;
      if (kt < KT) *(f4_t *)&Ht[l16 * (K + 4) + 16 * kt + 4 * g4] = H[p];
    }
    // v of my column of the 16 x 16 tile [V][steps]: wave 0 and 1 the chunk's first and second 16 steps
    const bool tok = t0 + tt < a.T;
    const f4_t v = nv;
    lds_barrier();
    fetch(min(ch + 1, chunks - 1));
    // waves 0, 1: (K H)^T;  waves 2, 3: (Q H)^T
    const f4_t zero = {0.f, 0.f, 0.f, 0.f};
    f4_t xh = mma_rows(Ht + l16 * (K + 4) + 4 * g4, (wv < 2 ? ks : qs) + tt * (K + 4) + 4 * g4, K, zero);
    const float gm = ge[tt];
    if (wv < 2) {
      const float bt = be[tt];
#pragma unroll
      for (int x = 0; x < 4; ++x) Rt[(4 * g4 + x) * LC + tt] = bt * (v[x] - gm * xh[x]);
    }
    lds_barrier();
    f4_t u = zero;
    if (wv < 2) {
      u = mma_rows(Rt + l16 * LC + 4 * g4, Ts + tt * LC + 4 * g4, C, zero);
      const float gt = gl[tt];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        Ut[(4 * g4 + x) * LC + tt] = u[x];
        Wt[(4 * g4 + x) * LC + tt] = gt * u[x];
      }
    }
    lds_barrier();
    if (wv >= 2 && a.write_y) xh = mma_rows(Ut + l16 * LC + 4 * g4, Ps + tt * LC + 4 * g4, C, gm * xh);
    const float gc = ge[C - 1];
    f4_t H0[PW];
#pragma unroll
    for (int p = 0; p < PW; ++p) H0[p] = H[p];
#pragma unroll
    for (int p = 0; p < PW; ++p) {
      const int kt = wv + 4 * p;
      if (kt < KT)
        H[p] = mma_rows(kT + (16 * kt + l16) * LC + 4 * g4, Wt + l16 * LC + 4 * g4, C, gc * H[p]);
    }
    arrived();
    if (tok && wv >= 2 && a.write_y) store4<IO>(a.y, vbase + (size_t)(t0 + tt) * vrow, xh);
    if (tok && wv < 2 && rows_u) *(f4_t *)&rows_u[vbase + (size_t)(t0 + tt) * vrow] = u;
    if (states)
#pragma unroll
      for (int p = 0; p < PW; ++p) {
        const int kt = wv + 4 * p;
        if (kt < KT)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            states[(((size_t)unit * chunks + ch) * K + 16 * kt + 4 * g4 + x) * a.V + vb * VB + l16] = H0[p][x];
      }
    lds_barrier();
  }
  if (a.HT)
#pragma unroll
    for (int p = 0; p < PW; ++p) {
      const int kt = wv + 4 * p;
      if (kt < KT)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          a.HT[((size_t)unit * K + 16 * kt + 4 * g4 + x) * a.V + vb * VB + l16] = H[p][x];
    }
}

// ------------------------------------------------------------------ backward, chunks in reverse order
template <typename IO, int K>
__global__ void __launch_bounds__(256, 2)
    delta_bwd_kernel(DeltaArgs a, int chunks, const float *__restrict__ gates, const float *__restrict__ mats,
                     float *__restrict__ states, float *__restrict__ rows_z) {
  constexpr int KT = K / 16, PW = (KT + 3) / 4;
  extern __shared__ __align__(16) float lds[];
  float *ks = lds, *qT = ks + C * (K + 4), *kT = qT + K * LC, *Ht = kT + K * LC, *Yt = Ht + VB * (K + 4);
  float *Wt = Yt + VB * LC, *Ut = Wt + VB * LC, *Zt = Ut + VB * LC, *Tt = Zt + VB * LC, *Pt = Tt + C * LC;
  float *ge = Pt + C * LC, *gl = ge + C, *be = gl + C;
  int unit, vb;
  if (!delta_map(a.B * a.N, a.V / VB, unit, vb)) return;
  const int b = unit / a.N, n = unit - b * a.N, nq = n / (a.N / a.Nqk);
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g4 = lane >> 4;
  const size_t qrow = (size_t)a.Nqk * K, qbase = (size_t)b * a.T * qrow + (size_t)nq * K;
  const size_t vrow = (size_t)a.N * a.V, vbase = (size_t)b * a.T * vrow + (size_t)n * a.V + vb * VB + 4 * g4;

  f4_t D[PW];
#pragma unroll
  for (int p = 0; p < PW; ++p) {
    const int kt = wv + 4 * p;
#pragma unroll
    for (int x = 0; x < 4; ++x)
      D[p][x] = a.dHT && kt < KT ? a.dHT[((size_t)unit * K + 16 * kt + 4 * g4 + x) * a.V + vb * VB + l16] : 0.f;
  }
  // The next chunk's inputs, in flight for a whole chunk and taken before this one's results are stored: the counter
  // that a wait for loads looks at counts stores as well, in order.
  const int tt = 16 * (wv & 1) + l16;
  Rows<IO, K> q, k;
  f4_t tm, pm, nv;
  float gv = 0.f;
  auto fetch = [&](int ch) {
    const int t0 = ch * C;
    const size_t at = (size_t)unit * chunks + ch;
    q.load(a.q, qbase, qrow, t0, a.T);
    k.load(a.k, qbase, qrow, t0, a.T);
    nv = load4<IO>(a.dy, vbase + (size_t)(t0 + tt) * vrow, t0 + tt < a.T);
    tm = *(const f4_t *)(mats + at * 2 * C * C + 4 * tid);
    pm = *(const f4_t *)(mats + at * 2 * C * C + C * C + 4 * tid);
    if (tid < 2 * C) gv = gates[at * 4 * C + tid];
    else if (tid < 3 * C) gv = t0 + tid - 2 * C < a.T ? a.beta[((size_t)b * a.T + t0 + tid - 2 * C) * a.N + n] : 0.f;
  };
  auto arrived = [&]() {
    q.pin();
    k.pin();
    asm volatile("" : "+v"(tm), "+v"(pm), "+v"(nv), "+v"(gv));
  };
  if (chunks > 0) {
    fetch(chunks - 1);
    arrived();
  }
  for (int ch = chunks - 1; ch >= 0; --ch) {
    const int t0 = ch * C;
    q.store(nullptr, qT);
    k.store(ks, kT);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      Tt[(4 * (tid & 7) + x) * LC + (tid >> 3)] = tm[x];
      Pt[(4 * (tid & 7) + x) * LC + (tid >> 3)] = pm[x];
    }
    if (tid < 3 * C) ge[tid] = gv;
#pragma unroll
    for (int p = 0; p < PW; ++p) {
      const int kt = wv + 4 * p;
      if (kt < KT) *(f4_t *)&Ht[l16 * (K + 4) + 16 * kt + 4 * g4] = D[p];
    }
    const bool tok = t0 + tt < a.T;
    const f4_t dy = nv;
    lds_barrier();
    const float gm = ge[tt], bt = be[tt];
    if (wv < 2)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        Yt[(4 * g4 + x) * LC + tt] = dy[x];
        Wt[(4 * g4 + x) * LC + tt] = gm * dy[x];
      }
    lds_barrier();
    fetch(max(ch - 1, 0));
    const f4_t zero = {0.f, 0.f, 0.f, 0.f};
    if (wv < 2) {
      f4_t u = mma_rows(Ht + l16 * (K + 4) + 4 * g4, ks + tt * (K + 4) + 4 * g4, K, zero);
      u = mma_rows(Yt + l16 * LC + 4 * g4, Pt + tt * LC + 4 * g4, C, gl[tt] * u);
#pragma unroll
      for (int x = 0; x < 4; ++x) Ut[(4 * g4 + x) * LC + tt] = u[x];
    }
    lds_barrier();
    f4_t z = zero;
    if (wv < 2) {
      z = mma_rows(Ut + l16 * LC + 4 * g4, Tt + tt * LC + 4 * g4, C, zero);
#pragma unroll
      for (int x = 0; x < 4; ++x) Zt[(4 * g4 + x) * LC + tt] = -bt * gm * z[x];
    }
    lds_barrier();
    const float gc = ge[C - 1];
    f4_t D0[PW];
#pragma unroll
    for (int p = 0; p < PW; ++p) D0[p] = D[p];
#pragma unroll
    for (int p = 0; p < PW; ++p) {
      const int kt = wv + 4 * p;
      if (kt < KT) {
        D[p] = mma_rows(qT + (16 * kt + l16) * LC + 4 * g4, Wt + l16 * LC + 4 * g4, C, gc * D[p]);
        D[p] = mma_rows(kT + (16 * kt + l16) * LC + 4 * g4, Zt + l16 * LC + 4 * g4, C, D[p]);
      }
    }
    arrived();
    if (tok && wv < 2) {
      *(f4_t *)&rows_z[vbase + (size_t)(t0 + tt) * vrow] = z;
      store4<IO>(a.dv, vbase + (size_t)(t0 + tt) * vrow, bt * z);
    }
#pragma unroll
    for (int p = 0; p < PW; ++p) {
      const int kt = wv + 4 * p;
      if (kt < KT)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          states[(((size_t)unit * chunks + ch) * K + 16 * kt + 4 * g4 + x) * a.V + vb * VB + l16] = D0[p][x];
    }
    lds_barrier();
  }
  if (a.dH0)
#pragma unroll
    for (int p = 0; p < PW; ++p) {
      const int kt = wv + 4 * p;
      if (kt < KT)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          a.dH0[((size_t)unit * K + 16 * kt + 4 * g4 + x) * a.V + vb * VB + l16] = D[p][x];
    }
}

// ------------------------------------------------------------------ dq, dk, dg, dbeta of one chunk
// Waves own column tiles wave, wave + 4 of K for both 16-step halves, and tile `wave` of S1 and S2.
// Operands over V come straight from memory, four neighbours a lane.
template <typename IO, int K>
__global__ void __launch_bounds__(256, 2)
    delta_grad_kernel(DeltaArgs a, int chunks, const float *__restrict__ gates, const float *__restrict__ states,
                      const float *__restrict__ rows_u, const float *__restrict__ dstates,
                      const float *__restrict__ rows_z, float *__restrict__ dq_heads, float *__restrict__ dk_heads) {
  constexpr int KT = K / 16, PW = (KT + 3) / 4;
  extern __shared__ __align__(16) float lds[];
  float *qT = lds, *kT = qT + K * LC, *S1 = kT + K * LC, *S1t = S1 + C * LC, *S2 = S1t + C * LC, *S2t = S2 + C * LC;
  float *ge = S2t + C * LC, *gl = ge + C, *hi = gl + C, *lo = hi + C, *be = lo + C, *red = be + C;  // red [4][2][C] + [4]
  const int unit = blockIdx.x / chunks, ch = blockIdx.x - unit * chunks, t0 = ch * C;
  const int b = unit / a.N, n = unit - b * a.N, nq = n / (a.N / a.Nqk);
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g4 = lane >> 4;
  const size_t qrow = (size_t)a.Nqk * K, qbase = (size_t)b * a.T * qrow + (size_t)nq * K;
  const size_t vrow = (size_t)a.N * a.V, vbase = (size_t)b * a.T * vrow + (size_t)n * a.V;
  const size_t at = (size_t)blockIdx.x;
  {
    Rows<IO, K> x;
    x.load(a.q, qbase, qrow, t0, a.T);
    x.store(nullptr, qT);
    x.load(a.k, qbase, qrow, t0, a.T);
    x.store(nullptr, kT);
    if (tid < 4 * C) ge[tid] = gates[at * 4 * C + tid];
    else if (tid < 5 * C) be[tid - 4 * C] = t0 + tid - 4 * C < a.T ? a.beta[((size_t)b * a.T + t0 + tid - 4 * C) * a.N + n] : 0.f;
  }
  const f4_t zero = {0.f, 0.f, 0.f, 0.f};
  const int r = wv >> 1, c = wv & 1;
  f4_t s1 = zero, s2 = zero, dq[PW][2], asks[PW][2], kept[PW][2];
#pragma unroll
  for (int p = 0; p < PW; ++p)
#pragma unroll
    for (int h = 0; h < 2; ++h) dq[p][h] = asks[p][h] = kept[p][h] = zero;
  float zv = 0.f, hd = 0.f;  // Z.v of step tid / 8 over vectors tid % 8, ..; <H, dH> over my tiles
  for (int e = 0; e < a.V; e += 16) {
    f4_t y[2], u[2], z[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int t = t0 + 16 * h + l16;
      const size_t o = vbase + (size_t)t * vrow + e + 4 * g4;
      y[h] = load4<IO>(a.dy, o, t < a.T);
      u[h] = load4<float>(rows_u, o, t < a.T);
      z[h] = load4<float>(rows_z, o, t < a.T);
    }
    s1 = mma(r ? y[1] : y[0], c ? u[1] : u[0], s1);
    s2 = mma(r ? z[1] : z[0], c ? u[1] : u[0], s2);
#pragma unroll
    for (int p = 0; p < PW; ++p) {
      const int kt = wv + 4 * p;
      if (kt < KT) {
        const size_t o = (at * K + 16 * kt + l16) * a.V + e + 4 * g4;
        const f4_t h0 = *(const f4_t *)(states + o), h1 = *(const f4_t *)(dstates + o);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          dq[p][h] = mma(h0, y[h], dq[p][h]);
          asks[p][h] = mma(h0, z[h], asks[p][h]);
          kept[p][h] = mma(h1, u[h], kept[p][h]);
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) hd = fmaf(h0[x], h1[x], hd);
      }
    }
  }
  settle(s1);
  settle(s2);
#pragma unroll
  for (int p = 0; p < PW; ++p)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      settle(dq[p][h]);
      settle(asks[p][h]);
      settle(kept[p][h]);
    }
  {
    const int t = t0 + (tid >> 3);
    for (int e = 4 * (tid & 7); e < a.V; e += 32) {
      const size_t o = vbase + (size_t)t * vrow + e;
      const f4_t z = load4<float>(rows_z, o, t < a.T), v = load4<IO>(a.v, o, t < a.T);
#pragma unroll
      for (int x = 0; x < 4; ++x) zv = fmaf(z[x], v[x], zv);
    }
#pragma unroll
    for (int d = 1; d < 8; d *= 2) zv += __shfl_xor(zv, d, 64);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) hd += __shfl_xor(hd, d, 64);
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const int i = 16 * r + 4 * g4 + x, j = 16 * c + l16;
    const float e = exp2_((hi[i] - hi[j]) + (lo[i] - lo[j]));
    const float p1 = j <= i ? e * s1[x] : 0.f, p2 = j < i ? e * s2[x] : 0.f;
    S1[i * LC + j] = p1;
    S1t[j * LC + i] = p1;
    S2[i * LC + j] = -p2;
    S2t[j * LC + i] = -be[i] * p2;
  }
  __syncthreads();
  const bool heads = a.N != a.Nqk;
  float dG[2] = {0.f, 0.f}, kb[2] = {0.f, 0.f};
#pragma unroll
  for (int p = 0; p < PW; ++p) {
    const int kt = wv + 4 * p;
    if (kt < KT) {
      const float *qr = qT + (16 * kt + l16) * LC + 4 * g4, *kr = kT + (16 * kt + l16) * LC + 4 * g4;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int i = 16 * h + l16, t = t0 + i;
        const float gm = ge[i], gt = gl[i], bt = be[i];
        const f4_t d = mma_rows(kr, S1 + i * LC + 4 * g4, C, gm * dq[p][h]);
        const f4_t s = mma_rows(kr, S2 + i * LC + 4 * g4, C, -gm * asks[p][h]);
        f4_t w = mma_rows(qr, S1t + i * LC + 4 * g4, C, gt * kept[p][h]);
        w = mma_rows(kr, S2t + i * LC + 4 * g4, C, w);
        f4_t o;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int kk = 16 * kt + 4 * g4 + x;
          const float qv = qT[kk * LC + i], kv = kT[kk * LC + i];
          o[x] = fmaf(bt, s[x], w[x]);
          dG[h] = fmaf(qv, d[x], dG[h]);
          dG[h] = fmaf(kv, fmaf(bt, s[x], -w[x]), dG[h]);
          kb[h] = fmaf(kv, s[x], kb[h]);
        }
        if (t < a.T) {
          const size_t m = ((size_t)b * a.T + t) * (heads ? a.N : a.Nqk) * K + (size_t)(heads ? n : nq) * K + 16 * kt + 4 * g4;
          if (heads) {
            *(f4_t *)&dq_heads[m] = d;
            *(f4_t *)&dk_heads[m] = o;
          } else {
            store4<IO>(a.dq, m, d);
            store4<IO>(a.dk, m, o);
          }
        }
      }
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    dG[h] += __shfl_xor(dG[h], 16, 64);
    dG[h] += __shfl_xor(dG[h], 32, 64);
    kb[h] += __shfl_xor(kb[h], 16, 64);
    kb[h] += __shfl_xor(kb[h], 32, 64);
    if (g4 == 0) {
      red[(wv * 2 + 0) * C + 16 * h + l16] = dG[h];
      red[(wv * 2 + 1) * C + 16 * h + l16] = kb[h];
    }
  }
  if (lane == 0) red[8 * C + wv] = hd;
  if ((tid & 7) == 0) red[8 * C + 4 + (tid >> 3)] = zv;
  // what the chunk's own steps add to <H_C, dH>: the sum over j of e^{G_C - G_j} k_j.(dH U_j), of which the
  // waves hold their columns
  float tail = 0.f;
#pragma unroll
  for (int p = 0; p < PW; ++p) {
    const int kt = wv + 4 * p;
    if (kt < KT)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          tail = fmaf(gl[16 * h + l16] * kT[(16 * kt + 4 * g4 + x) * LC + 16 * h + l16], kept[p][h][x], tail);
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) tail += __shfl_xor(tail, d, 64);
  if (lane == 0) red[9 * C + 4 + wv] = tail;
  __syncthreads();
  if (tid < 64) {  // one wave: the sums over the steps behind, in 64 bits
    double s = 0.0;
    float db = 0.f;
    if (lane < C) {
      for (int w = 0; w < 4; ++w) {
        s += (double)red[(2 * w) * C + lane];
        db += red[(2 * w + 1) * C + lane];
      }
      db += red[8 * C + 4 + lane];
    }
    if (lane == C - 1)
      for (int w = 0; w < 4; ++w) s += (double)ge[C - 1] * red[8 * C + w] + red[9 * C + 4 + w];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const double o = __shfl_down(s, d, 64);
      if (lane + d < 64) s += o;
    }
    if (lane < C && t0 + lane < a.T) {
      const size_t o = ((size_t)b * a.T + t0 + lane) * a.N + n;
      ((IO *)a.dg)[o] = from_f32<IO>((float)s);
      ((IO *)a.dbeta)[o] = from_f32<IO>(db);
    }
  }
}
constexpr int lds_grad(int K) { return (2 * K * LC + 4 * C * LC + 5 * C + 9 * C + 8) * 4; }

// ------------------------------------------------------------------ launches
// Gates, T and P stand behind the states and U of the checkpoints where there are any (the backward takes them from
// there), else in the workspace.
Ws carve(const DeltaLayout &l, char *p, char *ckpt) {
  Ws w;
  char *m = ckpt ? ckpt + l.states + l.rows : p;
  w.gates = (float *)m;
  w.mats = (float *)(m + l.gates);
  if (!ckpt) p += l.gates + l.mats;
  w.states = (float *)p;
  w.rows = (float *)(p += l.states);
  w.dqh = (float *)(p += l.rows);
  w.dkh = (float *)(p += l.heads);
  return w;
}

template <typename IO>
hipError_t prep(const DeltaArgs &a, const DeltaLayout &l, const Ws &w, hipStream_t s) {
  hipLaunchKernelGGL(delta_prep_kernel<IO>, dim3((unsigned)(a.B * a.N) * (unsigned)l.chunks), dim3(256), 0, s, a,
                     l.chunks, w.gates, w.mats);
  return hipGetLastError();
}
template <typename IO, int K>
hipError_t scan(const DeltaArgs &a, const DeltaLayout &l, const Ws &w, hipStream_t s) {
  hipError_t e = set_max_lds_once(delta_fwd_kernel<IO, K>, lds_fwd(K));
  if (e != hipSuccess) return e;
  float *states = (float *)a.ckpt, *rows = a.ckpt ? (float *)(a.ckpt + l.states) : nullptr;
  hipLaunchKernelGGL((delta_fwd_kernel<IO, K>), dim3(delta_grid(a.B * a.N, a.V / VB)), dim3(256), lds_fwd(K), s, a,
                     l.chunks, w.gates, w.mats, states, rows);
  return hipGetLastError();
}
template <typename IO, int K>
hipError_t back(const DeltaArgs &a, const DeltaLayout &l, const Ws &w, hipStream_t s) {
  hipError_t e = set_max_lds_once(delta_bwd_kernel<IO, K>, lds_bwd(K));
  if (e == hipSuccess) e = set_max_lds_once(delta_grad_kernel<IO, K>, lds_grad(K));
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((delta_bwd_kernel<IO, K>), dim3(delta_grid(a.B * a.N, a.V / VB)), dim3(256), lds_bwd(K), s, a,
                     l.chunks, w.gates, w.mats, w.states, w.rows);
  if ((e = hipGetLastError()) != hipSuccess || l.chunks == 0) return e;
  hipLaunchKernelGGL((delta_grad_kernel<IO, K>), dim3((unsigned)(a.B * a.N) * (unsigned)l.chunks), dim3(256),
                     lds_grad(K), s, a, l.chunks, w.gates, (const float *)a.ckpt, (const float *)(a.ckpt + l.states),
                     w.states, w.rows, w.dqh, w.dkh);
  return hipGetLastError();
}
#define M2RNN_DELTA_K(F_, ...)                       \
  switch (a.K) {                                     \
    case 16: e = F_<IO, 16>(__VA_ARGS__); break;     \
    case 32: e = F_<IO, 32>(__VA_ARGS__); break;     \
    case 64: e = F_<IO, 64>(__VA_ARGS__); break;     \
    default: e = F_<IO, 128>(__VA_ARGS__); break;    \
  }
template <typename IO>
hipError_t fwd_t(const DeltaArgs &a, hipStream_t s) {
  const DeltaLayout l = delta_f32_layout(a);
  const Ws w = carve(l, a.ws, a.ckpt);
  hipError_t e = l.chunks > 0 ? prep<IO>(a, l, w, s) : hipSuccess;
  if (e != hipSuccess) return e;
  M2RNN_DELTA_K(scan, a, l, w, s)
  return e;
}
template <typename IO>
hipError_t bwd_t(const DeltaArgs &a, hipStream_t s) {
  const DeltaLayout l = delta_f32_layout(a);
  const Ws w = carve(l, a.ws, a.ckpt);
  hipError_t e = hipSuccess;
  if (a.own_ckpt && l.chunks > 0) {
    DeltaArgs f = a;
    f.write_y = 0;
    f.HT = nullptr;
    if ((e = prep<IO>(a, l, w, s)) != hipSuccess) return e;
    M2RNN_DELTA_K(scan, f, l, w, s)
    if (e != hipSuccess) return e;
  }
  M2RNN_DELTA_K(back, a, l, w, s)
  if (e != hipSuccess || l.chunks == 0 || a.N == a.Nqk) return e;
  BwdArgs h = {};
  h.B = a.B; h.T = a.T; h.N = a.N; h.Nqk = a.Nqk; h.K = a.K; h.io = a.io;
  if ((e = generic_head_group_sum(h, w.dqh, a.dq, s)) != hipSuccess) return e;
  return generic_head_group_sum(h, w.dkh, a.dk, s);
}
#undef M2RNN_DELTA_K

}  // namespace

DeltaLayout delta_f32_layout(const DeltaArgs &a) {
  DeltaLayout l;
  l.C = C;
  l.kept = true;
  l.chunks = ceil_div(a.T, C);
  const size_t n = (size_t)a.B * a.N * l.chunks, steps = (size_t)a.B * a.T * a.N;
  l.gates = align256(n * 4 * C * sizeof(float));
  l.mats = align256(n * 2 * C * C * sizeof(float));
  l.states = align256(n * a.K * a.V * sizeof(float));
  l.rows = align256(steps * a.V * sizeof(float));
  l.carry = l.exps = l.dexps = 0;
  l.heads = a.N != a.Nqk ? align256(steps * a.K * sizeof(float)) : 0;
  return l;
}
hipError_t delta_f32_fwd(const DeltaArgs &a, hipStream_t s) {
  return a.io == 0 ? fwd_t<float>(a, s) : fwd_t<__hip_bfloat16>(a, s);
}
hipError_t delta_f32_bwd(const DeltaArgs &a, hipStream_t s) {
  return a.io == 0 ? bwd_t<float>(a, s) : bwd_t<__hip_bfloat16>(a, s);
}

}  // namespace m2rnn
