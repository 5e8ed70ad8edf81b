// Gated delta rule of bf16 io, chunks of 64 steps on the 16x16x32 matrix instructions.  The lines of the rule by
// chunks stand in m2rnn_delta.hpp.
//
//   delta_half_prep_kernel   one workgroup per chunk: gates, T and P             -> workspace
//   delta_half_fwd_kernel    one workgroup per state and VB columns of V, chunks in order -> y, HT, (H, U); few long
//                            sequences in several launches, T and P of the next one's chunks beside them
//   delta_half_bwd_kernel    the same, backwards                                  -> dv, dH0, dH and Z
//   delta_half_grad_kernel   one workgroup per chunk                              -> dq, dk, dg, dbeta
//
// Operands.  q, k, v, dy are bf16 and exact as fp16 beside the largest of their chunk.  Everything that reaches a
// state enters its product as an fp16 pair hi + lo of 22 bits, so that states and their gradients, which are
// fp32, are as good as that; what only reaches a bf16 result is one fp16 value of 11 bits.  T is formed in fp32.
//
// Powers of two.  No magnitude is given, and fp16 has few exponents: every operand is brought near one by a power of two of
// its chunk (H, U, dH, dy, Z: of its workgroup's columns too), which its products are given back in fp32.  They come
// from the largest finite entries of q, k, beta and P (found with T) and of v, H, dy and dH (by the chains), and
// of sums, U and Z, from bounds that hold while the rule does not expand.  What is below 2^-25 of the largest is lost.
//
// Layout.  Products are D = A B^T: a lane gives eight elements of row (lane % 16) of a factor, and holds rows
// 4 (lane / 16) .. + 3 of column lane % 16 of D.  Which eight of the 32 that are contracted is free, as long as both
// factors agree: over K and V they are neighbours, 8 (lane / 16) .. + 7; over steps the two groups of four that
// the lane holds in D of the two 16-step tiles, 4 (lane / 16) .. + 3 and 16 further, so that what is a result is an
// operand as it stands.  LDS arrays with steps side by side keep them in that order (`place`).
// What one kernel hands to another (T, P, H, U, dH, Z) is stored as the operands that the reader needs, 16 bytes
// a lane, 1 KB an operand: no reader goes through LDS for it.
#include "m2rnn_delta.hpp"

#include <algorithm>
#include <type_traits>

namespace m2rnn {
namespace {

constexpr int C = 64;
constexpr int LC = C + 8;       // halfs per row of an LDS array with a chunk's steps side by side
// Floats per chunk: e^G, e^{G_C - G}, G / ln 2 as hi, lo, beta, and as ints at kTops the exponents (floor log2) of the
// largest |k|, |beta|, |P| and |q|
constexpr int kTops = 5 * C, kGates = kTops + 16;
// (Backward: e^G over om = 2^floor(G_0 / ln 2).  e^G goes into fp16 operands there, all of it can be as small as
// the first step's gate, and the gradient of the state in front is then as small: om is put back in fp32.)
__device__ __forceinline__ float gate_unit(float hi0) { return exp2_(floorf(hi0)); }

typedef __bf16 b8_t __attribute__((ext_vector_type(8)));
typedef _Float16 half_t;

__device__ __forceinline__ f4_t mfma_bf16(u4_t a, u4_t b, f4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8_t, a), __builtin_bit_cast(b8_t, b), c, 0, 0, 0);
}
// two floats, rounded to nearest even, as fp16
__device__ __forceinline__ uint32_t pack2_h(float a, float b) {
  typedef float f2_t __attribute__((ext_vector_type(2)));
  const f2_t x = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, h2_t));
}
__device__ __forceinline__ u2_t pack4_h(f4_t x) { return u2_t{pack2_h(x[0], x[1]), pack2_h(x[2], x[3])}; }
// 2^e, no more than 2^127
__device__ __forceinline__ float two_to(int e) { return __builtin_amdgcn_ldexpf(1.f, min(e, 127)); }
// eight bf16 values times s, as fp16
__device__ __forceinline__ h8_t bf16_to_h8(u4_t w, float s) {
  u4_t r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = w[i];
    r[i] = pack2_h(s * __builtin_bit_cast(float, x << 16), s * __builtin_bit_cast(float, x & 0xFFFF0000u));
  }
  return __builtin_bit_cast(h8_t, r);
}
// eight bf16 values as fp16
__device__ __forceinline__ h8_t bf16_to_h8(u4_t w) {
  u4_t r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = w[i];
    r[i] = pack2_h(__builtin_bit_cast(float, x << 16), __builtin_bit_cast(float, x & 0xFFFF0000u));
  }
  return __builtin_bit_cast(h8_t, r);
}
// Keys and queries of a chunk whose largest entry has an exponent e far from zero come as fp16 over 2^e, others as they
// are: entries of 2^-17 and more are exact then, and below them 2^-25 is lost, 2^-21 of the largest key's entry at most,
// 2^-18 of the largest query's (K^{-1/2} of a unit vector's, for which there is more room).
__device__ __forceinline__ bool far_key(int e) { return e < -4 || e > 10; }
__device__ __forceinline__ bool far_query(int e) { return e < -7 || e > 10; }
template <bool FAR, int N>
__device__ __forceinline__ void rows_to_h8(const u4_t (&w)[N], int e, h8_t (&x)[N]) {
  const float s = two_to(-e);
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = FAR ? bf16_to_h8(w[i], s) : bf16_to_h8(w[i]);
}
__device__ __forceinline__ f4_t fma4(float a, f4_t b, f4_t c) {
  return f4_t{fmaf(a, b[0], c[0]), fmaf(a, b[1], c[1]), fmaf(a, b[2], c[2]), fmaf(a, b[3], c[3])};
}
// four floats as fp16 hi and lo parts
struct Pair4 {
  u2_t hi, lo;
};
__device__ __forceinline__ Pair4 split4(f4_t x) {
  Pair4 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    // (hi to nearest: on its own it is the operand of what becomes bf16, y among it, and cut towards zero it would
    // make all of that smaller by 2^-12)
    const uint32_t hi = pack2_h(x[2 * i], x[2 * i + 1]);
    float l0, l1;
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(l0) : "v"(hi), "v"(x[2 * i]));
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(l1) : "v"(hi), "v"(x[2 * i + 1]));
    r.hi[i] = hi;
    r.lo[i] = pack2_h(l0, l1);
  }
  return r;
}
__device__ __forceinline__ h8_t ld8(const half_t *p) { return *(const h8_t *)p; }

// The largest finite magnitude of a wave's values, of which `each` calls back with all that a lane has.  Infinities
// and NaN do not count: they are no measure for the values beside them.  (fmaxf passes over a NaN; an infinity, which
// is rare, costs a second pass without it.)
template <typename F>
__device__ __forceinline__ float wave_top(F each) {
  float top = 0.f;
  each([&](float x) { top = fmaxf(top, fabsf(x)); });
  top = group_max_nonneg<64>(top);
  if (__builtin_bit_cast(int, top) == 0x7F800000) {
    top = 0.f;
    each([&](float x) { top = fabsf(x) < __builtin_inff() ? fmaxf(top, fabsf(x)) : top; });
    top = group_max_nonneg<64>(top);
  }
  return top;
}
template <typename F, int M, int N>
__device__ __forceinline__ void all_of(const f4_t (&x)[M][N], F put) {
#pragma unroll
  for (int i = 0; i < M * N * 4; ++i) put(x[i / (4 * N)][i / 4 % N][i % 4]);
}
template <typename F, int M>
__device__ __forceinline__ void all_of(const f4_t (&x)[M], F put) {
#pragma unroll
  for (int i = 0; i < M * 4; ++i) put(x[i / 4][i % 4]);
}
// the exponent of the largest of four waves' tops, the same in all lanes and so in a scalar register; such that 2^e and
// 2^-e are both normal numbers
__device__ __forceinline__ int exponent_in_range(int e) { return min(max(e, -126), 126); }
__device__ __forceinline__ int exponent_of(u4_t tops) {
  const uint32_t top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
  return exponent_in_range(ilog2f(__builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(top))));
}
__device__ __forceinline__ int exponent_of(f4_t tops) { return exponent_of(__builtin_bit_cast(u4_t, tops)); }
// eight bf16 magnitudes into the largest finite ones so far, two at a time, as bits + 0x80: what is not finite is
// negative then.  Start from kNoBf16Top.
typedef short s2_t __attribute__((ext_vector_type(2)));
typedef unsigned short us2_t __attribute__((ext_vector_type(2)));
constexpr short kNoBf16Top = 0x80;
__device__ __forceinline__ s2_t bf16_top(u4_t w, s2_t top) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const us2_t x = __builtin_bit_cast(us2_t, w[i] & 0x7FFF7FFFu) + us2_t{0x80, 0x80};
    top = __builtin_elementwise_max(top, __builtin_bit_cast(s2_t, x));
  }
  return top;
}
__device__ __forceinline__ float bf16_top_value(s2_t top) {
  return __builtin_bit_cast(float, (uint32_t)(max((int)top.x, (int)top.y) - 0x80) << 16);
}
__device__ __forceinline__ h8_t tr8(const half_t *p0, const half_t *p1) {
  const h4_t a = lds_ld_tr((const lchar *)p0, 0), b = lds_ld_tr((const lchar *)p1, 0);
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
// Where the steps 16 tile + 4 (lane / 16) .. + 3 lie in an LDS row
__device__ __forceinline__ int place(int tile) { return 32 * (tile >> 1) + 8 * ((threadIdx.x & 63) >> 4) + 4 * (tile & 1); }
// The operand whose 16 rows are columns c0 .. c0 + 15 of an LDS array whose rows are steps, contracted over the
// steps r0 .. r0 + 31
__device__ __forceinline__ h8_t ld8_steps(const half_t *base, int ld, int r0, int c0) {
  const int lane = threadIdx.x & 63, d = lane & 15, g = lane >> 4;
  const half_t *p = base + (r0 + 4 * g + (d >> 2)) * ld + c0 + 4 * (d & 3);
  return tr8(p, p + 16 * ld);
}
// The operand whose 16 rows are columns c0 .. c0 + 15 of an LDS array, contracted over its rows r0 .. r0 + 31
__device__ __forceinline__ h8_t ld8_tr(const half_t *base, int ld, int r0, int c0) {
  const int lane = threadIdx.x & 63, d = lane & 15, g = lane >> 4;
  const half_t *p = base + (r0 + 8 * g + (d >> 2)) * ld + c0 + 4 * (d & 3);
  return tr8(p, p + 4 * ld);
}

// ------------------------------------------------------------------ gates, T, P of one chunk
// T and P of a chunk: [row tile 4][32 columns 2][hi, lo][lane][8].  BWD: of their transposes.
constexpr size_t kMat = 4 * 2 * 2 * 64 * 8;  // halfs
__device__ __forceinline__ int mat_at(int tile, int kb, int part) { return (((tile * 2 + kb) * 2 + part) * 64) * 8; }
// the bytes of a lane's part of it, or beyond the buffer (reads as zero) where the block is zero
__device__ __forceinline__ uint32_t mat_bytes(int tile, int kb, int part, bool there) {
  return there ? 2 * mat_at(tile, kb, part) + 16 * (threadIdx.x & 63) : 2 * (uint32_t)kMat;
}

__device__ __forceinline__ f4_t mma_f32(f4_t a, f4_t b, f4_t c) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
  return c;
}

// The inverse of I + A by blocks of 16: the diagonal blocks row by row, then
//     [ T0 0 ; -T1 A10 T0  T1 ]   for the two pairs of neighbours, and the same with blocks of 32,
// whose products run on the fp32 matrix instructions; T takes the place of A in LDS block by block.
// What bounds it is latency: all loads are issued at once, and 24 KB of LDS leave room for six workgroups per CU.
// 8 x 4096 steps, 16 heads of 64 x 64: 69 us forward, 93 backward (3.5 TB/s, mostly of T and P).
struct PrepLds {
  float As[C][C + 4], Xt[C / 2][C / 2 + 4], hi[C], lo[C], be[C], tops[12];
};
template <int K, bool BWD>
__device__ __forceinline__ void prep_chunk(const DeltaArgs &a, int chunks, int unit, int ch, float *gates, half_t *mats,
                                           PrepLds &lds) {
  constexpr int LA = C + 4, KB = K / 32;
  auto &As = lds.As;
  auto &Xt = lds.Xt;
  float *hi = lds.hi, *lo = lds.lo, *be = lds.be;
  const size_t slot = (size_t)unit * chunks + ch;
  const int b = unit / a.N, n = unit - b * a.N, nq = n / (a.N / a.Nqk);
  const int t0 = ch * C, lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int d = lane & 15, g4 = lane >> 4;
  // forward: wave = tile of i, over j <= i, D[j][i];  backward: wave = tile of j, over i >= j, D[i][j]
  const size_t row = (size_t)a.Nqk * K, base = (size_t)b * a.T * row + (size_t)nq * K + 8 * g4;
  const unsigned short *q = (const unsigned short *)a.q, *k = (const unsigned short *)a.k;
  auto at = [&](int tile) { return base + (size_t)min(t0 + 16 * tile + d, a.T - 1) * row; };
  u4_t kw[KB], qw[KB], ko[3][KB], qo[3][KB];
#pragma unroll
  for (int e = 0; e < KB; ++e) {
    kw[e] = *(const u4_t *)(k + at(wv) + 32 * e);
    qw[e] = *(const u4_t *)(q + at(wv) + 32 * e);
  }
#pragma unroll
  for (int o = 0; o < 3; ++o)
    if (BWD ? wv + 1 + o < 4 : o < wv)
#pragma unroll
      for (int e = 0; e < KB; ++e) {
        ko[o][e] = *(const u4_t *)(k + at(BWD ? wv + 1 + o : o) + 32 * e);
        if (BWD) qo[o][e] = *(const u4_t *)(q + at(wv + 1 + o) + 32 * e);
      }
  if (wv == 0) {
    const bool in = t0 + lane < a.T;
    const size_t e = ((size_t)b * a.T + (in ? t0 + lane : 0)) * a.N + n;
    const float beta = in ? a.beta[e] : 0.f;
    const GateSum G = gate_sum(in ? a.g[e] : 0.f);
    const float ghi = __shfl(G.hi, C - 1, 64), glo = __shfl(G.lo, C - 1, 64);
    hi[lane] = G.hi;
    lo[lane] = G.lo;
    be[lane] = beta;
    float *gt = gates + slot * kGates;
    gt[lane] = BWD ? exp2_((G.hi - floorf(__shfl(G.hi, 0, 64))) + G.lo) : exp2_(G.hi) * exp2_(G.lo);
    gt[C + lane] = exp2_((ghi - G.hi) + (glo - G.lo));
    gt[2 * C + lane] = G.hi;
    gt[3 * C + lane] = G.lo;
    gt[4 * C + lane] = beta;
    const float top = wave_top([&](auto put) { put(beta); });
    if (lane == 0) ((int *)gt)[kTops + 1] = exponent_in_range(ilog2f(top));
  }
  s2_t ktop = {kNoBf16Top, kNoBf16Top}, qtop = ktop;
#pragma unroll
  for (int e = 0; e < KB; ++e) {
    ktop = bf16_top(kw[e], ktop);
    qtop = bf16_top(qw[e], qtop);
  }
  const float kmax = group_max_nonneg<64>(bf16_top_value(ktop)), qmax = group_max_nonneg<64>(bf16_top_value(qtop));
  if (lane == 0) {
    lds.tops[wv] = kmax;
    lds.tops[4 + wv] = qmax;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    // (keys or queries that are all zero, as behind the end of a padded sequence, need no power of two: as near one)
    auto exponent = [](f4_t tops) { return tops[0] + tops[1] + tops[2] + tops[3] == 0.f ? 0 : exponent_of(tops); };
    int *tops = (int *)(gates + slot * kGates) + kTops;
    tops[0] = exponent(*(const f4_t *)lds.tops);
    tops[3] = exponent(*(const f4_t *)(lds.tops + 4));
  }
  f4_t ps[4];  // P's four columns (rows, transposed) per tile
  const int mine = 16 * wv + d;
  auto tile = [&](int o, const u4_t *kt, const u4_t *qt) {
    f4_t kk = {0.f, 0.f, 0.f, 0.f}, qk = kk;
#pragma unroll
    for (int e = 0; e < KB; ++e) {
      kk = mfma_bf16(kt[e], kw[e], kk);
      qk = BWD ? mfma_bf16(qt[e], kw[e], qk) : mfma_bf16(kt[e], qw[e], qk);
    }
    settle(kk);
    settle(qk);
    f4_t am, p;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int r = 16 * o + 4 * g4 + x, i = BWD ? r : mine, j = BWD ? mine : r;
      const float e = exp2_((hi[i] - hi[j]) + (lo[i] - lo[j]));
      am[x] = j < i ? be[i] * e * kk[x] : 0.f;
      p[x] = j <= i ? e * qk[x] : 0.f;
      if (BWD) As[i][j] = am[x];
    }
    if (!BWD) *(f4_t *)&As[mine][16 * o + 4 * g4] = am;
    return p;
  };
#pragma unroll
  for (int o = 0; o < 4; ++o) {
    f4_t p = {0.f, 0.f, 0.f, 0.f};
    if (o == wv) p = tile(o, kw, qw);
    else if (BWD ? o > wv : o < wv) {
      // (the register arrays are indexed by constants: one case per distance)
      if constexpr (!BWD) {
        if (o < 3) p = tile(o, ko[o < 3 ? o : 0], nullptr);
      } else {
#pragma unroll
        for (int x = 0; x < 3; ++x)
          if (o - wv - 1 == x) p = tile(o, ko[x], qo[x]);
      }
    }
    ps[o] = p;
  }
  const float pmax = wave_top([&](auto put) { all_of(ps, put); });
  if (lane == 0) lds.tops[8 + wv] = pmax;
  __syncthreads();
  const int ep = exponent_of(*(const f4_t *)(lds.tops + 8));
  if (threadIdx.x == 0) ((int *)(gates + slot * kGates))[kTops + 2] = ep;
  // P over its largest entry, an operand's halves as they are
  u2_t ph[4], pl[4];
#pragma unroll
  for (int o = 0; o < 4; ++o) {
    const f4_t p = two_to(-ep) * ps[o];
    if (BWD) {
      const Pair4 s = split4(p);
      ph[o] = s.hi;
      pl[o] = s.lo;
    } else {
      ph[o] = pack4_h(p);
    }
  }
  if (lane < 16) {
    float x[16];
    float *A0 = &As[16 * wv][16 * wv];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float s[4] = {d == i ? 1.f : 0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < i; ++j) s[j & 3] = fmaf(-A0[i * LA + j], x[j], s[j & 3]);
      x[i] = (s[0] + s[1]) + (s[2] + s[3]);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) A0[i * LA + d] = x[i];
  }
  __syncthreads();
  const f4_t zero = {0.f, 0.f, 0.f, 0.f};
  // rows of an array as one factor, columns as the other
  auto cols = [&](int r, int c) { return f4_t{As[r][c], As[r + 1][c], As[r + 2][c], As[r + 3][c]}; };
  auto rows = [&](int r, int c) { return *(const f4_t *)&As[r][c]; };
  auto put = [&](int r, int c, f4_t x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) As[r + i][c] = -x[i];
  };
  if (wv < 2) {  // neighbours: block (2 wv + 1, 2 wv)
    const int r = 32 * wv + 16, c = 32 * wv;
    f4_t x = mma_f32(rows(r + d, c + 4 * g4), cols(c + 4 * g4, c + d), zero);
    settle(x);
    *(f4_t *)&Xt[16 * wv + d][4 * g4] = x;  // (read by this wave alone)
    x = mma_f32(rows(r + d, r + 4 * g4), *(const f4_t *)&Xt[16 * wv + d][4 * g4], zero);
    settle(x);
    put(r + 4 * g4, c + d, x);
  }
  __syncthreads();
  const int r = wv >> 1, c = wv & 1;  // tile (2 + r, c)
  {
    f4_t x = mma_f32(rows(32 + 16 * r + d, 16 + 4 * g4), cols(16 + 4 * g4, 16 * c + d), zero);
    if (c == 0) x = mma_f32(rows(32 + 16 * r + d, 4 * g4), cols(4 * g4, d), x);
    settle(x);
    *(f4_t *)&Xt[16 * c + d][16 * r + 4 * g4] = x;
  }
  __syncthreads();
  {
    f4_t x = mma_f32(rows(32 + 16 * r + d, 32 + 4 * g4), *(const f4_t *)&Xt[16 * c + d][4 * g4], zero);
    if (r == 1) x = mma_f32(rows(48 + d, 48 + 4 * g4), *(const f4_t *)&Xt[16 * c + d][16 + 4 * g4], x);
    settle(x);
    put(32 + 16 * r + 4 * g4, 16 * c + d, x);
  }
  __syncthreads();
  half_t *Tm = mats + slot * 2 * kMat, *Pm = Tm + kMat;
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    if (BWD ? (kb == 0 && wv >= 2) : (kb == 1 && wv < 2)) continue;  // (zero)
    Pair4 t[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int c0 = 32 * kb + 16 * u + 4 * g4;
      f4_t x = BWD ? cols(c0, mine) : rows(mine, c0);
#pragma unroll
      for (int v = 0; v < 4; ++v)
        if (BWD ? c0 + v < mine : c0 + v > mine) x[v] = 0.f;  // (tiles beyond the diagonal have not been written)
      t[u] = split4(x);
    }
    auto join = [](u2_t x, u2_t y) { return u4_t{x.x, x.y, y.x, y.y}; };
    *(u4_t *)(Tm + mat_at(wv, kb, 0) + lane * 8) = join(t[0].hi, t[1].hi);
    *(u4_t *)(Tm + mat_at(wv, kb, 1) + lane * 8) = join(t[0].lo, t[1].lo);
    *(u4_t *)(Pm + mat_at(wv, kb, 0) + lane * 8) = join(ph[2 * kb], ph[2 * kb + 1]);
    if (BWD) *(u4_t *)(Pm + mat_at(wv, kb, 1) + lane * 8) = join(pl[2 * kb], pl[2 * kb + 1]);
  }
}
// the chunks c0 .. c1 - 1 of all units
template <int K, bool BWD>
__global__ void __launch_bounds__(256, BWD && K == 128 ? 3 : 4)
    delta_half_prep_kernel(DeltaArgs a, int chunks, int c0, int c1, float *__restrict__ gates, half_t *__restrict__ mats) {
  __shared__ __align__(16) PrepLds lds;
  const int n = c1 - c0, unit = blockIdx.x / n;
  prep_chunk<K, BWD>(a, chunks, unit, c0 + (int)blockIdx.x - unit * n, gates, mats, lds);
}

// ------------------------------------------------------------------ the kernels that run in order
// A workgroup of four waves has VB columns of one state.  In products over steps wave w has the chunk's steps
// 16 w .. 16 w + 15; of the state it has KTW row tiles times VTW column tiles, in fp32 registers throughout.
//
// What bounds them is the chain of a chunk: three products, each of which needs the one before from all waves.
// So every operand of a product is read from LDS before its first instruction, what is off the chain (Q H, Q^T W,
// results on their way out) lies in the shadow of such reads, and the next chunk's loads are in flight for a whole
// chunk.  They are taken into the registers that use them before this chunk's results are stored: the counter that
// a wait for loads looks at counts stores as well, in order.
template <int K, int VB>
struct Scan {
  static constexpr int KB = K / 32, KT = K / 16, VT = VB / 16;
  static constexpr int KTW = KT >= 4 ? KT / 4 : 1, VTW = KT >= 4 ? VT : 1;
  static constexpr int LK = K + 8;
  // row tile i and column tile j of wave w; with K = 32 two waves share a row tile (and with VB = 16 two have none)
  static __device__ __forceinline__ int kt(int w, int i) { return KT >= 4 ? w + 4 * i : w % KT; }
  static __device__ __forceinline__ int vt(int w, int j) { return KT >= 4 ? j : (w / KT) % VT; }
  static __device__ __forceinline__ bool on(int w) { return KT >= 4 || w / KT < VT; }
};
// Where the operand that holds 16 rows x 32 columns of V goes: [V / 32][tiles][lane][8]; with VB = 16 a
// workgroup has one half of the lanes, and its two halves the same.
template <int VB>
__device__ __forceinline__ size_t frag_at(int part, int tiles, int tile) {
  const int lane = threadIdx.x & 63;
  if constexpr (VB == 32) return ((size_t)(part * tiles + tile) * 64 + lane) * 8;
  else return ((size_t)((part >> 1) * tiles + tile) * 64 + (lane & 31) + 32 * (part & 1)) * 8;
}
// that operand, from an LDS array [VB][ld]: its rows are the columns c0 .. c0 + 15 (STEPS: c0 a tile of steps)
template <int VB, bool STEPS>
__device__ __forceinline__ h8_t frag_of(const half_t *base, int ld, int c0) {
  const int lane = threadIdx.x & 63, d = lane & 15, g = VB == 32 ? lane >> 4 : (lane >> 4) & 1;
  const int c = STEPS ? 32 * (c0 >> 1) + 4 * (c0 & 1) + 8 * (d & 3) : c0 + 4 * (d & 3);
  const half_t *p = base + (8 * g + (d >> 2)) * ld + c;
  return tr8(p, p + 4 * ld);
}
// Values that have arrived, in registers here and now (see above)
template <typename X>
__device__ __forceinline__ void pin(X &x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void pin8(h8_t &x) {
  u4_t y = __builtin_bit_cast(u4_t, x);
  pin(y);
  x = __builtin_bit_cast(h8_t, y);
}

// Nothing moves across: a load stays behind the last use of the registers that it fills
__device__ __forceinline__ void hold() { __builtin_amdgcn_sched_barrier(0); }

// A chunk's rows of a [T][row] tensor through a buffer that ends with the sequence: what lies behind the last step
// reads as zero and is not written, without a branch, and a lane's offset is the same for all chunks.
struct Rows {
  char *base;
  uint32_t row;  // bytes
  int T;
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t at(int ch) const {
    return __builtin_amdgcn_make_buffer_rsrc(base + (size_t)ch * C * row, 0, min(C, T - ch * C) * row, 0x00027000);
  }
};
__device__ __forceinline__ u4_t buf_ld(__amdgpu_buffer_rsrc_t r, uint32_t o) {
  return __builtin_amdgcn_raw_buffer_load_b128(r, o, 0, 0);
}
__device__ __forceinline__ h8_t buf_h8(__amdgpu_buffer_rsrc_t r, uint32_t o) { return __builtin_bit_cast(h8_t, buf_ld(r, o)); }
__device__ __forceinline__ void buf_st(__amdgpu_buffer_rsrc_t r, uint32_t o, u2_t x) {
  __builtin_amdgcn_raw_buffer_store_b64(x, r, o, 0, 0);
}
struct Place {  // of a workgroup
  Rows q, k, v, o;  // o: y or dv, laid out as v (v or dy)
  char *mats;
  const float *gates;
  // T (part 0) and P (part 1) of a chunk
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t mat(int ch, int part) const {
    return __builtin_amdgcn_make_buffer_rsrc(mats + ((size_t)ch * 2 + part) * (2 * kMat), 0, 2 * kMat, 0x00027000);
  }
  __device__ __forceinline__ Place(const DeltaArgs &a, const void *v_, void *o_, int unit, int col, int chunks,
                                   const float *gates_, const half_t *mats_) {
    const int b = unit / a.N, n = unit - b * a.N, nq = n / (a.N / a.Nqk);
    const uint32_t qr = (uint32_t)a.Nqk * a.K * 2, vr = (uint32_t)a.N * a.V * 2;
    const size_t qo = (size_t)b * a.T * qr + (size_t)nq * a.K * 2, vo = (size_t)b * a.T * vr + ((size_t)n * a.V + col) * 2;
    q = Rows{(char *)a.q + qo, qr, a.T};
    k = Rows{(char *)a.k + qo, qr, a.T};
    v = Rows{(char *)v_ + vo, vr, a.T};
    o = Rows{(char *)o_ + vo, vr, a.T};
    mats = (char *)(mats_ + (size_t)unit * chunks * 2 * kMat);
    gates = gates_ + (size_t)unit * chunks * kGates;
  }
};
// What the wave's steps need of the gates, one float a lane in one load, through LDS to the lanes that use it
struct Gates {
  float *at;  // 64 of the wave
  static __device__ __forceinline__ uint32_t offset(int wv) {
    const int lane = threadIdx.x & 63, i = lane & 15;
    return 4 * (lane < 16 ? 16 * wv + i : lane < 32 ? C + 16 * wv + i : lane < 48 ? 4 * C + 16 * wv + i
                : i == 0 ? C - 1 : i == 1 ? 2 * C : kTops + ((i - 2) & 3));
  }
  __device__ __forceinline__ f4_t four(int which) const { return *(const f4_t *)(at + 16 * which + 4 * ((threadIdx.x & 63) >> 4)); }
  __device__ __forceinline__ float one(int which) const { return at[16 * which + (threadIdx.x & 15)]; }
  __device__ __forceinline__ float last() const { return at[48]; }    // e^G of the chunk's last step
  __device__ __forceinline__ float first() const { return at[49]; }   // hi of its first
  // (the tops from the lanes that have loaded them)
  static __device__ __forceinline__ int top(float x, int i) { return __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 50 + i); }
};
// A wave's 16 steps of VB columns, eight a lane as loaded, through LDS to four steps of one column per lane and
// column tile, as in D[step][column]
template <int VB>
struct Turn {
  static constexpr int LD = VB + 8, HALFS = 16 * LD;  // per wave
  half_t *at;
  __device__ __forceinline__ void put(u4_t x) const {
    const int lane = threadIdx.x & 63, g = VB == 32 ? lane >> 4 : (lane >> 4) & 1;
    *(u4_t *)(at + (lane & 15) * LD + 8 * g) = x;
  }
  __device__ __forceinline__ f4_t get(int t) const {
    const int lane = threadIdx.x & 63, d = lane & 15, g = lane >> 4;
    const u2_t x = __builtin_bit_cast(u2_t, lds_ld_tr((const lchar *)(at + (4 * g + (d >> 2)) * LD + 16 * t + 4 * (d & 3)), 0));
    return f4_t{__builtin_bit_cast(float, x.x << 16), __builtin_bit_cast(float, x.x & 0xFFFF0000u),
                __builtin_bit_cast(float, x.y << 16), __builtin_bit_cast(float, x.y & 0xFFFF0000u)};
  }
};

template <int K, int VB>
constexpr int lds_fwd() { return (C * (K + 8) + 2 * VB * (K + 8) + 5 * VB * LC + 4 * Turn<VB>::HALFS) * 2 + 4 * 64 * 4 + 12 * 4; }

// The largest |H| (upper 16 bits, cut to them as bf16) and |v| of a workgroup, infinities among them, in two halves of
// a word, a word for every wave, to LDS and from there.
__device__ __forceinline__ uint32_t max_halves(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2_t, a), __builtin_bit_cast(us2_t, b)));
}
template <int M, int N, int VT>
__device__ __forceinline__ void top_of_wave(uint32_t *red, const f4_t (&H)[M][N], const f4_t (&v)[VT], int wv) {
  float th = 0.f, tw = 0.f;
  all_of(H, [&](float x) { th = fmaxf(th, fabsf(x)); });
  all_of(v, [&](float x) { tw = fmaxf(tw, fabsf(x)); });
  uint32_t t = (__builtin_bit_cast(uint32_t, th) & 0xFFFF0000u) | (__builtin_bit_cast(uint32_t, tw) >> 16);
  t = max_halves(t, __builtin_amdgcn_update_dpp(0, t, 0xB1, 0xF, 0xF, false));   // quad_perm [1,0,3,2]
  t = max_halves(t, __builtin_amdgcn_update_dpp(0, t, 0x4E, 0xF, 0xF, false));   // quad_perm [2,3,0,1]
  t = max_halves(t, __builtin_amdgcn_update_dpp(0, t, 0x141, 0xF, 0xF, false));  // row_half_mirror
  t = max_halves(t, __builtin_amdgcn_update_dpp(0, t, 0x140, 0xF, 0xF, false));  // row_mirror
  t = max_halves(t, __builtin_amdgcn_update_dpp(0, t, 0x142, 0xA, 0xF, false));  // row_bcast:15: rows 1 and 3 also those before
  t = max_halves(t, __builtin_amdgcn_update_dpp(0, t, 0x143, 0xC, 0xF, false));  // row_bcast:31: the last row all
  if ((threadIdx.x & 63) == 63) red[wv] = t;
}
__device__ __forceinline__ uint32_t top_of_all(const uint32_t *red) {
  const u4_t m = *(const u4_t *)red;
  return __builtin_amdgcn_readfirstlane(max_halves(max_halves(m[0], m[1]), max_halves(m[2], m[3])));
}
// the exponent of the lower 16 bits of x as bf16
__device__ __forceinline__ int top_exponent(uint32_t x) { return max((int)(x >> 7 & 255u) - 127, -126); }
// the same without what is not finite, as floats: four words of H, four of v
template <int M, int N, int VT>
__device__ __forceinline__ void finite_tops(uint32_t *red, const f4_t (&H)[M][N], const f4_t (&v)[VT], int wv) {
  const float th = wave_top([&](auto put) { all_of(H, put); }), tw = wave_top([&](auto put) { all_of(v, put); });
  if ((threadIdx.x & 63) == 0) {
    red[wv] = __builtin_bit_cast(uint32_t, th);
    red[4 + wv] = __builtin_bit_cast(uint32_t, tw);
  }
}
__device__ __forceinline__ bool not_finite(uint32_t tops) {
  return (tops & 0x7F800000u) == 0x7F800000u || (tops & 0x7F80u) == 0x7F80u;
}

// Forward.  The state lies in registers over 2^eh and enters as that; R and U are over 2^er.  Both stay while the largest
// entries (of U its bound) are between 2^-2 and 2^13 (2^-3 and 2^4) of them.  That is known to all waves only behind the
// barrier that hands the state over: where it does not hold any more, all is scaled anew and handed over again (a few
// times at a sequence's start).

// What a launch of the forward does: the chunks c0 .. c1 - 1 of all states, from H0 to HT, in its first `scans`
// workgroups, and T and P of the chunks c1 .. c2 - 1, which the next launch reads, in the others.
struct Part {
  int c0, c1, c2;
  unsigned scans;
  const float *H0;
  float *HT;
};
// Y: y is wanted;  CKPT: the chunks' states and U are.  8 x 4096 steps, 16 heads of 64 x 64: 167 us, 2.6 a chunk on
// 256 workgroups (3.4 TB/s); 65 536 steps, 32 of 64 x 64 without checkpoints: 1.4 a chunk on 128 of them,
// T and P of later chunks beside it.  K = 64, VB = 32: three workgroups fit into a CU's LDS, and are given registers for it
// (64 sequences of 64 steps, 16 heads, a call without checkpoints 37.2 -> 35.1).
template <int K, int VB, bool Y, bool CKPT>
__global__ void __launch_bounds__(256, VB == 32 && K == 64 ? 3 : 2)
    delta_half_fwd_kernel(DeltaArgs a, int chunks, Part p, float *gates, half_t *mats, half_t *__restrict__ states,
                          half_t *__restrict__ rows_u, int *__restrict__ exps) {
  using S = Scan<K, VB>;
  constexpr int KB = S::KB, KT = S::KT, VT = S::VT, KTW = S::KTW, VTW = S::VTW, LK = S::LK;
  extern __shared__ __align__(16) char lds[];
  half_t *ks = (half_t *)lds, *Ht = ks + C * LK, *Hl = Ht + VB * LK, *Rt = Hl + VB * LK, *Rl = Rt + VB * LC;
  half_t *Ut = Rl + VB * LC, *Wt = Ut + VB * LC, *Wl = Wt + VB * LC, *turn = Wl + VB * LC;
  uint32_t *red = (uint32_t *)(turn + 4 * Turn<VB>::HALFS) + 4 * 64;
  int unit, part;
  if (blockIdx.x >= p.scans) {
    const int i = blockIdx.x - p.scans, n = p.c2 - p.c1;
    unit = i / n;
    prep_chunk<K, false>(a, chunks, unit, p.c1 + i - unit * n, gates, mats, *(PrepLds *)lds);
    return;
  }
  if (!delta_map(a.B * a.N, a.V / VB, unit, part)) return;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int d = lane & 15, g4 = lane >> 4;
  const Turn<VB> tv{turn + wv * Turn<VB>::HALFS};
  const Gates gs{(float *)(turn + 4 * Turn<VB>::HALFS) + 64 * wv};
  // T and P are lower triangular: the first two waves have no steps above 31, and read zeros there without a memory
  // access (a branch around their products would not make the other two waves faster)
  const bool two = wv >= 2;
  const Place in(a, a.v, a.y, unit, part * VB, chunks, gates, mats);
  const f4_t zero = {0.f, 0.f, 0.f, 0.f};
  const size_t state0 = (size_t)unit * K * a.V + part * VB + d;  // element (0, d) of my columns
  const uint32_t oq = (16 * wv + d) * in.q.row + 16 * g4, og = Gates::offset(wv);
  const uint32_t ov = (16 * wv + d) * in.v.row + 16 * (VB == 32 ? g4 : g4 & 1), oy = (16 * wv + d) * in.v.row + 8 * g4;

  f4_t H[KTW][VTW];
#pragma unroll
  for (int i = 0; i < KTW; ++i)
#pragma unroll
    for (int j = 0; j < VTW; ++j) H[i][j] = zero;
  if (p.H0)
#pragma unroll
    for (int i = 0; i < KTW; ++i)
#pragma unroll
      for (int j = 0; j < VTW; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          H[i][j][x] = p.H0[state0 + (size_t)(16 * S::kt(wv, i) + 4 * g4 + x) * a.V + 16 * S::vt(wv, j)];
  // (here, and not at the head of the loop, which would then wait for everything at every chunk)
#pragma unroll
  for (int i = 0; i < KTW; ++i)
#pragma unroll
    for (int j = 0; j < VTW; ++j) settle(H[i][j]);
  // The next chunk's, in the order of their use: k, v and gates in its first product, T in its second, q and P last.
  // Each load is issued behind the last use of its registers and so has most of a chunk to arrive.
  u4_t nk[KB], nq[KB], nv;
  h8_t Tf[4], Pf[2];  // [32 steps][hi, lo];  [32 steps]
  float ng;
  auto fetch1 = [&](int ch) {
    const auto k = in.k.at(ch), v = in.v.at(ch);
#pragma unroll
    for (int i = 0; i < KB; ++i) nk[i] = buf_ld(k, oq + 64 * i);
    nv = buf_ld(v, ov);
    ng = *(const float *)((const char *)(in.gates + (size_t)ch * kGates) + og);
  };
  auto fetch2 = [&](int ch) {
    const auto m = in.mat(ch, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) Tf[i] = buf_h8(m, mat_bytes(wv, i >> 1, i & 1, i < 2 || two));
  };
  auto fetch3 = [&](int ch) {
    const auto m = in.mat(ch, 1), q = in.q.at(ch);
#pragma unroll
    for (int i = 0; i < KB; ++i) nq[i] = buf_ld(q, oq + 64 * i);
#pragma unroll
    for (int i = 0; i < 2; ++i) Pf[i] = buf_h8(m, mat_bytes(wv, i, 0, i < 1 || two));
  };
  h8_t kf[KB];
  f4_t vf[VT], ge, gl, be;
  float g1, gc;
  int ek, eb, ep, eq, eh = 0, er = 0;
  auto take_keys = [&](auto far) {
    rows_to_h8<decltype(far)::value>(nk, ek, kf);
#pragma unroll
    for (int i = 0; i < KB; ++i) pin8(kf[i]);
  };
  auto take1 = [&](auto far) {
    tv.put(nv);
    gs.at[lane] = ng;
    ek = Gates::top(ng, 0); eb = Gates::top(ng, 1); ep = Gates::top(ng, 2); eq = Gates::top(ng, 3);
    take_keys(far);
#pragma unroll
    for (int t = 0; t < VT; ++t) vf[t] = tv.get(t);
    ge = gs.four(0); gl = gs.four(1); be = gs.four(2); g1 = gs.one(0); gc = gs.last();
  };
  auto put_state = [&]() {
    if (S::on(wv))
#pragma unroll
      for (int i = 0; i < KTW; ++i)
#pragma unroll
        for (int j = 0; j < VTW; ++j) {
          const Pair4 x = split4(H[i][j]);
          const int o = (16 * S::vt(wv, j) + d) * LK + 16 * S::kt(wv, i) + 4 * g4;
          *(u2_t *)&Ht[o] = x.hi;
          *(u2_t *)&Hl[o] = x.lo;
        }
  };
  if (p.c0 < p.c1) {
    fetch1(p.c0);
    fetch2(p.c0);
    if (Y) fetch3(p.c0);
    take1(std::false_type());
  }
  auto get_state = [&](h8_t(&hh)[VT][KB], h8_t(&hl)[VT][KB]) {
#pragma unroll
    for (int i = 0; i < KB; ++i)
#pragma unroll
      for (int t = 0; t < VT; ++t) {
        const int o = (16 * t + d) * LK + 32 * i + 8 * g4;
        hh[t][i] = ld8(Ht + o);
        hl[t][i] = ld8(Hl + o);
      }
  };
  // For R, which is no larger than sqrt(K) times this (and U not by much more while the rule does not expand)
  auto scale_of_u = [&](int et, int ev) { return exponent_in_range(eb + max(ev, ek + et)); };
  // The state counts as no smaller than 2^-24 of that, of which nothing would be left beside it.
  auto scale_of_state = [&](int et, int tu) { return max(exponent_in_range(et), tu - 24); };
  // The exponents of the largest finite |H| and |v|
  auto measure = [&](int &et, int &ev) {
    finite_tops(red + 4, H, vf, wv);
    lds_barrier();
    et = eh + exponent_of(*(const u4_t *)(red + 4));
    ev = exponent_of(*(const u4_t *)(red + 8));
  };
  auto rescale = [&](int to) {
#pragma unroll
    for (int i = 0; i < KTW; ++i)
#pragma unroll
      for (int j = 0; j < VTW; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x) H[i][j][x] = __builtin_amdgcn_ldexpf(H[i][j][x], eh - to);
    eh = to;
  };
  if (p.c0 < p.c1) {
    top_of_wave(red + 4, H, vf, wv);
    lds_barrier();
    const uint32_t tops = top_of_all(red + 4);
    if (!not_finite(tops)) {  // (else the first chunk measures again)
      const int et = top_exponent(tops >> 16);
      er = scale_of_u(et, top_exponent(tops));
      rescale(scale_of_state(et, er));
    }
  }
  const int w = place(wv);
  auto is_far = [&]() { return far_key(ek) || (Y && far_query(eq)); };
  // the chunks from ch on; without FAR up to one whose keys or queries are far from one.  Returns the next chunk.
  auto run_chunks = [&](auto far, int ch) __attribute__((always_inline)) {
    constexpr bool FAR = decltype(far)::value;
    while (ch < p.c1) {
      const int next = min(ch + 1, p.c1 - 1), kx = FAR ? ek : 0, qx = FAR ? eq : 0;
      put_state();
#pragma unroll
      for (int i = 0; i < KB; ++i) *(h8_t *)&ks[(16 * wv + d) * LK + 32 * i + 8 * g4] = kf[i];
      top_of_wave(red, H, vf, wv);
      lds_barrier();  // the state is there, and k of the chunk before has been read
      // R = beta (v - e^G K H): D[step][column]
      const uint32_t tops = top_of_all(red);
      h8_t hh[VT][KB], hl[VT][KB];
      f4_t x[VT], xl[VT];
      auto keys_with_state = [&]() {
#pragma unroll
        for (int t = 0; t < VT; ++t) x[t] = xl[t] = zero;
#pragma unroll
        for (int i = 0; i < KB; ++i)
#pragma unroll
          for (int t = 0; t < VT; ++t) {
            x[t] = mfma_k32(kf[i], hh[t][i], x[t]);
            xl[t] = mfma_k32(kf[i], hl[t][i], xl[t]);
          }
      };
      get_state(hh, hl);
      fetch1(next);
      keys_with_state();
      f4_t gh = two_to(eh + kx) * ge, br = two_to(-er) * be;
      int et = eh + top_exponent(tops >> 16), ev = top_exponent(tops), tu = scale_of_u(et, ev);
      int want = scale_of_state(et, tu);
      if (not_finite(tops) | (want < eh - 2) | (want > eh + 13) | (tu < er - 3) | (tu > er + 4)) {  // (the same in all waves)
        measure(et, ev);
        er = scale_of_u(et, ev);
        rescale(scale_of_state(et, er));
        put_state();
        lds_barrier();
        get_state(hh, hl);
        keys_with_state();
        gh = two_to(eh + kx) * ge;
        br = two_to(-er) * be;
      }
#pragma unroll
      for (int t = 0; t < VT; ++t) {
        const Pair4 s = split4(br * (vf[t] - gh * (x[t] + xl[t])));
        *(u2_t *)&Rt[(16 * t + d) * LC + w] = s.hi;
        *(u2_t *)&Rl[(16 * t + d) * LC + w] = s.lo;
      }
      lds_barrier();
      // U = T R: D[step][column];  off the chain (Q H)^T: D[column][step]
      h8_t rh[VT][2], rl[VT][2], hs[KTW], kT[KTW][2];
      f4_t y[VT], u[VT], ul[VT];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int t = 0; t < VT; ++t) {
          const int o = (16 * t + d) * LC + 32 * kb + 8 * g4;
          rh[t][kb] = ld8(Rt + o);
          rl[t][kb] = ld8(Rl + o);
        }
      if (CKPT)
#pragma unroll
        for (int i = 0; i < KTW; ++i) hs[i] = frag_of<VB, false>(Ht, LK, 16 * S::kt(wv, i));
#pragma unroll
      for (int i = 0; i < KTW; ++i)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) kT[i][kb] = ld8_steps(ks, LK, 32 * kb, 16 * S::kt(wv, i));
#pragma unroll
      for (int t = 0; t < VT; ++t) y[t] = u[t] = ul[t] = zero;
#pragma unroll
      for (int t = 0; t < VT; ++t) {
        u[t] = mfma_k32(Tf[0], rh[t][0], u[t]);
        ul[t] = mfma_k32(Tf[1], rh[t][0], ul[t]);
        ul[t] = mfma_k32(Tf[0], rl[t][0], ul[t]);
        u[t] = mfma_k32(Tf[2], rh[t][1], u[t]);
        ul[t] = mfma_k32(Tf[3], rh[t][1], ul[t]);
        ul[t] = mfma_k32(Tf[2], rl[t][1], ul[t]);
      }
      hold();
      fetch2(next);
      hold();
#pragma unroll
      for (int t = 0; t < VT; ++t) {
        settle(u[t]);
        settle(ul[t]);
        const f4_t uu = u[t] + ul[t];
        const Pair4 s = split4(gl * uu);
        *(u2_t *)&Wt[(16 * t + d) * LC + w] = s.hi;
        *(u2_t *)&Wl[(16 * t + d) * LC + w] = s.lo;
        *(u2_t *)&Ut[(16 * t + d) * LC + w] = pack4_h(uu);
      }
      lds_barrier();
      // H = e^{G_C} H + K^T W: D[row][column];  y = e^G (Q H)^T + (P U)^T
      h8_t wh[VTW][2], wl[VTW][2], uf[VT][2], us;
      const float gy = two_to(eh + qx) * g1, rp = two_to(er + ep), rus = two_to(er + kx - eh);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int j = 0; j < VTW; ++j) {
          const int o = (16 * S::vt(wv, j) + d) * LC + 32 * kb + 8 * g4;
          wh[j][kb] = ld8(Wt + o);
          wl[j][kb] = ld8(Wl + o);
        }
      if (Y) {
        h8_t qf[KB];
        rows_to_h8<FAR>(nq, eq, qf);
#pragma unroll
        for (int i = 0; i < KB; ++i)
#pragma unroll
          for (int t = 0; t < VT; ++t) y[t] = mfma_k32(hh[t][i], qf[i], y[t]);
      }
      f4_t kw[KTW][VTW], hg[KTW][VTW];
#pragma unroll
      for (int i = 0; i < KTW; ++i)
#pragma unroll
        for (int j = 0; j < VTW; ++j) hg[i][j] = gc * H[i][j];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < KTW; ++i)
#pragma unroll
          for (int j = 0; j < VTW; ++j) {
            kw[i][j] = mfma_k32(kT[i][kb], wl[j][kb], kb ? kw[i][j] : zero);
            kw[i][j] = mfma_k32(kT[i][kb], wh[j][kb], kw[i][j]);
          }
#pragma unroll
      for (int i = 0; i < KTW; ++i)
#pragma unroll
        for (int j = 0; j < VTW; ++j) {
          settle(kw[i][j]);
          H[i][j] = fma4(rus, kw[i][j], hg[i][j]);
        }
      if (Y) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int t = 0; t < VT; ++t) uf[t][kb] = ld8(Ut + (16 * t + d) * LC + 32 * kb + 8 * g4);
#pragma unroll
        for (int t = 0; t < VT; ++t) {
          u[t] = mfma_k32(uf[t][0], Pf[0], zero);
          u[t] = mfma_k32(uf[t][1], Pf[1], u[t]);
        }
        hold();
        fetch3(next);
        hold();
#pragma unroll
        for (int t = 0; t < VT; ++t) {
          settle(u[t]);
          y[t] = gy * y[t] + rp * u[t];
        }
      }
      if (CKPT) us = frag_of<VB, true>(Ut, LC, wv);
      take1(far);
      if (Y) {
        const auto o = in.o.at(ch);
#pragma unroll
        for (int t = 0; t < VT; ++t)
          buf_st(o, oy + 32 * t, u2_t{pack2_bf16(y[t][0], y[t][1]), pack2_bf16(y[t][2], y[t][3])});
      }
      if (CKPT) {
        const size_t at = (size_t)unit * chunks + ch;
        if (KT >= 4 || wv < KT)
#pragma unroll
          for (int i = 0; i < KTW; ++i) *(h8_t *)(states + at * K * a.V + frag_at<VB>(part, KT, S::kt(wv, i))) = hs[i];
        *(h8_t *)(rows_u + at * C * a.V + frag_at<VB>(part, 4, wv)) = us;
        // (lanes behind the buffer's end write nothing; a branch would make the next loads wait for all stores)
        __builtin_amdgcn_raw_buffer_store_b32(lane ? er : eh, __builtin_amdgcn_make_buffer_rsrc(exps + (at * (a.V / VB) + part) * 2,
                                              0, 8, 0x00027000), 4 * (int)threadIdx.x, 0, 0);
      }
      ++ch;
      if (!FAR && is_far()) break;
    }
    return ch;
  };
  int ch = p.c0;
  if (ch < p.c1 && !is_far()) ch = run_chunks(std::false_type(), ch);
  if (ch < p.c1) {
    take_keys(std::true_type());
    run_chunks(std::true_type(), ch);
  }
  rescale(0);
  if (p.HT && S::on(wv))
#pragma unroll
    for (int i = 0; i < KTW; ++i)
#pragma unroll
      for (int j = 0; j < VTW; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          p.HT[state0 + (size_t)(16 * S::kt(wv, i) + 4 * g4 + x) * a.V + 16 * S::vt(wv, j)] = H[i][j][x];
}

// Backward, chunks in reverse order.  As in the forward dH lies in registers over 2^ed and enters as that, dy over 2^ey, dU
// and Z over 2^ez.  8 x 4096 steps, 16 heads of 64 x 64: 217 us, 3.4 a chunk (3.8 TB/s).
// (own_z: Z has room of its own, and the waves need not wait for each other before the next chunk's inputs come; with K = 128
// and VB = 32 it takes W's place, so that two workgroups fit into a CU's LDS: 4 x 64 steps of 32 heads 16.2 -> 12.4 us)
template <int K, int VB>
constexpr bool own_z() { return K != 128 || VB != 32; }
template <int K, int VB>
constexpr int lds_bwd() { return (2 * C * (K + 8) + 2 * VB * (K + 8) + (own_z<K, VB>() ? 7 : 5) * VB * LC + 4 * Turn<VB>::HALFS) * 2 + 4 * 64 * 4 + 12 * 4; }

template <int K, int VB>
__global__ void __launch_bounds__(256, 2)
    delta_half_bwd_kernel(DeltaArgs a, int chunks, const float *__restrict__ gates, const half_t *__restrict__ mats,
                          half_t *__restrict__ dstates, half_t *__restrict__ rows_z, u4_t *__restrict__ exps) {
  using S = Scan<K, VB>;
  constexpr int KB = S::KB, KT = S::KT, VT = S::VT, KTW = S::KTW, VTW = S::VTW, LK = S::LK;
  extern __shared__ __align__(16) char lds[];
  half_t *ks = (half_t *)lds, *qs = ks + C * LK, *Ht = qs + C * LK, *Hl = Ht + VB * LK, *Yt = Hl + VB * LK;
  half_t *Wt = Yt + VB * LC, *Wl = Wt + VB * LC, *Ut = Wl + VB * LC, *Ul = Ut + VB * LC;
  half_t *Zt = own_z<K, VB>() ? Ul + VB * LC : Wt, *Zl = Zt + VB * LC, *turn = (own_z<K, VB>() ? Zl : Ul) + VB * LC;
  uint32_t *red = (uint32_t *)(turn + 4 * Turn<VB>::HALFS) + 4 * 64;
  int unit, part;
  if (!delta_map(a.B * a.N, a.V / VB, unit, part)) return;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int d = lane & 15, g4 = lane >> 4;
  const Turn<VB> ty{turn + wv * Turn<VB>::HALFS};
  const Gates gs{(float *)(turn + 4 * Turn<VB>::HALFS) + 64 * wv};
  const bool two = wv < 2;  // (transposed: the last two waves have no steps below 32)
  const Place in(a, a.dy, a.dv, unit, part * VB, chunks, gates, mats);
  const uint32_t oq = (16 * wv + d) * in.q.row + 16 * g4, og = Gates::offset(wv);
  const uint32_t ov = (16 * wv + d) * in.v.row + 16 * (VB == 32 ? g4 : g4 & 1), oo = (16 * wv + d) * in.v.row + 8 * g4;
  const f4_t zero = {0.f, 0.f, 0.f, 0.f};
  const size_t state0 = (size_t)unit * K * a.V + part * VB + d;

  f4_t D[KTW][VTW];
#pragma unroll
  for (int i = 0; i < KTW; ++i)
#pragma unroll
    for (int j = 0; j < VTW; ++j) D[i][j] = zero;
  if (a.dHT)
#pragma unroll
    for (int i = 0; i < KTW; ++i)
#pragma unroll
      for (int j = 0; j < VTW; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          D[i][j][x] = a.dHT[state0 + (size_t)(16 * S::kt(wv, i) + 4 * g4 + x) * a.V + 16 * S::vt(wv, j)];
  // (here, and not at the head of the loop, which would then wait for everything at every chunk)
#pragma unroll
  for (int i = 0; i < KTW; ++i)
#pragma unroll
    for (int j = 0; j < VTW; ++j) settle(D[i][j]);
  u4_t nk[KB], nq[KB], ny;
  h8_t Tf[4], Pf[4];  // [32 steps, the later ones first][hi, lo]
  float ng;
  auto fetch1 = [&](int ch) {
    const auto k = in.k.at(ch), q = in.q.at(ch), y = in.v.at(ch);
    ny = buf_ld(y, ov);
    ng = *(const float *)((const char *)(in.gates + (size_t)ch * kGates) + og);
#pragma unroll
    for (int i = 0; i < KB; ++i) {
      nk[i] = buf_ld(k, oq + 64 * i);
      nq[i] = buf_ld(q, oq + 64 * i);
    }
  };
  auto fetch2 = [&](int ch) {
    const auto m = in.mat(ch, 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) Pf[i] = buf_h8(m, mat_bytes(wv, 1 - (i >> 1), i & 1, i < 2 || two));
  };
  auto fetch3 = [&](int ch) {
    const auto m = in.mat(ch, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) Tf[i] = buf_h8(m, mat_bytes(wv, 1 - (i >> 1), i & 1, i < 2 || two));
  };
  h8_t kf[KB], qf[KB];
  f4_t yf[VT], ge, gl, be;
  float b1, gc, om;
  int ek, eb, ep, eq, ed = 0, ey = 0, ez = 0;
  auto take_rows = [&](auto far) {
    rows_to_h8<decltype(far)::value>(nk, ek, kf);
    rows_to_h8<decltype(far)::value>(nq, eq, qf);
#pragma unroll
    for (int i = 0; i < KB; ++i) {
      pin8(kf[i]);
      pin8(qf[i]);
    }
  };
  auto take1 = [&](auto far) {
    ty.put(ny);
    gs.at[lane] = ng;
    ek = Gates::top(ng, 0); eb = Gates::top(ng, 1); ep = Gates::top(ng, 2); eq = Gates::top(ng, 3);
    take_rows(far);
#pragma unroll
    for (int t = 0; t < VT; ++t) yf[t] = ty.get(t);
    ge = gs.four(0); gl = gs.four(1); be = gs.four(2); b1 = gs.one(2);
    om = gate_unit(gs.first());
    gc = om * gs.last();
  };
  const int w = place(wv);
  auto put_in = [&]() {
    const float sy = two_to(-ey);
    if (S::on(wv))
#pragma unroll
      for (int i = 0; i < KTW; ++i)
#pragma unroll
        for (int j = 0; j < VTW; ++j) {
          const Pair4 x = split4(D[i][j]);
          const int o = (16 * S::vt(wv, j) + d) * LK + 16 * S::kt(wv, i) + 4 * g4;
          *(u2_t *)&Ht[o] = x.hi;
          *(u2_t *)&Hl[o] = x.lo;
        }
#pragma unroll
    for (int t = 0; t < VT; ++t) {
      const int o = (16 * t + d) * LC + w;
      const f4_t y = sy * yf[t];
      const Pair4 x = split4(ge * y);
      *(u2_t *)&Yt[o] = pack4_h(y);
      *(u2_t *)&Wt[o] = x.hi;
      *(u2_t *)&Wl[o] = x.lo;
    }
  };
  // For dU, from the exponents of the largest |dH| and |dy|; dH counts as no smaller than 2^-24 of what a chunk adds to it
  auto scale_of_z = [&](int td, int ty) { return exponent_in_range(max(td + ek, ty + ep)); };
  auto scale_of_dh = [&](int td, int ty, int tz) {
    return max(exponent_in_range(td), exponent_in_range(max(ty + eq, tz + eb + ek)) - 24);
  };
  auto measure = [&](int &td, int &ty) {
    finite_tops(red + 4, D, yf, wv);
    lds_barrier();
    td = ed + exponent_of(*(const u4_t *)(red + 4));
    ty = exponent_of(*(const u4_t *)(red + 8));
  };
  auto rescale = [&](int to) {
#pragma unroll
    for (int i = 0; i < KTW; ++i)
#pragma unroll
      for (int j = 0; j < VTW; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x) D[i][j][x] = __builtin_amdgcn_ldexpf(D[i][j][x], ed - to);
    ed = to;
  };
  if (chunks > 0) {
    fetch1(chunks - 1);
    fetch2(chunks - 1);
    fetch3(chunks - 1);
    take1(std::false_type());
    top_of_wave(red + 4, D, yf, wv);
    lds_barrier();
    const uint32_t tops = top_of_all(red + 4);
    if (!not_finite(tops)) {  // (else the first chunk measures again)
      const int td = top_exponent(tops >> 16);
      ey = top_exponent(tops);
      ez = scale_of_z(td, ey);
      rescale(scale_of_dh(td, ey, ez));
    }
  }
  auto is_far = [&]() { return far_key(ek) || far_query(eq); };
  // the chunks from ch down, as in the forward
  auto run_chunks = [&](auto far, int ch) __attribute__((always_inline)) {
    constexpr bool FAR = decltype(far)::value;
    while (ch >= 0) {
      const int next = max(ch - 1, 0), kx = FAR ? ek : 0, qx = FAR ? eq : 0;
      put_in();
#pragma unroll
      for (int i = 0; i < KB; ++i) {
        *(h8_t *)&ks[(16 * wv + d) * LK + 32 * i + 8 * g4] = kf[i];
        *(h8_t *)&qs[(16 * wv + d) * LK + 32 * i + 8 * g4] = qf[i];
      }
      top_of_wave(red, D, yf, wv);
      lds_barrier();  // (of the chunk before only Z may still be read)
      // dU = P^T dY + e^{G_C - G} K dH: D[step][column]
      const uint32_t tops = top_of_all(red);
      h8_t hh[VT][KB], hl[VT][KB], yy[VT][2];
      auto get_in = [&]() {
#pragma unroll
        for (int i = 0; i < KB; ++i)
#pragma unroll
          for (int t = 0; t < VT; ++t) {
            const int o = (16 * t + d) * LK + 32 * i + 8 * g4;
            hh[t][i] = ld8(Ht + o);
            hl[t][i] = ld8(Hl + o);
          }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int t = 0; t < VT; ++t) yy[t][kb] = ld8(Yt + (16 * t + d) * LC + 32 * kb + 8 * g4);
      };
      f4_t u[VT], ul[VT], py[VT];
      auto products = [&]() {
#pragma unroll
        for (int t = 0; t < VT; ++t) u[t] = ul[t] = py[t] = zero;
#pragma unroll
        for (int i = 0; i < KB; ++i)
#pragma unroll
          for (int t = 0; t < VT; ++t) {
            u[t] = mfma_k32(kf[i], hh[t][i], u[t]);
            ul[t] = mfma_k32(kf[i], hl[t][i], ul[t]);
          }
#pragma unroll
        for (int t = 0; t < VT; ++t) {
          py[t] = mfma_k32(Pf[0], yy[t][1], py[t]);
          py[t] = mfma_k32(Pf[1], yy[t][1], py[t]);
          py[t] = mfma_k32(Pf[2], yy[t][0], py[t]);
          py[t] = mfma_k32(Pf[3], yy[t][0], py[t]);
        }
      };
      get_in();
      fetch1(next);
      products();
      f4_t glz = two_to(ed + kx - ez) * gl;
      float pz = two_to(ey + ep - ez);
      int td = ed + top_exponent(tops >> 16), ty_ = top_exponent(tops), tz = scale_of_z(td, ty_);
      int want = scale_of_dh(td, ty_, tz);
      if (not_finite(tops) | (want < ed - 2) | (want > ed + 13) | (ty_ < ey - 2) | (ty_ > ey + 13) | (tz < ez - 3) |
          (tz > ez + 4)) {  // (the same in all waves)
        measure(td, ey);
        ez = scale_of_z(td, ey);
        rescale(scale_of_dh(td, ey, ez));
        put_in();
        lds_barrier();
        get_in();
        products();
        glz = two_to(ed + kx - ez) * gl;
        pz = two_to(ey + ep - ez);
      }
      hold();
      fetch2(next);
      hold();
#pragma unroll
      for (int t = 0; t < VT; ++t) {
        settle(u[t]);
        settle(ul[t]);
        settle(py[t]);
        const Pair4 x = split4(glz * (u[t] + ul[t]) + pz * py[t]);
        *(u2_t *)&Ut[(16 * t + d) * LC + w] = x.hi;
        *(u2_t *)&Ul[(16 * t + d) * LC + w] = x.lo;
      }
      // (what Q^T e^G dY needs)
      h8_t hs[KTW], xT[KTW][2], wh[VTW][2], wl[VTW][2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int j = 0; j < VTW; ++j) {
          const int o = (16 * S::vt(wv, j) + d) * LC + 32 * kb + 8 * g4;
          wh[j][kb] = ld8(Wt + o);
          wl[j][kb] = ld8(Wl + o);
        }
#pragma unroll
        for (int i = 0; i < KTW; ++i) xT[i][kb] = ld8_steps(qs, LK, 32 * kb, 16 * S::kt(wv, i));
      }
#pragma unroll
      for (int i = 0; i < KTW; ++i) hs[i] = frag_of<VB, false>(Ht, LK, 16 * S::kt(wv, i));
      lds_barrier();
      // Z = T^T dU as D[step][column] for the state, and as D[column][step] for what is written
      h8_t uh[VT][2], uo[VT][2];
#pragma unroll
      for (int kb = 1; kb >= 0; --kb)
#pragma unroll
        for (int t = 0; t < VT; ++t) {
          const int o = (16 * t + d) * LC + 32 * kb + 8 * g4;
          uh[t][kb] = ld8(Ut + o);
          uo[t][kb] = ld8(Ul + o);
        }
      f4_t acc[KTW][VTW];
#pragma unroll
      for (int i = 0; i < KTW; ++i)
#pragma unroll
        for (int j = 0; j < VTW; ++j) {
          acc[i][j] = zero;
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) {
            acc[i][j] = mfma_k32(xT[i][kb], wl[j][kb], acc[i][j]);
            acc[i][j] = mfma_k32(xT[i][kb], wh[j][kb], acc[i][j]);
          }
        }
      f4_t x[VT], xl[VT], z[VT];
#pragma unroll
      for (int t = 0; t < VT; ++t) {
        x[t] = mfma_k32(Tf[0], uh[t][1], zero);
        xl[t] = mfma_k32(Tf[1], uh[t][1], zero);
        xl[t] = mfma_k32(Tf[0], uo[t][1], xl[t]);
        x[t] = mfma_k32(Tf[2], uh[t][0], x[t]);
        xl[t] = mfma_k32(Tf[3], uh[t][0], xl[t]);
        xl[t] = mfma_k32(Tf[2], uo[t][0], xl[t]);
      }
      const f4_t bg = -two_to(-eb) * (be * ge);
#pragma unroll
      for (int t = 0; t < VT; ++t) {
        settle(x[t]);
        settle(xl[t]);
        const Pair4 y = split4(bg * (x[t] + xl[t]));
        *(u2_t *)&Zt[(16 * t + d) * LC + w] = y.hi;
        *(u2_t *)&Zl[(16 * t + d) * LC + w] = y.lo;
      }
#pragma unroll
      for (int i = 0; i < KTW; ++i)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) xT[i][kb] = ld8_steps(ks, LK, 32 * kb, 16 * S::kt(wv, i));
      lds_barrier();
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int j = 0; j < VTW; ++j) {
          const int o = (16 * S::vt(wv, j) + d) * LC + 32 * kb + 8 * g4;
          wh[j][kb] = ld8(Zt + o);
          wl[j][kb] = ld8(Zl + o);
        }
#pragma unroll
      for (int t = 0; t < VT; ++t) {
        z[t] = mfma_k32(uo[t][1], Tf[0], zero);
        z[t] = mfma_k32(uh[t][1], Tf[1], z[t]);
        z[t] = mfma_k32(uh[t][1], Tf[0], z[t]);
        z[t] = mfma_k32(uo[t][0], Tf[2], z[t]);
        z[t] = mfma_k32(uh[t][0], Tf[3], z[t]);
        z[t] = mfma_k32(uh[t][0], Tf[2], z[t]);
      }
      hold();
      fetch3(next);
      hold();
#pragma unroll
      for (int t = 0; t < VT; ++t) settle(z[t]);
      const float backq = om * two_to(ey + qx - ed), backk = om * two_to(ez + eb + kx - ed);
#pragma unroll
      for (int i = 0; i < KTW; ++i)
#pragma unroll
        for (int j = 0; j < VTW; ++j) {
          settle(acc[i][j]);
          D[i][j] = gc * D[i][j] + backq * acc[i][j];
        }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < KTW; ++i)
#pragma unroll
          for (int j = 0; j < VTW; ++j) {
            acc[i][j] = mfma_k32(xT[i][kb], wl[j][kb], kb ? acc[i][j] : zero);
            acc[i][j] = mfma_k32(xT[i][kb], wh[j][kb], acc[i][j]);
          }
#pragma unroll
      for (int i = 0; i < KTW; ++i)
#pragma unroll
        for (int j = 0; j < VTW; ++j) {
          settle(acc[i][j]);
          D[i][j] = fma4(backk, acc[i][j], D[i][j]);
        }
      const float bz = b1 * two_to(ez);
      take1(far);
      const size_t at = (size_t)unit * chunks + ch;
      const auto o = in.o.at(ch);
#pragma unroll
      for (int t = 0; t < VT; ++t) {
        // (a lane's four columns are half of the eight that the operand's lane d + 16 (column / 8) holds)
        const int c = (VB == 32 ? 0 : 16 * (part & 1)) + 16 * t + 4 * g4, v32 = VB == 32 ? part : part >> 1;
        *(u2_t *)(rows_z + at * C * a.V + ((size_t)(v32 * 4 + wv) * 64 + d + 16 * (c >> 3)) * 8 + (c & 7)) = pack4_h(z[t]);
        const f4_t dv = bz * z[t];
        buf_st(o, oo + 32 * t, u2_t{pack2_bf16(dv[0], dv[1]), pack2_bf16(dv[2], dv[3])});
      }
      if (KT >= 4 || wv < KT)
#pragma unroll
        for (int i = 0; i < KTW; ++i) *(h8_t *)(dstates + at * K * a.V + frag_at<VB>(part, KT, S::kt(wv, i))) = hs[i];
      // (lanes behind the buffer's end write nothing; a branch would make the next loads wait for all stores)
      __builtin_amdgcn_raw_buffer_store_b128(u4_t{(uint32_t)ed, (uint32_t)ez, (uint32_t)ey, 0u}, __builtin_amdgcn_make_buffer_rsrc(
                                             exps + at * (a.V / VB) + part, 0, 16, 0x00027000), 16 * (int)threadIdx.x, 0, 0);
      if (!own_z<K, VB>()) lds_barrier();
      --ch;
      if (!FAR && is_far()) break;
    }
    return ch;
  };
  int ch = chunks - 1;
  if (ch >= 0 && !is_far()) ch = run_chunks(std::false_type(), ch);
  if (ch >= 0) {
    take_rows(std::true_type());
    run_chunks(std::true_type(), ch);
  }
  rescale(0);
  if (a.dH0 && S::on(wv))
#pragma unroll
    for (int i = 0; i < KTW; ++i)
#pragma unroll
      for (int j = 0; j < VTW; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          a.dH0[state0 + (size_t)(16 * S::kt(wv, i) + 4 * g4 + x) * a.V + 16 * S::vt(wv, j)] = D[i][j][x];
}

// ------------------------------------------------------------------ dq, dk, dg, dbeta of one chunk
// Wave w has the chunk's steps 16 w .. 16 w + 15 and all of K: D[row of K][step].  S1 and S2 go through LDS to
// the operands that the last products take.  With V <= 64 the products with H and dH come after that, in a loop of
// their own: with all loads of a short loop in flight the two are faster (8 x 4096 steps, 16 heads of 64 x 64: 188 us,
// 4.4 TB/s, against 198 in one).  With more blocks of 32 columns the second reading of y, z and U costs more than that
// gives (4 x 8192, 8 of 128 x 128: 294 us against 225 in one loop).
template <int K>
constexpr int lds_grad() { return (2 * C * (K + 8) + 2 * C * LC + C) * 2 + (6 * C + 4 * 4) * 4; }

__device__ __forceinline__ float dot8(h8_t a, h8_t b, float c) {
#pragma unroll
  for (int i = 0; i < 8; i += 2)
    c = __builtin_amdgcn_fdot2(h2_t{a[i], a[i + 1]}, h2_t{b[i], b[i + 1]}, c, false);
  return c;
}
template <int K, int V32>
__global__ void __launch_bounds__(256, K <= 64 ? 3 : 2)
    delta_half_grad_kernel(DeltaArgs a, int chunks, int vbs, const float *__restrict__ gates,
                           const half_t *__restrict__ states, const half_t *__restrict__ rows_u,
                           const int *__restrict__ exps, const half_t *__restrict__ dstates, const half_t *__restrict__ rows_z,
                           const u4_t *__restrict__ dexps, float *__restrict__ dq_heads, float *__restrict__ dk_heads) {
  constexpr int KB = K / 32, KT = K / 16, LK = K + 8;
  constexpr bool ONE = V32 > 2;
  extern __shared__ __align__(16) char lds[];
  half_t *ks = (half_t *)lds, *qs = ks + C * LK, *S1 = qs + C * LK, *S2 = S1 + C * LC, *bh = S2 + C * LC;
  float *ge = (float *)(bh + C), *red = ge + 5 * C;  // e^G, e^{G_C - G}, hi, lo, beta;  [4][4] and dG [C]
  const int unit = blockIdx.x / chunks, ch = blockIdx.x - unit * chunks, t0 = ch * C;
  const int b = unit / a.N, n = unit - b * a.N, nq = n / (a.N / a.Nqk);
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int d = lane & 15, g4 = lane >> 4, i = 16 * wv + d, own = t0 + i;
  const size_t at = (size_t)blockIdx.x;
  const Place in(a, a.dy, a.dv, unit, 0, chunks, gates, nullptr);
  const Rows v_{(char *)a.v + (in.v.base - (char *)a.dy), in.v.row, a.T};
  const auto rq = in.q.at(ch), rk = in.k.at(ch), ry = in.v.at(ch), rv = v_.at(ch);
  const uint32_t oq = i * in.q.row + 16 * g4, ov = i * in.v.row + 16 * g4;
  const f4_t zero = {0.f, 0.f, 0.f, 0.f};
  // (everything that depends on nothing: in flight together)
  u4_t qr[KB], kr[KB];
#pragma unroll
  for (int e = 0; e < KB; ++e) {
    kr[e] = buf_ld(rk, oq + 64 * e);
    qr[e] = buf_ld(rq, oq + 64 * e);
  }
  const half_t *U = rows_u + at * C * a.V + lane * 8, *Z = rows_z + at * C * a.V + (size_t)wv * 512 + lane * 8;
  const half_t *h0 = states + at * K * a.V + lane * 8, *h1 = dstates + at * K * a.V + lane * 8;
  // What comes for a block of columns (one of `blocks`) has a power of two of its own; the chunk's common one is the
  // largest.  Each 16 lanes have the blocks' factors to it: of the states, of U, of dH and of Z.
  const int blocks = a.V / vbs, lb = lane & 15;
  const bool there = lb < blocks;
  const int ey = there ? (int)dexps[at * blocks + lb][2] : -1000;
  const int el = !there ? -1000 : lane < 32 ? exps[(at * blocks + lb) * 2 + (lane >> 4)] : (int)dexps[at * blocks + lb][(lane >> 4) - 2];
  auto row_top = [](int e) { return __builtin_bit_cast(int, group_max_nonneg<16>(__builtin_bit_cast(float, e + 1000))) - 1000; };
  const int et = row_top(el), eY = __builtin_amdgcn_readlane(row_top(ey), 0);
  const int eh = __builtin_amdgcn_readlane(et, 0), eu = __builtin_amdgcn_readlane(et, 16);
  const int eD = __builtin_amdgcn_readlane(et, 32), eZ = __builtin_amdgcn_readlane(et, 48);
  const int fl = __builtin_bit_cast(unsigned short, (half_t)two_to(el - et));
  auto own_factor = [&](int kind, int vb) {
    const int at = 16 * kind + (vbs == 32 ? vb : 2 * vb);
    int f;
    if (ONE) f = __shfl(fl, at + (vbs == 32 ? 0 : g4 >> 1), 64);
    else f = vbs == 32 || g4 < 2 ? __builtin_amdgcn_readlane(fl, at) : __builtin_amdgcn_readlane(fl, at + 1);  // (at: a constant)
    const half_t h = __builtin_bit_cast(half_t, (unsigned short)f);
    return h8_t{h, h, h, h, h, h, h, h};
  };
  const int *gt_tops = (const int *)gates + at * kGates + kTops;
  const int eb = gt_tops[1], ek = far_key(gt_tops[0]) ? gt_tops[0] : 0, eq = far_query(gt_tops[3]) ? gt_tops[3] : 0;
  const float sy = two_to(-eY), sb = two_to(-eb);

  {
    h8_t x[KB];
    if (ek) rows_to_h8<true>(kr, ek, x);
    else rows_to_h8<false>(kr, 0, x);
#pragma unroll
    for (int e = 0; e < KB; ++e) *(h8_t *)&ks[i * LK + 32 * e + 8 * g4] = x[e];
    if (eq) rows_to_h8<true>(qr, eq, x);
    else rows_to_h8<false>(qr, 0, x);
#pragma unroll
    for (int e = 0; e < KB; ++e) *(h8_t *)&qs[i * LK + 32 * e + 8 * g4] = x[e];
  }
  for (int x = threadIdx.x; x < kTops; x += 256) {
    const float g = gates[at * kGates + x];
    ge[x] = g;
    if (x >= 4 * C) bh[x - 4 * C] = (half_t)(sb * g);
  }

  f4_t s1[4], s2[4], dq[KT], as[KT], kept[KT];
#pragma unroll
  for (int j = 0; j < 4; ++j) s1[j] = s2[j] = zero;
#pragma unroll
  for (int x = 0; x < KT; ++x) dq[x] = as[x] = kept[x] = zero;
  float zv = 0.f, hd = 0.f;
  auto with_states = [&](int vb, h8_t y, h8_t z, h8_t u) {
    const h8_t fd = own_factor(2, vb), uf = u * (fd * own_factor(1, vb));
    const h8_t fh = own_factor(0, vb), yh = y * fh, zh = z * fh;
    float hb = 0.f;
#pragma unroll
    for (int x = 0; x < KT; ++x) {
      const h8_t x0 = ld8(h0 + (vb * KT + x) * 512), x1 = ld8(h1 + (vb * KT + x) * 512);
      dq[x] = mfma_k32(x0, yh, dq[x]);
      as[x] = mfma_k32(x0, zh, as[x]);
      kept[x] = mfma_k32(x1, uf, kept[x]);
      if ((x & 3) == wv) hb = dot8(x0, x1, hb);
    }
    hd = fmaf((float)fd[0] * (float)fh[0], hb, hd);
  };
#pragma unroll
  for (int vb = 0; vb < (ONE ? 1 : V32); ++vb)
#pragma unroll 1
    for (int vo = vb; vo < (ONE ? V32 : vb + 1); ++vo) {
      const h8_t z = ld8(Z + vo * 2048) * own_factor(3, vo), y = bf16_to_h8(buf_ld(ry, ov + 64 * vo), sy);
      float vv[8];
      bf16x8_to_f32(buf_ld(rv, ov + 64 * vo), vv);
#pragma unroll
      for (int x = 0; x < 8; ++x) zv = fmaf((float)z[x], vv[x], zv);
      const h8_t fu = own_factor(1, vo), yu = y * fu, zu = z * fu;
      h8_t u = {};
#pragma unroll
      for (int j = 0; j < 4; ++j) {  // D[j][i], of which j <= i counts
        if (ONE && j > wv) break;
        u = ld8(U + (vo * 4 + j) * 512);
        s1[j] = mfma_k32(u, yu, s1[j]);
        s2[j] = mfma_k32(u, zu, s2[j]);
      }
      if (ONE) with_states(vo, y, z, u);  // (the last u is my own)
    }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    settle(s1[j]);
    settle(s2[j]);
  }
  __syncthreads();
  // S1, S2 masked; their largest entries, so that they can be fp16 whatever U is
  const float ghi = ge[2 * C + i], glo = ge[3 * C + i];
#pragma unroll
  for (int jt = 0; jt < 4; ++jt)
    {
      const f4_t h = *(const f4_t *)&ge[2 * C + 16 * jt + 4 * g4], l = *(const f4_t *)&ge[3 * C + 16 * jt + 4 * g4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int j = 16 * jt + 4 * g4 + x;
        const float e = exp2_((ghi - h[x]) + (glo - l[x]));
        s1[jt][x] = j <= i ? e * s1[jt][x] : 0.f;
        s2[jt][x] = j < i ? -e * s2[jt][x] : 0.f;
      }
    }
  const float top1 = wave_top([&](auto put) {
#pragma unroll
    for (int jt = 0; jt < 4; ++jt)
#pragma unroll
      for (int x = 0; x < 4; ++x) put(s1[jt][x]);
  });
  const float top2 = wave_top([&](auto put) {
#pragma unroll
    for (int jt = 0; jt < 4; ++jt)
#pragma unroll
      for (int x = 0; x < 4; ++x) put(s2[jt][x]);
  });
  zv += __shfl_xor(zv, 16, 64);
  zv += __shfl_xor(zv, 32, 64);
  if (lane == 0) {
    red[wv] = top1;
    red[4 + wv] = top2;
  }
  __syncthreads();
  const int x1 = exponent_of(*(const f4_t *)red), x2 = exponent_of(*(const f4_t *)(red + 4));
  const float ss1 = two_to(-x1), ss2 = two_to(-x2), bt = ge[4 * C + i], gt = ge[C + i];
  const float om = gate_unit(ge[2 * C]), gm = om * ge[i];
#pragma unroll
  for (int jt = 0; jt < 4; ++jt) {  // (the last tile of an even wave's pair is zero)
    const int o = i * LC + 16 * jt + 4 * g4;
    *(u2_t *)&S1[o] = pack4_h(ss1 * s1[jt]);
    *(u2_t *)&S2[o] = pack4_h(ss2 * s2[jt]);
  }

  if (!ONE)
#pragma unroll
    for (int vb = 0; vb < V32; ++vb) {
      with_states(vb, bf16_to_h8(buf_ld(ry, ov + 64 * vb), sy), ld8(Z + vb * 2048) * own_factor(3, vb), ld8(U + (vb * 4 + wv) * 512));
    }
#pragma unroll
  for (int x = 0; x < KT; ++x) {
    settle(dq[x]);
    settle(as[x]);
    settle(kept[x]);
  }
#pragma unroll
  for (int m = 1; m < 64; m *= 2) hd += __shfl_xor(hd, m, 64);
  if (lane == 0) red[8 + wv] = hd;
  __syncthreads();
  const bool heads = a.N != a.Nqk;
  // every product with the powers of two that its factors came without
  const float cq = gm * two_to(eh + eY), ca = -gm * two_to(eh + eZ), ck = gt * two_to(eu + eD);
  const float c1k = two_to(x1 + eu + eY + ek), c1q = two_to(x1 + eu + eY + eq), c2 = two_to(x2 + eu + eZ + ek);
  const float cb = two_to(x2 + eu + eZ + eb + ek);
  float dGq = 0.f, dGk = 0.f, kb1 = 0.f, tail = 0.f;
  h8_t row1[2], row2[2], col1[2], colb[2];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    row1[kb] = ld8(S1 + i * LC + 32 * kb + 8 * g4);
    row2[kb] = ld8(S2 + i * LC + 32 * kb + 8 * g4);
    col1[kb] = ld8_tr(S1, LC, 32 * kb, 16 * wv);
    colb[kb] = ld8_tr(S2, LC, 32 * kb, 16 * wv) * ld8(bh + 32 * kb + 8 * g4);
  }
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    const f4_t kd = kept[kt];
    f4_t x = zero, y = zero, w = zero, wb = zero;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const h8_t kT = ld8_tr(ks, LK, 32 * kb, 16 * kt), qT = ld8_tr(qs, LK, 32 * kb, 16 * kt);
      x = mfma_k32(kT, row1[kb], x);
      y = mfma_k32(kT, row2[kb], y);
      w = mfma_k32(qT, col1[kb], w);
      wb = mfma_k32(kT, colb[kb], wb);
    }
    settle(x);
    settle(y);
    settle(w);
    settle(wb);
    const h4_t qv = *(const h4_t *)&qs[i * LK + 16 * kt + 4 * g4], kv = *(const h4_t *)&ks[i * LK + 16 * kt + 4 * g4];
    f4_t o;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float q_ = (float)qv[r], k_ = (float)kv[r];
      x[r] = fmaf(c1k, x[r], cq * dq[kt][r]);
      y[r] = fmaf(c2, y[r], ca * as[kt][r]);
      w[r] = fmaf(c1q, w[r], fmaf(cb, wb[r], ck * kd[r]));
      o[r] = fmaf(bt, y[r], w[r]);
      dGq = fmaf(q_, x[r], dGq);
      dGk = fmaf(k_, fmaf(bt, y[r], -w[r]), dGk);
      kb1 = fmaf(k_, y[r], kb1);
      tail = fmaf(ck * k_, kd[r], tail);
    }
    if (own < a.T) {
      const size_t m = ((size_t)b * a.T + own) * (heads ? a.N : a.Nqk) * K + (size_t)(heads ? n : nq) * K + 16 * kt + 4 * g4;
      if (heads) {
        *(f4_t *)&dq_heads[m] = x;
        *(f4_t *)&dk_heads[m] = o;
      } else {
        *(u2_t *)((unsigned short *)a.dq + m) = u2_t{pack2_bf16(x[0], x[1]), pack2_bf16(x[2], x[3])};
        *(u2_t *)((unsigned short *)a.dk + m) = u2_t{pack2_bf16(o[0], o[1]), pack2_bf16(o[2], o[3])};
      }
    }
  }
  const float k1 = two_to(ek);
  float dG = fmaf(two_to(eq), dGq, k1 * dGk);
  kb1 *= k1;
  tail *= k1;
  dG += __shfl_xor(dG, 16, 64);
  dG += __shfl_xor(dG, 32, 64);
  kb1 += __shfl_xor(kb1, 16, 64);
  kb1 += __shfl_xor(kb1, 32, 64);
#pragma unroll
  for (int m = 1; m < 64; m *= 2) tail += __shfl_xor(tail, m, 64);
  if (lane == 0) red[12 + wv] = tail;
  if (g4 == 0) red[16 + i] = dG;
  if (g4 == 0 && own < a.T)
    ((__hip_bfloat16 *)a.dbeta)[((size_t)b * a.T + own) * a.N + n] = __float2bfloat16(two_to(eZ) * zv + kb1);
  __syncthreads();
  if (wv == 0) {  // sums over the steps behind, in 64 bits; <H_C, dH> at the last one
    double s = (double)red[16 + lane];
    if (lane == C - 1)
      for (int w = 0; w < 4; ++w) s += (double)(om * ge[C - 1]) * two_to(eh + eD) * red[8 + w] + red[12 + w];
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
      const double o = __shfl_down(s, m, 64);
      if (lane + m < 64) s += o;
    }
    if (t0 + lane < a.T)
      ((__hip_bfloat16 *)a.dg)[((size_t)b * a.T + t0 + lane) * a.N + n] = __float2bfloat16((float)s);
  }
}

// dq and dk of heads that share q and k: the sums over the heads of a group, in increasing order.  Memory-bound:
// 8 x 1000 steps, 12 heads of K = 64 on 4: 9.8 us, 5.9 TB/s with what the caches still hold.
__global__ void __launch_bounds__(256)
    delta_half_heads_kernel(const float *__restrict__ dq_heads, const float *__restrict__ dk_heads, void *__restrict__ dq,
                            void *__restrict__ dk, size_t vecs, int K4, int rep) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < vecs; i += (size_t)gridDim.x * 256) {
    const size_t row = i / K4, c = i - row * K4;  // four elements of [B T Nqk][K]
    const float *src = (blockIdx.y ? dk_heads : dq_heads) + (row * rep * K4 + c) * 4;
    f4_t s = *(const f4_t *)src;
    for (int r = 1; r < rep; ++r) s += *(const f4_t *)(src + (size_t)r * K4 * 4);
    *(u2_t *)((unsigned short *)(blockIdx.y ? dk : dq) + 4 * i) = u2_t{pack2_bf16(s[0], s[1]), pack2_bf16(s[2], s[3])};
  }
}

// ------------------------------------------------------------------ launches
struct Ws {
  float *gates, *carry;
  half_t *mats, *dstates, *rows_z;
  u4_t *exps;
  float *dqh, *dkh;
};
Ws carve(const DeltaLayout &l, char *p) {
  Ws w;
  w.gates = (float *)p;
  w.mats = (half_t *)(p += l.gates);
  w.carry = (float *)(p += l.mats);
  w.dstates = (half_t *)(p += l.carry);
  w.rows_z = (half_t *)(p += l.states);
  w.exps = (u4_t *)(p += l.rows);
  w.dqh = (float *)(p += l.dexps);
  w.dkh = (float *)(p += l.heads);
  return w;
}

// Columns of V per workgroup of the kernels that run in order: 32, or 16 where that leaves half of the 256 CUs
// without one.  us, forward + backward of 1024 steps, 32 -> 16 columns, by the workgroups that there are with 32:
//                32           64          128          160          256          512
//   32 x 32    96 ->  84   104 ->  92   122 -> 112   130 -> 132   165 -> 167   329 -> 371
//   64 x 64   103 ->  84   114 ->  94   132 -> 114   138 -> 139   163 -> 165   300 -> 333
//  128 x 128  130 -> 108   135 -> 112   149 -> 126   165 -> 182   184 -> 199   355 -> 405
int columns(const DeltaArgs &a) {
  return a.B * a.N * (a.V / 32) <= 128 ? 16 : 32;
}
// Chunks per launch of the forward.  Where its chains have no more than half of the CUs, a long one goes in parts whose
// launches also form T and P of the next part, on the idle CUs: in parts of about 1024 chunks over all states, as many
// as run at once (longer ones keep the chains' CUs busy as well), and of 16 each at least, for a launch's 6 us.
// us, whole -> parts of half, once, twice as many: 65 536 steps of 32 states 64 x 64 1592 -> 1631, 1471, 1462; 32 768 of
// 16 of 64 x 128 675 -> 718, 679, 670; of 8 of 128 x 128 823 -> 837, 821, 819.  With chains on all 256 CUs there is
// nothing to gain (8 x 4096 steps, 16 of 64 x 64: 231 -> 228 to 241).
int part_chunks(const DeltaArgs &a, int chunks) {
  const int units = a.B * a.N;
  if (units == 0 || units * (a.V / columns(a)) > 128) return chunks;
  return std::min(chunks, std::max(16, 1024 / units));
}

template <bool BWD>
hipError_t prep(const DeltaArgs &a, const DeltaLayout &l, int c0, int c1, const Ws &w, hipStream_t s) {
  const dim3 grid((unsigned)(a.B * a.N) * (unsigned)(c1 - c0));
  if (a.K == 32) hipLaunchKernelGGL((delta_half_prep_kernel<32, BWD>), grid, dim3(256), 0, s, a, l.chunks, c0, c1, w.gates, w.mats);
  else if (a.K == 64) hipLaunchKernelGGL((delta_half_prep_kernel<64, BWD>), grid, dim3(256), 0, s, a, l.chunks, c0, c1, w.gates, w.mats);
  else hipLaunchKernelGGL((delta_half_prep_kernel<128, BWD>), grid, dim3(256), 0, s, a, l.chunks, c0, c1, w.gates, w.mats);
  return hipGetLastError();
}
template <int K, int VB, bool Y, bool CKPT>
hipError_t fwd_go(const DeltaArgs &a, const DeltaLayout &l, const Ws &w, hipStream_t s) {
  constexpr int lds = std::max<int>(lds_fwd<K, VB>(), sizeof(PrepLds));
  hipError_t e = set_max_lds_once(delta_half_fwd_kernel<K, VB, Y, CKPT>, lds);
  const int step = part_chunks(a, l.chunks);
  if (e == hipSuccess && l.chunks > 0) e = prep<false>(a, l, 0, step, w, s);
  Part p = {0, 0, 0, delta_grid(a.B * a.N, a.V / VB), a.H0, nullptr};
  do {
    if (e != hipSuccess) return e;
    p.c1 = std::min(p.c0 + step, l.chunks);
    p.c2 = std::min(p.c1 + step, l.chunks);
    p.HT = p.c1 < l.chunks ? w.carry : a.HT;
    hipLaunchKernelGGL((delta_half_fwd_kernel<K, VB, Y, CKPT>), dim3(p.scans + (unsigned)(a.B * a.N) * (unsigned)(p.c2 - p.c1)),
                       dim3(256), lds, s, a, l.chunks, p, w.gates, w.mats, (half_t *)a.ckpt,
                       a.ckpt ? (half_t *)(a.ckpt + l.states) : nullptr,
                       a.ckpt ? (int *)(a.ckpt + l.states + l.rows) : nullptr);
    e = hipGetLastError();
    p.c0 = p.c1;
    p.H0 = w.carry;
  } while (p.c0 < l.chunks);
  return e;
}
template <int K, int VB>
hipError_t fwd_kv(const DeltaArgs &a, const DeltaLayout &l, const Ws &w, hipStream_t s) {
  if (!a.write_y) return fwd_go<K, VB, false, true>(a, l, w, s);
  return a.ckpt ? fwd_go<K, VB, true, true>(a, l, w, s) : fwd_go<K, VB, true, false>(a, l, w, s);
}
template <int K, int V32>
hipError_t grad_go(const DeltaArgs &a, const DeltaLayout &l, const Ws &w, int vb, hipStream_t s) {
  constexpr int lds = lds_grad<K>();
  const hipError_t e = set_max_lds_once(delta_half_grad_kernel<K, V32>, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((delta_half_grad_kernel<K, V32>), dim3((unsigned)(a.B * a.N) * (unsigned)l.chunks), dim3(256), lds, s,
                     a, l.chunks, vb, w.gates, (const half_t *)a.ckpt, (const half_t *)(a.ckpt + l.states),
                     (const int *)(a.ckpt + l.states + l.rows), w.dstates, w.rows_z, w.exps, w.dqh, w.dkh);
  return hipGetLastError();
}
template <int K, int VB>
hipError_t bwd_kv(const DeltaArgs &a, const DeltaLayout &l, const Ws &w, hipStream_t s) {
  constexpr int lds = lds_bwd<K, VB>();
  hipError_t e = set_max_lds_once(delta_half_bwd_kernel<K, VB>, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((delta_half_bwd_kernel<K, VB>), dim3(delta_grid(a.B * a.N, a.V / VB)), dim3(256), lds, s, a, l.chunks, w.gates, w.mats, w.dstates, w.rows_z, w.exps);
  if ((e = hipGetLastError()) != hipSuccess || l.chunks == 0) return e;
  switch (a.V) {
    case 32: return grad_go<K, 1>(a, l, w, VB, s);
    case 64: return grad_go<K, 2>(a, l, w, VB, s);
    case 128: return grad_go<K, 4>(a, l, w, VB, s);
    default: return grad_go<K, 8>(a, l, w, VB, s);
  }
}
template <int K>
hipError_t fwd_k(const DeltaArgs &a, const DeltaLayout &l, const Ws &w, hipStream_t s) {
  return columns(a) == 32 ? fwd_kv<K, 32>(a, l, w, s) : fwd_kv<K, 16>(a, l, w, s);
}
template <int K>
hipError_t bwd_k(const DeltaArgs &a, const DeltaLayout &l, const Ws &w, hipStream_t s) {
  return columns(a) == 32 ? bwd_kv<K, 32>(a, l, w, s) : bwd_kv<K, 16>(a, l, w, s);
}
hipError_t scan(const DeltaArgs &a, const DeltaLayout &l, const Ws &w, hipStream_t s) {
  return a.K == 32 ? fwd_k<32>(a, l, w, s) : a.K == 64 ? fwd_k<64>(a, l, w, s) : fwd_k<128>(a, l, w, s);
}

}  // namespace

// (K = 16 and V = 16 fill half an operand; they run on the fp32 kernels)
bool delta_half_serves(int K, int V, int io) { return io == 1 && K >= 32 && V >= 32; }

DeltaLayout delta_half_layout(const DeltaArgs &a) {
  DeltaLayout l;
  l.C = C;
  l.kept = false;
  l.chunks = ceil_div(a.T, C);
  const size_t n = (size_t)a.B * a.N * l.chunks, steps = (size_t)a.B * a.T * a.N;
  l.gates = align256(n * kGates * sizeof(float));
  l.mats = align256(n * 2 * kMat * sizeof(half_t));
  l.carry = part_chunks(a, l.chunks) < l.chunks ? align256((size_t)a.B * a.N * a.K * a.V * sizeof(float)) : 0;
  l.states = align256(n * a.K * a.V * sizeof(half_t));
  l.rows = align256(n * C * a.V * sizeof(half_t));
  l.exps = align256(n * (a.V / 16) * 2 * sizeof(int));
  l.dexps = align256(n * (a.V / 16) * sizeof(u4_t));
  l.heads = a.N != a.Nqk ? align256(steps * a.K * sizeof(float)) : 0;
  return l;
}
hipError_t delta_half_fwd(const DeltaArgs &a, hipStream_t s) {
  const DeltaLayout l = delta_half_layout(a);
  const Ws w = carve(l, a.ws);
  return scan(a, l, w, s);
}
hipError_t delta_half_bwd(const DeltaArgs &a, hipStream_t s) {
  const DeltaLayout l = delta_half_layout(a);
  const Ws w = carve(l, a.ws);
  hipError_t e;
  if (a.own_ckpt && l.chunks > 0) {
    DeltaArgs f = a;
    f.write_y = 0;
    f.HT = nullptr;
    if ((e = delta_half_fwd(f, s)) != hipSuccess) return e;
  }
  if (l.chunks > 0 && (e = prep<true>(a, l, 0, l.chunks, w, s)) != hipSuccess) return e;
  e = a.K == 32 ? bwd_k<32>(a, l, w, s) : a.K == 64 ? bwd_k<64>(a, l, w, s) : bwd_k<128>(a, l, w, s);
  if (e != hipSuccess || l.chunks == 0 || a.N == a.Nqk) return e;
  const size_t vecs = (size_t)a.B * a.T * a.Nqk * (a.K / 4);
  const size_t blocks = (vecs + 255) / 256;
  hipLaunchKernelGGL(delta_half_heads_kernel, dim3((unsigned)(blocks < (1u << 20) ? blocks : 1u << 20), 2), dim3(256), 0, s, w.dqh, w.dkh, a.dq,
                     a.dk, vecs, a.K / 4, a.N / a.Nqk);
  return hipGetLastError();
}

}  // namespace m2rnn
