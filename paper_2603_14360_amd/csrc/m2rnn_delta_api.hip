// Host side of the gated delta rule's entry points (include/m2rnn.h): validation, sizes and the choice of
// kernels.
#include "../../include/m2rnn.h"

#include "m2rnn_delta.hpp"

using namespace m2rnn;

namespace {

m2rnn_status check(const m2rnn_desc *d) {
  if (!d) return M2RNN_ERR_NULL;
  if (d->io != M2RNN_F32 && d->io != M2RNN_BF16) return M2RNN_ERR_DTYPE;
  if (d->B < 0 || d->T < 0 || d->N < 1 || d->Nqk < 1 || d->N % d->Nqk != 0) return M2RNN_ERR_SHAPE;
  const auto dim = [](int x) { return x == 16 || x == 32 || x == 64 || x == 128; };
  if (!dim(d->K) || !(dim(d->V) || d->V == 256) || d->flags != 0) return M2RNN_ERR_SHAPE;
  if ((double)d->B * (d->T > 0 ? d->T : 1) * d->N * d->K * d->V > 1e15) return M2RNN_ERR_SHAPE;
  // (units times parts or chunks are workgroups of 256 threads, of which a launch has fewer than 2^32; for the parts
  // delta_grid counts units in eights)
  const double units = (double)d->B * d->N, most = (1 << 24) - 1;
  if (units > (1 << 20) - 8 || units * (d->T / 32 + 1) > most) return M2RNN_ERR_SHAPE;
  // (a chunk's rows are reached by 31-bit byte offsets)
  if ((double)d->N * d->V >= (1 << 23) || (double)d->Nqk * d->K >= (1 << 23)) return M2RNN_ERR_SHAPE;
  if (d->chunk != 0) return M2RNN_ERR_CHUNK;
  return M2RNN_OK;
}

DeltaArgs args_of(const m2rnn_desc *d) {
  DeltaArgs a = {};
  a.B = d->B; a.T = d->T; a.N = d->N; a.Nqk = d->Nqk; a.K = d->K; a.V = d->V; a.io = d->io;
  a.write_y = 1;
  return a;
}
bool half(const DeltaArgs &a) { return delta_half_serves(a.K, a.V, a.io); }
DeltaLayout layout(const DeltaArgs &a) { return half(a) ? delta_half_layout(a) : delta_f32_layout(a); }
hipError_t run_fwd(const DeltaArgs &a, hipStream_t s) { return half(a) ? delta_half_fwd(a, s) : delta_f32_fwd(a, s); }
hipError_t run_bwd(const DeltaArgs &a, hipStream_t s) { return half(a) ? delta_half_bwd(a, s) : delta_f32_bwd(a, s); }

size_t ckpt_bytes(const DeltaLayout &l) { return l.states + l.rows + l.exps + (l.kept ? l.gates + l.mats : 0); }
size_t ws_bytes(const DeltaLayout &l, int bwd) {
  // (a backward finds what is kept with the checkpoints there)
  const size_t fwd = (bwd && l.kept ? 0 : l.gates + l.mats) + l.carry;
  return bwd ? fwd + l.states + l.rows + l.dexps + 2 * l.heads + (bwd >= 2 ? ckpt_bytes(l) : 0) : fwd;
}
bool few_steps(const m2rnn_desc *d) { return d->T <= delta_step_most((double)d->B * d->N, d->K, d->V); }
// A forward of so many steps needs no workspace: without one it runs step by step, whatever is faster.
bool needs_no_room(const m2rnn_desc *d) { return d->T <= (d->io == M2RNN_BF16 ? 12 : 16); }
bool misaligned(const void *p) { return ((uintptr_t)p & 15u) != 0; }

}  // namespace

extern "C" {

size_t m2rnn_delta_ckpt_bytes(const m2rnn_desc *desc) {
  return check(desc) == M2RNN_OK ? ckpt_bytes(layout(args_of(desc))) : 0;
}

size_t m2rnn_delta_workspace_bytes(const m2rnn_desc *desc, int bwd) {
  return check(desc) == M2RNN_OK ? ws_bytes(layout(args_of(desc)), bwd) : 0;
}

const char *m2rnn_delta_route_string(const m2rnn_desc *desc, int bwd) {
  if (check(desc) != M2RNN_OK) return "invalid descriptor";
  if (!bwd && few_steps(desc)) return "step";
  return half(args_of(desc)) ? "chunk64<half>" : "chunk32<f32>";
}

m2rnn_status m2rnn_delta_fwd(const m2rnn_desc *desc, const void *q, const void *k, const void *v, const float *g,
                             const float *beta, const float *H0, void *y, float *HT, void *ckpt, void *workspace,
                             size_t workspace_bytes, void *hip_stream) {
  const m2rnn_status st = check(desc);
  if (st != M2RNN_OK) return st;
  if (desc->B > 0 && desc->T > 0 && (!q || !k || !v || !g || !beta || !y)) return M2RNN_ERR_NULL;
  for (const void *p : {q, k, v, (const void *)g, (const void *)beta, (const void *)H0, (const void *)y,
                        (const void *)HT, (const void *)ckpt, (const void *)workspace})
    if (misaligned(p)) return M2RNN_ERR_ALIGN;
  DeltaArgs a = args_of(desc);
  a.q = q; a.k = k; a.v = v; a.g = g; a.beta = beta; a.H0 = H0; a.y = y; a.HT = HT;
  a.ckpt = (char *)ckpt; a.ws = (char *)workspace;
  size_t need = ws_bytes(layout(a), 0);
  const bool room = workspace && workspace_bytes >= need;
  const bool step = !ckpt && (few_steps(desc) || (!room && needs_no_room(desc)));
  if (step) need = 0;
  if (need > 0 && (!workspace || workspace_bytes < need)) return workspace ? M2RNN_ERR_WORKSPACE : M2RNN_ERR_NULL;
  if (desc->B == 0) return M2RNN_OK;
  hipStream_t s = (hipStream_t)hip_stream;
  return (step ? delta_step_fwd(a, s) : run_fwd(a, s)) == hipSuccess ? M2RNN_OK : M2RNN_ERR_HIP;
}

m2rnn_status m2rnn_delta_bwd(const m2rnn_desc *desc, const void *q, const void *k, const void *v, const float *g,
                             const float *beta, const float *H0, const void *ckpt, const void *dy, const float *dHT,
                             void *dq, void *dk, void *dv, void *dg, void *dbeta, float *dH0, void *workspace,
                             size_t workspace_bytes, void *hip_stream) {
  const m2rnn_status st = check(desc);
  if (st != M2RNN_OK) return st;
  if (desc->B > 0 && desc->T > 0 && (!q || !k || !v || !g || !beta || !dy || !dq || !dk || !dv || !dg || !dbeta))
    return M2RNN_ERR_NULL;
  for (const void *p : {q, k, v, (const void *)g, (const void *)beta, (const void *)H0, ckpt, dy, (const void *)dHT,
                        (const void *)dq, (const void *)dk, (const void *)dv, (const void *)dg, (const void *)dbeta,
                        (const void *)dH0, (const void *)workspace})
    if (misaligned(p)) return M2RNN_ERR_ALIGN;
  DeltaArgs a = args_of(desc);
  const DeltaLayout l = layout(a);
  const size_t need = ws_bytes(l, ckpt ? 1 : 2);
  if (need > 0 && (!workspace || workspace_bytes < need)) return workspace ? M2RNN_ERR_WORKSPACE : M2RNN_ERR_NULL;
  if (desc->B == 0) return M2RNN_OK;
  a.q = q; a.k = k; a.v = v; a.g = g; a.beta = beta; a.H0 = H0; a.dy = dy; a.dHT = dHT;
  a.dq = dq; a.dk = dk; a.dv = dv; a.dg = dg; a.dbeta = dbeta; a.dH0 = dH0; a.ws = (char *)workspace;
  // (only read where it is the caller's)
  a.ckpt = ckpt ? (char *)const_cast<void *>(ckpt) : a.ws + ws_bytes(l, 1);
  a.own_ckpt = !ckpt;
  return run_bwd(a, (hipStream_t)hip_stream) == hipSuccess ? M2RNN_OK : M2RNN_ERR_HIP;
}

}  // extern "C"
