// fc.hip -- FC column shard forward and backward (sec. 3.1: a LINEAR layer
// split to 1/K of its outputs, run on the batch the modulo layer gathers;
// its backward yields this shard's partial gradient over the full input).
//
//   forward   Y   = X * W_sh (+ b) (ReLU)       [m x ns] = [m x kin][kin x ns]
//   backward  dXp = G * W_sh^T                  [m x kin]
//             dW  = (dW +) X^T * G              [kin x ns]
//             db  = (db +) column sums of G     [ns]
// with G = dY, or dY * [mask > 0] (ReLU of this shard's output).
//
// One GEMM kernel on the bf16 MFMA (gemm_split, fc_gemm.hpp) serves the three
// products.  fp32 operands are split in three bf16 parts (split_bf16.hpp, six
// MFMAs per product); bf16 operands are their own first part, so their products
// are exact with one MFMA, and y and dx_partial are rounded to nearest-even on
// store.  Sums, dW and db are fp32.  The backward's bias gradient is added up
// inside the dW product.  Tile shapes and reduction splits are chosen per shape
// (gemm_plan).
#include "fc_gemm.hpp"

using namespace sb;

static sb_status fc_check(const sb_fc_desc* d) {
  if (!d) return SB_ERR_INVALID_ARG;
  if (d->m <= 0 || d->k_in <= 0 || d->n_shard <= 0) return SB_ERR_INVALID_ARG;
  if (d->ldx < d->k_in || d->ldy < d->n_shard) return SB_ERR_INVALID_ARG;
  if (d->flags & ~SB_FUSE_RELU) return SB_ERR_INVALID_ARG;
  if (d->dtype != SB_F32 && d->dtype != SB_BF16) return SB_ERR_INVALID_ARG;
  return SB_OK;
}

// The plans of the three products: Y, dX partial, dW.
static GemmPlan plan_y(const sb_fc_desc* d) {
  return product_plan(d->m, d->n_shard, d->k_in, d->ldx, true, d->n_shard, false,
                      (int)sbh::dsize(d->dtype));
}
static GemmPlan plan_dx(const sb_fc_desc* d) {
  return product_plan(d->m, d->k_in, d->n_shard, d->ldy, true, d->n_shard, true,
                      (int)sbh::dsize(d->dtype));
}
static GemmPlan plan_dw(const sb_fc_desc* d) {
  return product_plan(d->k_in, d->n_shard, d->m, d->ldx, false, d->ldy, false,
                      (int)sbh::dsize(d->dtype));
}

extern "C" size_t sb_fc_workspace_bytes(const sb_fc_desc* d, int pass) {
  if (fc_check(d) != SB_OK) return (size_t)-1;
  if (pass == SB_FC_FWD) return plan_y(d).ws_bytes;
  if (pass == SB_FC_BWD)   // dX partial, then dW: the two share the workspace
    return std::max(plan_dx(d).ws_bytes, plan_dw(d).ws_bytes);
  return (size_t)-1;
}

// Forward on operands of type E (fp32, or bf16 bits with a bf16 output).
template <class E>
static sb_status fc_fwd_run(const sb_fc_desc* d, const GemmPlan& p, const void* x, const void* w,
                            const float* b, void* y, void* ws, size_t ws_bytes, hipStream_t st) {
  GemmArgs g{};
  g.a = x; g.lda = d->ldx; g.amask = nullptr;
  g.b = w; g.ldb = d->n_shard; g.bmask = nullptr;
  g.c = y; g.ldc = d->ldy;
  g.M = d->m; g.N = d->n_shard; g.K = d->k_in;
  g.bias = b; g.relu = (d->flags & SB_FUSE_RELU) ? 1 : 0; g.accumulate = 0;
  return gemm_run<true, false, E, E>(g, p, (float*)ws, ws_bytes, st);
}

extern "C" sb_status sb_fc_shard_fwd(const sb_fc_desc* d, const void* x, const void* w,
                                     const float* b, void* y, void* ws, size_t ws_bytes,
                                     void* stream) {
  sb_status s = fc_check(d);
  if (s != SB_OK) return s;
  if (!x || !w || !y) return SB_ERR_INVALID_ARG;
  const size_t es = d->dtype == SB_BF16 ? 2 : 4;
  size_t xb = ((size_t)(d->m - 1) * d->ldx + d->k_in) * es;
  size_t yb = ((size_t)(d->m - 1) * d->ldy + d->n_shard) * es;
  size_t wb = (size_t)d->k_in * d->n_shard * es;
  if (sbh::overlaps(y, yb, x, xb) || sbh::overlaps(y, yb, w, wb) ||
      sbh::overlaps(y, yb, b, b ? d->n_shard * sizeof(float) : 0))
    return SB_ERR_INVALID_ARG;
  // The workspace (split partials) must not overlap any operand.
  const GemmPlan p = plan_y(d);
  const size_t need = p.ws_bytes;
  if (need > 0 && (sbh::overlaps(ws, need, x, xb) || sbh::overlaps(ws, need, w, wb) ||
                   sbh::overlaps(ws, need, y, yb) ||
                   sbh::overlaps(ws, need, b, b ? d->n_shard * sizeof(float) : 0)))
    return SB_ERR_INVALID_ARG;
  hipStream_t st = sbh::stream_of(stream);
  s = d->dtype == SB_BF16 ? fc_fwd_run<u16>(d, p, x, w, b, y, ws, ws_bytes, st)
                          : fc_fwd_run<float>(d, p, x, w, b, y, ws, ws_bytes, st);
  if (s != SB_OK) return s;
  return sbh::launch_status();
}

// Backward on operands of type E: dx_partial has type E, dW and db fp32.
// db is added up inside the dW product.
template <class E>
static sb_status fc_bwd_run(const sb_fc_desc* d, const GemmPlan& px, const GemmPlan& pw,
                            const void* x, const void* w, const void* dy, const void* mask,
                            void* dxp, float* dw, float* db, int accumulate, void* ws,
                            size_t ws_bytes, hipStream_t st) {
  sb_status s;
  if (dxp) {
    GemmArgs g{};
    g.a = dy; g.lda = d->ldy; g.amask = mask;
    g.b = w; g.ldb = d->n_shard; g.bmask = nullptr;
    g.c = dxp; g.ldc = d->ldx;
    g.M = d->m; g.N = d->k_in; g.K = d->n_shard;
    s = gemm_run<true, true, E, E>(g, px, (float*)ws, ws_bytes, st);
    if (s != SB_OK) return s;
  }
  GemmArgs g{};
  g.a = x; g.lda = d->ldx; g.amask = nullptr;
  g.b = dy; g.ldb = d->ldy; g.bmask = mask;
  g.c = dw; g.ldc = d->n_shard;
  g.M = d->k_in; g.N = d->n_shard; g.K = d->m;
  g.accumulate = accumulate;
  g.colsum = db; g.colsum_acc = accumulate;
  return gemm_run<false, false, E, float>(g, pw, (float*)ws, ws_bytes, st);
}

extern "C" sb_status sb_fc_shard_bwd(const sb_fc_desc* d, const void* x, const void* w,
                                     const void* dy, const void* mask, void* dxp, float* dw,
                                     float* db, int accumulate, void* ws, size_t ws_bytes,
                                     void* stream) {
  sb_status s = fc_check(d);
  if (s != SB_OK) return s;
  if (d->flags != 0) return SB_ERR_INVALID_ARG;
  if (!x || !w || !dy || !dw) return SB_ERR_INVALID_ARG;
  if (accumulate != 0 && accumulate != 1) return SB_ERR_INVALID_ARG;
  const size_t es = d->dtype == SB_BF16 ? 2 : 4;
  size_t xb = ((size_t)(d->m - 1) * d->ldx + d->k_in) * es;
  size_t yb = ((size_t)(d->m - 1) * d->ldy + d->n_shard) * es;
  size_t wb = (size_t)d->k_in * d->n_shard * es;
  size_t dwb = (size_t)d->k_in * d->n_shard * sizeof(float);
  size_t dbb = (size_t)d->n_shard * sizeof(float);
  const void* ins[4] = {x, w, dy, mask};
  size_t insb[4] = {xb, wb, yb, mask ? yb : 0};
  void* outs[3] = {dxp, dw, db};
  size_t outsb[3] = {dxp ? xb : 0, dwb, db ? dbb : 0};
  for (int o = 0; o < 3; ++o) {
    for (int i = 0; i < 4; ++i)
      if (sbh::overlaps(outs[o], outsb[o], ins[i], insb[i])) return SB_ERR_INVALID_ARG;
    for (int o2 = o + 1; o2 < 3; ++o2)
      if (sbh::overlaps(outs[o], outsb[o], outs[o2], outsb[o2])) return SB_ERR_INVALID_ARG;
  }
  const GemmPlan px = plan_dx(d), pw = plan_dw(d);
  const size_t need = std::max(px.ws_bytes, pw.ws_bytes);
  if (need > 0 && (!ws || ws_bytes < need)) return SB_ERR_WORKSPACE;
  // The workspace (split partials) must not overlap any operand.
  if (need > 0) {
    for (int i = 0; i < 4; ++i)
      if (sbh::overlaps(ws, need, ins[i], insb[i])) return SB_ERR_INVALID_ARG;
    for (int o = 0; o < 3; ++o)
      if (sbh::overlaps(ws, need, outs[o], outsb[o])) return SB_ERR_INVALID_ARG;
  }
  hipStream_t st = sbh::stream_of(stream);
  s = d->dtype == SB_BF16
          ? fc_bwd_run<u16>(d, px, pw, x, w, dy, mask, dxp, dw, db, accumulate, ws, ws_bytes, st)
          : fc_bwd_run<float>(d, px, pw, x, w, dy, mask, dxp, dw, db, accumulate, ws, ws_bytes, st);
  if (s != SB_OK) return s;
  return sbh::launch_status();
}
