// gated.hip -- gated FC column shard forward and backward (sec. 3.1 Layer
// Partitioning: a dense layer split to 1/K of its outputs on the gathered batch;
// here the layer's ReLU is a gate).
//
//   forward   a = x Wg + bg,  u = x Wu + bu,  y = act(a) u
//   backward  da = dy u act'(a),  du = dy act(a)
//             dx  = da Wg^T + du Wu^T                       [m x kin]
//             dWg = x^T da,  dWu = x^T du,  db their column sums
//
// The products run on gemm_split (fc_gemm.hpp); a and u are kept in fp32.  The
// weight gradients are fp32 also where x is bf16: da and du go into their
// products as three bf16 parts, which hold all 24 bits, so a gradient is off by
// the rounding of its fp32 sums and not by 2^-9 of every term.  dx of the bf16
// path is rounded to bf16 itself and takes their first parts.
#include "fc_gemm.hpp"

#include <cmath>

namespace sb {

// The activation and its derivative.
__device__ __forceinline__ void gate_act(int act, float a, float& f, float& df) {
  switch (act) {
    case SB_ACT_SIGMOID: {
      f = 1.f / (1.f + expf(-a));
      df = f * (1.f - f);
      break;
    }
    case SB_ACT_SILU: {
      const float p = 1.f / (1.f + expf(-a));
      f = a * p;
      df = p * (1.f + a * (1.f - p));
      break;
    }
    case SB_ACT_GELU: {
      const float c = 0.5f + 0.5f * erff(a * 0.70710678118654752f);
      f = a * c;
      df = c + a * expf(-0.5f * a * a) * 0.39894228040143268f;
      break;
    }
    case SB_ACT_GELU_TANH: {
      const float r = 0.79788456080286536f;
      const float t = tanhf(r * (a + 0.044715f * a * a * a));
      f = 0.5f * a * (1.f + t);
      df = 0.5f * (1.f + t) + 0.5f * a * (1.f - t * t) * r * (1.f + 0.134145f * a * a);
      break;
    }
    default:
      f = a > 0.f ? a : 0.f;
      df = a > 0.f ? 1.f : 0.f;
  }
}

template <class E>
__global__ __launch_bounds__(256) void gated_act_fwd(int m, int n, int act,
                                                     const float* __restrict__ pre, E* y, int ldy) {
  const size_t mn = (size_t)m * n;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < mn; i += (size_t)gridDim.x * 256) {
    float f, df;
    gate_act(act, pre[i], f, df);
    const size_t r = i / n;
    Elem<E>::store(y, r * ldy + (i - r * n), f * pre[mn + i]);
  }
}

// da and du, dense [m][n]: fp32, or the three parts of each (part p of da at
// p * m * n, of du at (3 + p) * m * n).
template <class E>
__global__ __launch_bounds__(256) void gated_act_bwd(int m, int n, int act,
                                                     const float* __restrict__ pre,
                                                     const E* __restrict__ dy, int ldy, E* d) {
  const size_t mn = (size_t)m * n;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < mn; i += (size_t)gridDim.x * 256) {
    float f, df;
    gate_act(act, pre[i], f, df);
    const size_t r = i / n;
    const float g = Elem<E>::load(dy, r * ldy + (i - r * n));
    const float v[2] = {g * pre[mn + i] * df, g * f};
    if constexpr (sizeof(E) == 4) {
      d[i] = v[0];
      d[mn + i] = v[1];
    } else {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const u16 h = f32_to_bf16(v[q]);
        float rest = v[q] - bf16_to_f32(h);
        // An infinite or NaN first part is the whole value.
        if ((h & 0x7f80u) == 0x7f80u) rest = 0.f;
        const u16 mid = f32_to_bf16(rest);
        rest -= bf16_to_f32(mid);
        d[(3 * q) * mn + i] = h;
        d[(3 * q + 1) * mn + i] = mid;
        d[(3 * q + 2) * mn + i] = f32_to_bf16(rest);
      }
    }
  }
}

__global__ __launch_bounds__(256) void gated_round_dx(int m, int k, const float* __restrict__ s,
                                                      u16* dx, int ldx) {
  const size_t mk = (size_t)m * k;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < mk; i += (size_t)gridDim.x * 256) {
    const size_t r = i / k;
    dx[r * ldx + (i - r * k)] = f32_to_bf16(s[i]);
  }
}

static unsigned gated_blocks(size_t count) {
  return (unsigned)std::min<size_t>((count + 255) / 256, 65536);
}

// A workspace's parts, each from a multiple of 256 bytes on.
struct GatedSpace {
  size_t d, dx, gemm, bytes;               // offsets: da and du (or a and u), dx in fp32, splits
};

static GemmPlan gated_plan_y(const sb_gated_desc* d) {
  return product_plan(d->m, d->n_shard, d->k_in, d->ldx, true, d->n_shard, false,
                      (int)sbh::dsize(d->dtype));
}
static GemmPlan gated_plan_dx(const sb_gated_desc* d) {
  return product_plan(d->m, d->k_in, d->n_shard, d->n_shard, true, d->n_shard, true,
                      (int)sbh::dsize(d->dtype));
}
static GemmPlan gated_plan_dw(const sb_gated_desc* d) {
  return product_plan(d->k_in, d->n_shard, d->m, d->ldx, false, d->n_shard, false,
                      (int)sbh::dsize(d->dtype));
}

static GatedSpace gated_space(const sb_gated_desc* d, int pass, bool pre) {
  const size_t mn = (size_t)d->m * d->n_shard;
  GatedSpace s{};
  if (pass == SB_FC_FWD) {
    s.gemm = pre ? 0 : round_up(mn * 8, 256);
    s.bytes = s.gemm + gated_plan_y(d).ws_bytes;
  } else {
    s.dx = round_up(mn * (d->dtype == SB_BF16 ? 12 : 8), 256);
    s.gemm = s.dx + (d->dtype == SB_BF16 ? round_up((size_t)d->m * d->k_in * 4, 256) : 0);
    s.bytes = s.gemm + std::max(gated_plan_dx(d).ws_bytes, gated_plan_dw(d).ws_bytes);
  }
  return s;
}

static sb_status gated_check(const sb_gated_desc* d) {
  if (!d) return SB_ERR_INVALID_ARG;
  if (d->m <= 0 || d->k_in <= 0 || d->n_shard <= 0) return SB_ERR_INVALID_ARG;
  if (d->ldx < d->k_in || d->ldy < d->n_shard) return SB_ERR_INVALID_ARG;
  if (d->dtype != SB_F32 && d->dtype != SB_BF16) return SB_ERR_INVALID_ARG;
  if (d->act < SB_ACT_SIGMOID || d->act > SB_ACT_RELU) return SB_ERR_INVALID_ARG;
  // The kernels' ranges are below 2^31 bytes.
  const int64_t es = (int64_t)sbh::dsize(d->dtype), top = 1ll << 31;
  if (((int64_t)(d->m - 1) * d->ldx + d->k_in) * es >= top ||
      ((int64_t)(d->m - 1) * d->ldy + d->n_shard) * es >= top ||
      (int64_t)d->k_in * d->n_shard * es >= top)
    return SB_ERR_UNSUPPORTED;
  return SB_OK;
}

struct Span { const void* p; size_t bytes; };

static bool spans_meet(const Span* a, int na, const Span* b, int nb) {
  for (int i = 0; i < na; ++i)
    for (int j = 0; j < nb; ++j)
      if (sbh::overlaps(a[i].p, a[i].bytes, b[j].p, b[j].bytes)) return true;
  return false;
}

template <class E>
static sb_status gated_fwd_run(const sb_gated_desc* d, const void* x, const void* const* w,
                               const float* const* b, void* y, float* pre, char* ws,
                               size_t ws_bytes, hipStream_t st) {
  const size_t mn = (size_t)d->m * d->n_shard;
  const GatedSpace sp = gated_space(d, SB_FC_FWD, pre != nullptr);
  if (!pre) pre = (float*)ws;
  for (int q = 0; q < 2; ++q) {
    GemmArgs g{};
    g.a = x; g.lda = d->ldx;
    g.b = w[q]; g.ldb = d->n_shard;
    g.c = pre + q * mn; g.ldc = d->n_shard;
    g.M = d->m; g.N = d->n_shard; g.K = d->k_in;
    g.bias = b[q];
    const sb_status s = gemm_run<true, false, E, float>(g, gated_plan_y(d), (float*)(ws + sp.gemm),
                                                        ws_bytes - sp.gemm, st);
    if (s != SB_OK) return s;
  }
  gated_act_fwd<E><<<gated_blocks(mn), 256, 0, st>>>(d->m, d->n_shard, d->act, pre, (E*)y, d->ldy);
  return SB_OK;
}

template <class E>
static sb_status gated_bwd_run(const sb_gated_desc* d, const void* x, const void* const* w,
                               const float* pre, const void* dy, void* dx, float* const* dw,
                               float* const* db, int accumulate, char* ws, size_t ws_bytes,
                               hipStream_t st) {
  constexpr bool B16 = sizeof(E) == 2;
  constexpr int NP = B16 ? 3 : 1;
  const size_t mn = (size_t)d->m * d->n_shard;
  const GatedSpace sp = gated_space(d, SB_FC_BWD, true);
  float* split = (float*)(ws + sp.gemm);
  const size_t split_bytes = ws_bytes - sp.gemm;
  E* dd = (E*)ws;                          // part p of da at p * mn, of du at (NP + p) * mn
  gated_act_bwd<E><<<gated_blocks(mn), 256, 0, st>>>(d->m, d->n_shard, d->act, pre, (const E*)dy,
                                                     d->ldy, dd);
  if (dx) {
    float* sum = B16 ? (float*)(ws + sp.dx) : (float*)dx;
    const int ld = B16 ? d->k_in : d->ldx;
    for (int q = 0; q < 2; ++q) {
      GemmArgs g{};
      g.a = dd + (size_t)q * NP * mn; g.lda = d->n_shard;
      g.b = w[q]; g.ldb = d->n_shard;
      g.c = sum; g.ldc = ld;
      g.M = d->m; g.N = d->k_in; g.K = d->n_shard;
      g.accumulate = q;
      const sb_status s = gemm_run<true, true, E, float>(g, gated_plan_dx(d), split, split_bytes, st);
      if (s != SB_OK) return s;
    }
    if (B16)
      gated_round_dx<<<gated_blocks((size_t)d->m * d->k_in), 256, 0, st>>>(d->m, d->k_in, sum,
                                                                           (u16*)dx, d->ldx);
  }
  for (int q = 0; q < 2; ++q)
    for (int p = NP - 1; p >= 0; --p) {    // the smallest parts first
      GemmArgs g{};
      g.a = x; g.lda = d->ldx;
      g.b = dd + (size_t)(q * NP + p) * mn; g.ldb = d->n_shard;
      g.c = dw[q]; g.ldc = d->n_shard;
      g.M = d->k_in; g.N = d->n_shard; g.K = d->m;
      g.accumulate = p < NP - 1 ? 1 : accumulate;
      g.colsum = db[q]; g.colsum_acc = g.accumulate;
      const sb_status s = gemm_run<false, false, E, float>(g, gated_plan_dw(d), split, split_bytes, st);
      if (s != SB_OK) return s;
    }
  return SB_OK;
}

}  // namespace sb

using namespace sb;

extern "C" size_t sb_gated_workspace_bytes(const sb_gated_desc* d, int pass) {
  if (gated_check(d) != SB_OK || (pass != SB_FC_FWD && pass != SB_FC_BWD)) return (size_t)-1;
  return gated_space(d, pass, false).bytes;
}

extern "C" sb_status sb_gated_shard_fwd(const sb_gated_desc* d, const void* x, const void* w_gate,
                                        const void* w_up, const float* b_gate, const float* b_up,
                                        void* y, float* pre, void* ws, size_t ws_bytes,
                                        void* stream) {
  sb_status s = gated_check(d);
  if (s != SB_OK) return s;
  if (!x || !w_gate || !w_up || !y) return SB_ERR_INVALID_ARG;
  const size_t es = sbh::dsize(d->dtype), nb = (size_t)d->n_shard * 4;
  const size_t wb = (size_t)d->k_in * d->n_shard * es;
  const size_t need = gated_space(d, SB_FC_FWD, pre != nullptr).bytes;
  const Span ins[5] = {{x, ((size_t)(d->m - 1) * d->ldx + d->k_in) * es}, {w_gate, wb},
                       {w_up, wb}, {b_gate, nb}, {b_up, nb}};
  const Span outs[3] = {{y, ((size_t)(d->m - 1) * d->ldy + d->n_shard) * es},
                        {pre, (size_t)d->m * d->n_shard * 8}, {ws, need}};
  if (spans_meet(outs, 3, ins, 5) || spans_meet(outs, 1, outs + 1, 2) ||
      spans_meet(outs + 1, 1, outs + 2, 1))
    return SB_ERR_INVALID_ARG;
  if (need > 0 && (!ws || ws_bytes < need)) return SB_ERR_WORKSPACE;
  const void* w[2] = {w_gate, w_up};
  const float* b[2] = {b_gate, b_up};
  hipStream_t st = sbh::stream_of(stream);
  s = d->dtype == SB_BF16 ? gated_fwd_run<u16>(d, x, w, b, y, pre, (char*)ws, ws_bytes, st)
                          : gated_fwd_run<float>(d, x, w, b, y, pre, (char*)ws, ws_bytes, st);
  return s != SB_OK ? s : sbh::launch_status();
}

extern "C" sb_status sb_gated_shard_bwd(const sb_gated_desc* d, const void* x, const void* w_gate,
                                        const void* w_up, const float* pre, const void* dy,
                                        void* dx, float* dw_gate, float* dw_up, float* db_gate,
                                        float* db_up, int accumulate, void* ws, size_t ws_bytes,
                                        void* stream) {
  sb_status s = gated_check(d);
  if (s != SB_OK) return s;
  if (!x || !w_gate || !w_up || !pre || !dy || !dw_gate || !dw_up) return SB_ERR_INVALID_ARG;
  if (accumulate != 0 && accumulate != 1) return SB_ERR_INVALID_ARG;
  const size_t es = sbh::dsize(d->dtype), nb = (size_t)d->n_shard * 4;
  const size_t xb = ((size_t)(d->m - 1) * d->ldx + d->k_in) * es;
  const size_t wn = (size_t)d->k_in * d->n_shard;
  const size_t need = gated_space(d, SB_FC_BWD, true).bytes;
  const Span ins[5] = {{x, xb}, {w_gate, wn * es}, {w_up, wn * es},
                       {pre, (size_t)d->m * d->n_shard * 8},
                       {dy, ((size_t)(d->m - 1) * d->ldy + d->n_shard) * es}};
  const Span outs[6] = {{dx, xb}, {dw_gate, wn * 4}, {dw_up, wn * 4}, {db_gate, nb}, {db_up, nb},
                        {ws, need}};
  if (spans_meet(outs, 6, ins, 5)) return SB_ERR_INVALID_ARG;
  for (int i = 0; i < 5; ++i)
    if (spans_meet(outs + i, 1, outs + i + 1, 5 - i)) return SB_ERR_INVALID_ARG;
  if (need > 0 && (!ws || ws_bytes < need)) return SB_ERR_WORKSPACE;
  const void* w[2] = {w_gate, w_up};
  float* dw[2] = {dw_gate, dw_up};
  float* db[2] = {db_gate, db_up};
  hipStream_t st = sbh::stream_of(stream);
  s = d->dtype == SB_BF16 ? gated_bwd_run<u16>(d, x, w, pre, dy, dx, dw, db, accumulate, (char*)ws,
                                               ws_bytes, st)
                          : gated_bwd_run<float>(d, x, w, pre, dy, dx, dw, db, accumulate,
                                                 (char*)ws, ws_bytes, st);
  return s != SB_OK ? s : sbh::launch_status();
}
