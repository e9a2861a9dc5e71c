// gated.hip -- gated FC column shard forward and backward (sec. 3.1 Layer
// Partitioning: a dense layer split to 1/K of its outputs on the gathered batch;
// here the layer's ReLU is a gate).
//
//   forward   a = x Wg + bg,  u = x Wu + bu,  y = act(a) u
//   backward  da = dy u act'(a),  du = dy act(a)
//             dx  = da Wg^T + du Wu^T                       [m x kin]
//             dWg = x^T da,  dWu = x^T du,  db their column sums
//
// bf16 runs on gemm_dual (gemm_dual.hpp): both projections, the activation and the
// product are one kernel, dx and the two weight gradients one each.  fp32 runs on
// gemm_split (fc_gemm.hpp).  a and u are kept in fp32.  The weight gradients are fp32
// also where x is bf16: da and du go into their products as three bf16 parts, which
// hold all 24 bits, so a gradient is off by the rounding of its fp32 sums and not by
// 2^-9 of every term.  dx of the bf16 path is rounded to bf16 itself and takes their
// first parts.
#include "fc_gemm.hpp"
#include "gemm_dual.hpp"

#include <cmath>

namespace sb {

__global__ __launch_bounds__(256) void gated_act_fwd(int m, int n, int act,
                                                     const float* __restrict__ pre, float* y,
                                                     int ldy) {
  const size_t mn = (size_t)m * n;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < mn; i += (size_t)gridDim.x * 256) {
    float f, df;
    gate_act(act, pre[i], f, df);
    const size_t r = i / n;
    y[r * ldy + (i - r * n)] = f * pre[mn + i];
  }
}

// da and du, dense [m][n] each.
__global__ __launch_bounds__(256) void gated_act_bwd(int m, int n, int act,
                                                     const float* __restrict__ pre,
                                                     const float* __restrict__ dy, int ldy,
                                                     float* d) {
  const size_t mn = (size_t)m * n;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < mn; i += (size_t)gridDim.x * 256) {
    float f, df;
    gate_act(act, pre[i], f, df);
    const size_t r = i / n;
    const float g = dy[r * ldy + (i - r * n)];
    d[i] = g * pre[mn + i] * df;
    d[mn + i] = g * f;
  }
}

// ---- bf16 -----------------------------------------------------------------
// da and du as three parts each, rows of np (n rounded up to 8, zeros behind n): part
// p of da at p * m * np, of du at (3 + p) * m * np.  A block has 256 columns of
// kActRows rows, a lane four columns of every fourth row, and leaves its columns' sums
// (of the whole values) in sums [row block][2][np].
constexpr int kActRows = 32;

__global__ __launch_bounds__(256) void gated_act_bwd_parts(int m, int n, int np, int act,
                                                           const float* __restrict__ pre,
                                                           const u16* __restrict__ dy, int ldy,
                                                           u16* __restrict__ d,
                                                           float* __restrict__ sums, int vec) {
  __shared__ f4 part[2][4][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int c = blockIdx.x * 256 + lane * 4;
  const size_t mn = (size_t)m * n, plane = (size_t)m * np;
  const int r1 = min(m, (int)(blockIdx.y + 1) * kActRows);
  f4 s[2] = {f4{0.f, 0.f, 0.f, 0.f}, f4{0.f, 0.f, 0.f, 0.f}};
  for (int r = blockIdx.y * kActRows + w; r < r1 && c < np; r += 4) {
    const float* pa = pre + (size_t)r * n + c;
    const u16* pd = dy + (size_t)r * ldy + c;
    f4 a = f4{0.f, 0.f, 0.f, 0.f}, u = a, g = a;
    if (vec && c < n) {                              // n a multiple of 4
      a = *reinterpret_cast<const f4*>(pa);
      u = *reinterpret_cast<const f4*>(pa + mn);
      g = Elem<u16>::load4(pd);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < n) {
          a[e] = pa[e];
          u[e] = pa[mn + e];
          g[e] = bf16_to_f32(pd[e]);
        }
    }
    f4 v[2];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float f, df;
      gate_act(act, a[e], f, df);
      v[0][e] = c + e < n ? g[e] * u[e] * df : 0.f;
      v[1][e] = c + e < n ? g[e] * f : 0.f;
    }
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      s[q] += v[q];
      f4 rest = v[q];
#pragma unroll
      for (int p = 0; p < 3; ++p) {
        u16* o = d + (3 * q + p) * plane + (size_t)r * np + c;
        uint2 b;
        b.x = f32x2_to_bf16x2(rest[0], rest[1]);
        b.y = f32x2_to_bf16x2(rest[2], rest[3]);
        *reinterpret_cast<uint2*>(o) = b;
        const f4 h = Elem<u16>::load4(reinterpret_cast<const u16*>(&b));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          // An infinite or NaN first part is the whole value.
          const bool whole = (__float_as_uint(h[e]) & 0x7f800000u) == 0x7f800000u;
          rest[e] = whole ? 0.f : rest[e] - h[e];
        }
      }
    }
  }
  if (!sums) return;
  part[0][w][lane] = s[0];
  part[1][w][lane] = s[1];
  __syncthreads();
  if (w < 2 && c < np) {
    const f4 t = (part[w][0][lane] + part[w][1][lane]) + (part[w][2][lane] + part[w][3][lane]);
    *reinterpret_cast<f4*>(sums + ((size_t)blockIdx.y * 2 + w) * np + c) = t;
  }
}

// db of the gate (block row 0) and the other projection: a wave has 64 columns and
// every fourth of the row blocks' sums.
__global__ __launch_bounds__(256) void gated_bias_sums(const float* __restrict__ sums, int chunks,
                                                       int n, int np, float* db_gate, float* db_up,
                                                       int accumulate) {
  __shared__ float part[4][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int c = blockIdx.x * 64 + lane, q = blockIdx.y;
  float v = 0.f;
  if (c < n)
    for (int r = w; r < chunks; r += 4) v += sums[((size_t)r * 2 + q) * np + c];
  part[w][lane] = v;
  __syncthreads();
  float* db = q ? db_up : db_gate;
  if (w || c >= n || !db) return;
  v = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
  db[c] = accumulate ? db[c] + v : v;
}

// Rows of `cols` elements, `ld` apart, to rows of cp (a multiple of 8), zeros behind.
// grid.y: up to two matrices.
__global__ __launch_bounds__(256) void gated_pack(const u16* a, const u16* b, size_t rows, int cols,
                                                  int ld, int cp, u16* to) {
  const u16* from = blockIdx.y ? b : a;
  u16* out = to + blockIdx.y * rows * cp;
  const size_t pieces = rows * (cp / 8);
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (size_t)gridDim.x * 256) {
    const size_t r = i / (cp / 8);
    const int c = (int)(i - r * (cp / 8)) * 8;
    u16 v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c + e < cols ? from[r * ld + c + e] : (u16)0;
    u4v o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (uint32_t)v[2 * e] | (uint32_t)v[2 * e + 1] << 16;
    *reinterpret_cast<u4v*>(out + r * cp + c) = o;
  }
}

// Sums of the splits' partials, four columns of a row a lane.  FWD: [split][2][M][N] to
// y and pre; DW: to the two gradients; DX: [split][M][N] to dx.
__device__ __forceinline__ f4 split_quad(const float* p, int splits, size_t stride, int n, int N) {
  f4 v = f4{0.f, 0.f, 0.f, 0.f};
  if (N % 4 == 0) return split_sum4(p, splits, stride, 0);
  for (int s = 0; s < splits; ++s)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < N) v[e] += p[(size_t)s * stride + e];
  return v;
}

template <DualKind KIND>
__global__ __launch_bounds__(256) void gated_split_sum(DualArgs g, int act) {
  const int quads = cdiv(g.N, 4);
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  const int m = (int)(i / quads), n = (int)(i - (size_t)m * quads) * 4;
  if (m >= g.M) return;
  const size_t plane = (size_t)g.M * g.N, at = (size_t)m * g.N + n;
  if constexpr (KIND == kDualDx) {
    const f4 v = split_quad(g.part + at, g.splits, plane, n, g.N);
    u16* o = (u16*)g.c[0] + (size_t)m * g.ldc + n;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < g.N) o[e] = f32_to_bf16(v[e]);
  } else {
    const f4 a = split_quad(g.part + at, g.splits, 2 * plane, n, g.N);
    const f4 u = split_quad(g.part + plane + at, g.splits, 2 * plane, n, g.N);
    if constexpr (KIND == kDualFwd) {
      gate_store<u16>(act, a, u, n, g.N, g.bias[0], g.bias[1],
                      g.pre ? g.pre + (size_t)m * g.N : nullptr, plane,
                      (u16*)g.c[0] + (size_t)m * g.ldc);
    } else {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        float* o = (float*)g.c[q] + (size_t)m * g.ldc + n;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = q ? u[e] : a[e];
          if (n + e < g.N) o[e] = g.accumulate ? o[e] + x : x;
        }
      }
    }
  }
}

// Tile and split of a product: the least estimated time.
struct DualPlan { int f, mt, nt, splits, stages; size_t ws_bytes; };

static DualPlan dual_plan(DualKind kind, int M, int N, int K, int segs) {
  DualPlan best{};
  double best_t = 0;
  const int total = cdiv(K, 32) * segs;
  for (int f = 4; f >= 2; f -= 2) {
    const int mt = cdiv(M, 64 * f), nt = cdiv(N, kind == kDualDx ? 64 * f : 32 * f);
    const int64_t tiles = (int64_t)mt * nt;
    for (int s = 1; s <= 16 && s <= total; ++s) {
      const int stages = cdiv(total, s);
      if (cdiv(total, stages) != s) continue;
      const int64_t blocks = tiles * s;
      const int64_t per_cu = (blocks + 255) / 256;
      const double bytes = (double)M * N * (kind == kDualDx ? 4 : 8);
      double t = s > 1 ? 4.0 + bytes * (2 * s + 1) / 5e6 : 0.0;
      t += f == 4 ? per_cu * (5.0 + stages * (blocks > 192 ? 1.04 : 0.75))
                  : 3.0 * ((per_cu + 2) / 3) + stages * (per_cu > 1 ? 0.33 * per_cu : 0.29);
      if (best_t == 0 || t < best_t) {
        best_t = t;
        best = DualPlan{f, mt, nt, s, stages, s > 1 ? (size_t)s * (size_t)bytes : 0};
      }
    }
  }
  return best;
}

template <int F, DualKind KIND, int ACT>
static void dual_launch_t(const DualArgs& g, hipStream_t st) {
  typedef DualTile<F> T;
  static std::once_flag once;
  std::call_once(once, [] {
    (void)hipFuncSetAttribute((const void*)gemm_dual<T, KIND, ACT>,
                              hipFuncAttributeMaxDynamicSharedMemorySize, (int)T::LDS_BYTES);
  });
  gemm_dual<T, KIND, ACT><<<(unsigned)(g.mt * g.nt * g.splits), 256, T::LDS_BYTES, st>>>(g);
}
template <DualKind KIND, int ACT>
static void dual_launch(int f, const DualArgs& g, hipStream_t st) {
  if (f == 4) dual_launch_t<4, KIND, ACT>(g, st);
  else dual_launch_t<2, KIND, ACT>(g, st);
}

// One product under its plan: unsplit it ends in its outputs, split in the workspace,
// from where gated_split_sum takes it.
template <DualKind KIND>
static void dual_run(DualArgs g, const DualPlan& p, int act, float* part, hipStream_t st) {
  g.mt = p.mt; g.nt = p.nt; g.splits = p.splits; g.stages = p.stages;
  g.part = part;
  if (KIND != kDualFwd || p.splits > 1) {
    dual_launch<KIND, 0>(p.f, g, st);
  } else {
    switch (act) {
      case SB_ACT_SIGMOID: dual_launch<kDualFwd, SB_ACT_SIGMOID>(p.f, g, st); break;
      case SB_ACT_SILU: dual_launch<kDualFwd, SB_ACT_SILU>(p.f, g, st); break;
      case SB_ACT_GELU: dual_launch<kDualFwd, SB_ACT_GELU>(p.f, g, st); break;
      case SB_ACT_GELU_TANH: dual_launch<kDualFwd, SB_ACT_GELU_TANH>(p.f, g, st); break;
      default: dual_launch<kDualFwd, SB_ACT_RELU>(p.f, g, st);
    }
  }
  if (p.splits > 1) {
    const size_t quads = (size_t)g.M * cdiv(g.N, 4);
    gated_split_sum<KIND><<<(unsigned)((quads + 255) / 256), 256, 0, st>>>(g, act);
  }
}

static unsigned gated_blocks(size_t count) {
  return (unsigned)std::min<size_t>((count + 255) / 256, 65536);
}

static int up8(int n) { return (n + 7) / 8 * 8; }
static bool at16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Which bf16 operands have to be laid out anew for 16-byte pieces: x as rows of the
// forward's reduction, x as lines of the weight gradient's, the weights.
struct GatedPacks { bool x, lines, w; };
static GatedPacks gated_packs(const sb_gated_desc* d, bool x_at16, bool w_at16) {
  // (An odd k_in would end the last line inside the 4 bytes that ranges count in.)
  const bool lines = d->ldx % 8 != 0 || d->k_in % 2 != 0 || !x_at16;
  return GatedPacks{lines || d->k_in % 8 != 0, lines, d->n_shard % 8 != 0 || !w_at16};
}

// A workspace's parts, each from a multiple of 256 bytes on (offsets).
struct GatedSpace {
  size_t d, x, w, sums, split, bytes;
};

static DualPlan gated_plan(const sb_gated_desc* d, DualKind kind) {
  if (kind == kDualFwd) return dual_plan(kind, d->m, d->n_shard, d->k_in, 1);
  if (kind == kDualDx) return dual_plan(kind, d->m, d->k_in, up8(d->n_shard), 2);
  return dual_plan(kind, d->k_in, d->n_shard, d->m, 3);
}

static GemmPlan gated_plan_y(const sb_gated_desc* d) {
  return product_plan(d->m, d->n_shard, d->k_in, d->ldx, true, d->n_shard, false, 4);
}
static GemmPlan gated_plan_dx(const sb_gated_desc* d) {
  return product_plan(d->m, d->k_in, d->n_shard, d->n_shard, true, d->n_shard, true, 4);
}
static GemmPlan gated_plan_dw(const sb_gated_desc* d) {
  return product_plan(d->k_in, d->n_shard, d->m, d->ldx, false, d->n_shard, false, 4);
}

// pre: whether the forward has a place for a and u of the caller's.
static GatedSpace gated_space(const sb_gated_desc* d, int pass, const GatedPacks& k, bool pre) {
  const size_t m = d->m, mn = m * d->n_shard, np = up8(d->n_shard);
  GatedSpace s{};
  size_t at = 0;
  auto take = [&](size_t& part, size_t bytes) {
    part = at;
    at += round_up(bytes, 256);
  };
  if (d->dtype == SB_F32) {
    take(s.d, pass == SB_FC_FWD && pre ? 0 : mn * 8);
    take(s.split, pass == SB_FC_FWD ? gated_plan_y(d).ws_bytes
                                    : std::max(gated_plan_dx(d).ws_bytes, gated_plan_dw(d).ws_bytes));
  } else {
    if (pass == SB_FC_BWD) {
      take(s.d, m * np * 12);
      take(s.sums, (size_t)cdiv(d->m, kActRows) * np * 8);
    }
    if (pass == SB_FC_FWD ? k.x : k.lines) take(s.x, m * up8(d->k_in) * 2);
    if (k.w) take(s.w, (size_t)d->k_in * np * 4);
    take(s.split, pass == SB_FC_FWD
                      ? gated_plan(d, kDualFwd).ws_bytes
                      : std::max(gated_plan(d, kDualDx).ws_bytes, gated_plan(d, kDualDw).ws_bytes));
  }
  s.bytes = at;
  return s;
}

static sb_status gated_check(const sb_gated_desc* d) {
  if (!d) return SB_ERR_INVALID_ARG;
  if (d->m <= 0 || d->k_in <= 0 || d->n_shard <= 0) return SB_ERR_INVALID_ARG;
  if (d->ldx < d->k_in || d->ldy < d->n_shard) return SB_ERR_INVALID_ARG;
  if (d->dtype != SB_F32 && d->dtype != SB_BF16) return SB_ERR_INVALID_ARG;
  if (d->flags & ~SB_UNALIGNED) return SB_ERR_INVALID_ARG;
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

static sb_status gated_fwd_f32(const sb_gated_desc* d, const void* x, const void* const* w,
                               const float* const* b, void* y, float* pre, char* ws,
                               const GatedSpace& sp, hipStream_t st) {
  const size_t mn = (size_t)d->m * d->n_shard;
  if (!pre) pre = (float*)(ws + sp.d);
  for (int q = 0; q < 2; ++q) {
    GemmArgs g{};
    g.a = x; g.lda = d->ldx;
    g.b = w[q]; g.ldb = d->n_shard;
    g.c = pre + q * mn; g.ldc = d->n_shard;
    g.M = d->m; g.N = d->n_shard; g.K = d->k_in;
    g.bias = b[q];
    const sb_status s = gemm_run<true, false, float, float>(
        g, gated_plan_y(d), (float*)(ws + sp.split), sp.bytes - sp.split, st);
    if (s != SB_OK) return s;
  }
  gated_act_fwd<<<gated_blocks(mn), 256, 0, st>>>(d->m, d->n_shard, d->act, pre, (float*)y, d->ldy);
  return SB_OK;
}

static sb_status gated_bwd_f32(const sb_gated_desc* d, const void* x, const void* const* w,
                               const float* pre, const void* dy, void* dx, float* const* dw,
                               float* const* db, int accumulate, char* ws, const GatedSpace& sp,
                               hipStream_t st) {
  const size_t mn = (size_t)d->m * d->n_shard, split_bytes = sp.bytes - sp.split;
  float* split = (float*)(ws + sp.split);
  float* dd = (float*)(ws + sp.d);
  gated_act_bwd<<<gated_blocks(mn), 256, 0, st>>>(d->m, d->n_shard, d->act, pre, (const float*)dy,
                                                  d->ldy, dd);
  for (int q = 0; q < 2 && dx; ++q) {
    GemmArgs g{};
    g.a = dd + q * mn; g.lda = d->n_shard;
    g.b = w[q]; g.ldb = d->n_shard;
    g.c = dx; g.ldc = d->ldx;
    g.M = d->m; g.N = d->k_in; g.K = d->n_shard;
    g.accumulate = q;
    const sb_status s = gemm_run<true, true, float, float>(g, gated_plan_dx(d), split, split_bytes, st);
    if (s != SB_OK) return s;
  }
  for (int q = 0; q < 2; ++q) {
    GemmArgs g{};
    g.a = x; g.lda = d->ldx;
    g.b = dd + q * mn; g.ldb = d->n_shard;
    g.c = dw[q]; g.ldc = d->n_shard;
    g.M = d->k_in; g.N = d->n_shard; g.K = d->m;
    g.accumulate = accumulate;
    g.colsum = db[q]; g.colsum_acc = accumulate;
    const sb_status s = gemm_run<false, false, float, float>(g, gated_plan_dw(d), split, split_bytes, st);
    if (s != SB_OK) return s;
  }
  return SB_OK;
}

// The weights as lines of 16-byte pieces, np apart.
static void gated_weights(const sb_gated_desc* d, const void* const* w, const u16** to, bool pack,
                          char* ws, const GatedSpace& sp, hipStream_t st) {
  const int np = up8(d->n_shard);
  to[0] = (const u16*)w[0];
  to[1] = (const u16*)w[1];
  if (!pack) return;
  u16* out = (u16*)(ws + sp.w);
  gated_pack<<<dim3(gated_blocks((size_t)d->k_in * np / 8), 2), 256, 0, st>>>(
      to[0], to[1], d->k_in, d->n_shard, d->n_shard, np, out);
  to[0] = out;
  to[1] = out + (size_t)d->k_in * np;
}
static const u16* gated_rows(const sb_gated_desc* d, const void* x, bool pack, int* ld, char* ws,
                             const GatedSpace& sp, hipStream_t st) {
  *ld = d->ldx;
  if (!pack) return (const u16*)x;
  const int kp = up8(d->k_in);
  u16* out = (u16*)(ws + sp.x);
  gated_pack<<<dim3(gated_blocks((size_t)d->m * kp / 8), 1), 256, 0, st>>>(
      (const u16*)x, nullptr, d->m, d->k_in, d->ldx, kp, out);
  *ld = kp;
  return out;
}

static void gated_fwd_b16(const sb_gated_desc* d, const void* x, const void* const* w,
                          const float* const* b, void* y, float* pre, const GatedPacks& packs,
                          char* ws, const GatedSpace& sp, hipStream_t st) {
  const int np = up8(d->n_shard);
  DualArgs g{};
  g.a[0] = gated_rows(d, x, packs.x, &g.lda, ws, sp, st);
  const u16* wp[2];
  gated_weights(d, w, wp, packs.w, ws, sp, st);
  g.b[0][0] = wp[0]; g.b[1][0] = wp[1];
  g.ldb = np;
  g.M = d->m; g.N = d->n_shard; g.K = packs.x ? up8(d->k_in) : d->k_in; g.segs = 1;
  g.a_bytes = (uint32_t)(((size_t)(d->m - 1) * g.lda + g.K) * 2);
  g.b_bytes = (uint32_t)((size_t)d->k_in * np * 2);
  g.c[0] = y; g.ldc = d->ldy;
  g.bias[0] = b[0]; g.bias[1] = b[1];
  g.pre = pre;
  dual_run<kDualFwd>(g, gated_plan(d, kDualFwd), d->act, (float*)(ws + sp.split), st);
}

static void gated_bwd_b16(const sb_gated_desc* d, const void* x, const void* const* w,
                          const float* pre, const void* dy, void* dx, float* const* dw,
                          float* const* db, int accumulate, const GatedPacks& packs, char* ws,
                          const GatedSpace& sp, hipStream_t st) {
  const int np = up8(d->n_shard), chunks = cdiv(d->m, kActRows);
  const size_t plane = (size_t)d->m * np;
  u16* parts = (u16*)(ws + sp.d);
  float* split = (float*)(ws + sp.split);
  float* sums = db[0] || db[1] ? (float*)(ws + sp.sums) : nullptr;
  const int vec = d->n_shard % 4 == 0 && at16(pre) && d->ldy % 4 == 0 && ((uintptr_t)dy & 7) == 0;
  gated_act_bwd_parts<<<dim3(cdiv(np, 256), chunks), 256, 0, st>>>(
      d->m, d->n_shard, np, d->act, pre, (const u16*)dy, d->ldy, parts, sums, vec);
  if (sums)
    gated_bias_sums<<<dim3(cdiv(d->n_shard, 64), 2), 256, 0, st>>>(sums, chunks, d->n_shard, np,
                                                                   db[0], db[1], accumulate);
  if (dx) {
    DualArgs g{};
    const u16* wp[2];
    gated_weights(d, w, wp, packs.w, ws, sp, st);
    for (int q = 0; q < 2; ++q) {
      g.a[q] = parts + 3 * q * plane;
      g.b[0][q] = wp[q];
    }
    g.lda = g.ldb = np;
    g.M = d->m; g.N = d->k_in; g.K = np; g.segs = 2;
    g.a_bytes = (uint32_t)(plane * 2);
    g.b_bytes = (uint32_t)((size_t)d->k_in * np * 2);
    g.c[0] = dx; g.ldc = d->ldx;
    dual_run<kDualDx>(g, gated_plan(d, kDualDx), 0, split, st);
  }
  DualArgs g{};
  const u16* xp = gated_rows(d, x, packs.lines, &g.lda, ws, sp, st);
  for (int p = 0; p < 3; ++p) {                      // the smallest parts first
    g.a[p] = xp;
    for (int q = 0; q < 2; ++q) g.b[q][p] = parts + (3 * q + 2 - p) * plane;
  }
  g.ldb = np;
  g.M = d->k_in; g.N = d->n_shard; g.K = d->m; g.segs = 3;
  g.a_bytes = (uint32_t)(((size_t)(d->m - 1) * g.lda + (packs.lines ? g.lda : d->k_in)) * 2);
  g.b_bytes = (uint32_t)(plane * 2);
  g.c[0] = dw[0]; g.c[1] = dw[1]; g.ldc = d->n_shard;
  g.accumulate = accumulate;
  dual_run<kDualDw>(g, gated_plan(d, kDualDw), 0, split, st);
}

}  // namespace sb

using namespace sb;

extern "C" size_t sb_gated_workspace_bytes(const sb_gated_desc* d, int pass) {
  if (gated_check(d) != SB_OK || (pass != SB_FC_FWD && pass != SB_FC_BWD)) return (size_t)-1;
  const bool at = !(d->flags & SB_UNALIGNED);
  return gated_space(d, pass, gated_packs(d, at, at), false).bytes;
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
  const GatedPacks packs = gated_packs(d, at16(x), at16(w_gate) && at16(w_up));
  const GatedSpace sp = gated_space(d, SB_FC_FWD, packs, pre != nullptr);
  const size_t need = sp.bytes;
  const Span ins[5] = {{x, ((size_t)(d->m - 1) * d->ldx + d->k_in) * es}, {w_gate, wb},
                       {w_up, wb}, {b_gate, nb}, {b_up, nb}};
  const Span outs[3] = {{y, ((size_t)(d->m - 1) * d->ldy + d->n_shard) * es},
                        {pre, (size_t)d->m * d->n_shard * 8}, {ws, need}};
  if (spans_meet(outs, 3, ins, 5) || spans_meet(outs, 1, outs + 1, 2) ||
      spans_meet(outs + 1, 1, outs + 2, 1))
    return SB_ERR_INVALID_ARG;
  if (need > 0 && (!ws || ws_bytes < need)) return SB_ERR_WORKSPACE;
  if (need > 0 && !at16(ws)) return SB_ERR_INVALID_ARG;
  const void* w[2] = {w_gate, w_up};
  const float* b[2] = {b_gate, b_up};
  hipStream_t st = sbh::stream_of(stream);
  if (d->dtype == SB_BF16) gated_fwd_b16(d, x, w, b, y, pre, packs, (char*)ws, sp, st);
  else s = gated_fwd_f32(d, x, w, b, y, pre, (char*)ws, sp, st);
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
  const GatedPacks packs = gated_packs(d, at16(x), at16(w_gate) && at16(w_up));
  const GatedSpace sp = gated_space(d, SB_FC_BWD, packs, true);
  const size_t need = sp.bytes;
  const Span ins[5] = {{x, xb}, {w_gate, wn * es}, {w_up, wn * es},
                       {pre, (size_t)d->m * d->n_shard * 8},
                       {dy, ((size_t)(d->m - 1) * d->ldy + d->n_shard) * es}};
  const Span outs[6] = {{dx, xb}, {dw_gate, wn * 4}, {dw_up, wn * 4}, {db_gate, nb}, {db_up, nb},
                        {ws, need}};
  if (spans_meet(outs, 6, ins, 5)) return SB_ERR_INVALID_ARG;
  for (int i = 0; i < 5; ++i)
    if (spans_meet(outs + i, 1, outs + i + 1, 5 - i)) return SB_ERR_INVALID_ARG;
  if (need > 0 && (!ws || ws_bytes < need)) return SB_ERR_WORKSPACE;
  if (need > 0 && !at16(ws)) return SB_ERR_INVALID_ARG;
  const void* w[2] = {w_gate, w_up};
  float* dw[2] = {dw_gate, dw_up};
  float* db[2] = {db_gate, db_up};
  hipStream_t st = sbh::stream_of(stream);
  if (d->dtype == SB_BF16)
    gated_bwd_b16(d, x, w, pre, dy, dx, dw, db, accumulate, packs, (char*)ws, sp, st);
  else
    s = gated_bwd_f32(d, x, w, pre, dy, dx, dw, db, accumulate, (char*)ws, sp, st);
  return s != SB_OK ? s : sbh::launch_status();
}
