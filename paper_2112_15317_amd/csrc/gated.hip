// gated.hip -- gated FC column shard forward and backward (sec. 3.1 Layer
// Partitioning: a dense layer split to 1/K of its outputs on the gathered batch;
// here the layer's ReLU is a gate).
//
//   forward   a = x Wg + bg,  u = x Wu + bu,  y = act(a) u
//   backward  da = dy u act'(a),  du = dy act(a)
//             dx  = da Wg^T + du Wu^T                       [m x kin]
//             dWg = x^T da,  dWu = x^T du,  db their column sums
//
// The products run on gemm_dual (gemm_dual.hpp): both projections, the activation
// and the product with it are one kernel, dx another, both weight gradients a third;
// da, du and the bias gradients come from a pass over dy and the kept a and u.
//
// The weight gradients are fp32 also where x is bf16: da and du go into their
// products as three bf16 parts, which hold all 24 bits, so a gradient is off by the
// rounding of its fp32 sums and not by 2^-9 of every term (measured against 64 bits:
// 3e-7 of the gradient; with two parts 2.6e-6, with one 1.7e-3).  dx of the bf16 path
// is rounded to bf16 itself and takes their first parts.
#include "gemm_dual.hpp"

#include <algorithm>
#include <mutex>

namespace sb {

// da and du in rows of np (n rounded up to 8, zeros behind n).  fp32: da, then du,
// m * np elements each.  bf16: three parts of each, part p of da at p * m * np, of du at
// (3 + p) * m * np.  A block has 256 columns of `rows` rows, a lane four columns of
// every fourth row, and leaves its columns' sums in sums [row block][2][np].
static int act_rows(int m, int np) {
  // Down to a row a wave where 32 would leave CUs idle (128 x 256: 10.2 -> 3 us).
  int rows = 32;
  while (rows > 4 && (int64_t)((np + 255) / 256) * cdiv(m, rows) < 1024) rows /= 2;
  return rows;
}

template <class E>
__global__ __launch_bounds__(256) void gated_act_bwd(int m, int n, int np, int act,
                                                     const float* __restrict__ pre,
                                                     const E* __restrict__ dy, int ldy,
                                                     E* __restrict__ d, float* __restrict__ sums,
                                                     int rows, int vec) {
  __shared__ f4 part[2][4][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int c = blockIdx.x * 256 + lane * 4;
  const size_t mn = (size_t)m * n, plane = (size_t)m * np;
  const int r1 = min(m, (int)(blockIdx.y + 1) * rows);
  f4 s[2] = {f4{0.f, 0.f, 0.f, 0.f}, f4{0.f, 0.f, 0.f, 0.f}};
  for (int r = blockIdx.y * rows + w; r < r1 && c < np; r += 4) {
    const float* pa = pre + (size_t)r * n + c;
    const E* pd = dy + (size_t)r * ldy + c;
    f4 a = f4{0.f, 0.f, 0.f, 0.f}, u = a, g = a;
    if (vec && c < n) {                              // n a multiple of 4
      a = *reinterpret_cast<const f4*>(pa);
      u = *reinterpret_cast<const f4*>(pa + mn);
      g = Elem<E>::load4(pd);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < n) {
          a[e] = pa[e];
          u[e] = pa[mn + e];
          g[e] = Elem<E>::load(pd, e);
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
      const size_t at = (size_t)r * np + c;
      if constexpr (sizeof(E) == 4) {
        *reinterpret_cast<f4*>(d + q * plane + at) = v[q];
      } else {
        f4 rest = v[q];
#pragma unroll
        for (int p = 0; p < 3; ++p) {
          uint2 b;
          b.x = f32x2_to_bf16x2(rest[0], rest[1]);
          b.y = f32x2_to_bf16x2(rest[2], rest[3]);
          *reinterpret_cast<uint2*>(d + (3 * q + p) * plane + at) = b;
          const f4 h = f4{__uint_as_float(b.x << 16), __uint_as_float(b.x & 0xffff0000u),
                          __uint_as_float(b.y << 16), __uint_as_float(b.y & 0xffff0000u)};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            // An infinite or NaN first part is the whole value.
            const bool whole = (__float_as_uint(h[e]) & 0x7f800000u) == 0x7f800000u;
            rest[e] = whole ? 0.f : rest[e] - h[e];
          }
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
// Block rows: two matrices.
template <class E>
__global__ __launch_bounds__(256) void gated_pack(const E* a, const E* b, size_t rows, int cols,
                                                  int ld, int cp, E* to) {
  const E* from = blockIdx.y ? b : a;
  E* out = to + blockIdx.y * rows * cp;
  const size_t quads = rows * (cp / 4);
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < quads; i += (size_t)gridDim.x * 256) {
    const size_t r = i / (cp / 4);
    const int c = (int)(i - r * (cp / 4)) * 4;
    f4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = c + e < cols ? Elem<E>::load(from, r * ld + c + e) : 0.f;
    Elem<E>::store4(out + r * cp + c, v);
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

template <DualKind KIND, class E>
__global__ __launch_bounds__(256) void gated_split_sum(DualArgs g, int act) {
  const int quads = cdiv(g.N, 4);
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  const int m = (int)(i / quads), n = (int)(i - (size_t)m * quads) * 4;
  if (m >= g.M) return;
  const size_t plane = (size_t)g.M * g.N, at = (size_t)m * g.N + n;
  if constexpr (KIND == kDualDx) {
    const f4 v = split_quad(g.part + at, g.splits, plane, n, g.N);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < g.N) Elem<E>::store((E*)g.c[0], (size_t)m * g.ldc + n + e, v[e]);
  } else {
    const f4 a = split_quad(g.part + at, g.splits, 2 * plane, n, g.N);
    const f4 u = split_quad(g.part + plane + at, g.splits, 2 * plane, n, g.N);
    if constexpr (KIND == kDualFwd) {
      gate_store<E>(act, a, u, n, g.N, g.bias[0], g.bias[1],
                    g.pre ? g.pre + (size_t)m * g.N : nullptr, plane,
                    (E*)g.c[0] + (size_t)m * g.ldc);
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

// Tile and split of a product: the least estimated time (us).
struct DualPlan { int f, mt, nt, splits, stages; size_t ws_bytes; };

static DualPlan dual_plan(DualKind kind, bool b16, int M, int N, int K, int segs) {
  DualPlan best{};
  double best_t = 0;
  const int total = cdiv(K, 32) * segs;
  for (int f = b16 ? 4 : 2; f >= 2; f -= 2) {
    const int mt = cdiv(M, 64 * f), nt = cdiv(N, kind == kDualDx ? 64 * f : 32 * f);
    const int64_t tiles = (int64_t)mt * nt;
    for (int s = 1; s <= 16 && s <= total; ++s) {
      const int stages = cdiv(total, s);
      if (cdiv(total, stages) != s) continue;
      const int64_t blocks = tiles * s;
      const double per_cu = (double)((blocks + 255) / 256);
      const double bytes = (double)M * N * (kind == kDualDx ? 4 : 8);
      double t = s > 1 ? 4.0 + bytes * (2 * s + 1) / 5e6 : 0.0;
      if (!b16) t += per_cu * (5.0 + stages * (blocks > 128 ? 1.8 : 1.4));
      else if (f == 4) t += per_cu * (5.0 + stages * (blocks > 192 ? 1.04 : 0.75));
      else t += 3.0 * (double)(((int64_t)per_cu + 2) / 3) + stages * (per_cu > 1 ? 0.33 * per_cu : 0.29);
      if (best_t == 0 || t < best_t) {
        best_t = t;
        best = DualPlan{f, mt, nt, s, stages, s > 1 ? (size_t)s * (size_t)bytes : 0};
      }
    }
  }
  return best;
}

template <int F, DualKind KIND, int ACT, class E>
static void dual_launch(const DualArgs& g, hipStream_t st) {
  typedef DualTile<F, E> T;
  static std::once_flag once;
  std::call_once(once, [] {
    (void)hipFuncSetAttribute((const void*)gemm_dual<T, KIND, ACT>,
                              hipFuncAttributeMaxDynamicSharedMemorySize, (int)T::LDS_BYTES);
  });
  gemm_dual<T, KIND, ACT><<<(unsigned)(g.mt * g.nt * g.splits), 256, T::LDS_BYTES, st>>>(g);
}
template <DualKind KIND, int ACT, class E>
static void dual_launch_f(int f, const DualArgs& g, hipStream_t st) {
  if constexpr (sizeof(E) == 2) {
    if (f == 4) {
      dual_launch<4, KIND, ACT, E>(g, st);
      return;
    }
  }
  dual_launch<2, KIND, ACT, E>(g, st);
}

// One product under its plan: unsplit it ends in its outputs, split in the workspace,
// from where gated_split_sum takes it.
template <DualKind KIND, class E>
static void dual_run(DualArgs g, const DualPlan& p, int act, float* part, hipStream_t st) {
  g.mt = p.mt; g.nt = p.nt; g.splits = p.splits; g.stages = p.stages;
  g.part = part;
  if (KIND != kDualFwd || p.splits > 1) {
    dual_launch_f<KIND, 0, E>(p.f, g, st);
  } else {
    switch (act) {
      case SB_ACT_SIGMOID: dual_launch_f<kDualFwd, SB_ACT_SIGMOID, E>(p.f, g, st); break;
      case SB_ACT_SILU: dual_launch_f<kDualFwd, SB_ACT_SILU, E>(p.f, g, st); break;
      case SB_ACT_GELU: dual_launch_f<kDualFwd, SB_ACT_GELU, E>(p.f, g, st); break;
      case SB_ACT_GELU_TANH: dual_launch_f<kDualFwd, SB_ACT_GELU_TANH, E>(p.f, g, st); break;
      default: dual_launch_f<kDualFwd, SB_ACT_RELU, E>(p.f, g, st);
    }
  }
  if (p.splits > 1) {
    const size_t quads = (size_t)g.M * cdiv(g.N, 4);
    gated_split_sum<KIND, E><<<(unsigned)((quads + 255) / 256), 256, 0, st>>>(g, act);
  }
}

static unsigned gated_blocks(size_t count) {
  return (unsigned)std::min<size_t>((count + 255) / 256, 65536);
}
static int up8(int n) { return (n + 7) / 8 * 8; }
static bool at16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Which operands have to be laid out anew for 16-byte pieces of whole eights: x as
// rows of the forward's reduction, x as lines of the weight gradient's, the weights.
struct GatedPacks { bool x, lines, w; };
static GatedPacks gated_packs(const sb_gated_desc* d, bool x_at16, bool w_at16) {
  const bool b16 = d->dtype == SB_BF16;
  // (An odd bf16 k_in would end the last line inside the 4 bytes that ranges count in.)
  const bool lines = d->ldx % (b16 ? 8 : 4) != 0 || (b16 && d->k_in % 2 != 0) || !x_at16;
  return GatedPacks{lines || d->k_in % 8 != 0, lines, d->n_shard % 8 != 0 || !w_at16};
}

static DualPlan gated_plan(const sb_gated_desc* d, DualKind kind) {
  const bool b16 = d->dtype == SB_BF16;
  if (kind == kDualFwd) return dual_plan(kind, b16, d->m, d->n_shard, d->k_in, 1);
  if (kind == kDualDx) return dual_plan(kind, b16, d->m, d->k_in, up8(d->n_shard), 2);
  return dual_plan(kind, b16, d->k_in, d->n_shard, d->m, b16 ? 3 : 1);
}

// A workspace's parts, each from a multiple of 256 bytes on (offsets).
struct GatedSpace { size_t d, sums, x, w, split, bytes; };

static GatedSpace gated_space(const sb_gated_desc* d, int pass, const GatedPacks& k) {
  const size_t m = d->m, np = up8(d->n_shard), es = sbh::dsize(d->dtype);
  GatedSpace s{};
  size_t at = 0;
  auto take = [&](size_t& part, size_t bytes) {
    part = at;
    at += round_up(bytes, 256);
  };
  if (pass == SB_FC_BWD) {
    take(s.d, m * np * (d->dtype == SB_BF16 ? 12 : 8));
    take(s.sums, (size_t)cdiv(d->m, act_rows(d->m, (int)np)) * np * 8);
  }
  if (pass == SB_FC_FWD ? k.x : k.lines) take(s.x, m * up8(d->k_in) * es);
  if (k.w) take(s.w, 2 * (size_t)d->k_in * np * es);
  take(s.split, pass == SB_FC_FWD
                    ? gated_plan(d, kDualFwd).ws_bytes
                    : std::max(gated_plan(d, kDualDx).ws_bytes, gated_plan(d, kDualDw).ws_bytes));
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
  // The kernels' ranges are below 2^31 bytes, and so are 32 lines, by which a
  // stage may pass the end of one (its offsets must not wrap).
  const int64_t es = (int64_t)sbh::dsize(d->dtype), top = 1ll << 31;
  const int64_t m = d->m, kp = ((int64_t)d->k_in + 7) / 8 * 8, np = ((int64_t)d->n_shard + 7) / 8 * 8;
  if (m * std::max<int64_t>(d->ldx, kp) * es >= top || m * std::max<int64_t>(d->ldy, np) * es >= top ||
      d->k_in * np * es >= top || 32 * std::max<int64_t>({d->ldx, kp, np}) * es >= top)
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

// The weights as lines of whole eights, np apart.
template <class E>
static void gated_weights(const sb_gated_desc* d, const void* const* w, const void** to, bool pack,
                          char* ws, const GatedSpace& sp, hipStream_t st) {
  const int np = up8(d->n_shard);
  to[0] = w[0];
  to[1] = w[1];
  if (!pack) return;
  E* out = (E*)(ws + sp.w);
  gated_pack<E><<<dim3(gated_blocks((size_t)d->k_in * np / 4), 2), 256, 0, st>>>(
      (const E*)w[0], (const E*)w[1], d->k_in, d->n_shard, d->n_shard, np, out);
  to[0] = out;
  to[1] = out + (size_t)d->k_in * np;
}
// x, and its stride and width.
template <class E>
static const void* gated_x(const sb_gated_desc* d, const void* x, bool pack, int* ld, int* width,
                           char* ws, const GatedSpace& sp, hipStream_t st) {
  *ld = d->ldx;
  *width = d->k_in;
  if (!pack) return x;
  *ld = *width = up8(d->k_in);
  E* out = (E*)(ws + sp.x);
  gated_pack<E><<<dim3(gated_blocks((size_t)d->m * *ld / 4), 1), 256, 0, st>>>(
      (const E*)x, nullptr, d->m, d->k_in, d->ldx, *ld, out);
  return out;
}

template <class E>
static void gated_fwd_run(const sb_gated_desc* d, const void* x, const void* const* w,
                          const float* const* b, void* y, float* pre, const GatedPacks& packs,
                          char* ws, const GatedSpace& sp, hipStream_t st) {
  const int np = up8(d->n_shard);
  DualArgs g{};
  const void* wp[2];
  g.a[0] = gated_x<E>(d, x, packs.x, &g.lda, &g.K, ws, sp, st);
  gated_weights<E>(d, w, wp, packs.w, ws, sp, st);
  g.b[0][0] = wp[0]; g.b[1][0] = wp[1];
  g.ldb = np;
  g.M = d->m; g.N = d->n_shard; g.segs = 1;
  g.a_bytes = (uint32_t)(((size_t)(d->m - 1) * g.lda + g.K) * sizeof(E));
  g.b_bytes = (uint32_t)((size_t)d->k_in * np * sizeof(E));
  g.c[0] = y; g.ldc = d->ldy;
  g.bias[0] = b[0]; g.bias[1] = b[1];
  g.pre = pre;
  dual_run<kDualFwd, E>(g, gated_plan(d, kDualFwd), d->act, (float*)(ws + sp.split), st);
}

template <class E>
static void gated_bwd_run(const sb_gated_desc* d, const void* x, const void* const* w,
                          const float* pre, const void* dy, void* dx, float* const* dw,
                          float* const* db, int accumulate, const GatedPacks& packs, char* ws,
                          const GatedSpace& sp, hipStream_t st) {
  constexpr int NP = sizeof(E) == 2 ? 3 : 1;
  const int np = up8(d->n_shard), rows = act_rows(d->m, np), chunks = cdiv(d->m, rows);
  const size_t plane = (size_t)d->m * np;
  E* parts = (E*)(ws + sp.d);
  float* split = (float*)(ws + sp.split);
  float* sums = db[0] || db[1] ? (float*)(ws + sp.sums) : nullptr;
  const int vec = d->n_shard % 4 == 0 && at16(pre) && d->ldy % 4 == 0 &&
                  ((uintptr_t)dy & (4 * sizeof(E) - 1)) == 0;
  gated_act_bwd<E><<<dim3(cdiv(np, 256), chunks), 256, 0, st>>>(
      d->m, d->n_shard, np, d->act, pre, (const E*)dy, d->ldy, parts, sums, rows, vec);
  if (sums)
    gated_bias_sums<<<dim3(cdiv(d->n_shard, 64), 2), 256, 0, st>>>(sums, chunks, d->n_shard, np,
                                                                   db[0], db[1], accumulate);
  if (dx) {
    DualArgs g{};
    const void* wp[2];
    gated_weights<E>(d, w, wp, packs.w, ws, sp, st);
    for (int q = 0; q < 2; ++q) {
      g.a[q] = parts + NP * q * plane;
      g.b[0][q] = wp[q];
    }
    g.lda = g.ldb = np;
    g.M = d->m; g.N = d->k_in; g.K = np; g.segs = 2;
    g.a_bytes = (uint32_t)(plane * sizeof(E));
    g.b_bytes = (uint32_t)((size_t)d->k_in * np * sizeof(E));
    g.c[0] = dx; g.ldc = d->ldx;
    dual_run<kDualDx, E>(g, gated_plan(d, kDualDx), 0, split, st);
  }
  DualArgs g{};
  int width;
  const void* xp = gated_x<E>(d, x, packs.lines, &g.lda, &width, ws, sp, st);
  for (int p = 0; p < NP; ++p) {                     // the smallest parts first
    g.a[p] = xp;
    for (int q = 0; q < 2; ++q) g.b[q][p] = parts + (NP * q + NP - 1 - p) * plane;
  }
  g.ldb = np;
  g.M = d->k_in; g.N = d->n_shard; g.K = d->m; g.segs = NP;
  g.a_bytes = (uint32_t)(((size_t)(d->m - 1) * g.lda + width) * sizeof(E));
  g.b_bytes = (uint32_t)(plane * sizeof(E));
  g.c[0] = dw[0]; g.c[1] = dw[1]; g.ldc = d->n_shard;
  g.accumulate = accumulate;
  dual_run<kDualDw, E>(g, gated_plan(d, kDualDw), 0, split, st);
}

}  // namespace sb

using namespace sb;

extern "C" size_t sb_gated_workspace_bytes(const sb_gated_desc* d, int pass) {
  if (gated_check(d) != SB_OK || (pass != SB_FC_FWD && pass != SB_FC_BWD)) return (size_t)-1;
  const bool at = !(d->flags & SB_UNALIGNED);
  return gated_space(d, pass, gated_packs(d, at, at)).bytes;
}

extern "C" sb_status sb_gated_shard_fwd(const sb_gated_desc* d, const void* x, const void* w_gate,
                                        const void* w_up, const float* b_gate, const float* b_up,
                                        void* y, float* pre, void* ws, size_t ws_bytes,
                                        void* stream) {
  const sb_status s = gated_check(d);
  if (s != SB_OK) return s;
  if (!x || !w_gate || !w_up || !y) return SB_ERR_INVALID_ARG;
  const size_t es = sbh::dsize(d->dtype), nb = (size_t)d->n_shard * 4;
  const size_t wb = (size_t)d->k_in * d->n_shard * es;
  const GatedPacks packs = gated_packs(d, at16(x), at16(w_gate) && at16(w_up));
  const GatedSpace sp = gated_space(d, SB_FC_FWD, packs);
  const Span ins[5] = {{x, ((size_t)(d->m - 1) * d->ldx + d->k_in) * es}, {w_gate, wb},
                       {w_up, wb}, {b_gate, nb}, {b_up, nb}};
  const Span outs[3] = {{y, ((size_t)(d->m - 1) * d->ldy + d->n_shard) * es},
                        {pre, (size_t)d->m * d->n_shard * 8}, {ws, sp.bytes}};
  if (spans_meet(outs, 3, ins, 5) || spans_meet(outs, 1, outs + 1, 2) ||
      spans_meet(outs + 1, 1, outs + 2, 1))
    return SB_ERR_INVALID_ARG;
  if (sp.bytes > 0 && (!ws || ws_bytes < sp.bytes)) return SB_ERR_WORKSPACE;
  if (sp.bytes > 0 && !at16(ws)) return SB_ERR_INVALID_ARG;
  const void* w[2] = {w_gate, w_up};
  const float* b[2] = {b_gate, b_up};
  const auto run = d->dtype == SB_BF16 ? gated_fwd_run<u16> : gated_fwd_run<float>;
  run(d, x, w, b, y, pre, packs, (char*)ws, sp, sbh::stream_of(stream));
  return sbh::launch_status();
}

extern "C" sb_status sb_gated_shard_bwd(const sb_gated_desc* d, const void* x, const void* w_gate,
                                        const void* w_up, const float* pre, const void* dy,
                                        void* dx, float* dw_gate, float* dw_up, float* db_gate,
                                        float* db_up, int accumulate, void* ws, size_t ws_bytes,
                                        void* stream) {
  const sb_status s = gated_check(d);
  if (s != SB_OK) return s;
  if (!x || !w_gate || !w_up || !pre || !dy || !dw_gate || !dw_up) return SB_ERR_INVALID_ARG;
  if (accumulate != 0 && accumulate != 1) return SB_ERR_INVALID_ARG;
  const size_t es = sbh::dsize(d->dtype), nb = (size_t)d->n_shard * 4;
  const size_t xb = ((size_t)(d->m - 1) * d->ldx + d->k_in) * es;
  const size_t wn = (size_t)d->k_in * d->n_shard;
  const GatedPacks packs = gated_packs(d, at16(x), at16(w_gate) && at16(w_up));
  const GatedSpace sp = gated_space(d, SB_FC_BWD, packs);
  const Span ins[5] = {{x, xb}, {w_gate, wn * es}, {w_up, wn * es},
                       {pre, (size_t)d->m * d->n_shard * 8},
                       {dy, ((size_t)(d->m - 1) * d->ldy + d->n_shard) * es}};
  const Span outs[6] = {{dx, xb}, {dw_gate, wn * 4}, {dw_up, wn * 4}, {db_gate, nb}, {db_up, nb},
                        {ws, sp.bytes}};
  if (spans_meet(outs, 6, ins, 5)) return SB_ERR_INVALID_ARG;
  for (int i = 0; i < 5; ++i)
    if (spans_meet(outs + i, 1, outs + i + 1, 5 - i)) return SB_ERR_INVALID_ARG;
  if (!ws || ws_bytes < sp.bytes) return SB_ERR_WORKSPACE;
  if (!at16(ws)) return SB_ERR_INVALID_ARG;
  const void* w[2] = {w_gate, w_up};
  float* dw[2] = {dw_gate, dw_up};
  float* db[2] = {db_gate, db_up};
  const auto run = d->dtype == SB_BF16 ? gated_bwd_run<u16> : gated_bwd_run<float>;
  run(d, x, w, pre, dy, dx, dw, db, accumulate, packs, (char*)ws, sp, sbh::stream_of(stream));
  return sbh::launch_status();
}
