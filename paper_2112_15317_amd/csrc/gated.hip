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
// and the product with it are one kernel, dx and both weight gradients another;
// da, du and the bias gradients come from a pass over dy and the kept a and u.
//
// The weight gradients are fp32 also where x is bf16: da and du go into their
// products as three bf16 parts, which hold all 24 bits, so a gradient is off by the
// rounding of its fp32 sums and not by 2^-9 of every term (measured against 64 bits over
// 2048 rows: 2.5e-7 of the gradient; with two parts 2.6e-6, with one 1.7e-3).  dx of the
// bf16 path is rounded to bf16 itself and takes their first two parts, 16 bits: with one,
// it was 2.3e-3 off where the rounding of its result alone is 1.7e-3, for a sixth less of
// a large step's time (4096 x 4096 x 8192: 2881 us, 2432 with one).
#include "gemm_dual.hpp"

#include <algorithm>
#include <cmath>
#include <mutex>

namespace sb {

// A 16- or 8-byte access need not lie on 16 or 8 bytes.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
// Elements p[0] .. p[3], those from `left` on 0; at any address.
template <class E>
__device__ __forceinline__ f4 load_quad(const E* p, int left) {
  f4 v = f4{0.f, 0.f, 0.f, 0.f};
  if (left >= 4) {
    if constexpr (sizeof(E) == 4) {
      const u32x4 t = *reinterpret_cast<const u32x4_any*>(p);
      v = f4{__uint_as_float(t[0]), __uint_as_float(t[1]), __uint_as_float(t[2]), __uint_as_float(t[3])};
    } else {
      const u32x2_any t = *reinterpret_cast<const u32x2_any*>(p);
      v = f4{__uint_as_float(t[0] << 16), __uint_as_float(t[0] & 0xffff0000u),
             __uint_as_float(t[1] << 16), __uint_as_float(t[1] & 0xffff0000u)};
    }
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < left) v[e] = Elem<E>::load(p, e);
  }
  return v;
}

// Up to three matrices: rows of `cols` elements, `ld` apart, to rows of cp (a multiple
// of 8), zeros behind.  Matrix q has blocks block0[q] .. block0[q + 1] - 1.
struct PackTasks {
  const void* from[3];
  void* to[3];
  int rows[3], cols[3], ld[3], cp[3], block0[4];
  int count;
};
template <class E>
__device__ __forceinline__ void pack_rows(const PackTasks& t, int block) {
  const int q = block >= t.block0[2] ? 2 : block >= t.block0[1] ? 1 : 0;
  const int cols = t.cols[q], cp = t.cp[q];
  const E* from = (const E*)t.from[q];
  E* out = (E*)t.to[q];
  const size_t quads = (size_t)t.rows[q] * (cp / 4);
  const size_t step = (size_t)(t.block0[q + 1] - t.block0[q]) * 256;
  for (size_t i = (size_t)(block - t.block0[q]) * 256 + threadIdx.x; i < quads; i += step) {
    const uint32_t r = (uint32_t)i / (uint32_t)(cp / 4);     // (quads are below 2^29)
    const int c = (int)((uint32_t)i - r * (cp / 4)) * 4;
    Elem<E>::store4(out + (size_t)r * cp + c, load_quad<E>(from + (size_t)r * t.ld[q] + c, cols - c));
  }
}
template <class E>
__global__ __launch_bounds__(256) void gated_pack(PackTasks t) {
  pack_rows<E>(t, blockIdx.x);
}

// da and du in rows of np (n rounded up to 8, zeros behind n).  D fp32: da, then du,
// m * np elements each.  bf16: three parts of each, part p of da at p * m * np, of du at
// (3 + p) * m * np.  A block has 256 columns of `rows` rows, a lane four columns of
// every fourth row.  Its columns' sums are db where it has all rows, else they go to
// sums [row block][2][np].  The blocks behind pack the operands of the products to come
// (each launch less is 4 us to a caller that does not capture its calls).
static int act_rows(int m, int np) {
  // 32 rows, fewer where that would leave CUs idle (128 x 256: 10.2 -> 3.7 us), but all
  // of them up to 32, which saves the launch that joins the sums.
  int rows = 32;
  if (m > rows)
    while (rows > 4 && (int64_t)((np + 255) / 256) * cdiv(m, rows) < 1024) rows /= 2;
  return rows;
}

template <class E, class D>
__global__ __launch_bounds__(256) void gated_act_bwd(int m, int n, int np, int act,
                                                     const float* __restrict__ pre,
                                                     const E* __restrict__ dy, int ldy,
                                                     D* __restrict__ d, BiasSums bias, int rows,
                                                     int chunks, PackTasks packs) {
  __shared__ f4 part[2][4][64];
  const int by = blockIdx.x % chunks, bx = blockIdx.x / chunks;
  if (bx * 256 >= np) {
    pack_rows<E>(packs, blockIdx.x - cdiv(np, 256) * chunks);
    return;
  }
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int c = bx * 256 + lane * 4;
  const size_t mn = (size_t)m * n, plane = (size_t)m * np;
  const int r1 = min(m, (by + 1) * rows);
  f4 s[2] = {f4{0.f, 0.f, 0.f, 0.f}, f4{0.f, 0.f, 0.f, 0.f}};
  for (int r = by * rows + w; r < r1 && c < np; r += 4) {
    const float* pa = pre + (size_t)r * n + c;
    const f4 a = load_quad<float>(pa, n - c), u = load_quad<float>(pa + mn, n - c);
    const f4 g = load_quad<E>(dy + (size_t)r * ldy + c, n - c);
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
      if constexpr (sizeof(D) == 4) {
        *reinterpret_cast<f4*>(d + q * plane + at) = v[q];
      } else {
        // An infinite or NaN first part is the whole value; a finite value's is not past
        // bf16's largest, to which those above it would not round.
        constexpr float most = 0x1.fep127f;
        f4 rest, part;
        bool whole[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          rest[e] = v[q][e];
          whole[e] = (__float_as_uint(rest[e]) & 0x7f800000u) == 0x7f800000u;
          part[e] = whole[e] ? rest[e] : fminf(fmaxf(rest[e], -most), most);
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) {
          uint2 b;
          b.x = f32x2_to_bf16x2(part[0], part[1]);
          b.y = f32x2_to_bf16x2(part[2], part[3]);
          *reinterpret_cast<uint2*>(d + (3 * q + p) * plane + at) = b;
          const f4 h = f4{__uint_as_float(b.x << 16), __uint_as_float(b.x & 0xffff0000u),
                          __uint_as_float(b.y << 16), __uint_as_float(b.y & 0xffff0000u)};
#pragma unroll
          for (int e = 0; e < 4; ++e) rest[e] = part[e] = whole[e] ? 0.f : rest[e] - h[e];
        }
      }
    }
  }
  if (!bias.sums && !bias.db[0] && !bias.db[1]) return;
  part[0][w][lane] = s[0];
  part[1][w][lane] = s[1];
  __syncthreads();
  if (w >= 2 || c >= np) return;
  const f4 t = (part[w][0][lane] + part[w][1][lane]) + (part[w][2][lane] + part[w][3][lane]);
  if (bias.sums) {
    *reinterpret_cast<f4*>(bias.sums + ((size_t)by * 2 + w) * np + c) = t;
  } else if (float* db = w ? bias.db[1] : bias.db[0]) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < n) db[c + e] = bias.accumulate ? db[c + e] + t[e] : t[e];
  }
}

// ---- few rows --------------------------------------------------------------
// Up to kFewRows rows (a model that answers, the last rows of a batch): the weights are
// read once and bound the time, and tiles of 128 rows would be mostly zeros.  Products
// on the vector ALU, whole pieces of a weight's line a lane, sums in fp32.
constexpr int kFewRows = 8;

// A piece: eight (bf16) or four (fp32) consecutive elements, at any address (a 16-byte
// access need not lie on 16 bytes).  Where fewer are left the piece that ends with the
// last one is taken and its first elements, which another piece has, are set to 0 (bounds
// for each element took 8 us of the 12 of 164 x 287): so a row has a piece's elements.
template <class E> constexpr int kFewWidth = 16 / (int)sizeof(E);
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
template <class E, int N = kFewWidth<E>>
__device__ __forceinline__ u32x4 few_piece(const E* p) {
  if constexpr (N * sizeof(E) == 16) {
    return *reinterpret_cast<const u32x4_any*>(p);
  } else {
    static_assert(N * sizeof(E) == 8, "half a piece");
    const u32x2_any t = *reinterpret_cast<const u32x2_any*>(p);
    return u32x4{t[0], t[1], 0, 0};
  }
}
// Two bf16 products and s.  (Rounded once or twice: within 2^-23 of the three terms.  A
// product of a subnormal factor, below 2^-126 of the other, keeps 16 bits or more.)
__device__ __forceinline__ float few_dot(uint32_t a, uint32_t b, float s) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, a), __builtin_bit_cast(bf16x2, b), s,
                                         false);
}
// Its first `skip` elements 0.
template <class E>
__device__ __forceinline__ u32x4 few_without(u32x4 t, int skip) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(E) == 4) t[i] = i < skip ? 0 : t[i];
    else t[i] &= 2 * i + 1 < skip ? 0 : 2 * i < skip ? 0xffff0000u : 0xffffffffu;
  }
  return t;
}
// The value of the lane N further on in a row of 16.
template <int N>
__device__ __forceinline__ float row_turned(float v) {
  const int i = __float_as_int(v);
  return __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0x120 + N, 0xf, 0xf, false));
}

// Sums over a wave's four rows of 16 lanes, of four values at once: row 0 of the result
// has the first, row 1 the third, row 2 the second, row 3 the fourth.  (Swapping halves
// of two registers adds up two values in the instructions of one.)
__device__ __forceinline__ float halves_sum(float a, float b) {
  const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return __uint_as_float(t[0]) + __uint_as_float(t[1]);
}
__device__ __forceinline__ float rows_sum(float a, float b, float c, float d) {
  const float p = halves_sum(a, b), q = halves_sum(c, d);
  const auto t = __builtin_amdgcn_permlane16_swap(__float_as_uint(p), __float_as_uint(q), false, false);
  return __uint_as_float(t[0]) + __uint_as_float(t[1]);
}

struct FewArgs {
  const void *x, *w[2];
  const float* bias[2];
  void* y;
  float *pre, *part;                                 // part: splits > 1, as DualArgs'
  int m, n, k, ldx, ldy, pitch, act;
  int strips, splits, lines;                         // lines of k a split
};

// Forward of M rows: a block has the columns of L lanes (16 L bytes of a line of each
// weight) and a split's lines, J at a time for each L lanes: 2 J loads of 16 bytes are
// under way in a lane, and x is a piece for J lines.  L = 8 takes whole lines of the
// caches.  L = 4 takes half of them and so does half the work a block one after the other,
// but what the caches read twice bounds it from a few MB on.  One row of bf16 weights
// (in a captured graph): 1024 x 1024 3.8 us (one line of k at a time a lane, reduced by
// shuffles: 5.5), 4096 x 1024 7.1 (24.1), 4096 x 4096 16.4 (4.1 TB/s); eight rows of
// 4096 x 4096 20.0.
template <class E, int M> constexpr int kFewLines = sizeof(E) == 2 && M == 8 ? 4 : kFewWidth<E>;
template <class E, int M, int L>
__global__ __launch_bounds__(512) void gated_few_fwd(FewArgs g) {
  constexpr int V = kFewWidth<E>, J = kFewLines<E, M>, C = L * V, NV = 2 * M * V, TH = 512, W = TH / 64;
  __shared__ float part[W][NV][L];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int strip = blockIdx.x % g.strips, split = blockIdx.x / g.strips;
  const int c0 = strip * C + lane % L * V, c = min(c0, g.n - V);
  const int k1 = min(g.k, (split + 1) * g.lines);
  const E* x = (const E*)g.x;
  float acc[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) acc[i] = 0.f;
  if (c0 < g.n) {
    for (int kk = split * g.lines + threadIdx.x / L * J; kk < k1; kk += TH / L * J) {
      const int skip = max(kk + J - k1, 0), k0 = kk - skip;
      u32x4 w[2][J];
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int q = 0; q < 2; ++q) w[q][j] = few_piece<E>((const E*)g.w[q] + (size_t)(k0 + j) * g.n + c);
      u32x4 xs[M];                                   // J elements
#pragma unroll
      for (int r = 0; r < M; ++r)
        xs[r] = few_piece<E, J>(x + (size_t)min(r, g.m - 1) * g.ldx + k0);
      if (skip) {                                    // of both: each may be infinite
#pragma unroll
        for (int r = 0; r < M; ++r) xs[r] = few_without<E>(xs[r], skip);
#pragma unroll
        for (int j = 0; j < J - 1; ++j)
#pragma unroll
          for (int q = 0; q < 2; ++q)
            if (j < skip) w[q][j] = u32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          if constexpr (sizeof(E) == 2) {
            // Two lines at a time, as x has them.
#pragma unroll
            for (int j = 0; j < J; j += 2) {
              const uint32_t v = __builtin_amdgcn_perm(w[q][j + 1][e / 2], w[q][j][e / 2],
                                                       e % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
              for (int r = 0; r < M; ++r) {
                float& s = acc[(q * M + r) * V + e];
                s = few_dot(v, xs[r][j / 2], s);
              }
            }
          } else {
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
              for (int r = 0; r < M; ++r) {
                float& s = acc[(q * M + r) * V + e];
                s = fmaf(__uint_as_float(xs[r][j]), __uint_as_float(w[q][j][e]), s);
              }
          }
        }
    }
  }
  const int row = lane / 16;
#pragma unroll
  for (int i = 0; i < NV; i += 4) {
    float v = rows_sum(acc[i], acc[i + 1], acc[i + 2], acc[i + 3]);
    if constexpr (L <= 8) v += row_turned<8>(v);
    if constexpr (L <= 4) v += row_turned<4>(v);
    if constexpr (L <= 2) v += row_turned<2>(v);
    if (lane % 16 < L) part[wave][i + row / 2 + row % 2 * 2][lane % 16] = v;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < g.m * C; i += TH) {
    const int r = i / C, at = i % C, own = strip * C + at / V * V, col = min(own, g.n - V) + at % V;
    if (own >= g.n || col < own) continue;
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int w = 0; w < W; ++w) s[q] += part[w][(q * M + r) * V + at % V][at / V];
    if (g.splits > 1) {
#pragma unroll
      for (int q = 0; q < 2; ++q) g.part[(((size_t)split * 2 + q) * g.m + r) * g.pitch + col] = s[q];
      continue;
    }
    const float a = s[0] + (g.bias[0] ? g.bias[0][col] : 0.f);
    const float u = s[1] + (g.bias[1] ? g.bias[1][col] : 0.f);
    float f, df;
    gate_act(g.act, a, f, df);
    if (g.pre) {
      g.pre[(size_t)r * g.n + col] = a;
      g.pre[((size_t)g.m + r) * g.n + col] = u;
    }
    Elem<E>::store((E*)g.y, (size_t)r * g.ldy + col, f * u);
  }
}

// Backward of M rows, one launch: da and du of one or two rows are so few that every block
// forms those it needs (as a pass of their own and products on tiles: 2 x 1024 x 1280 bf16
// 17.2 us, like this 9.1).  From three rows on dx takes them from the pass over dy (8 x
// 2048 x 2048 fp32 30.0 us without it, 21.5 with it), the weight gradients' blocks,
// which need a strip of them, do not.
constexpr int kFewGates = 2;
constexpr int kFewDx = 16;                           // lines of k a block of dx
struct FewBwdArgs {
  const void *x, *w[2], *dy;
  const float* pre;
  void* dx;
  float *dw[2], *db[2];
  int m, n, k, ldx, ldy, act, accumulate;
  int first, strips, lines;                          // first: blocks of dx; lines of k a block behind
  const float* d[2]; int np;                         // da and du from the pass, M > kFewGates
};

// The dot product of a piece of a weight with as many fp32 values, and s.
template <class E>
__device__ __forceinline__ float few_dot_f32(u32x4 w, const f4 (&d)[kFewWidth<E> / 4], float s) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (sizeof(E) == 4) {
      s = fmaf(__uint_as_float(w[e]), d[0][e], s);
    } else {
      s = fmaf(__uint_as_float(w[e] << 16), d[e / 2][e % 2 * 2], s);
      s = fmaf(__uint_as_float(w[e] & 0xffff0000u), d[e / 2][e % 2 * 2 + 1], s);
    }
  }
  return s;
}

// da and du of four columns of a row, those from `left` on 0.
template <class E>
__device__ __forceinline__ void few_gates(const FewBwdArgs& g, int r, int c, int left, f4& da, f4& du) {
  const float* pa = g.pre + (size_t)r * g.n + c;
  const f4 a = load_quad<float>(pa, left), u = load_quad<float>(pa + (size_t)g.m * g.n, left);
  const f4 dy = load_quad<E>((const E*)g.dy + (size_t)r * g.ldy + c, left);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float f, df;
    gate_act(g.act, a[e], f, df);
    da[e] = e < left ? dy[e] * u[e] * df : 0.f;
    du[e] = e < left ? dy[e] * f : 0.f;
  }
}

// dx of rows whose da and du the pass has formed, in fp32: a wave has four lines of both
// weights, its lanes the columns, four at a time (bf16 lines in pieces of eight took 39 us
// for 8 x 2048 x 2048, 21 in fours: the loads of da and du, not the weights', wait then).
template <class E, int M>
__device__ __forceinline__ void few_dx_lines(const FewBwdArgs& g, int block) {
  constexpr int R = 4;
  const int lane = threadIdx.x & 63;
  const int k0 = (block * 4 + (threadIdx.x >> 6)) * R;
  float acc[R][M];
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int r = 0; r < M; ++r) acc[i][r] = 0.f;
  for (int c0 = lane * 4; c0 < g.n; c0 += 256) {
    const int skip = max(c0 + 4 - g.n, 0), c = c0 - skip;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      f4 w[R], d[M];
#pragma unroll
      for (int i = 0; i < R; ++i)
        w[i] = load_quad<E>((const E*)g.w[q] + (size_t)min(k0 + i, g.k - 1) * g.n + c, 4);
#pragma unroll
      for (int r = 0; r < M; ++r)
        d[r] = load_quad<float>(g.d[q] + (size_t)min(r, g.m - 1) * g.np + c, 4);
      if (skip) {
#pragma unroll
        for (int e = 0; e < 3; ++e) {
#pragma unroll
          for (int i = 0; i < R; ++i) w[i][e] = e < skip ? 0.f : w[i][e];
#pragma unroll
          for (int r = 0; r < M; ++r) d[r][e] = e < skip ? 0.f : d[r][e];
        }
      }
#pragma unroll
      for (int r = 0; r < M; ++r)
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][r] = fmaf(w[i][e], d[r][e], acc[i][r]);
    }
  }
  // The sums of four lines at once, in the four rows of lanes.
  const int row = lane / 16, at = k0 + row / 2 + row % 2 * 2;
#pragma unroll
  for (int r = 0; r < M; ++r) {
    float v = rows_sum(acc[0][r], acc[1][r], acc[2][r], acc[3][r]);
    v += row_turned<8>(v);
    v += row_turned<4>(v);
    v += row_turned<2>(v);
    v += row_turned<1>(v);
    if (lane % 16 == 0 && at < g.k && r < g.m) Elem<E>::store((E*)g.dx, (size_t)r * g.ldx + at, v);
  }
}

// dx of up to kFewGates rows: a block has kFewDx lines of both weights, each wave 64 pieces
// of them at a time, whose da and du it forms.  (With more rows that many
// activations a wave take longer than all the rest: 8 x 1024 x 1024 bf16 23.8 us for 12.6.)
template <class E, int M>
__device__ __forceinline__ void few_dx_block(const FewBwdArgs& g, int block, float* lds) {
  constexpr int V = kFewWidth<E>, R = kFewDx;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int k0 = block * R;
  float acc[R][M];
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int r = 0; r < M; ++r) acc[i][r] = 0.f;
  for (int b = wave * 64 * V; b < g.n; b += 4 * 64 * V) {
    const int c0 = b + lane * V, c = min(c0, g.n - V), skip = c0 - c;
    f4 d[2][M][V / 4];
#pragma unroll
    for (int r = 0; r < M; ++r)
#pragma unroll
      for (int i = 0; i < V / 4; ++i) {
        few_gates<E>(g, min(r, g.m - 1), c + 4 * i, 4, d[0][r][i], d[1][r][i]);
        if (skip) {
#pragma unroll
          for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) d[q][r][i][e] = 4 * i + e < skip ? 0.f : d[q][r][i][e];
        }
      }
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        u32x4 w = few_piece<E>((const E*)g.w[q] + (size_t)min(k0 + i, g.k - 1) * g.n + c);
        if (skip) w = few_without<E>(w, skip);
#pragma unroll
        for (int r = 0; r < M; ++r) acc[i][r] = few_dot_f32<E>(w, d[q][r], acc[i][r]);
      }
  }
  // The sums of four lines at once, in the four rows of lanes.
  const int row = lane / 16, at = row / 2 + row % 2 * 2;
#pragma unroll
  for (int i = 0; i < R; i += 4)
#pragma unroll
    for (int r = 0; r < M; ++r) {
      float v = rows_sum(acc[i][r], acc[i + 1][r], acc[i + 2][r], acc[i + 3][r]);
      v += row_turned<8>(v);
      v += row_turned<4>(v);
      v += row_turned<2>(v);
      v += row_turned<1>(v);
      if (lane % 16 == 0) lds[(wave * M + r) * R + i + at] = v;
    }
  __syncthreads();
  const int r = threadIdx.x / R, i = threadIdx.x % R;
  if (r < g.m && r < M && k0 + i < g.k)
    Elem<E>::store((E*)g.dx, (size_t)r * g.ldx + k0 + i,
                   (lds[r * R + i] + lds[(M + r) * R + i]) +
                       (lds[(2 * M + r) * R + i] + lds[(3 * M + r) * R + i]));
}

// The weight gradients of 256 columns and g.lines of k, eight lines a wave at a time, and
// the bias gradients beside the first of them.  What it writes bounds it.
template <class E, int M>
__device__ __forceinline__ void few_dw_block(const FewBwdArgs& g, int block, float* lds) {
  constexpr int V = kFewWidth<E>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c0 = block % g.strips * 256, c = c0 + lane * 4, k0 = block / g.strips * g.lines;
  for (int r = wave; r < g.m; r += 4) {
    f4 da, du;
    few_gates<E>(g, r, c, g.n - c, da, du);
    *reinterpret_cast<f4*>(lds + r * 256 + lane * 4) = da;
    *reinterpret_cast<f4*>(lds + (M + r) * 256 + lane * 4) = du;
  }
  __syncthreads();
  f4 d[2][M];
#pragma unroll
  for (int q = 0; q < 2; ++q)
#pragma unroll
    for (int r = 0; r < M; ++r)
      d[q][r] = r < g.m ? *reinterpret_cast<const f4*>(lds + (q * M + r) * 256 + lane * 4)
                        : f4{0.f, 0.f, 0.f, 0.f};
  if (k0 == 0 && wave == 0) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      f4 v = d[q][0];
#pragma unroll
      for (int r = 1; r < M; ++r) v += d[q][r];
      float* db = g.db[q];
      if (!db) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < g.n) db[c + e] = g.accumulate ? db[c + e] + v[e] : v[e];
    }
  }
  const int k1 = min(g.k, k0 + g.lines);
  for (int kk = k0 + wave * 8; kk < k1; kk += 32) {
    const int kx = min(kk, g.k - 8);                 // the last eight may be begun earlier
    u32x4 x[M][8 / V];
#pragma unroll
    for (int r = 0; r < M; ++r)
#pragma unroll
      for (int i = 0; i < 8 / V; ++i)
        x[r][i] = few_piece<E>((const E*)g.x + (size_t)min(r, g.m - 1) * g.ldx + kx + i * V);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (kx + j < kk) continue;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        f4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int r = 0; r < M; ++r) {
          if (r >= g.m) continue;
          const uint32_t t = x[r][j / V][sizeof(E) == 4 ? j % V : j / 2];
          const float xv = __uint_as_float(sizeof(E) == 4 ? t : j % 2 ? t & 0xffff0000u : t << 16);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = fmaf(xv, d[q][r][e], v[e]);
        }
        float* row = g.dw[q] + (size_t)(kx + j) * g.n + c;
        if (c + 4 <= g.n) {
          if (g.accumulate) v += load_quad<float>(row, 4);
          *reinterpret_cast<u32x4_any*>(row) = __builtin_bit_cast(u32x4, v);
        } else {
#pragma unroll
          for (int e = 0; e < 3; ++e)
            if (c + e < g.n) row[e] = g.accumulate ? row[e] + v[e] : v[e];
        }
      }
    }
  }
}

template <class E, int M>
__global__ __launch_bounds__(256) void gated_few_bwd(FewBwdArgs g) {
  __shared__ __attribute__((aligned(16))) float lds[2 * M * 256];
  if ((int)blockIdx.x < g.first) {
    if constexpr (M <= kFewGates) few_dx_block<E, M>(g, blockIdx.x, lds);
    else few_dx_lines<E, M>(g, blockIdx.x);
  } else few_dw_block<E, M>(g, (int)blockIdx.x - g.first, lds);
}

// Sums of the splits' partials (rows of g.pitch), four columns of a row a lane.  FWD:
// [split][2][M] to y and pre; DW: to the two gradients; DX: [split][M] to dx.  W waves
// share the splits of a quad (many splits are of small outputs, which are few lanes).
template <DualKind KIND, class E, int W>
__device__ __forceinline__ void split_sum_block(const DualArgs& g, int act, int block, f4* lds) {
  constexpr int Q = KIND == kDualDx ? 1 : 2, LANES = 256 / W;
  const uint32_t quads = g.pitch / 4;
  const int w = threadIdx.x / LANES, lane = threadIdx.x % LANES;
  const uint32_t i = (uint32_t)block * LANES + lane, row = i / quads;   // (below 2^30)
  const int m = (int)min(row, (uint32_t)g.M - 1), n = (int)(i - row * quads) * 4;
  const size_t plane = (size_t)g.M * g.pitch, at = (size_t)m * g.pitch + n;
  const int per = cdiv(g.splits, W), s0 = min(w * per, g.splits), s1 = min(s0 + per, g.splits);
  f4 v[Q];
#pragma unroll
  for (int q = 0; q < Q; ++q) v[q] = split_sum4(g.part + q * plane, s0, s1, Q * plane, at);
  if constexpr (W > 1) {
#pragma unroll
    for (int q = 0; q < Q; ++q) lds[(w * Q + q) * LANES + lane] = v[q];
    __syncthreads();
    if (w) return;
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int u = 1; u < W; ++u) v[q] += lds[(u * Q + q) * LANES + lane];
  }
  if (row >= (uint32_t)g.M) return;
  if constexpr (KIND == kDualDx) {
    put_quad((E*)g.c[0] + (size_t)m * g.ldc, v[0], n, g.N);
  } else if constexpr (KIND == kDualFwd) {
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (g.bias[q] && n + e < g.N) v[q][e] += g.bias[q][n + e];
    gate_store<E>(act, v[0], v[1], n, g.N, g.pre ? g.pre + (size_t)m * g.N : nullptr,
                  (size_t)g.M * g.N, (E*)g.c[0] + (size_t)m * g.ldc);
  } else {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      float* c = (float*)g.c[q] + (size_t)m * g.ldc;
      if (g.accumulate) v[q] += get_quad(c, n, g.N);
      put_quad(c, v[q], n, g.N);
    }
  }
}
template <class E, int W>
__global__ __launch_bounds__(256) void gated_split_sum(DualArgs g, int act) {
  __shared__ f4 lds[W > 1 ? 512 : 1];
  split_sum_block<kDualFwd, E, W>(g, act, blockIdx.x, lds);
}
// Of dx in the first blocks, of the weight gradients behind them.
template <class E, int W>
__global__ __launch_bounds__(256) void gated_split_sums(DualArgs dx, DualArgs dw, int first) {
  __shared__ f4 lds[W > 1 ? 512 : 1];
  if ((int)blockIdx.x < first) split_sum_block<kDualDx, E, W>(dx, 0, blockIdx.x, lds);
  else split_sum_block<kDualDw, E, W>(dw, 0, (int)blockIdx.x - first, lds);
}
static int split_sum_blocks(const DualArgs& g, int w) {
  return g.splits > 1 ? (int)(((size_t)g.M * (g.pitch / 4) + 256 / w - 1) / (256 / w)) : 0;
}

// Tile and split of a product: the least estimated time (us) over 256-row tiles (bf16) and
// 128-row ones and 1 to 64 ranges of the reduction.  A block costs its first stages and
// its output, then a stage at a time, the more the fuller the chip is (power, L2); up to
// three blocks of 128 rows share a CU, where one does not use it to the full; splits cost a
// launch and their partials' traffic.  Fitted to 8000 timings of the three products of 900
// shards in both types; the plan taken is 1.8 (bf16) or 1.2 % (fp32) slower than the best
// one on average, at most half as slow again (80 rows of 1280 by 128: 21 us for 13).
struct DualPlan { int f, mt, nt, splits, stages; size_t ws_bytes; };
struct DualCost { double block, alone, full, shared; };
static const DualCost kDualCost[3] = {{9.0, 0.56, 0.92, 0.92},         // bf16, 256 rows
                                      {4.8, 0.253, 0.338, 0.30},      // bf16, 128 rows
                                      {4.1, 0.92, 1.09, 1.09}};       // fp32, 128 rows

static DualPlan dual_plan(DualKind kind, bool b16, int M, int N, int K, int segs) {
  DualPlan best{};
  double best_t = 0;
  const int total = cdiv(K, 32) * segs;
  const double tb_s = b16 ? 8.24 : 5.72;
  const double bytes = (double)M * cdiv(N, 4) * 4 * (kind == kDualDx ? 4 : 8);
  for (int f = b16 ? 4 : 2; f >= 2; f -= 2) {
    const DualCost& c = kDualCost[!b16 ? 2 : f == 4 ? 0 : 1];
    const int share = b16 && f == 2 ? 3 : 1;
    const int mt = cdiv(M, 64 * f), nt = cdiv(N, kind == kDualDx ? 64 * f : 32 * f);
    const int64_t tiles = (int64_t)mt * nt;
    for (int s = 1; s <= 64 && s <= total; ++s) {
      const int stages = cdiv(total, s);
      if (cdiv(total, stages) != s) continue;
      const int64_t blocks = tiles * s;
      const double per_cu = (double)((blocks + 255) / 256);
      const double one = c.alone + (c.full - c.alone) * std::min(1.0, (double)blocks / 256);
      double t = s > 1 ? 3.2 + bytes * (2 * s + 1) / (tb_s * 1e6) : bytes / (tb_s * 1e6);
      if (share == 1) t += per_cu * (c.block + stages * one);
      else t += c.block * std::ceil(per_cu / share) + stages * (per_cu > 1 ? c.shared * per_cu : one);
      if (best_t == 0 || t < best_t) {
        best_t = t;
        best = DualPlan{f, mt, nt, s, stages, s > 1 ? (size_t)s * (size_t)bytes : 0};
      }
    }
  }
  return best;
}

// The plan of dx and the weight gradients in one launch: one tile, splits of each.  The
// time is the longest block's, or all blocks' over the chip where that is more (a
// fifth more where a CU takes one block after the other).  One launch instead of two,
// and one for both sums, saves a third of the time over 120 shards in both types (from
// 2 % at 593 x 2752 x 1984 fp32 to 43 % at 248 x 1024 x 384 bf16); the plan taken is
// 2 (fp32) or 7 % (bf16, with one part in dx) slower than the best on average over 270,
// mostly where all take 10 to 20 us.
struct GradPlan { DualPlan dx, dw; };

static GradPlan grad_plan(bool b16, int m, int k, int n) {
  static const int kSplits[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
  GradPlan best{};
  double best_t = 0;
  const int total[2] = {cdiv(n, 32) * (b16 ? 4 : 2), cdiv(m, 32) * (b16 ? 3 : 1)};
  const double bytes[2] = {(double)m * cdiv(k, 4) * 16, (double)k * cdiv(n, 4) * 32};
  const double tb_s = (b16 ? 8.24 : 5.72) * 1e6;
  for (int f = b16 ? 4 : 2; f >= 2; f -= 2) {
    const DualCost& c = kDualCost[!b16 ? 2 : f == 4 ? 0 : 1];
    const int share = b16 && f == 2 ? 3 : 1;
    const int mt[2] = {cdiv(m, 64 * f), cdiv(k, 64 * f)}, nt[2] = {cdiv(k, 64 * f), cdiv(n, 32 * f)};
    for (int s0 : kSplits) {
      for (int s1 : kSplits) {
        const int s[2] = {s0, s1};
        int stages[2];
        double blocks[2], t = 0.0;
        bool ok = true;
        for (int q = 0; q < 2; ++q) {
          stages[q] = cdiv(total[q], s[q]);
          ok = ok && cdiv(total[q], stages[q]) == s[q];
          blocks[q] = (double)mt[q] * nt[q] * s[q];
          t += s[q] > 1 ? 4.5 + bytes[q] * (2 * s[q] + 1) / tb_s : bytes[q] / tb_s;
        }
        if (!ok) continue;
        const double all = blocks[0] + blocks[1];
        const double one = c.alone + (c.full - c.alone) * std::min(1.0, all / 256);
        const double longest = c.block + std::max(stages[0], stages[1]) * one;
        double sat = 0.0;
        for (int q = 0; q < 2; ++q) sat += blocks[q] * (c.block / share + stages[q] * c.shared) / 256;
        if (share == 1) sat *= 1.2;
        t += all > 256 ? std::max(longest, sat) : longest;
        if (best_t == 0 || t < best_t) {
          best_t = t;
          DualPlan* p[2] = {&best.dx, &best.dw};
          for (int q = 0; q < 2; ++q)
            *p[q] = DualPlan{f, mt[q], nt[q], s[q], stages[q],
                             s[q] > 1 ? (size_t)s[q] * (size_t)bytes[q] : 0};
        }
      }
    }
  }
  return best;
}

template <int F, int ACT, class E>
static void fwd_launch(const DualArgs& g, hipStream_t st) {
  typedef DualTile<F, E> T;
  static std::once_flag once;
  std::call_once(once, [] {
    (void)hipFuncSetAttribute((const void*)gemm_dual_fwd<T, ACT>,
                              hipFuncAttributeMaxDynamicSharedMemorySize, (int)T::LDS_BYTES);
  });
  gemm_dual_fwd<T, ACT><<<(unsigned)(g.mt * g.nt * g.splits), T::THREADS, T::LDS_BYTES, st>>>(g);
}
template <int ACT, class E>
static void fwd_launch_f(int f, const DualArgs& g, hipStream_t st) {
  if (sizeof(E) == 2 && f == 4) fwd_launch<sizeof(E) == 2 ? 4 : 2, ACT, E>(g, st);
  else fwd_launch<2, ACT, E>(g, st);
}

static DualArgs dual_planned(DualArgs g, const DualPlan& p, float* part) {
  g.mt = p.mt; g.nt = p.nt; g.splits = p.splits; g.stages = p.stages;
  g.part = part;
  g.pitch = cdiv(g.N, 4) * 4;
  return g;
}

template <class E>
static void split_sum_fwd(const DualArgs& g, int act, hipStream_t st) {
  if (g.splits < 8) gated_split_sum<E, 1><<<split_sum_blocks(g, 1), 256, 0, st>>>(g, act);
  else gated_split_sum<E, 4><<<split_sum_blocks(g, 4), 256, 0, st>>>(g, act);
}

// The forward under its plan: unsplit it ends in its outputs, split in the workspace,
// from where gated_split_sum takes it (whichever activation the product was built for).
template <class E>
static void fwd_run(DualArgs g, const DualPlan& p, int act, float* part, hipStream_t st) {
  g = dual_planned(g, p, part);
  switch (p.splits > 1 ? SB_ACT_RELU : act) {
    case SB_ACT_SIGMOID: fwd_launch_f<SB_ACT_SIGMOID, E>(p.f, g, st); break;
    case SB_ACT_SILU: fwd_launch_f<SB_ACT_SILU, E>(p.f, g, st); break;
    case SB_ACT_GELU: fwd_launch_f<SB_ACT_GELU, E>(p.f, g, st); break;
    case SB_ACT_GELU_TANH: fwd_launch_f<SB_ACT_GELU_TANH, E>(p.f, g, st); break;
    default: fwd_launch_f<SB_ACT_RELU, E>(p.f, g, st);
  }
  if (p.splits > 1) split_sum_fwd<E>(g, act, st);
}

template <int F, class E>
static void grads_launch(const DualArgs& dx, const DualArgs& dw, const BiasSums& bias, hipStream_t st) {
  typedef DualTile<F, E> T;
  static std::once_flag once;
  std::call_once(once, [] {
    (void)hipFuncSetAttribute((const void*)gemm_dual_grads<T>,
                              hipFuncAttributeMaxDynamicSharedMemorySize, (int)T::LDS_BYTES);
  });
  const int first = dx.mt * dx.nt * dx.splits;
  const int last = first + dw.mt * dw.nt * dw.splits, sums = bias.sums ? cdiv(bias.n, 64) : 0;
  gemm_dual_grads<T><<<(unsigned)(last + sums), T::THREADS, T::LDS_BYTES, st>>>(dx, dw, first, bias);
}
// dx (not with an empty plan) and the weight gradients, and the bias gradients where there
// are sums of them to join.  part: dx's partials, then the others'.
template <class E>
static void grads_run(DualArgs dx, DualArgs dw, const BiasSums& bias, const GradPlan& p, char* part,
                      hipStream_t st) {
  dx = dual_planned(dx, p.dx, (float*)part);
  dw = dual_planned(dw, p.dw, (float*)(part + round_up(p.dx.ws_bytes, 256)));
  if (sizeof(E) == 2 && p.dw.f == 4) grads_launch<sizeof(E) == 2 ? 4 : 2, E>(dx, dw, bias, st);
  else grads_launch<2, E>(dx, dw, bias, st);
  const int w = std::max(dx.splits, dw.splits) < 8 ? 1 : 4;
  const int first = split_sum_blocks(dx, w), all = first + split_sum_blocks(dw, w);
  if (all == 0) return;
  if (w == 1) gated_split_sums<E, 1><<<all, 256, 0, st>>>(dx, dw, first);
  else gated_split_sums<E, 4><<<all, 256, 0, st>>>(dx, dw, first);
}

static int up8(int n) { return (n + 7) / 8 * 8; }
static bool at16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Whether the kernels for few rows take a call: lines and rows of a piece at least.
static bool few_rows(const sb_gated_desc* d) {
  return d->m <= kFewRows && d->n_shard >= 8 && d->k_in >= 8;
}

// Lanes a line and splits of their forward: the least estimated time (us).  Without
// splits: the start, M rows' ends, a block's rounds of J lines for each of its groups of
// lanes, M times as much work in them, and the weights' MB; splits cost a launch and the
// partials.  Fitted to 3800 timings of 360 shapes of 64 to 8192 (1 to 8 rows, both
// types); the plan taken is 3 (bf16) or 2 % (fp32) slower than the best on average.
struct FewPlan { int lanes, strips, splits, lines; size_t ws_bytes; };
static FewPlan few_plan(const sb_gated_desc* d) {
  static const double kCost[2][3][6] = {
      // start, of it a row, round, of it a row, MB, MB of partials
      {{1.95, 0.15, 0.37, 0.085, 0.251, 0}, {2.01, 0.205, 0.49, 0.049, 0.100, 0},
       {5.76, 0.091, 0.068, 0.12, 0.132, 1.17}},                      // fp32: 4 lanes, 8, 8 split
      {{1.46, 0.33, 1.35, 0.194, 0.240, 0}, {1.94, 0.34, 1.14, 0.188, 0.094, 0},
       {5.87, 0.16, 0.27, 0.344, 0.137, 1.29}}};                      // bf16
  const bool b16 = d->dtype == SB_BF16;
  const int es = b16 ? 2 : 4, v = 16 / es, M = d->m <= 2 ? d->m : d->m <= 4 ? 4 : 8;
  const int J = b16 && M == 8 ? 4 : v;                                // kFewLines
  const double mb = 2e-6 * d->k_in * d->n_shard * es;
  FewPlan best{};
  double best_t = 0;
  for (int lanes = 4; lanes <= 8; lanes *= 2) {
    for (int s = 1; s <= (lanes == 8 ? 32 : 1) && (s == 1 || d->k_in / s >= 16); s *= 2) {
      const double* c = kCost[b16][s > 1 ? 2 : lanes / 8];
      const int strips = cdiv(cdiv(d->n_shard, v), lanes), lines = cdiv(cdiv(d->k_in, s), J) * J;
      const int splits = cdiv(d->k_in, lines), group = 512 / lanes * J;
      const double rounds = cdiv(lines, group) * (double)J / v * std::max(1.0, strips * (double)splits / 256);
      const size_t part = splits > 1 ? (size_t)splits * 8 * d->m * cdiv(d->n_shard, 4) * 4 : 0;
      const double t = c[0] + c[1] * M + rounds * (c[2] + c[3] * M) + c[4] * mb + c[5] * 1e-6 * part;
      if (best_t == 0 || t < best_t) {
        best_t = t;
        best = FewPlan{lanes, strips, splits, lines, part};
      }
    }
  }
  return best;
}

// Which operands have to be laid out anew for 16-byte pieces of whole eights: x as
// rows of the forward's reduction, x as lines of the weight gradient's, the weights.
struct GatedPacks { bool x, lines, w; };
static GatedPacks gated_packs(const sb_gated_desc* d, bool x_at16, bool w_at16) {
  const bool b16 = d->dtype == SB_BF16, few = few_rows(d);
  // (An odd bf16 k_in would end the last line inside the 4 bytes that ranges count in.)
  const bool lines = d->ldx % (b16 ? 8 : 4) != 0 || (b16 && d->k_in % 2 != 0) || !x_at16;
  return GatedPacks{!few && (lines || d->k_in % 8 != 0), !few && lines,
                    !few && (d->n_shard % 8 != 0 || !w_at16)};
}

static DualPlan gated_plan_fwd(const sb_gated_desc* d) {
  return dual_plan(kDualFwd, d->dtype == SB_BF16, d->m, d->n_shard, d->k_in, 1);
}
static DualPlan gated_plan_dw(const sb_gated_desc* d) {   // without dx beside it
  const bool b16 = d->dtype == SB_BF16;
  return dual_plan(kDualDw, b16, d->k_in, d->n_shard, d->m, b16 ? 3 : 1);
}
static GradPlan gated_plan_grads(const sb_gated_desc* d) {
  return grad_plan(d->dtype == SB_BF16, d->m, d->k_in, up8(d->n_shard));
}

// A workspace's parts, each from a multiple of 256 bytes on (offsets).
struct GatedSpace { size_t d, sums, x, w, split, bytes; };

static GatedSpace gated_space(const sb_gated_desc* d, int pass, const GatedPacks& k) {
  const size_t m = d->m, np = up8(d->n_shard), es = sbh::dsize(d->dtype);
  const bool few = few_rows(d);
  GatedSpace s{};
  if (few && pass == SB_FC_BWD && d->m <= kFewGates) return s;
  size_t at = 0;
  auto take = [&](size_t& part, size_t bytes) {
    part = at;
    at += round_up(bytes, 256);
  };
  if (pass == SB_FC_BWD) {
    take(s.d, m * np * (d->dtype == SB_BF16 && !few ? 12 : 8));
    if (few) {
      s.bytes = at;
      return s;
    }
    take(s.sums, (size_t)cdiv(d->m, act_rows(d->m, (int)np)) * np * 8);
  }
  if (pass == SB_FC_FWD ? k.x : k.lines) take(s.x, m * up8(d->k_in) * es);
  if (k.w) take(s.w, 2 * (size_t)d->k_in * np * es);
  size_t split = 0;
  if (pass == SB_FC_FWD) {
    split = few ? few_plan(d).ws_bytes : gated_plan_fwd(d).ws_bytes;
  } else {
    const GradPlan p = gated_plan_grads(d);
    split = std::max(gated_plan_dw(d).ws_bytes, round_up(p.dx.ws_bytes, 256) + p.dw.ws_bytes);
  }
  take(s.split, split);
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

// The operands as the products take them, and what has to be laid out anew for that.
struct GatedOperands {
  const void *x, *w[2];
  int ldx, width, ldw;                               // width: of x's rows
  PackTasks packs;
};
template <class E>
static GatedOperands gated_operands(const sb_gated_desc* d, const void* x, const void* const* w,
                                    bool pack_x, bool pack_w, char* ws, const GatedSpace& sp) {
  GatedOperands o{x, {w[0], w[1]}, d->ldx, d->k_in, d->n_shard, {}};
  PackTasks& t = o.packs;
  auto add = [&](const void* from, void* to, int rows, int cols, int ld, int cp) {
    const int q = t.count++;
    t.from[q] = from; t.to[q] = to;
    t.rows[q] = rows; t.cols[q] = cols; t.ld[q] = ld; t.cp[q] = cp;
    const int blocks = (int)std::min<size_t>(((size_t)rows * cp / 4 + 255) / 256, 4096);
    for (int i = q + 1; i < 4; ++i) t.block0[i] = t.block0[q] + blocks;
  };
  if (pack_x) {
    o.x = ws + sp.x;
    o.ldx = o.width = up8(d->k_in);
    add(x, ws + sp.x, d->m, d->k_in, d->ldx, o.width);
  }
  if (pack_w) {
    o.ldw = up8(d->n_shard);
    for (int q = 0; q < 2; ++q) {
      E* to = (E*)(ws + sp.w) + q * (size_t)d->k_in * o.ldw;
      o.w[q] = to;
      add(w[q], to, d->k_in, d->n_shard, d->n_shard, o.ldw);
    }
  }
  return o;
}

template <class E, int M>
static void few_fwd(FewArgs g, int lanes, hipStream_t st) {
  const int blocks = g.strips * g.splits;
  if (lanes == 8) gated_few_fwd<E, M, 8><<<blocks, 512, 0, st>>>(g);
  else gated_few_fwd<E, M, 4><<<blocks, 512, 0, st>>>(g);
  if (g.splits == 1) return;
  DualArgs d{};
  d.M = g.m; d.N = g.n; d.pitch = g.pitch; d.splits = g.splits; d.part = g.part;
  d.bias[0] = g.bias[0]; d.bias[1] = g.bias[1];
  d.pre = g.pre; d.c[0] = g.y; d.ldc = g.ldy;
  split_sum_fwd<E>(d, g.act, st);
}

template <class E>
static void gated_fwd_run(const sb_gated_desc* d, const void* x, const void* const* w,
                          const float* const* b, void* y, float* pre, const GatedPacks& packs,
                          char* ws, const GatedSpace& sp, hipStream_t st) {
  if (few_rows(d)) {
    const FewPlan p = few_plan(d);
    FewArgs g{x, {w[0], w[1]}, {b[0], b[1]}, y, pre, (float*)(ws + sp.split), d->m, d->n_shard,
              d->k_in, d->ldx, d->ldy, cdiv(d->n_shard, 4) * 4, d->act, p.strips, p.splits, p.lines};
    if (d->m == 1) few_fwd<E, 1>(g, p.lanes, st);
    else if (d->m == 2) few_fwd<E, 2>(g, p.lanes, st);
    else if (d->m <= 4) few_fwd<E, 4>(g, p.lanes, st);
    else few_fwd<E, 8>(g, p.lanes, st);
    return;
  }
  const GatedOperands o = gated_operands<E>(d, x, w, packs.x, packs.w, ws, sp);
  if (o.packs.count) gated_pack<E><<<o.packs.block0[3], 256, 0, st>>>(o.packs);
  DualArgs g{};
  g.a[0] = o.x; g.lda = o.ldx;
  g.b[0][0] = o.w[0]; g.b[1][0] = o.w[1]; g.ldb = o.ldw;
  g.M = d->m; g.N = d->n_shard; g.K = o.width; g.segs = 1;
  g.a_bytes = (uint32_t)(((size_t)(d->m - 1) * g.lda + g.K) * sizeof(E));
  g.b_bytes = (uint32_t)((size_t)d->k_in * g.ldb * sizeof(E));
  g.c[0] = y; g.ldc = d->ldy;
  g.bias[0] = b[0]; g.bias[1] = b[1];
  g.pre = pre;
  fwd_run<E>(g, gated_plan_fwd(d), d->act, (float*)(ws + sp.split), st);
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
  const bool few = few_rows(d), pass = !few || (dx && d->m > kFewGates);
  const BiasSums bias{!few && (db[0] || db[1]) && chunks > 1 ? (float*)(ws + sp.sums) : nullptr,
                      {few ? nullptr : db[0], few ? nullptr : db[1]}, d->n_shard, np, chunks, accumulate};
  const GatedOperands o = gated_operands<E>(d, x, w, packs.lines, dx && packs.w, ws, sp);
  if (pass) {
    const unsigned blocks = (unsigned)(cdiv(np, 256) * chunks + o.packs.block0[3]);
    if (few)
      gated_act_bwd<E, float><<<blocks, 256, 0, st>>>(d->m, d->n_shard, np, d->act, pre, (const E*)dy,
                                                      d->ldy, (float*)parts, bias, rows, chunks, o.packs);
    else
      gated_act_bwd<E, E><<<blocks, 256, 0, st>>>(d->m, d->n_shard, np, d->act, pre, (const E*)dy,
                                                  d->ldy, parts, bias, rows, chunks, o.packs);
  }
  if (few) {
    const int strips = cdiv(d->n_shard, 256);
    int lines = 32;                                  // about 512 blocks and more
    while (lines < d->k_in && strips * (int64_t)cdiv(d->k_in, 2 * lines) >= 512) lines *= 2;
    const FewBwdArgs g{x, {w[0], w[1]}, dy, pre, dx, {dw[0], dw[1]}, {db[0], db[1]}, d->m,
                       d->n_shard, d->k_in, d->ldx, d->ldy, d->act, accumulate,
                       dx ? cdiv(d->k_in, kFewDx) : 0, strips, lines,
                       {(const float*)parts, (const float*)parts + plane}, np};
    const int blocks = g.first + strips * cdiv(d->k_in, lines);
    const auto kernel = d->m == 1 ? gated_few_bwd<E, 1> : d->m == 2 ? gated_few_bwd<E, 2>
                        : d->m <= 4 ? gated_few_bwd<E, 4> : gated_few_bwd<E, 8>;
    kernel<<<blocks, 256, 0, st>>>(g);
    return;
  }
  DualArgs gw{};
  for (int p = 0; p < NP; ++p) {                     // the smallest parts first
    gw.a[p] = o.x;
    for (int q = 0; q < 2; ++q) gw.b[q][p] = parts + (NP * q + NP - 1 - p) * plane;
  }
  gw.lda = o.ldx; gw.ldb = np;
  gw.M = d->k_in; gw.N = d->n_shard; gw.K = d->m; gw.segs = NP; gw.firsts = 1;
  gw.a_bytes = (uint32_t)(((size_t)(d->m - 1) * gw.lda + o.width) * sizeof(E));
  gw.b_bytes = (uint32_t)(plane * sizeof(E));
  gw.c[0] = dw[0]; gw.c[1] = dw[1]; gw.ldc = d->n_shard;
  gw.accumulate = accumulate;
  if (dx) {
    DualArgs gx{};
    constexpr int XP = sizeof(E) == 2 ? 2 : 1;       // parts, the second ones first
    for (int i = 0; i < 2 * XP; ++i) {
      const int q = i % 2, p = XP - 1 - i / 2;
      gx.a[i] = parts + (NP * q + p) * plane;
      gx.b[0][i] = gx.b[1][i] = o.w[q];
    }
    gx.lda = np; gx.ldb = o.ldw;                     // o.ldw is np: n_shard, or packed
    gx.M = d->m; gx.N = d->k_in; gx.K = np; gx.segs = 2 * XP; gx.firsts = 2;
    gx.a_bytes = (uint32_t)(plane * sizeof(E));
    gx.b_bytes = (uint32_t)((size_t)d->k_in * np * sizeof(E));
    gx.c[0] = dx; gx.ldc = d->ldx;
    grads_run<E>(gx, gw, bias, gated_plan_grads(d), ws + sp.split, st);
    return;
  }
  grads_run<E>(DualArgs{}, gw, bias, GradPlan{{}, gated_plan_dw(d)}, ws + sp.split, st);
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
  if (sp.bytes > 0 && (!ws || ws_bytes < sp.bytes)) return SB_ERR_WORKSPACE;
  if (sp.bytes > 0 && !at16(ws)) return SB_ERR_INVALID_ARG;
  const void* w[2] = {w_gate, w_up};
  float* dw[2] = {dw_gate, dw_up};
  float* db[2] = {db_gate, db_up};
  const auto run = d->dtype == SB_BF16 ? gated_bwd_run<u16> : gated_bwd_run<float>;
  run(d, x, w, pre, dy, dx, dw, db, accumulate, packs, (char*)ws, sp, sbh::stream_of(stream));
  return sbh::launch_status();
}
