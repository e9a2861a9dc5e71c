// gemm_dual.hpp -- products of the gated FC shard (gated.hip) on the 32x32x16 bf16
// MFMA, two weight matrices (or their gradients) at a time; fp32 operands as three
// bf16 parts each, six products of them (split_bf16.hpp).
//
//   FWD   gate and up = x * Wg, x * Wu          x [m][k], W [k][n]
//   DX    sum over q of d_q * W_q^T             d_q [m][n], W_q [kin][n]
//   DW    x^T * da and x^T * du                 x [m][kin], d [m][n]
//
// A block has 64 F rows (M) by 64 F columns: of FWD and DW 32 F columns of each
// of the two outputs (N), so the operand they share is staged once and the gate's
// value and the other projection's for one output element end in one wave.  Four
// waves, 2 x 2, or eight, 4 x 2, each with FA x F blocks of 32 x 32 in registers.
// The reduction is a list of segments of equal length (DX: one per weight matrix and bf16
// part of its d; DW: one per bf16 part of da and du), each in stages of 32.
//
// Three stages are in LDS: while stage t is multiplied, t + 2 is written from
// registers and t + 4 loaded, and t + 1 can already be read, so that the operands
// of the next 16 k are in registers before the current ones are used up.  An
// operand that is contiguous along k (x of FWD, both of DX) lies in LDS as rows
// of four 16-byte pieces and is read as such; one that is contiguous along its
// rows keeps its layout, and the transposing LDS read (ds_read_b64_tr_b16) gives a
// lane its column's four k.  Pieces are permuted so that neither the writes nor
// the reads meet in a bank: piece p of row r at p ^ r / 4 % 4, a column
// block of 16 of line k at block ^ k % 4.
//
// The weight (or d) is the MFMA's first operand, so a lane has four consecutive
// output columns of a row in four registers and stores them at once.
#pragma once

#include "gate.hpp"
#include "split_bf16.hpp"

namespace sb {

typedef short s4v __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));

enum DualKind { kDualFwd, kDualDx, kDualDw };

// E: float (three bf16 parts, F = 2) or bf16 bits.
template <int F_, class E_>
struct DualTile {
  typedef E_ E;
  static constexpr int F = F_, NP = sizeof(E) == 4 ? 3 : 1;
  // Waves by rows and columns, a wave's blocks of rows (of columns F), its threads'
  // pieces of an operand's stage.  Eight waves where two of them leave a SIMD room:
  // one wave issues an instruction every five or six cycles, and what an MFMA has
  // beside it (fp32: the splitting; bf16: reads, writes and their waits) is about as
  // many as fit then.  fp32, 512 x 1024 outputs of 4096 k: 62 -> 55 us; bf16 256-row
  // tiles: 8192 x 8192 of 4096 k 1123 -> 1085 us, 2048 x 2048 of 2048 k 61 -> 55 us.
  // Tiles of 128 rows in bf16, two or three blocks a CU, keep four: LDS bounds them,
  // and eight would read a half more.
  static constexpr int WM = NP == 3 || F == 4 ? 4 : 2, WN = 2, THREADS = 64 * WM * WN;
  static constexpr int FA = 2 * F / WM, PCS = 256 * F / THREADS;
  static constexpr int BM = 64 * F, RC = 32 * F;     // rows; columns of a region
  static constexpr int PART = BM * 32, OPER = NP * PART;   // elements of an operand's stage
  static constexpr int STAGE = 2 * OPER;
  static constexpr int PITCH = 32 * F + 4;           // floats a row of the output on its way
  static constexpr size_t LDS_OUT = (size_t)THREADS / 64 * 32 * PITCH * sizeof(float);
  static constexpr size_t LDS_IN = 3 * (size_t)STAGE * sizeof(u16);
  static constexpr size_t LDS_STAGES = LDS_IN > LDS_OUT ? LDS_IN : LDS_OUT;
  static constexpr size_t LDS_BYTES = LDS_STAGES + (NP == 3 ? 16 : 0);   // the redo flag
  static_assert(LDS_BYTES <= 160 * 1024, "one block per CU");
};

struct DualArgs {
  const void* a[4];                // per segment
  const void* b[2][4];             // per region (DX: region 0) and segment
  uint32_t a_bytes, b_bytes;       // ranges of the operands
  int lda, ldb;
  int M, N, K, segs;               // K: of a segment
  int firsts;                      // bf16 DX, DW: the last segments, which have the first parts
  int mt, nt, splits, stages;      // stages per split
  int pitch;                       // of partials' rows: N rounded up to 4
  float* part;                     // splits > 1: [split][2][M][N up to 4] (DX [split][M][..])
  void* c[2]; int ldc;             // DX: dx; DW: fp32 gradients; FWD: y in c[0]
  const float* bias[2];            // FWD
  float* pre;                      // FWD, may be null: [2][M][N]
  int accumulate;
};

__device__ __forceinline__ f16v mfma32(s8 a, s8 b, f16v c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ u32x4 load16(rsrc_t r, uint32_t off) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, 0));
}

// Eight elements on their way to LDS.
template <class E> struct DualPiece;
template <> struct DualPiece<u16> {
  u32x4 v;
  __device__ __forceinline__ void load(rsrc_t r, uint32_t off) { v = load16(r, off); }
  __device__ __forceinline__ void store(u16* to, int, uint32_t&) const {
    *reinterpret_cast<u32x4*>(to) = v;
  }
};
template <> struct DualPiece<float> {
  u32x4 v[2];
  __device__ __forceinline__ void load(rsrc_t r, uint32_t off) {
    v[0] = load16(r, off);
    v[1] = load16(r, off + 16);
  }
  // The three parts, `part` elements apart; lost as in split_pair.
  __device__ __forceinline__ void store(u16* to, int part, uint32_t& lost) const {
    f8v f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(v[e / 4][e % 4]);
    const Split8 t = split8(f, lost);
#pragma unroll
    for (int p = 0; p < 3; ++p) *reinterpret_cast<s8*>(to + p * part) = t.p[p];
  }
};

// A staged operand: KC contiguous along k, otherwise two regions of RC columns.
template <class T, bool KC>
struct DualStage {
  typedef typename T::E E;
  uint32_t off[T::PCS];            // byte offset of this lane's pieces at k = 0, or kOOB
  int lds[T::PCS];                 // their place (elements)
  uint32_t step;                   // bytes per k
  int k;                           // KC: the first k of all of them within a stage
  // Rows (KC) or columns from r0 on, `rows` of them; region 1 starts at r1.
  __device__ __forceinline__ void init(int tid, int ld, int rows, int r0, int r1) {
    step = (KC ? 1u : (uint32_t)ld) * (uint32_t)sizeof(E);
    k = KC ? tid % 4 * 8 : 0;
#pragma unroll
    for (int i = 0; i < T::PCS; ++i) {
      const int u = tid + T::THREADS * i;
      if constexpr (KC) {
        const int row = u / 4, p = u % 4;
        lds[i] = row * 32 + (p ^ (row >> 2 & 3)) * 8;
        off[i] = r0 + row < rows ? (uint32_t)((r0 + row) * ld + p * 8) * (uint32_t)sizeof(E) : kOOB;
      } else {
        constexpr int PR = T::RC / 8;                // pieces a line
        const int region = u / (128 * T::F), w = u % (128 * T::F), line = w / PR, p = w % PR;
        const int col = (region ? r1 : r0) + p * 8;
        lds[i] = region * (T::RC * 32) + line * T::RC + ((p / 2 ^ (line & 3)) * 2 + p % 2) * 8;
        off[i] = col < rows ? (uint32_t)(line * ld + col) * (uint32_t)sizeof(E) : kOOB;
      }
    }
  }
  // The region of a wave's piece i.
  __device__ static __forceinline__ int region(int wave, int i) {
    return (64 * wave + T::THREADS * i) / (128 * T::F);
  }
  // Piece i of the stage from k0 on (k0 < K); r: its region's resource.  Lines at
  // and past K lie behind the operand and read 0 by its range, as kOOB does at
  // any k; a row's pieces past K are left out here.
  __device__ __forceinline__ void load_one(rsrc_t r, int k0, int K, DualPiece<E> (&v)[T::PCS],
                                           int i) const {
    uint32_t o = off[i] + (uint32_t)k0 * step;
    if constexpr (KC) o = k0 + k < K ? o : kOOB;
    v[i].load(r, o);
  }
  __device__ __forceinline__ void store_one(u16* S, const DualPiece<E> (&v)[T::PCS], int i,
                                            uint32_t& lost) const {
    v[i].store(S + lds[i], T::PART, lost);
  }
};

// The two blocks of 16 columns of a region that fragment q (0 .. F - 1) takes.
template <int F>
__device__ __forceinline__ int pair_block(int q, int half) {
  return F == 4 ? q + 4 * half : 2 * q + half;
}

// Fragment of 32 rows (or columns) by 16 k.  place: this lane's first element
// for k = 0 of the stage (frag_place); step s of the stage.
template <class T, bool KC>
__device__ __forceinline__ int frag_place(int q, int lane, int row0) {
  if constexpr (KC) {
    const int row = row0 + q * 32 + lane % 32;
    return row * 32 + (((lane / 32) ^ (row >> 2 & 3)) * 8);
  } else {
    const int g = lane / 16, i = lane % 16;
    const int line = 8 * (g >> 1) + i / 4, block = pair_block<T::F>(q, g & 1);
    return line * T::RC + (block ^ (line & 3)) * 16 + (i % 4) * 4;
  }
}
template <class T, bool KC>
__device__ __forceinline__ s8 frag_read(const u16* S, int place, int s) {
  if constexpr (KC) {
    return *reinterpret_cast<const s8*>(S + (place ^ (s * 16)));    // piece + 2 of 4
  } else {
    typedef __attribute__((address_space(3))) s4v* lds4;
    const u16* p = S + place + s * 16 * T::RC;
    const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p));
    const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p + 4 * T::RC));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
}

// Four columns n .. n + 3 of a row, those below N.
template <class E>
__device__ __forceinline__ void put_quad(E* row, f4 v, int n, int N) {
  if (n + 4 <= N && ((uintptr_t)(row + n) & (4 * sizeof(E) - 1)) == 0) {
    Elem<E>::store4(row + n, v);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < N) Elem<E>::store(row, n + e, v[e]);
  }
}
__device__ __forceinline__ f4 get_quad(const float* row, int n, int N) {
  if (n + 4 <= N && ((uintptr_t)(row + n) & 15) == 0) return *reinterpret_cast<const f4*>(row + n);
  f4 v = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (n + e < N) v[e] = row[n + e];
  return v;
}

// ACT: FWD's activation (its code is unrolled over all the outputs of a lane).
// Block `block` of a product.
template <class T, DualKind KIND, int ACT>
__device__ __forceinline__ void dual_block(const DualArgs& g, int block, u16* lds) {
  typedef typename T::E E;
  constexpr int F = T::F, NP = T::NP, FA = T::FA, PCS = T::PCS;
  constexpr bool AKC = KIND != kDualDw, BKC = KIND == kDualDx;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % T::WM, wn = wave / T::WM;

  // Blocks are dealt to the 8 XCDs in contiguous ranges of an order in which 8 row
  // tiles take turns under one column tile, so what an XCD runs at a time is a
  // patch of the output that shares rows and columns in its L2.
  const int tiles = g.mt * g.nt, nb = tiles * g.splits;
  int h = block;
  if (nb % 8 == 0) h = (h % 8) * (nb / 8) + h / 8;
  const int split = h / tiles;
  h -= split * tiles;
  const int group = h / (8 * g.nt), in = h - group * 8 * g.nt;
  const int gm = min(8, g.mt - group * 8);
  const int mtile = group * 8 + in % gm, ntile = in / gm;
  const int m0 = mtile * T::BM, n0 = ntile * (KIND == kDualDx ? T::BM : T::RC);

  const int per_seg = cdiv(g.K, 32);
  const int t0 = split * g.stages, t1 = min(t0 + g.stages, per_seg * g.segs);
  const int nk = t1 - t0;

  DualStage<T, AKC> sa;
  DualStage<T, BKC> sb;
  sa.init(tid, g.lda, g.M, m0, m0 + T::RC);
  sb.init(tid, g.ldb, g.N, n0, n0);
  // The next stage to load.
  int seg = t0 / per_seg, k0 = (t0 - seg * per_seg) * 32;
  DualPiece<E> va[2][PCS], vb[2][PCS];
  uint32_t lost = 0;
  // The operands of its segment; its first k.  Stages past the block's last one, which
  // nothing multiplies, are empty ranges: their loads return 0 and read nothing.
  rsrc_t ra, rb, rc;
  int left = nk;
  auto segment = [&]() {
    const int s = min(seg, g.segs - 1);
    const uint32_t bytes_a = left > 0 ? g.a_bytes : 0, bytes_b = left > 0 ? g.b_bytes : 0;
    ra = make_rsrc(g.a[s], bytes_a);
    rb = make_rsrc(g.b[0][s], bytes_b);
    rc = make_rsrc(g.b[1][s], bytes_b);
  };
  segment();
  int ka;
  auto next = [&]() {
    ka = k0;
    k0 += 32;
    --left;
    if (k0 >= g.K) {
      k0 = 0;
      ++seg;
    }
  };
  auto turn = [&]() {
    if (k0 == 0 || left == 0) segment();
  };
  auto load_a = [&](DualPiece<E> (&x)[PCS], int i) { sa.load_one(ra, ka, g.K, x, i); };
  auto load_b = [&](DualPiece<E> (&x)[PCS], int i) {
    sb.load_one(!BKC && sb.region(wave, i) ? rc : rb, ka, g.K, x, i);
  };
  auto load = [&](DualPiece<E> (&xa)[PCS], DualPiece<E> (&xb)[PCS]) {
    next();
#pragma unroll
    for (int i = 0; i < PCS; ++i) {
      load_a(xa, i);
      load_b(xb, i);
    }
    turn();
  };
  auto store = [&](u16* S, const DualPiece<E> (&xa)[PCS], const DualPiece<E> (&xb)[PCS]) {
#pragma unroll
    for (int i = 0; i < PCS; ++i) {
      sa.store_one(S, xa, i, lost);
      sb.store_one(S + T::OPER, xb, i, lost);
    }
  };

  // Row block i of the wave: block gf + i of the tile's, F of them a region.
  const int gf = wm * FA;
  int pa[FA], pb[F];
#pragma unroll
  for (int i = 0; i < FA; ++i)
    pa[i] = AKC ? frag_place<T, true>(gf + i, lane, 0)
                : frag_place<T, false>((gf + i) % F, lane, 0) + (gf + i) / F * T::RC * 32;
#pragma unroll
  for (int i = 0; i < F; ++i) {
    if constexpr (BKC) pb[i] = T::OPER + frag_place<T, true>(i, lane, wn * T::RC);
    else pb[i] = T::OPER + (i / (F / 2)) * T::RC * 32 +
                 frag_place<T, false>(wn * (F / 2) + i % (F / 2), lane, 0);
  }
  // Output row of row c (0 .. 31) of the wave's block i.
  auto out_row = [&](int i, int c) {
    const int f = gf + i;
    return m0 + (AKC ? f * 32 + c : f / F * T::RC + pair_block<F>(f % F, c / 16) * 16 + c % 16);
  };
  // [column block][row block]; low: the sums of the five smaller products of the
  // parts, which are below 2^-8 of the sums they are added to at the end, so their
  // roundings do not count.  Sums stay here over the whole reduction: to empty them every
  // 128 k, as gemm_split does, takes as many registers again, which 256-row tiles do not
  // have.  What the 32x32x16 MFMA drops always downwards is less than its last bit: 8192
  // terms of one sign came out 3.6e-8 low on average and 4.3e-7 off (rms), 16384 terms
  // 9.4e-8 and 6.2e-7, in both types; terms of either sign -3e-9 and 5.4e-7, -4e-9 and
  // 7.8e-7 of the sums' size.
  f16v acc[F][FA], low[NP == 3 ? F : 1][NP == 3 ? FA : 1];
  auto clear = [](f16v& x) {
#pragma unroll
    for (int v = 0; v < 16; ++v) x[v] = 0.f;
  };
#pragma unroll
  for (int j = 0; j < F; ++j)
#pragma unroll
    for (int i = 0; i < FA; ++i) {
      clear(acc[j][i]);
      if constexpr (NP == 3) clear(low[j][i]);
    }

  load(va[0], vb[0]);
  load(va[1], vb[1]);
  store(lds, va[0], vb[0]);
  store(lds + T::STAGE, va[1], vb[1]);
  load(va[0], vb[0]);
  load(va[1], vb[1]);
  __syncthreads();

  s8 fa[2][FA][NP], fb[2][F][NP];
  auto read_a = [&](int c, const u16* S, int i, int p, int s) {
    fa[c][i][p] = frag_read<T, AKC>(S + p * T::PART, pa[i], s);
  };
  auto read_b = [&](int c, const u16* S, int j, int p, int s) {
    fb[c][j][p] = frag_read<T, BKC>(S + p * T::PART, pb[j], s);
  };
#pragma unroll
  for (int p = 0; p < NP; ++p) {
#pragma unroll
    for (int i = 0; i < FA; ++i) read_a(0, lds, i, p, 0);
#pragma unroll
    for (int j = 0; j < F; ++j) read_b(0, lds, j, p, 0);
  }
  // 16 k out of fragment set P: the MFMAs, and between them the reads of the next 16 k
  // from S (one fragment behind each of the first MFMAs, in the order of their use),
  // and, behind the others, pieces of the stage after the next one to LDS and the loads
  // that take their registers' place.
  auto step = [&](auto P, auto H, auto W, const u16* S, int s, u16* to) {
    constexpr int c = decltype(P)::value, half = decltype(H)::value, r = decltype(W)::value;
    if constexpr (NP == 1) {
#pragma unroll
      for (int n = 0; n < F * FA; ++n) {
        const int j = n / FA, i = n % FA;
        acc[j][i] = mfma32(fb[c][j][0], fa[c][i][0], acc[j][i]);
        if (n == 0) read_b(c ^ 1, S, 0, 0, s);
        else if (n <= FA) read_a(c ^ 1, S, n - 1, 0, s);
        else if (n < FA + F) read_b(c ^ 1, S, n - FA, 0, s);
        if (half == 0) {
          const int x = n - (F * FA - 2 * PCS);
          if (x >= 0 && x < PCS) {
            sa.store_one(to, va[r], x, lost);
            load_a(va[r], x);
          } else if (x >= PCS && x < 2 * PCS) {
            sb.store_one(to + T::OPER, vb[r], x - PCS, lost);
            load_b(vb[r], x - PCS);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      // Six products of two blocks; A's piece in a stage's first half, B's in its second.
      // An MFMA takes the time of eight instructions: behind each of the first nine a
      // fragment is read, behind each of the first eight half a pair of values is split
      // (six instructions), behind the others the piece is written, then loaded.  (Left
      // to the compiler the splitting came first, the MFMAs after it: 490 us for 2048 x
      // 4096 x 2048, 447 like this.)
      static_assert(NP == 1 || (F == 2 && FA == 1 && PCS == 1), "one piece of each operand");
      u32x4 t[3];                                    // the piece's parts
      float ra = 0.f, rb = 0.f;
      const DualPiece<E>& v = half == 0 ? va[r][0] : vb[r][0];
#pragma unroll
      for (int n = 0; n < 12; ++n) {
        const int q = n / 2, j = n % 2;
        f16v& sum = q == 5 ? acc[j][0] : low[j][0];
        sum = mfma32(fb[c][j][kSplitB[q]], fa[c][0][kSplitA[q]], sum);
        if (n < 9) {                                 // A 2, B 0, A 1, B 1, A 0, B 2
          if (n % 3 == 0) read_a(c ^ 1, S, 0, 2 - n / 3, s);
          else read_b(c ^ 1, S, n % 3 - 1, n / 3, s);
        }
        if (n < 8) {
          const int e = n / 2;
          if (n % 2 == 0) {
            ra = __uint_as_float(v.v[e / 2][e % 2 * 2]);
            rb = __uint_as_float(v.v[e / 2][e % 2 * 2 + 1]);
            t[0][e] = f32x2_to_bf16x2(ra, rb);
            ra -= __uint_as_float(t[0][e] << 16);
            rb -= __uint_as_float(t[0][e] & 0xffff0000u);
          } else {
            t[1][e] = f32x2_to_bf16x2(ra, rb);
            ra -= __uint_as_float(t[1][e] << 16);
            rb -= __uint_as_float(t[1][e] & 0xffff0000u);
            t[2][e] = f32x2_to_bf16x2(ra, rb);
            lost |= __float_as_uint(ra) | __float_as_uint(rb);
          }
        } else if (n < 11) {
          u16* at = half == 0 ? to + sa.lds[0] : to + T::OPER + sb.lds[0];
          *reinterpret_cast<u32x4*>(at + (n - 8) * T::PART) = t[n - 8];
        } else if (half == 0) {
          load_a(va[r], 0);
        } else {
          load_b(vb[r], 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  // A stage in buffer b0; b2 gets the stage after the next one.
  typedef std::integral_constant<int, 0> Zero;
  typedef std::integral_constant<int, 1> One;
  auto stage = [&](auto R, u16* b0, u16* b1, u16* b2) {
    next();
    step(Zero{}, Zero{}, R, b0, 1, b2);
    if (NP == 1) turn();
    step(One{}, One{}, R, b1, 0, b2);
    if (NP == 3) turn();
    __syncthreads();
  };
  u16 *b0 = lds, *b1 = lds + T::STAGE, *b2 = lds + 2 * T::STAGE;
  int t = 0;
  auto turns = [&](auto R) {                         // the stage whose set is R, if there is one
    if (t < nk) {
      stage(R, b0, b1, b2);
      u16* x = b0;
      b0 = b1;
      b1 = b2;
      b2 = x;
      ++t;
    }
  };
  while (t + 2 <= nk) {
    turns(Zero{});
    turns(One{});
  }
  turns(Zero{});

  // Whether the products are formed again on the fp32 MFMA, operands straight from memory:
  // those of an fp32 block with values that the parts do not carry, or with sums that are
  // not finite; those of a bf16 wave with infinities beside lower parts, which are 0 or of
  // either sign, so that their products would make a NaN of an infinite sum.  Only sums
  // that are not finite look for infinities: a NaN in dy puts the backward of 4096 x 4096 x
  // 8192 from 2.7 to 3.2 ms, nothing but NaN to 6.1; an infinity in x, found, to 27.
  constexpr bool PARTS = NP == 1 && KIND != kDualFwd;
  bool again = false;
  if constexpr (NP == 3 || PARTS) {
    float z = 0.f;                                   // stays 0 over finite values
#pragma unroll
    for (int j = 0; j < F; ++j)
#pragma unroll
      for (int i = 0; i < FA; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          if constexpr (NP == 3) acc[j][i][v] += low[j][i][v];
          z = fmaf(acc[j][i][v], 0.f, z);
        }
    if constexpr (NP == 3) {
      int* redo = reinterpret_cast<int*>(lds + T::LDS_STAGES / sizeof(u16));
      if (tid == 0) *redo = 0;
      __syncthreads();
      if ((lost & 0xffffu) || !(z == 0.f)) *redo = 1;
      __syncthreads();
      again = __builtin_amdgcn_readfirstlane(*redo);
    } else {
      again = __ballot(!(z == 0.f)) != 0;
    }
  }
  int ar[FA], bc[F];                                 // this lane's rows of A, columns of B
  if (__builtin_expect(again, 0)) {
    const int c = lane % 32;
#pragma unroll
    for (int i = 0; i < FA; ++i) ar[i] = out_row(i, c);
#pragma unroll
    for (int j = 0; j < F; ++j)
      bc[j] = n0 + (BKC ? wn * T::RC + j * 32 + c
                        : pair_block<F>(wn * (F / 2) + j % (F / 2), c / 16) * 16 + c % 16);
    if constexpr (PARTS) {
      bool found = false;                            // (DW's segments have the same x)
      for (int u = t0; u < (KIND == kDualDw ? min(t1, t0 + per_seg) : t1); ++u) {
        const int sg = u / per_seg, kb = (u - sg * per_seg) * 32, ke = min(g.K, kb + 32);
        if (sg >= g.segs - g.firsts) break;
        if constexpr (KIND == kDualDw) {
          const u16* A = (const u16*)g.a[sg];
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            const int k = kb + 2 * x + lane / 32;
#pragma unroll
            for (int i = 0; i < FA; ++i)
              found |= k < ke && ar[i] < g.M && (A[(size_t)k * g.lda + ar[i]] & 0x7fffu) == 0x7f80u;
          }
        } else {                                     // whole pieces: K is a multiple of 8
          const u16* B = (const u16*)g.b[0][sg];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int k = kb + 16 * x + lane / 32 * 8;
#pragma unroll
            for (int j = 0; j < F; ++j) {
              if (k >= ke || bc[j] >= g.N) continue;
              const u32x4 v = *reinterpret_cast<const u32x4*>(B + (size_t)bc[j] * g.ldb + k);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                found |= (v[e] & 0x7fffu) == 0x7f80u || (v[e] & 0x7fff0000u) == 0x7f800000u;
            }
          }
        }
      }
      again = __ballot(found) != 0;
    }
  }
  if (__builtin_expect(again, 0)) {
#pragma unroll
    for (int j = 0; j < F; ++j)
#pragma unroll
      for (int i = 0; i < FA; ++i) clear(acc[j][i]);
    for (int u = t0; u < t1; ++u) {
      const int sg = u / per_seg, kb = (u - sg * per_seg) * 32, ke = min(g.K, kb + 32);
      const E* A = (const E*)g.a[sg];
      // Beside a lower part, infinities and NaN of the other operand count as 0: the first
      // part, an infinite one too, has their terms' signs.
      const bool lower = PARTS && sg < g.segs - g.firsts;
      auto whole = [&](float v) {
        return lower && (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u ? 0.f : v;
      };
#pragma unroll 1
      for (int kk = kb; kk < ke; kk += 2) {
        const int k = kk + lane / 32;
        float av[FA];
#pragma unroll
        for (int i = 0; i < FA; ++i) {
          const size_t at = AKC ? (size_t)ar[i] * g.lda + k : (size_t)k * g.lda + ar[i];
          av[i] = k < ke && ar[i] < g.M ? Elem<E>::load(A, at) : 0.f;
          if constexpr (KIND == kDualDw) av[i] = whole(av[i]);
        }
#pragma unroll
        for (int j = 0; j < F; ++j) {
          // (The weights end at b_bytes, before K where FWD's rows of x are padded.)
          const E* B = (const E*)g.b[BKC ? 0 : j / (F / 2)][sg];
          const size_t at = BKC ? (size_t)bc[j] * g.ldb + k : (size_t)k * g.ldb + bc[j];
          float bv = k < ke && bc[j] < g.N && at < g.b_bytes / sizeof(E) ? Elem<E>::load(B, at) : 0.f;
          if constexpr (KIND == kDualDx) bv = whole(bv);
#pragma unroll
          for (int i = 0; i < FA; ++i)
            acc[j][i] = __builtin_amdgcn_mfma_f32_32x32x2f32(bv, av[i], acc[j][i], 0, 0, 0);
        }
      }
    }
  }

  // acc[j][i] element v: row lane % 32 of row block i, column 8 (v / 4) + 4 (lane / 32) +
  // v % 4 of column block j.  Stored from there an access would touch 64 lines, 16 bytes
  // each, and those of an epilogue with pre took 60 us a tile; so 32 rows at a time go
  // through the wave's own part of LDS (the last stage's reads are done), and out in
  // runs of 32 columns or more.
  constexpr int CW = KIND == kDualDx ? 32 * F : 16 * F;      // columns of an output
  constexpr int P = T::PITCH;
  float* W = reinterpret_cast<float*>(lds) + wave * 32 * P;
  auto rows_out = [&](auto I) {
    constexpr int i = decltype(I)::value;
    if constexpr (i < FA) {
#pragma unroll
      for (int j = 0; j < F; ++j)
#pragma unroll
        for (int v4 = 0; v4 < 4; ++v4) {
          f4 t;
#pragma unroll
          for (int e = 0; e < 4; ++e) t[e] = acc[j][i][v4 * 4 + e];
          *reinterpret_cast<f4*>(W + (lane % 32) * P + j * 32 + 8 * v4 + 4 * (lane / 32)) = t;
        }
    }
  };
  f4 bias[2] = {f4{0.f, 0.f, 0.f, 0.f}, f4{0.f, 0.f, 0.f, 0.f}};   // of a lane's columns
  if constexpr (KIND == kDualFwd) {
    const int o = lane % (CW / 4) * 4;
    const int n = n0 + (F == 4 ? wn * 32 + o / 32 * 64 + o % 32 : wn * 32 + o);
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (g.bias[q] && n + e < g.N) bias[q][e] = g.bias[q][n + e];
  }
  // One copy of the code that stores (the activations' is long); i is uniform.
#pragma unroll 1
  for (int i = 0; i < FA; ++i) {
    switch (i) {
      case 0: rows_out(Zero{}); break;
      case 1: rows_out(One{}); break;
      case 2: rows_out(std::integral_constant<int, 2>{}); break;
      default: rows_out(std::integral_constant<int, 3>{});
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int x = 0; x < CW / 8; ++x) {
      const int row = (x * 64 + lane) / (CW / 4), o = lane % (CW / 4) * 4;
      const int m = out_row(i, row);
      if constexpr (KIND == kDualDx) {
        const int n = n0 + wn * T::RC + o;
        const f4 v = *reinterpret_cast<const f4*>(W + row * P + o);
        if (m < g.M && n < g.N) {
          if (g.splits > 1) put_quad(g.part + ((size_t)split * g.M + m) * g.pitch, v, n, g.pitch);
          else put_quad((E*)g.c[0] + (size_t)m * g.ldc, v, n, g.N);
        }
      } else {
        // Output columns in order: F = 4 has its blocks' halves 64 columns apart.
        const int at = F == 4 ? o % 32 / 16 * 32 + o / 32 * 16 + o % 16 : o;
        const int n = n0 + (F == 4 ? wn * 32 + o / 32 * 64 + o % 32 : wn * 32 + o);
        f4 v[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) v[q] = *reinterpret_cast<const f4*>(W + row * P + q * CW + at);
        if (m < g.M && n < g.N) {
          if (KIND == kDualFwd && g.splits == 1) {
            gate_store<E>(ACT, v[0] + bias[0], v[1] + bias[1], n, g.N,
                          g.pre ? g.pre + (size_t)m * g.N : nullptr, (size_t)g.M * g.N,
                          (E*)g.c[0] + (size_t)m * g.ldc);
          } else if (g.splits > 1) {
#pragma unroll
            for (int q = 0; q < 2; ++q)
              put_quad(g.part + (((size_t)split * 2 + q) * g.M + m) * g.pitch, v[q], n, g.pitch);
          } else {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              float* c = (float*)g.c[q] + (size_t)m * g.ldc;
              if (g.accumulate) v[q] += get_quad(c, n, g.N);
              put_quad(c, v[q], n, g.N);
            }
          }
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

template <class T, int ACT>
__global__ __launch_bounds__(T::THREADS, 2) void gemm_dual_fwd(DualArgs g) {
  extern __shared__ u16 lds[];
  dual_block<T, kDualFwd, ACT>(g, blockIdx.x, lds);
}

// The bias gradients from `chunks` row blocks' sums ([chunk][2][np]): 64 columns of both
// a block, every second or fourth row block a wave (of four or eight).
struct BiasSums {
  float *sums, *db[2];                               // sums null: nothing to join
  int n, np, chunks, accumulate;
};
template <int THREADS>
__device__ __forceinline__ void bias_sum_block(const BiasSums& b, int block, float* part) {
  constexpr int W = THREADS / 128;                   // waves a gradient
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, q = w / W;
  const int c = block * 64 + lane;
  float v = 0.f;
  if (c < b.n)
#pragma unroll 8
    for (int r = w % W; r < b.chunks; r += W) v += b.sums[((size_t)r * 2 + q) * b.np + c];
  part[w * 64 + lane] = v;
  __syncthreads();
  float* db = q ? b.db[1] : b.db[0];
  if (w % W || c >= b.n || !db) return;
#pragma unroll
  for (int u = 1; u < W; ++u) v += part[(w + u) * 64 + lane];
  db[c] = b.accumulate ? db[c] + v : v;
}

// The products of the backward in one launch, the weight gradients' blocks behind dx's
// (none: first = 0), behind them the bias gradients': none reads what another writes, and
// small shards leave CUs idle in each.
template <class T>
__global__ __launch_bounds__(T::THREADS, 2) void gemm_dual_grads(DualArgs dx, DualArgs dw, int first,
                                                                 BiasSums bias) {
  extern __shared__ u16 lds[];
  const int block = blockIdx.x, last = first + dw.mt * dw.nt * dw.splits;
  if (block < first) dual_block<T, kDualDx, 0>(dx, block, lds);
  else if (block < last) dual_block<T, kDualDw, 0>(dw, block - first, lds);
  else bias_sum_block<T::THREADS>(bias, block - last, reinterpret_cast<float*>(lds));
}

}  // namespace sb
