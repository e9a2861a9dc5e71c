// token_logp.hip -- log-probabilities of given tokens, entropy and the most likely
// alternatives of rows of logits, and the logits' gradient.
//
// With M a row's largest logit and S = sum_c exp(z_c - M):
//   logp_c = (z_c - M) - log S,   H = log S - sum_c exp(z_c - M) (z_c - M) / S
// The largest term is left out of the sum, O = S - 1, and log S is log1p(O): where a
// row is sure of its token, logp and H are small and keep their bits.
//
// Backward: a gradient g on the log-probabilities of some classes and dH on the entropy give
//   dz_c = sum of g at c - p_c (sum of all g + dH (logp_c + H)).
//
// Rows of up to 1024 classes (a router's): 8 to 64 lanes have a row in registers and do
// everything in one launch.  Longer rows are cut into stretches, each held in a wave's
// registers so that z is read once: maximum, sums, and the stretch's best classes.  A
// block's waves have a row's stretches and join them in LDS; few very long rows have theirs
// over the whole chip, joined by a second launch.  Sums run in a fixed order.
//
// The best `top` classes of a stretch: every lane's maximum is known, and the
// top-th largest of those 64 is a bound that at least `top` elements reach and few
// others.  What reaches it goes to LDS and is ranked there.  Where too much does
// (many equal logits) or a NaN is about, the slow way takes one after another.
#include "rows.hpp"

#include <algorithm>
#include <cfloat>
#include <cmath>

namespace sb {

constexpr int kTopList = 256;          // classes of a stretch that are ranked in LDS
constexpr int kMaxStretches = 512;     // of a row
constexpr int kHeads = 4;              // of a stretch's list, read at once by the joining wave
constexpr int kNarrow = 1024;          // classes of a row in one launch
constexpr int kNarrowElems = 16;       // of a lane there
constexpr int kMoreTop = 2;            // fp32 classes there that are ranked beside the best
template <typename T> constexpr int kNarrowPieces = kNarrowElems / Piece<T>::N;
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
constexpr float kLeastPower = -1000.f; // in place of masked elements' -inf: 0 times it is 0
// Largest magnitude of a maximum M whose sums take powers of 2 against M log2 e rounded: that is
// off by 2^-4 at most, which a factor puts right.  (From 1.5e9 on it is off by up to 128, and a
// power, or the factor, is infinite or 0.  Larger ones take the sums against M itself: 2048 x
// 32000 bf16 without alternatives 29.6 us below, 31.2 above.)
constexpr float kMostSums = 0x1p20f;
// The same for M itself taken from the logits, in the best classes and the gradient.
constexpr float kMostPlain = 1e30f;

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// Whole numbers in the order of the logits: -0 is 0, any NaN above all.  0 is none.
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  const uint32_t o = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
  return v != v ? 0xffffffffu : o;
}
__device__ __forceinline__ float value_of(uint32_t o) {
  return o == 0xffffffffu ? NAN : __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
// Larger logits first, then lower classes.
__device__ __forceinline__ uint64_t key_of(uint32_t order, uint32_t cls) {
  return (uint64_t)order << 32 | (uint32_t)~cls;
}
__device__ __forceinline__ uint32_t class_of(uint64_t key) { return ~(uint32_t)key; }

// Reductions over a group of 8 to 64 lanes, which all get the result: within 16 lanes by
// moves inside the vector unit, beyond by swapped halves; no LDS, a fixed order.
template <int CTRL>
__device__ __forceinline__ uint32_t lane_move(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false);
}
struct Both {
  uint32_t a, b;
};
__device__ __forceinline__ Both swap16(uint32_t v) {
  const auto t = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return Both{t[0], t[1]};
}
__device__ __forceinline__ Both swap32(uint32_t v) {
  const auto t = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return Both{t[0], t[1]};
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140;

template <typename F>
__device__ __forceinline__ uint32_t group_reduce(uint32_t v, int lanes, F f) {
  v = f(v, lane_move<kXor1>(v));
  v = f(v, lane_move<kXor2>(v));
  v = f(v, lane_move<kMirror8>(v));
  if (lanes > 8) v = f(v, lane_move<kMirror16>(v));
  if (lanes > 16) {
    const Both t = swap16(v);
    v = f(t.a, t.b);
  }
  if (lanes > 32) {
    const Both t = swap32(v);
    v = f(t.a, t.b);
  }
  return v;
}
__device__ __forceinline__ float maximum(float a, float b) {   // NaN if one is
  return __builtin_elementwise_maximum(a, b);
}
__device__ __forceinline__ float group_max(float v, int lanes) {
  return __uint_as_float(group_reduce(__float_as_uint(v), lanes, [](uint32_t a, uint32_t b) {
    return __float_as_uint(maximum(__uint_as_float(a), __uint_as_float(b)));
  }));
}
__device__ __forceinline__ float group_sum(float v, int lanes) {
  return __uint_as_float(group_reduce(__float_as_uint(v), lanes, [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}
__device__ __forceinline__ uint32_t group_max(uint32_t v, int lanes) {
  return group_reduce(v, lanes, [](uint32_t a, uint32_t b) { return max(a, b); });
}
// The largest of 64-bit numbers: upper halves first, lower ones where those agree.
__device__ __forceinline__ uint64_t group_max(uint64_t v, int lanes) {
  const uint32_t hi = (uint32_t)(v >> 32), top = group_max(hi, lanes);
  return (uint64_t)top << 32 | group_max(hi == top ? (uint32_t)v : 0u, lanes);
}

struct LogpFwd {
  int m, classes, ldz, top, probs;
  int stretches;               // of a row
  const int32_t* targets;
  float *logp, *entropy, *stats;
  int32_t* top_ids;
  float* top_values;
  float* part;                 // [m][stretches][3]: maximum, sum without it, weighted sum
  uint64_t* keys;              // [m][stretches][top], in order, 0: none
};

// Sums of a lane's elements against the maximum mx of its row or stretch, whatever they
// are: o without the elements that equal it (their number is `equal`), s of
// exp(t) t.  Masked elements (-inf) give nothing.  A NaN ends up in o.
template <typename T, int P>
__device__ __forceinline__ void lane_sums(const Piece<T>* p, float mx, float& o, float& s,
                                          int& equal) {
  constexpr int N = Piece<T>::N;
  o = 0.f;
  s = 0.f;
  equal = 0;
  const float base = mx == -INFINITY ? 0.f : mx;
#pragma unroll
  for (int e = 0; e < P * N; ++e) {
    const float v = p[e / N].get(e % N);
    const float t = v - base;
    const float x = exp2_hw(t * kLog2e);
    const bool is_max = v == mx;
    equal += is_max ? 1 : 0;
    o += is_max ? 0.f : x;
    s += x > 0.f ? x * t : 0.f;
  }
}

// What a row gives once its maximum M, O = S - 1 and the weighted sum are known.
struct RowSums {
  float mx, sum, ls, h;
};
__device__ __forceinline__ RowSums row_sums(float mx, float o, float s) {
  RowSums r;
  r.mx = mx;
  // Nothing is left of a row of -inf alone: probabilities 0, entropy 0, log S -inf.
  const bool none = mx == -INFINITY && o == o;
  r.ls = none ? -INFINITY : mx == INFINITY ? NAN : log1pf(o);
  r.sum = mx == INFINITY ? NAN : 1.f + o;
  r.h = none ? 0.f : r.ls - s / r.sum;
  return r;
}
__device__ __forceinline__ float row_logp(const RowSums& r, float z) {
  return z == -INFINITY && r.ls == r.ls ? -INFINITY : (z - r.mx) - r.ls;
}

// exp(row_logp), without the logarithm's rounding: that is 2^-20 of a probability of 1e-8.
__device__ __forceinline__ float row_prob(const RowSums& r, float z) {
  return z == -INFINITY && r.ls == r.ls ? 0.f : expf(z - r.mx) / r.sum;
}

template <typename T>
__device__ __forceinline__ float target_logp(const RowSums& r, const T* z, int target,
                                             int classes) {
  if (target < 0) return 0.f;
  if (target >= classes) return NAN;
  return row_logp(r, Elem<T>::load(z, target));
}

// P pieces of a lane: pieces lane, lane + lanes, ... of the row from `first` on.
// Elements past the row are -inf.
template <typename T> __device__ __forceinline__ uint32_t minus_inf();
template <> __device__ __forceinline__ uint32_t minus_inf<float>() { return 0xff800000u; }
template <> __device__ __forceinline__ uint32_t minus_inf<u16>() { return 0xff80ff80u; }

template <typename T, int P>
__device__ __forceinline__ void load_row(const T* row, int classes, int first, int lane, int lanes,
                                         Piece<T>* p) {
  constexpr int N = Piece<T>::N;
  if (first + P * N * lanes <= classes) {
#pragma unroll
    for (int u = 0; u < P; ++u) p[u].load(row + first + (lane + u * lanes) * N, N, N);
    return;
  }
  const uint32_t none = minus_inf<T>();
#pragma unroll
  for (int u = 0; u < P; ++u) {
    const int left = classes - (first + (lane + u * lanes) * N);
    p[u].raw = u4{none, none, none, none};
    if (left > 0) p[u].load(row + classes - left, left, classes);
  }
#pragma unroll
  for (int u = 0; u < P; ++u) {
    const int left = classes - (first + (lane + u * lanes) * N);
    if (left <= 0 || left >= N) continue;
    if (classes >= N) {
      p[u].settle(left, classes, none);
    } else {
      float v[N];
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = e < left ? p[u].get(e) : -INFINITY;
      p[u].set(v);
    }
  }
}
template <typename T>
__device__ __forceinline__ int class_at(int first, int lane, int lanes, int e) {
  constexpr int N = Piece<T>::N;
  return first + (lane + e / N * lanes) * N + e % N;
}

// Outputs of one of a row's best classes.
__device__ __forceinline__ void give_top(const LogpFwd& b, const RowSums& r, size_t row, int rank,
                                         uint64_t key) {
  const float z = value_of((uint32_t)(key >> 32));
  b.top_ids[row * b.top + rank] = (int32_t)class_of(key);
  b.top_values[row * b.top + rank] = b.probs ? row_prob(r, z) : row_logp(r, z);
}

// ------------------------------------------------------------- narrow rows --
// The best classes one after another, whatever the logits.
template <typename T>
__device__ __forceinline__ void narrow_top_exact(const LogpFwd& b, const RowSums& r, const T* zr,
                                                 size_t row, int lane, int lanes) {
  constexpr int N = Piece<T>::N, E = kNarrowElems;
  Piece<T> p[E / N];
  load_row<T, E / N>(zr, b.classes, 0, lane, lanes, p);
  uint32_t order[E];
#pragma unroll
  for (int e = 0; e < E; ++e)
    order[e] = class_at<T>(0, lane, lanes, e) < b.classes ? order_of(p[e / N].get(e % N)) : 0;
#pragma unroll 1
  for (int k = 0; k < b.top; ++k) {
    uint32_t best = order[0];
#pragma unroll
    for (int e = 1; e < E; ++e) best = max(best, order[e]);
    int at = 0;                               // the first of them: classes grow with e
#pragma unroll
    for (int e = E - 1; e >= 0; --e) at = order[e] == best ? e : at;
    const uint64_t key = best ? key_of(best, class_at<T>(0, lane, lanes, at)) : 0;
    const uint64_t most = group_max(key, lanes);
    const int gone = key == most ? at : -1;
#pragma unroll
    for (int e = 0; e < E; ++e) order[e] = e == gone ? 0 : order[e];
    if (lane == (k & (lanes - 1))) give_top(b, r, row, k, most);
  }
}

// Instructions and the chain of a wave's steps bound it (4096 waves, four on a SIMD): 32768 x
// 128 fp32 5 to 6 us without alternatives, 12.2 with the best eight, 9.8 of bf16.
template <typename T>
__global__ __launch_bounds__(256) void logp_narrow_fwd(LogpFwd b, int shift,
                                                       const T* __restrict__ z) {
  constexpr int N = Piece<T>::N, P = kNarrowPieces<T>, E = P * N;
  __shared__ uint64_t lists[256 / 8][SB_LOGP_MAX_TOP + kMoreTop];
  const int lanes = 1 << shift, lane = threadIdx.x & (lanes - 1);
  const size_t row = ((size_t)blockIdx.x * 256 + threadIdx.x) >> shift;
  if (row >= (size_t)b.m) return;             // whole groups leave together
  const T* zr = z + row * (size_t)b.ldz;
  Piece<T> p[P];
  load_row<T, P>(zr, b.classes, 0, lane, lanes, p);
  float v[E];
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = p[e / N].get(e % N);
  float mx = v[0];
#pragma unroll
  for (int e = 1; e < E; ++e) mx = maximum(mx, v[e]);
  mx = group_max(mx, lanes);
  float o, s;
  int equal;
  lane_sums<T, P>(p, mx, o, s, equal);
  o = group_sum(o, lanes);
  s = group_sum(s, lanes);
  const float others = group_sum((float)equal, lanes) - 1.f;
  if (mx != -INFINITY) o += others;           // (else the -inf elements are all that is there)
  const RowSums r = row_sums(mx, o, s);
  if (lane == 0) {
    b.stats[row * 2] = r.mx;
    b.stats[row * 2 + 1] = r.ls;
    if (b.entropy) b.entropy[row] = r.h;
    if (b.logp) b.logp[row] = target_logp(r, zr, b.targets ? b.targets[row] : -1, b.classes);
  }
  if (!b.top) return;
  // Logit and class in one number, the class in its lowest bits: no two are equal, and the next
  // best is what lies closest below the last one.  A bf16 logit has room beside a class; an
  // fp32 one loses bits, so two more than `top` are taken and ranked by all they have.  Where
  // the last of them does not lie below the best ones in the bits that are left, the wave
  // takes the slow way (one such wave and the launch would wait for it).
  constexpr bool whole = std::is_same<T, u16>::value;
  const uint32_t mask = whole ? 0xffffu : (uint32_t)(E * lanes) - 1;
  const int taken = whole ? b.top : min(b.top + kMoreTop, b.classes);
  uint32_t key[E];
#pragma unroll
  for (int e = 0; e < E; ++e)                 // (past the row: -inf behind any class of it)
    key[e] = (order_of(v[e]) & ~mask) | (mask - class_at<T>(0, lane, lanes, e));
  uint64_t* list = lists[threadIdx.x >> shift];
  uint32_t last = 0, kept = 0;                // by lane j: the best class j of those at hand
  for (int k = 0; k < taken; ++k) {
    uint32_t most = key[0] - last;            // (first: all of them are above 0)
#pragma unroll
    for (int e = 1; e < E; ++e) most = max(most, key[e] - last);
    last += group_max(most, lanes);
    const int j = k & (lanes - 1);
    if (lane == j) kept = last;
    if (j != lanes - 1 && k != taken - 1) continue;
    if (lane <= j) {
      const uint32_t c = mask - (kept & mask);
      const uint64_t full = key_of(order_of(Elem<T>::load(zr, c)), c);
      if constexpr (whole) give_top(b, r, row, k - j + lane, full);
      else list[k - j + lane] = full;
    }
  }
  if constexpr (whole) return;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  bool sure = true;
  for (int i = lane; i < taken; i += lanes) {
    const uint64_t mine = list[i];
    int rank = 0;
    for (int j = 0; j < taken; ++j) rank += list[j] > mine ? 1 : 0;
    if (rank < b.top) give_top(b, r, row, rank, mine);
    if (rank == b.top - 1)
      sure = taken == b.classes || ((uint32_t)(mine >> 32) & ~mask) > (last & ~mask);
  }
  if (__all(sure)) return;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // it writes there again
  narrow_top_exact(b, r, zr, row, lane, lanes);
}

// ---------------------------------------------------------------- long rows --
// A bound that at least k (>= 1) of the 64 lanes' numbers reach, and few more: the k-th
// largest of their upper halves.
__device__ __forceinline__ uint32_t wave_kth(uint32_t v, int k) {
  uint32_t got = 0;
#pragma unroll
  for (int b = 31; b >= 16; --b) {
    const uint32_t t = got | 1u << b;
    if (__popcll(__ballot(v >= t)) >= k) got = t;
  }
  return got;
}

// The best `top` of `count` <= kTopList different keys in LDS, in order; `give` gets each
// rank and key.  One wave.
template <typename F>
__device__ __forceinline__ void rank_list(const uint64_t* list, int count, int top, int lane,
                                          F give) {
  for (int i = lane; i < count; i += 64) {
    const uint64_t mine = list[i];
    int rank = 0;
    for (int j = 0; j < count; ++j) rank += list[j] > mine ? 1 : 0;
    if (rank < top) give(rank, mine);
  }
}

// best: the largest of each of the lane's pieces; lm: of the lane.
template <typename T, int P>
__device__ __forceinline__ void stretch_top(const LogpFwd& b, const T* row, const Piece<T>* p,
                                            const float* best, float lm, bool plain, int first,
                                            int lane, uint64_t* list, uint64_t* out) {
  constexpr int N = Piece<T>::N;
  int count = kTopList + 1;
  if (plain) {
    const uint32_t bound = wave_kth(order_of(lm), b.top);
    const float least = value_of(bound);      // (upper halves above -inf's are no NaN's)
    if (least > -INFINITY) {
      count = 0;
#pragma unroll
      for (int u = 0; u < P; ++u) {
        if (!__ballot(best[u] >= least)) continue;
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float v = p[u].get(e);
          const uint64_t mask = __ballot(v >= least);
          if (!mask) continue;
          const int at = count + __popcll(mask & ((1ull << lane) - 1));
          if (v >= least && at < kTopList)
            list[at] = key_of(order_of(v), class_at<T>(first, lane, 64, u * N + e));
          count += __popcll(mask);
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  if (count <= kTopList) {
    rank_list(list, count, b.top, lane, [&](int rank, uint64_t key) { out[rank] = key; });
    return;
  }
  uint64_t last = ~0ull;
#pragma unroll 1
  for (int k = 0; k < b.top; ++k) {
    uint64_t most = 0;
    const int end = min(b.classes, first + P * N * 64);
#pragma unroll 1
    for (int c = first + lane; c < end; c += 64) {
      const uint64_t key = key_of(order_of(Elem<T>::load(row, c)), c);
      // (A NaN in class 0 has the largest key there is.)
      if ((k == 0 || key < last) && key > most) most = key;
    }
    last = group_max(most, 64);
    if (lane == 0) out[k] = last;
  }
}

// Sums of a stretch without its largest element, for a maximum M of up to kMostSums.
// Powers of 2: exp(z - M) = 2^(z log2 e - c) * fix, c = M log2 e rounded and fix its
// error's power, so that an element costs one fused product.  Every lane sums all it has; the
// first lane that has the maximum does not count, and its elements are summed by all lanes
// once more, without the maximum.
template <typename T, int P>
__device__ __forceinline__ void stretch_sums(const Piece<T>* p, float mx, float lm, int lane,
                                             u4* share, float& o, float& s) {
  constexpr int N = Piece<T>::N, E = P * N;
  const float c = mx * kLog2e, err = fmaf(mx, kLog2e, -c);
  float sx = 0.f, sy = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float y = fmaxf(fmaf(p[e / N].get(e % N), kLog2e, -c), kLeastPower);
    const float x = exp2_hw(y);
    sx += x;
    sy = fmaf(x, y, sy);
  }
  const int leader = __ffsll((unsigned long long)__ballot(lm == mx)) - 1;
  if (lane == leader) {
#pragma unroll
    for (int u = 0; u < P; ++u) share[u] = p[u].raw;
    sx = sy = 0.f;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const float v = lane < E ? Elem<T>::load(reinterpret_cast<const T*>(share), lane) : -INFINITY;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  if (lane != __ffsll((unsigned long long)__ballot(v == mx)) - 1) {
    const float y = fmaxf(fmaf(v, kLog2e, -c), kLeastPower);
    const float x = exp2_hw(y);
    sx += x;
    sy = fmaf(x, y, sy);
  }
  sx = group_sum(sx, 64);
  sy = group_sum(sy, 64);
  const float fix = exp2_hw(-err);
  o = sx * fix;
  s = kLn2 * (fix * fmaf(-err, sx, sy));
}

// A stretch by one wave: its maximum and sums to part[3], its best classes to keys[top].
template <typename T, int P>
__device__ __forceinline__ void stretch(const LogpFwd& b, const T* zr, int first, int lane,
                                        uint64_t* list, float* part, uint64_t* keys) {
  constexpr int N = Piece<T>::N;
  Piece<T> p[P];
  load_row<T, P>(zr, b.classes, first, lane, 64, p);
  float best[P], lm = 0.f;
#pragma unroll
  for (int u = 0; u < P; ++u) {
    best[u] = p[u].get(0);
#pragma unroll
    for (int e = 1; e < N; ++e) best[u] = maximum(best[u], p[u].get(e));
    lm = u ? maximum(lm, best[u]) : best[u];
    // (Unpacked again for the sums: kept as fp32 they would cost half of the waves.)
    asm volatile("" : "+v"(p[u].raw));
  }
  const float mx = group_max(lm, 64);
  const bool plain = fabsf(mx) < kMostPlain;       // not where a NaN is
  float o, s;
  if (fabsf(mx) <= kMostSums) {
    stretch_sums<T, P>(p, mx, lm, lane, reinterpret_cast<u4*>(list), o, s);
  } else {
    int equal;
    lane_sums<T, P>(p, mx, o, s, equal);
    o = group_sum(o, 64);
    s = group_sum(s, 64);
    const float others = group_sum((float)equal, 64) - 1.f;
    if (mx != -INFINITY) o += others;
  }
  if (lane == 0) {
    part[0] = mx;
    part[1] = o;
    part[2] = s;
  }
  if (b.top) stretch_top<T, P>(b, zr, p, best, lm, plain, first, lane, list, keys);
}

// One wave joins a row's stretches.  A stretch's list is in order: with d = `depth` and q
// lists of which the d-th entry reaches a bound, q d classes do.  Latency bounds it: the heads
// of a lane's list are read before the bound is known (333 rows of 25 stretches, best 20:
// 6.2 -> 5.2 us).  counter: LDS.
template <typename T>
__device__ __forceinline__ void join_row(const LogpFwd& b, const T* zr, size_t row,
                                         const float* part, const uint64_t* keys, int lane,
                                         uint64_t* list, int* counter) {
  const int target = b.logp ? b.targets[row] : -1;
  // (Read ahead of the sums; a class past the row is told by its number later.)
  const float zt = target >= 0 && target < b.classes ? Elem<T>::load(zr, target) : 0.f;
  const int lists = min(b.stretches, 64);
  const int depth = min(b.top, max(1, (2 * b.top + lists - 1) / lists));
  // What the lane's first stretch gave is read once, all of it on its way together.
  const int mine = min(lane, b.stretches - 1);
  const float m0 = part[mine * 3], o0 = part[mine * 3 + 1], s0 = part[mine * 3 + 2];
  uint64_t heads[kHeads], deep = 0;             // the best d-th entry of the lane's lists
  if (b.top) {
    const uint64_t* from = keys + (size_t)mine * b.top;
#pragma unroll
    for (int i = 0; i < kHeads; ++i) heads[i] = from[min(i, b.top - 1)];
    for (int p = lane; p < b.stretches; p += 64)
      deep = max(deep, keys[(size_t)p * b.top + depth - 1]);
  }
  if (lane == 0) *counter = 0;
  float mx = lane < b.stretches ? m0 : -INFINITY;
  for (int p = lane + 64; p < b.stretches; p += 64) mx = maximum(mx, part[p * 3]);
  const float all = group_max(mx, 64);
  uint32_t who = lane < b.stretches && m0 == all ? lane : ~0u;
  for (int p = lane + 64; p < b.stretches; p += 64)   // the first stretch that has it
    if (who == ~0u && part[p * 3] == all) who = p;
  who = ~group_max(~who, 64);
  float o = 0.f, s = 0.f;
  for (int p = lane; p < b.stretches; p += 64) {
    float pm = m0, po = o0, ps = s0;
    if (p != lane) {
      pm = part[p * 3];
      po = part[p * 3 + 1];
      ps = part[p * 3 + 2];
    }
    if (pm == -INFINITY) continue;              // nothing
    const float t = pm - all, f = exp2_hw(t * kLog2e);
    o += (uint32_t)p == who ? po : f * (1.f + po);
    s += f > 0.f ? f * (ps + t * (1.f + po)) : 0.f;
  }
  o = group_sum(o, 64);
  s = group_sum(s, 64);
  const RowSums r = row_sums(all, o, s);
  if (lane == 0) {
    b.stats[row * 2] = r.mx;
    b.stats[row * 2 + 1] = r.ls;
    if (b.entropy) b.entropy[row] = r.h;
    if (b.logp) b.logp[row] = target < 0 ? 0.f : target >= b.classes ? NAN : row_logp(r, zt);
  }
  if (!b.top) return;
  const uint32_t bound = wave_kth((uint32_t)(deep >> 32), (b.top + depth - 1) / depth);
  for (int p = lane; p < b.stretches; p += 64) {
    const uint64_t* from = keys + (size_t)p * b.top;
    bool more = true;
    for (int at = 0; more && at < b.top; at += kHeads) {
      if (p != lane || at)
#pragma unroll
        for (int i = 0; i < kHeads; ++i) heads[i] = from[min(at + i, b.top - 1)];
#pragma unroll
      for (int i = 0; i < kHeads; ++i) {
        const uint64_t key = heads[i];
        more = more && at + i < b.top && key != 0 && (uint32_t)(key >> 32) >= bound;
        if (!more) continue;
        // (Their order in the list does not matter: every one is ranked.)
        const int to = atomicAdd(counter, 1);
        if (to < kTopList) list[to] = key;
      }
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int count = *counter;
  if (count <= kTopList) {
    rank_list(list, count, b.top, lane,
              [&](int rank, uint64_t key) { give_top(b, r, row, rank, key); });
    return;
  }
  // Many equal ones: the best of a lane's heads, again and again.
  uint64_t taken = 0;                           // 8 bits for each of a lane's (at most 8) lists
  for (int k = 0; k < b.top; ++k) {
    uint64_t best = 0;
    int from = 0;
    for (int p = lane, i = 0; p < b.stretches; p += 64, ++i) {
      const int at = (int)(taken >> (8 * i)) & 255;
      const uint64_t key = at < b.top ? keys[(size_t)p * b.top + at] : 0;
      if (key > best) {
        best = key;
        from = i;
      }
    }
    const uint64_t most = group_max(best, 64);
    if (best == most && most) taken += 1ull << (8 * from);
    if (lane == 0) give_top(b, r, row, k, most);
  }
}

// A row by one block, a stretch a wave; the first wave joins them in LDS.  2048 x 32000 bf16
// (131 MB) in 38.5 us: loads and sums of all waves fall together, two blocks a CU.
struct RowShare {
  size_t part, keys, bytes;    // offsets in LDS, behind a list for each wave
};
__host__ __device__ inline RowShare row_share(int waves, int stretches, int top) {
  RowShare s;
  s.keys = (size_t)waves * kTopList * 8;
  s.part = s.keys + (size_t)stretches * top * 8;
  s.bytes = s.part + ((size_t)stretches * 3 + 1) * 4;
  return s;
}

template <typename T, int P>
__global__ __launch_bounds__(1024) void logp_row_fwd(LogpFwd b, const T* __restrict__ z) {
  constexpr int E = P * Piece<T>::N;
  extern __shared__ uint64_t lists[];
  const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const RowShare at = row_share(waves, b.stretches, b.top);
  uint64_t* keys = lists + at.keys / 8;
  float* part = reinterpret_cast<float*>(lists) + at.part / 4;
  const size_t row = blockIdx.x;
  const T* zr = z + row * (size_t)b.ldz;
  stretch<T, P>(b, zr, wave * (E * 64), lane, lists + wave * kTopList, part + wave * 3,
                keys + wave * b.top);
  __syncthreads();
  if (wave) return;
  join_row(b, zr, row, part, keys, lane, lists,
           reinterpret_cast<int*>(part + b.stretches * 3));
}

// Longer rows: a stretch a wave anywhere on the chip, joined by a second launch.  HBM bounds it
// where there are many: 4096 x 131072 bf16 with the best eight (1.07 GB) 235 us, 4.6 TB/s, and
// 8 us of joining.
template <typename T, int P>
__global__ __launch_bounds__(256) void logp_stretch_fwd(LogpFwd b, const T* __restrict__ z) {
  constexpr int E = P * Piece<T>::N;
  __shared__ uint64_t list[4][kTopList];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const size_t unit = (size_t)blockIdx.x * 4 + wave;
  const size_t row = unit / (unsigned)b.stretches;
  if (row >= (size_t)b.m) return;
  const int first = (int)(unit - row * b.stretches) * (E * 64);
  stretch<T, P>(b, z + row * (size_t)b.ldz, first, lane, list[wave], b.part + unit * 3,
                b.keys + unit * b.top);
}

template <typename T>
__global__ __launch_bounds__(256) void logp_join(LogpFwd b, const T* __restrict__ z) {
  __shared__ uint64_t list[4][kTopList];
  __shared__ int counts[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const size_t row = (size_t)blockIdx.x * 4 + wave;
  if (row >= (size_t)b.m) return;
  join_row(b, z + row * (size_t)b.ldz, row, b.part + row * b.stretches * 3,
           b.keys + row * b.stretches * b.top, lane, list[wave], &counts[wave]);
}

// ----------------------------------------------------------------- backward --
struct LogpBwd {
  int m, classes, ldz, top, probs;
  int stretches;
  const float *stats, *entropy;
  const int32_t* targets;
  const float *dlogp, *dentropy;
  const int32_t* top_ids;
  const float *top_values, *dtop;
};

// What a row's gradient needs: logp = z - mx - ls; dhh = dH H, all = the sum of g.
struct RowGrad {
  float mx, ls, dh, dhh, all;
  int target;
  float g;                     // at the target
  bool bad;                    // a target past the classes: a row of NaN
};
__device__ __forceinline__ RowGrad row_grad(const LogpBwd& b, size_t row) {
  RowGrad r;
  r.mx = b.stats[row * 2];
  r.ls = b.stats[row * 2 + 1];
  r.dh = b.dentropy ? b.dentropy[row] : 0.f;
  r.dhh = b.dentropy ? r.dh * b.entropy[row] : 0.f;
  r.target = b.dlogp ? b.targets[row] : -1;
  r.g = r.target >= 0 ? b.dlogp[row] : 0.f;
  r.bad = r.target >= b.classes;
  r.all = r.g;
  return r;
}
// Gradient of a row's k-th alternative on its log-probability; its class in id.
__device__ __forceinline__ float top_grad(const LogpBwd& b, size_t row, int k, int& id) {
  id = b.top_ids[row * b.top + k];
  const float d = b.dtop[row * b.top + k];
  if (id < 0 || id >= b.classes) return 0.f;
  if (!b.probs) return d;
  const float p = b.top_values[row * b.top + k];
  return p == 0.f ? 0.f : d * p;
}
// dz of a class that has the gradient g itself (0 for most) and the others `others` in all.  (As
// all - g they lose what is small beside g, and a sure row has little else.)
__device__ __forceinline__ float class_grad(const RowGrad& r, float z, float g, float others) {
  const float lp = (z - r.mx) - r.ls;
  const float p = exp2_hw(lp * kLog2e);
  const float d = p > 0.f ? p * (others + fmaf(r.dh, lp, r.dhh)) : p == 0.f ? 0.f : p;
  return (g != 0.f ? -g * expm1f(lp) : 0.f) - d;
}

// The same for classes without a gradient of their own, in rows of an ordinary M and
// log S: with t = z - M (exact where z is near M: sure rows keep their bits),
// dz = -2^(t log2 e - l) (a + dH t).
struct PlainGrad {
  float mx, l, a, dh;
  __device__ __forceinline__ explicit PlainGrad(const RowGrad& r)
      : mx(r.mx), l(r.ls * kLog2e), a(r.all + fmaf(-r.dh, r.ls, r.dhh)), dh(r.dh) {}
  __device__ __forceinline__ float operator()(float z) const {
    const float t = fmaxf(z - mx, kLeastPower);
    return -exp2_hw(fmaf(t, kLog2e, -l)) * fmaf(dh, t, a);
  }
};

// Whether a row takes PlainGrad: ordinary stats and no target past the classes.
__device__ __forceinline__ bool is_plain(const RowGrad& r) {
  return fabsf(r.mx) < kMostPlain && r.ls == r.ls && !r.bad;
}
// N elements of such a row, or of any other one.
template <int N, typename T>
__device__ __forceinline__ Piece<T> grad_piece(const RowGrad& r, const PlainGrad& grad, bool plain,
                                               const Piece<T>& z) {
  float d[N];
  if (plain) {
#pragma unroll
    for (int e = 0; e < N; ++e) d[e] = grad(z.get(e));
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      d[e] = r.bad ? NAN : r.ls == -INFINITY ? 0.f : class_grad(r, z.get(e), 0.f, r.all);
  }
  Piece<T> q;
  q.set(d);
  return q;
}

// The classes with a gradient of their own (alternatives, then the target) are a row's
// entries; lane l has entries l, l + lanes, ...  Their logits are read before the row is
// written (dz may be z), and they are written again behind it.  32768 x 128 fp32 through eight
// alternatives (34 MB) in 7.5 us.
template <typename T>
__global__ __launch_bounds__(256) void logp_narrow_bwd(LogpBwd b, int shift, const T* z, T* dz) {
  constexpr int N = Piece<T>::N, P = kNarrowPieces<T>;
  constexpr int ENTRIES = SB_LOGP_MAX_TOP + 1, MORE = (ENTRIES + 7) / 8;
  __shared__ int ids[256 / 8][ENTRIES];
  __shared__ float gs[256 / 8][ENTRIES];
  const int lanes = 1 << shift, lane = threadIdx.x & (lanes - 1);
  const size_t row = ((size_t)blockIdx.x * 256 + threadIdx.x) >> shift;
  if (row >= (size_t)b.m) return;
  int* id = ids[threadIdx.x >> shift];
  float* g = gs[threadIdx.x >> shift];
  const T* zr = z + row * (size_t)b.ldz;
  T* out = dz + row * (size_t)b.ldz;
  Piece<T> p[P];
  load_row<T, P>(zr, b.classes, 0, lane, lanes, p);
  RowGrad r = row_grad(b, row);
  const int tops = b.dtop ? b.top : 0, entries = tops + (r.target >= 0 && !r.bad ? 1 : 0);
  float all = 0.f;
  for (int k = lane; k < entries; k += lanes) {
    int c = r.target;
    const float gk = k < tops ? top_grad(b, row, k, c) : r.g;
    if (k < tops) all += gk;
    id[k] = c;
    g[k] = gk;
  }
  r.all += group_sum(all, lanes);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  float special[MORE];
#pragma unroll
  for (int i = 0; i < MORE; ++i) {
    const int k = i * lanes + lane;
    if (k >= entries) break;
    const int c = id[k];
    const float z0 = c >= 0 && c < b.classes ? Elem<T>::load(zr, c) : 0.f;
    float sum = 0.f, others = 0.f;              // of all that name this class, and of the rest
    for (int j = 0; j < entries; ++j) {
      sum += id[j] == c ? g[j] : 0.f;
      others += id[j] == c ? 0.f : g[j];
    }
    special[i] = r.ls == -INFINITY ? 0.f : class_grad(r, z0, sum, others);
  }
  const bool plain = __all(is_plain(r));
  const PlainGrad grad(r);
#pragma unroll
  for (int u = 0; u < P; ++u) {
    const int c = (lane + u * lanes) * N;
    const Piece<T> q = grad_piece<N>(r, grad, plain, p[u]);
    if (c < b.classes) q.store(out + c, b.classes - c);
  }
  // Behind what this wave has just written there.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
  for (int i = 0; i < MORE; ++i) {
    const int k = i * lanes + lane;
    if (k >= entries || r.bad) break;
    const int c = id[k];
    if (c >= 0 && c < b.classes) Elem<T>::store(out, c, special[i]);
  }
}

// A stretch of a long row, one a wave.  Lane l < top has alternative l, lane `top` the
// target: those in the stretch are read before the stretch is written (dz may be z)
// and written again behind it.  HBM bounds it: 4096 x 131072 bf16 (2.15 GB) in 370 us,
// 5.8 TB/s.
template <typename T, int P>
__global__ __launch_bounds__(256) void logp_stretch_bwd(LogpBwd b, const T* z, T* dz) {
  constexpr int N = Piece<T>::N, E = P * N;
  const int lane = threadIdx.x & 63;
  const size_t unit = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const size_t row = unit / (unsigned)b.stretches;
  if (row >= (size_t)b.m) return;
  const int first = (int)(unit - row * b.stretches) * (E * 64);
  const T* zr = z + row * (size_t)b.ldz;
  T* out = dz + row * (size_t)b.ldz;
  Piece<T> p[P];
  load_row<T, P>(zr, b.classes, first, lane, 64, p);
  RowGrad r = row_grad(b, row);
  const int tops = b.dtop ? b.top : 0;
  int id = -1;
  float g = 0.f;
  if (lane < tops) g = top_grad(b, row, lane, id);
  r.all += group_sum(g, 64);
  if (lane == tops && !r.bad) {
    id = r.target;
    g = r.g;
  }
  const bool mine = id >= first && id < min(b.classes, first + E * 64);
  const bool any = __ballot(mine) != 0;
  float special = 0.f;
  if (any) {
    const float z0 = mine ? Elem<T>::load(zr, id) : 0.f;
    float sum = 0.f, others = 0.f;              // of all that name this class, and of the rest
    for (int k = 0; k <= tops; ++k) {
      const float gk = __shfl(g, k, 64);
      const bool same = __shfl(id, k, 64) == id;
      sum += same ? gk : 0.f;
      others += same ? 0.f : gk;
    }
    special = r.ls == -INFINITY ? 0.f : class_grad(r, z0, sum, others);
  }
  const bool plain = is_plain(r);
  const PlainGrad grad(r);
#pragma unroll
  for (int u = 0; u < P; ++u) {
    const int c = first + (lane + u * 64) * N;
    const Piece<T> q = grad_piece<N>(r, grad, plain, p[u]);
    if (c < b.classes) q.store(out + c, b.classes - c);
  }
  if (any && !r.bad) {
    // Behind what this wave has just written there.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (mine) Elem<T>::store(out, id, special);
  }
}

}  // namespace sb

namespace {

// 16-byte pieces of a row that a lane holds, stretches of a row, and in the forward the
// waves of a row's block (0: stretches anywhere, joined by a second launch).
struct LogpPlan {
  int pieces, stretches, waves;
};
constexpr int kEnough = 4096;          // stretches: four waves for each SIMD

LogpPlan logp_plan(const sb_token_logp_desc* d, bool fwd) {
  const int per = 64 * 16 / (int)sbh::dsize(d->dtype);
  auto stretches = [&](int pieces) { return sb::cdiv(d->classes, per * pieces); };
  LogpPlan p{8, stretches(8), 0};
  const int64_t all = (int64_t)d->m * p.stretches;
  // A block a row saves the second launch: one row of 32000 bf16 8.4 us and not 4.2 + 4.4
  // and the time between, 2048 rows 40.5 and not 38.0 + 4.9.  More than 8 waves of long
  // stretches hold up one another where there are many rows: 333 rows of 50001 fp32 in blocks
  // of 13 waves took 31 us, apart 17.5 + 6.1.  Up to 16 of shorter ones are better while the
  // chip has few blocks to go on with (those 2048 rows 38.2), and shortest where rows are few.
  if (fwd && p.stretches <= (all < kEnough ? 16 : 8)) {
    if (all < 8 * kEnough && stretches(4) <= 16) p.pieces = 4;
    while (all < kEnough && p.pieces > 1 && stretches(p.pieces / 2) <= 16) p.pieces /= 2;
    p.waves = p.stretches = stretches(p.pieces);
    return p;
  }
  // Long stretches where there are enough of them (these 333 rows with 1, 2 and 8 pieces a
  // lane: 35, 24 and 17.5 us), short ones else.
  while (p.pieces > 1 && (int64_t)d->m * p.stretches < kEnough &&
         stretches(p.pieces / 2) <= sb::kMaxStretches) {
    p.pieces /= 2;
    p.stretches = stretches(p.pieces);
  }
  return p;
}

bool narrow(const sb_token_logp_desc* d) { return d->classes <= sb::kNarrow; }
int narrow_shift(const sb_token_logp_desc* d) {
  int s = 3;
  while (sb::kNarrowElems << s < d->classes) ++s;
  return s;
}

sb_status logp_check(const sb_token_logp_desc* d) {
  if (!d || d->m < 0 || d->classes < 1 || d->ldz < d->classes || d->top < 0 ||
      d->top > SB_LOGP_MAX_TOP || d->top > d->classes)
    return SB_ERR_INVALID_ARG;
  if ((d->dtype != SB_F32 && d->dtype != SB_BF16) || (d->flags & ~SB_TOP_PROBS))
    return SB_ERR_INVALID_ARG;
  if (d->classes > 1 << 20 || d->m >= 1 << 30) return SB_ERR_UNSUPPORTED;
  const size_t lanes =
      narrow(d) ? (size_t)d->m << narrow_shift(d)
                : (size_t)d->m * 64 *
                      std::max(logp_plan(d, true).stretches, logp_plan(d, false).stretches);
  return lanes < sb::kLaunchLanes - 256 ? SB_OK : SB_ERR_UNSUPPORTED;
}

size_t logp_part_bytes(const sb_token_logp_desc* d, const LogpPlan& p) {
  return sb::round_up((size_t)d->m * p.stretches * 3 * 4, 256);
}

bool off(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

template <typename T>
sb_status logp_fwd(const sb_token_logp_desc* d, const sb::LogpFwd& b, const LogpPlan& p, const T* z,
                   hipStream_t st) {
  if (narrow(d)) {
    const int shift = narrow_shift(d);
    const size_t blocks = (((size_t)d->m << shift) + 255) / 256;
    sb::logp_narrow_fwd<T><<<(unsigned)blocks, 256, 0, st>>>(b, shift, z);
    return sbh::launch_status();
  }
  if (p.waves) {
    const unsigned threads = 64 * p.waves;
    const size_t lds = sb::row_share(p.waves, p.stretches, d->top).bytes;
    switch (p.pieces) {
      case 8: sb::logp_row_fwd<T, 8><<<d->m, threads, lds, st>>>(b, z); break;
      case 4: sb::logp_row_fwd<T, 4><<<d->m, threads, lds, st>>>(b, z); break;
      case 2: sb::logp_row_fwd<T, 2><<<d->m, threads, lds, st>>>(b, z); break;
      default: sb::logp_row_fwd<T, 1><<<d->m, threads, lds, st>>>(b, z); break;
    }
    return sbh::launch_status();
  }
  const size_t blocks = ((size_t)d->m * p.stretches + 3) / 4;
  switch (p.pieces) {
    case 8: sb::logp_stretch_fwd<T, 8><<<(unsigned)blocks, 256, 0, st>>>(b, z); break;
    case 4: sb::logp_stretch_fwd<T, 4><<<(unsigned)blocks, 256, 0, st>>>(b, z); break;
    case 2: sb::logp_stretch_fwd<T, 2><<<(unsigned)blocks, 256, 0, st>>>(b, z); break;
    default: sb::logp_stretch_fwd<T, 1><<<(unsigned)blocks, 256, 0, st>>>(b, z); break;
  }
  sb::logp_join<T><<<(unsigned)sb::cdiv(d->m, 4), 256, 0, st>>>(b, z);
  return sbh::launch_status();
}

template <typename T>
sb_status logp_bwd(const sb_token_logp_desc* d, const sb::LogpBwd& b, const LogpPlan& p, const T* z,
                   T* dz, hipStream_t st) {
  if (narrow(d)) {
    const int shift = narrow_shift(d);
    const size_t blocks = (((size_t)d->m << shift) + 255) / 256;
    sb::logp_narrow_bwd<T><<<(unsigned)blocks, 256, 0, st>>>(b, shift, z, dz);
    return sbh::launch_status();
  }
  const size_t blocks = ((size_t)d->m * p.stretches + 3) / 4;
  switch (p.pieces) {
    case 8: sb::logp_stretch_bwd<T, 8><<<(unsigned)blocks, 256, 0, st>>>(b, z, dz); break;
    case 4: sb::logp_stretch_bwd<T, 4><<<(unsigned)blocks, 256, 0, st>>>(b, z, dz); break;
    case 2: sb::logp_stretch_bwd<T, 2><<<(unsigned)blocks, 256, 0, st>>>(b, z, dz); break;
    default: sb::logp_stretch_bwd<T, 1><<<(unsigned)blocks, 256, 0, st>>>(b, z, dz); break;
  }
  return sbh::launch_status();
}

}  // namespace

extern "C" size_t sb_token_logp_workspace_bytes(const sb_token_logp_desc* d) {
  if (logp_check(d) != SB_OK) return (size_t)-1;
  if (narrow(d) || d->m == 0) return 0;
  const LogpPlan p = logp_plan(d, true);
  if (p.waves) return 0;
  return logp_part_bytes(d, p) + sb::round_up((size_t)d->m * p.stretches * d->top * 8, 256);
}

extern "C" sb_status sb_token_logp_fwd(const sb_token_logp_desc* d, const void* z,
                                       const int32_t* targets, float* logp, float* entropy,
                                       float* stats, int32_t* top_ids, float* top_values,
                                       void* workspace, size_t workspace_bytes, void* stream) {
  const sb_status s = logp_check(d);
  if (s != SB_OK) return s;
  if (d->m == 0) return SB_OK;
  const size_t e = sbh::dsize(d->dtype), m = (size_t)d->m;
  if (!z || !stats || (logp && !targets) || (d->top > 0 && (!top_ids || !top_values)))
    return SB_ERR_INVALID_ARG;
  if (off(z, e) || off(targets, 4) || off(logp, 4) || off(entropy, 4) || off(stats, 4) ||
      off(top_ids, 4) || off(top_values, 4) || off(workspace, 16))
    return SB_ERR_INVALID_ARG;
  const size_t need = sb_token_logp_workspace_bytes(d);
  const size_t zb = ((m - 1) * d->ldz + d->classes) * e, tb = m * d->top * 4;
  const void* outs[6] = {logp, entropy, stats, d->top ? top_ids : nullptr,
                         d->top ? top_values : nullptr, workspace};
  const size_t ob[6] = {m * 4, m * 4, m * 8, tb, tb, need};
  for (int i = 0; i < 6; ++i) {
    if (sbh::overlaps(outs[i], ob[i], z, zb) || sbh::overlaps(outs[i], ob[i], targets, m * 4))
      return SB_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (sbh::overlaps(outs[i], ob[i], outs[j], ob[j])) return SB_ERR_INVALID_ARG;
  }
  if (need && (!workspace || workspace_bytes < need)) return SB_ERR_WORKSPACE;
  const LogpPlan p = logp_plan(d, true);
  sb::LogpFwd b{};
  b.m = d->m;
  b.classes = d->classes;
  b.ldz = d->ldz;
  b.top = d->top;
  b.probs = (d->flags & SB_TOP_PROBS) != 0;
  b.stretches = p.stretches;
  b.targets = targets;
  b.logp = logp;
  b.entropy = entropy;
  b.stats = stats;
  b.top_ids = top_ids;
  b.top_values = top_values;
  b.part = (float*)workspace;
  b.keys = (uint64_t*)((char*)workspace + logp_part_bytes(d, p));
  if (d->dtype == SB_BF16)
    return logp_fwd(d, b, p, (const sb::u16*)z, sbh::stream_of(stream));
  return logp_fwd(d, b, p, (const float*)z, sbh::stream_of(stream));
}

extern "C" sb_status sb_token_logp_bwd(const sb_token_logp_desc* d, const void* z,
                                       const float* stats, const int32_t* targets,
                                       const float* dlogp, const float* entropy,
                                       const float* dentropy, const int32_t* top_ids,
                                       const float* top_values, const float* dtop, void* dz,
                                       void* stream) {
  const sb_status s = logp_check(d);
  if (s != SB_OK) return s;
  if (d->m == 0) return SB_OK;
  const size_t e = sbh::dsize(d->dtype), m = (size_t)d->m;
  if (!z || !stats || !dz || (dlogp && !targets) || (dentropy && !entropy) ||
      (dtop && (d->top == 0 || !top_ids || ((d->flags & SB_TOP_PROBS) && !top_values))))
    return SB_ERR_INVALID_ARG;
  if (off(z, e) || off(dz, e) || off(stats, 4) || off(targets, 4) || off(dlogp, 4) ||
      off(entropy, 4) || off(dentropy, 4) || off(top_ids, 4) || off(top_values, 4) || off(dtop, 4))
    return SB_ERR_INVALID_ARG;
  const size_t zb = ((m - 1) * d->ldz + d->classes) * e, tb = m * d->top * 4;
  const void* ins[8] = {stats, targets, dlogp, entropy, dentropy, top_ids, top_values, dtop};
  const size_t ib[8] = {m * 8, m * 4, m * 4, m * 4, m * 4, tb, tb, tb};
  if (dz != z && sbh::overlaps(dz, zb, z, zb)) return SB_ERR_INVALID_ARG;
  for (int i = 0; i < 8; ++i)
    if (sbh::overlaps(dz, zb, ins[i], ib[i])) return SB_ERR_INVALID_ARG;
  const LogpPlan p = logp_plan(d, false);
  sb::LogpBwd b{};
  b.m = d->m;
  b.classes = d->classes;
  b.ldz = d->ldz;
  b.top = d->top;
  b.probs = (d->flags & SB_TOP_PROBS) != 0;
  b.stretches = p.stretches;
  b.stats = stats;
  b.entropy = entropy;
  b.targets = targets;
  b.dlogp = dlogp;
  b.dentropy = dentropy;
  b.top_ids = top_ids;
  b.top_values = top_values;
  b.dtop = dtop;
  if (d->dtype == SB_BF16)
    return logp_bwd(d, b, p, (const sb::u16*)z, (sb::u16*)dz, sbh::stream_of(stream));
  return logp_bwd(d, b, p, (const float*)z, (float*)dz, sbh::stream_of(stream));
}
