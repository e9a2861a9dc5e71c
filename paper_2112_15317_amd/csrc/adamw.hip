// adamw.hip -- the AdamW step over many tensors, moments in fp32 or in bytes
// (in place of the SGD step of sec. 4: what an MP group's worker does with the
// gradients of its conv layers and FC shards).
//
// Per element, in fp32 and in this order:
//   m = b1 m + (1 - b1) g,   v = b2 v + (1 - b2) g^2,   g = scale * gradient
//   w = keep w - (lr / (1 - b1^t)) m / (sqrt(v) (1 - b2^t)^-1/2 + eps)
// keep = 1 - lr * decay; the host forms the factors in fp64.  The products of m
// and v are rounded before their sum (no fused multiply-add), so that the bytes
// below are the same wherever they are formed.
//
// Moments in bytes.  A positive fp32 pattern's upper 11 bits below the sign are
// a rank: 8 ranks an octave, equally spaced within one.  A byte says how far a
// value's rank lies below the largest one of its block of 256 elements, so that a
// block needs one reference and no division: coding is a shift, an addition and
// a subtraction.  7 bits of it (m, with the sign) reach 15 octaves down, 8 (v)
// reach 31, the same as 15 of sqrt(v); a v below that takes the lowest code and
// not zero, which would turn m / sqrt(v) into m / eps.
//
// Rounding is random (up with the probability of the bits left out, so its mean
// is the value), because b2 = 0.999 changes v by 0.1 % a step and ranks are 6 to
// 12 % apart: rounded to nearest, v would never move.  The 16 random bits of each
// moment are halves of a hash of seed, step and element number.
//
// The kernel is a stream: 28 bytes an element (16 with moments in bytes), 2 more
// for the bf16 copy.  A wave takes 256 consecutive elements at a time, four a
// lane in 16-byte pieces, so that a block of bytes is one wave's and its largest
// rank a reduction over the lanes; a lane has all its loads under way before the
// first store.
//
// All tensors take one launch: their addresses lie in a table in device memory (the
// plan), written once.  As kernel arguments, 40 tensors a launch, 300 tensors of 40 M
// elements took 316 us, in one launch 219.  Blocks of tensor t are block0[t] ..
// block0[t+1]-1; a wave finds its tensor by counting, 64 entries at a time, those that
// start by its block.
#include "sb_internal.hpp"

#include <algorithm>
#include <cmath>

namespace sb {

// Groups of 4 elements per lane: two where moments are bytes and there are very many
// elements (134 M of them 406 us with one, 392 with two, 443 with four; 300 tensors of
// 40 M elements 158, 140, 161), else one (8 M elements 27.4 us, 30.0 with two; fp32 moments
// as fast with one, two and four).
constexpr int kAdamwGroups = 2;
constexpr size_t kAdamwMany = 24u << 20;
constexpr int kAdamwChunk = 40;              // tensors a launch writes into a plan

struct AdamwTensor {
  float* w;
  u16* copy;
  const float* g;
  void *m, *v;
  int16_t *m_top, *v_top;
  uint64_t first;
  size_t n;
  float scale, decay;
  int block0;
};

// A plan: the tensors' first blocks, then the tensors.
__host__ __device__ constexpr size_t plan_tensors(int count) {
  return round_up((size_t)count * sizeof(int), 256);
}

struct AdamwChunk {
  AdamwTensor t[kAdamwChunk];
  int first, count, total;                   // tensors first .. first + count - 1 of total
};
static_assert(sizeof(AdamwChunk) <= 4096, "kernel arguments");

__global__ __launch_bounds__(64) void adamw_plan_kernel(AdamwChunk c, char* plan) {
  const int i = threadIdx.x;
  if (i >= c.count) return;
  ((int*)plan)[c.first + i] = c.t[i].block0;
  ((AdamwTensor*)(plan + plan_tensors(c.total)))[c.first + i] = c.t[i];
}

struct AdamwStep {
  const char* plan;
  const int32_t* steps_done;
  double lr, beta1, beta2;
  float b1, c1, b2, c2, eps, rate, vscale;   // rate, vscale: of step, without a counter
  uint32_t seed;
  int step, count;
  int fast;                                  // eps hides subnormal v: see fast_root
};

__host__ __device__ inline uint32_t mix32(uint32_t x) {
  x ^= x >> 16;
  x *= 0x9e3779b9u;
  x ^= x >> 15;
  x *= 0xb7e15163u;
  return x ^ (x >> 16);
}

// Whether w's move takes the hardware's root and reciprocal (a step each, a quarter of
// the instructions).  They read a subnormal v as 0: its root, below 2^-63, times the bias
// factor, at most 1 / sqrt(1 - beta2), has to be below an eighth of half a step (2^-24)
// of eps.  A denominator from 2^126 on would have no reciprocal: eps is far below that,
// and the rest of it, below 2^64 times 2^27.
inline bool fast_root(double eps, double beta2) {
  return eps >= 0x1p-36 / std::sqrt(1.0 - beta2) && eps <= 0x1p100;
}

// beta^t by squaring.
__host__ __device__ inline double int_power(double b, uint32_t t) {
  double p = 1.0;
  for (; t; t >>= 1) {
    if (t & 1) p *= b;
    b *= b;
  }
  return p;
}

__device__ __forceinline__ float rank_value(int rank) {
  return rank > 0 ? __uint_as_float((uint32_t)rank << 20) : 0.f;
}

// The rank a magnitude's pattern is rounded to: up if the 20 bits below it and
// the random ones carry.  Finite values stay finite.
__device__ __forceinline__ int rank_of(uint32_t bits, uint32_t noise) {
  const int r = min((int)((bits + noise * 16 + 8) >> 20), 0x7f7);
  return bits < 0x7f800000u ? r : min((int)(bits >> 20), 0x7fc);   // infinity 7f8, quiet NaNs 7fc
}

// The largest of both halves over the wave.
__device__ __forceinline__ uint32_t wave_max2(uint32_t v) {
  typedef uint16_t us2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    const uint32_t u = (uint32_t)__shfl_xor((int)v, o, 64);
    v = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, v),
                                                               __builtin_bit_cast(us2, u)));
  }
  return v;
}

// Four elements, those below n.  Tensors may be views that start at any element: a 4-, 8-
// or 16-byte access need not lie on as many bytes.
template <class T>
__device__ __forceinline__ auto adamw_load4(const T* p, size_t i, size_t n) {
  typedef T V __attribute__((ext_vector_type(4)));
  typedef T Any __attribute__((ext_vector_type(4), aligned(sizeof(T))));
  V v = {0, 0, 0, 0};
  if (i + 4 <= n) {
    v = *reinterpret_cast<const Any*>(p + i);
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (i + e < n) v[e] = p[i + e];
  }
  return v;
}
template <class T, class V>
__device__ __forceinline__ void adamw_store4(T* p, size_t i, size_t n, V v) {
  typedef T Any __attribute__((ext_vector_type(4), aligned(sizeof(T))));
  if (i + 4 <= n) {
    *reinterpret_cast<Any*>(p + i) = v;
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (i + e < n) p[i + e] = v[e];
  }
}

typedef uint8_t b4 __attribute__((ext_vector_type(4)));
typedef u16 h4 __attribute__((ext_vector_type(4)));

template <bool BYTES, int U>
__global__ __launch_bounds__(256) void adamw_kernel(AdamwStep b) {
  typedef typename std::conditional<BYTES, uint8_t, float>::type S;
  typedef typename std::conditional<BYTES, b4, f4>::type S4;
  const int blk = blockIdx.x;
  int ti = -1;                               // the last tensor whose blocks start by blk
  const int* block0 = (const int*)b.plan;
  for (int i = 0; i < b.count; i += 64) {
    const int at = i + (threadIdx.x & 63);
    ti += __popcll(__ballot(at < b.count && block0[min(at, b.count - 1)] <= blk));
  }
  ti = __builtin_amdgcn_readfirstlane(ti);
  // (Constant memory to the compiler: the tensor's entry then loads into scalars.)
  typedef const __attribute__((address_space(4))) AdamwTensor* Entry;
  const auto& t = ((Entry)(uintptr_t)(b.plan + plan_tensors(b.count)))[ti];
  const size_t n = t.n;
  const size_t base = (size_t)(blk - t.block0) * (1024 * U) + threadIdx.x * 4;
  const S *m = (const S*)t.m, *v = (const S*)t.v;
  f4 w4[U], g4[U];
  S4 m4[U], v4[U];
  int mtop[U], vtop[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const size_t i = base + u * 1024;
    g4[u] = adamw_load4<float>(t.g, i, n);
    m4[u] = adamw_load4<S>(m, i, n);
    v4[u] = adamw_load4<S>(v, i, n);
    w4[u] = adamw_load4<float>(t.w, i, n);
    if constexpr (BYTES) {
      mtop[u] = i < n ? t.m_top[i / 256] : 0;
      vtop[u] = i < n ? t.v_top[i / 256] : 0;
    }
  }
  float rate = b.rate, vscale = b.vscale;
  const float keep = (float)(1.0 - b.lr * (double)t.decay);
  uint32_t step = (uint32_t)b.step;
  if (b.steps_done) {
    step = (uint32_t)max(1, b.step + *b.steps_done);
    rate = (float)(b.lr / (1.0 - int_power(b.beta1, step)));
    vscale = (float)(1.0 / sqrt(1.0 - int_power(b.beta2, step)));
  }
  const uint32_t key = mix32(b.seed + step * 0x9e3779b9u);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const size_t i = base + u * 1024;
    if (i - threadIdx.x % 64 * 4 >= n) return;   // whole waves leave together
    f4 nm, nv, nw;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma clang fp contract(off)
      float om, ov;
      if constexpr (BYTES) {
        const int mc = m4[u][e] & 127, vc = v4[u][e];
        om = rank_value(mc ? mtop[u] + mc - 127 : 0);
        om = m4[u][e] > 127 ? -om : om;
        ov = rank_value(vc ? vtop[u] + vc - 255 : 0);
      } else {
        om = m4[u][e];
        ov = v4[u][e];
      }
      const float g = g4[u][e] * t.scale;
      nm[e] = om * b.b1 + g * b.c1;
      nv[e] = ov * b.b2 + (g * g) * b.c2;
      if (b.fast)
        nw[e] = w4[u][e] * keep -
                rate * (nm[e] * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(nv[e]) * vscale + b.eps));
      else
        nw[e] = w4[u][e] * keep - rate * (nm[e] / (sqrtf(nv[e]) * vscale + b.eps));
    }
    adamw_store4<float>(t.w, i, n, nw);
    if (t.copy) {
      h4 c;
#pragma unroll
      for (int e = 0; e < 4; ++e) c[e] = f32_to_bf16(nw[e]);
      adamw_store4<u16>(t.copy, i, n, c);
    }
    if constexpr (!BYTES) {
      adamw_store4<float>((float*)t.m, i, n, nm);
      adamw_store4<float>((float*)t.v, i, n, nv);
    } else {
      const uint64_t at = t.first + i;       // its lower half may carry among the four
      const uint32_t lo = (uint32_t)at, hi = (uint32_t)(at >> 32);
      const uint32_t key0 = key ^ hi * 0x9e3779b9u, key1 = key ^ (hi + 1) * 0x9e3779b9u;
      int mr[4], vr[4];
      uint32_t top = 0;                      // m's largest rank above v's
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t h = mix32((lo + e) ^ (lo + e < lo ? key1 : key0));
        mr[e] = rank_of(__float_as_uint(nm[e]) & 0x7fffffffu, h & 0xffffu);
        vr[e] = rank_of(__float_as_uint(nv[e]) & 0x7fffffffu, h >> 16);
        if (i + e >= n) mr[e] = vr[e] = 0;
      }
      top = (uint32_t)max(max(mr[0], mr[1]), max(mr[2], mr[3])) << 16 |
            (uint32_t)max(max(vr[0], vr[1]), max(vr[2], vr[3]));
      top = wave_max2(top);
      const int mt = (int)(top >> 16), vt = (int)(top & 0xffffu);
      b4 mb, vb;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int mc = max(mr[e] - mt + 127, 0), vc = max(vr[e] - vt + 255, 1);
        mb[e] = (uint8_t)(mc | (mc > 0 && nm[e] < 0.f ? 128 : 0));
        vb[e] = (uint8_t)(nv[e] == 0.f ? 0 : vc);
      }
      adamw_store4<uint8_t>((uint8_t*)t.m, i, n, mb);
      adamw_store4<uint8_t>((uint8_t*)t.v, i, n, vb);
      if (threadIdx.x % 64 == 0) {
        t.m_top[i / 256] = (int16_t)mt;
        t.v_top[i / 256] = (int16_t)vt;
      }
    }
  }
}

__global__ void adamw_advance_kernel(int32_t* steps_done) { *steps_done += 1; }

// Four bytes of both moments a lane; a wave has one block's 256.
__global__ __launch_bounds__(256) void adamw_unpack_kernel(size_t n, const uint8_t* __restrict__ m,
                                                           const int16_t* __restrict__ m_top,
                                                           const uint8_t* __restrict__ v,
                                                           const int16_t* __restrict__ v_top,
                                                           float* __restrict__ m_out,
                                                           float* __restrict__ v_out) {
  const size_t i = (size_t)blockIdx.x * 1024 + threadIdx.x * 4;
  if (i >= n) return;
  if (m_out) {
    const b4 c = adamw_load4<uint8_t>(m, i, n);
    const int top = m_top[i / 256];
    f4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = rank_value((c[e] & 127) ? top + (c[e] & 127) - 127 : 0);
      o[e] = c[e] > 127 ? -x : x;
    }
    adamw_store4<float>(m_out, i, n, o);
  }
  if (v_out) {
    const b4 c = adamw_load4<uint8_t>(v, i, n);
    const int top = v_top[i / 256];
    f4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = rank_value(c[e] ? top + c[e] - 255 : 0);
    adamw_store4<float>(v_out, i, n, o);
  }
}

}  // namespace sb

namespace {

struct Range {
  uintptr_t at, end;
  bool out;
};

// Whether an output's range meets another one.  Sorted by their starts, a range
// meets an earlier one exactly if it starts before the furthest end so far.
bool outputs_meet(Range* r, int count) {
  std::sort(r, r + count, [](const Range& a, const Range& b) { return a.at < b.at; });
  uintptr_t in_end = 0, out_end = 0;
  for (int i = 0; i < count; ++i) {
    if (r[i].at < out_end || (r[i].out && r[i].at < in_end)) return true;
    uintptr_t& end = r[i].out ? out_end : in_end;
    end = std::max(end, r[i].end);
  }
  return false;
}

bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

}  // namespace

extern "C" size_t sb_adamw_plan_bytes(int count) {
  if (count < 1 || count > SB_ADAMW_MAX_TENSORS) return 0;
  return sb::plan_tensors(count) + (size_t)count * sizeof(sb::AdamwTensor);
}

extern "C" sb_status sb_adamw_make_plan(int moments, int count, const sb_adamw_tensor* tensors,
                                        void* plan, size_t plan_bytes, sb_adamw_plan* info,
                                        void* stream) {
  if (!tensors || !plan || !info || count < 1 || count > SB_ADAMW_MAX_TENSORS)
    return SB_ERR_INVALID_ARG;
  if ((moments != 8 && moments != 32) || !aligned(plan, 16)) return SB_ERR_INVALID_ARG;
  const size_t need = sb_adamw_plan_bytes(count);
  const bool bytes = moments == 8;
  Range r[7 * SB_ADAMW_MAX_TENSORS + 1];
  int ranges = 0;
  auto add = [&](const void* p, size_t size, bool out) {
    r[ranges++] = Range{(uintptr_t)p, (uintptr_t)p + size, out};
  };
  add(plan, need, true);
  size_t total = 0;
  int used = 0;
  for (int i = 0; i < count; ++i) {
    const sb_adamw_tensor& t = tensors[i];
    if (!std::isfinite(t.grad_scale) || !std::isfinite(t.decay)) return SB_ERR_INVALID_ARG;
    if (t.n == 0) continue;
    if (!t.w || !t.g || !t.m || !t.v || t.n >= (1ull << 40)) return SB_ERR_INVALID_ARG;
    if (!aligned(t.w, 4) || !aligned(t.g, 4) || !aligned(t.copy, 2)) return SB_ERR_INVALID_ARG;
    const size_t tops = (t.n + SB_ADAMW_BLOCK - 1) / SB_ADAMW_BLOCK;
    if (bytes) {
      if (!t.m_top || !t.v_top || !aligned(t.m_top, 2) || !aligned(t.v_top, 2))
        return SB_ERR_INVALID_ARG;
      add(t.m_top, tops * 2, true);
      add(t.v_top, tops * 2, true);
    } else if (!aligned(t.m, 4) || !aligned(t.v, 4)) {
      return SB_ERR_INVALID_ARG;
    }
    add(t.w, t.n * 4, true);
    add(t.g, t.n * 4, false);
    add(t.m, t.n * (bytes ? 1 : 4), true);
    add(t.v, t.n * (bytes ? 1 : 4), true);
    if (t.copy) add(t.copy, t.n * 2, true);
    ++used;
    total += t.n;
    // (A launch has fewer than 2^32 lanes, each of four elements or eight.)
    if (total >= (1ull << 33)) return SB_ERR_UNSUPPORTED;
  }
  if (outputs_meet(r, ranges)) return SB_ERR_INVALID_ARG;
  if (plan_bytes < need) return SB_ERR_WORKSPACE;
  sb::AdamwChunk c{};
  c.total = used;
  const int groups = bytes && total >= sb::kAdamwMany ? sb::kAdamwGroups : 1;
  const size_t block = 1024 * (size_t)groups;
  int64_t blocks = 0;
  for (int i = 0; i <= count; ++i) {
    if (c.count == sb::kAdamwChunk || (i == count && c.count)) {
      sb::adamw_plan_kernel<<<1, 64, 0, sbh::stream_of(stream)>>>(c, (char*)plan);
      const sb_status s = sbh::launch_status();
      if (s != SB_OK) return s;
      c.first += c.count;
      c.count = 0;
    }
    if (i == count) break;
    const sb_adamw_tensor& t = tensors[i];
    if (t.n == 0) continue;
    sb::AdamwTensor& o = c.t[c.count++];
    o.w = t.w; o.copy = (sb::u16*)t.copy; o.g = t.g; o.m = t.m; o.v = t.v;
    o.m_top = t.m_top; o.v_top = t.v_top; o.first = t.first; o.n = t.n;
    o.scale = t.grad_scale; o.decay = t.decay;
    o.block0 = (int)blocks;
    blocks += (int64_t)((t.n + block - 1) / block);
  }
  *info = sb_adamw_plan{used, moments, groups, (int)blocks};
  return SB_OK;
}

extern "C" sb_status sb_adamw_update(const sb_adamw_desc* d, const sb_adamw_plan* info,
                                     const void* plan, const int32_t* steps_done, void* stream) {
  if (!d || !info || !plan || !aligned(plan, 16)) return SB_ERR_INVALID_ARG;
  if (info->tensors < 0 || info->tensors > SB_ADAMW_MAX_TENSORS ||
      info->blocks < info->tensors || (info->tensors == 0 && info->blocks != 0) ||
      (info->moments != 8 && info->moments != 32) ||
      (info->groups != 1 && (info->groups != sb::kAdamwGroups || info->moments != 8)))
    return SB_ERR_INVALID_ARG;
  if (!std::isfinite(d->lr) || !std::isfinite(d->eps) || !(d->eps >= 0.0)) return SB_ERR_INVALID_ARG;
  if (!(d->beta1 >= 0.0 && d->beta1 < 1.0) || !(d->beta2 >= 0.0 && d->beta2 < 1.0))
    return SB_ERR_INVALID_ARG;
  if (d->step < 1 || !aligned(steps_done, 4)) return SB_ERR_INVALID_ARG;
  const double lr1 = d->lr / (1.0 - sb::int_power(d->beta1, (uint32_t)d->step));
  const double vs = 1.0 / std::sqrt(1.0 - sb::int_power(d->beta2, (uint32_t)d->step));
  if (!std::isfinite((float)lr1) || !std::isfinite((float)vs)) return SB_ERR_INVALID_ARG;
  if (info->blocks == 0) return SB_OK;
  sb::AdamwStep b{};
  b.plan = (const char*)plan;
  b.steps_done = steps_done;
  b.lr = d->lr; b.beta1 = d->beta1; b.beta2 = d->beta2;
  b.b1 = (float)d->beta1; b.c1 = (float)(1.0 - d->beta1);
  b.b2 = (float)d->beta2; b.c2 = (float)(1.0 - d->beta2);
  b.eps = (float)d->eps; b.rate = (float)lr1; b.vscale = (float)vs;
  b.seed = d->seed; b.step = d->step; b.count = info->tensors;
  b.fast = sb::fast_root(b.eps, d->beta2);
  const auto kernel = info->moments == 32 ? sb::adamw_kernel<false, 1>
                      : info->groups == 1 ? sb::adamw_kernel<true, 1>
                                          : sb::adamw_kernel<true, sb::kAdamwGroups>;
  kernel<<<(unsigned)info->blocks, 256, 0, sbh::stream_of(stream)>>>(b);
  return sbh::launch_status();
}

extern "C" sb_status sb_adamw_advance(int32_t* steps_done, void* stream) {
  if (!steps_done || !aligned(steps_done, 4)) return SB_ERR_INVALID_ARG;
  sb::adamw_advance_kernel<<<1, 1, 0, sbh::stream_of(stream)>>>(steps_done);
  return sbh::launch_status();
}

extern "C" sb_status sb_adamw_unpack(size_t n, const uint8_t* m, const int16_t* m_top,
                                     const uint8_t* v, const int16_t* v_top, float* m_out,
                                     float* v_out, void* stream) {
  if (n == 0) return SB_OK;
  if (n >= (1ull << 40)) return SB_ERR_INVALID_ARG;
  if (n >= (1ull << 34)) return SB_ERR_UNSUPPORTED;   // a launch has fewer than 2^32 lanes
  if ((m_out && (!m || !m_top)) || (v_out && (!v || !v_top))) return SB_ERR_INVALID_ARG;
  if (!aligned(m_out, 4) || !aligned(v_out, 4) || !aligned(m_top, 2) || !aligned(v_top, 2))
    return SB_ERR_INVALID_ARG;
  if (!m_out && !v_out) return SB_OK;
  const size_t tops = (n + SB_ADAMW_BLOCK - 1) / SB_ADAMW_BLOCK * 2;
  const void* in[4] = {m_out ? m : nullptr, m_out ? m_top : nullptr, v_out ? v : nullptr,
                       v_out ? v_top : nullptr};
  const size_t inb[4] = {n, tops, n, tops};
  for (int i = 0; i < 4; ++i)
    if (sbh::overlaps(m_out, n * 4, in[i], inb[i]) || sbh::overlaps(v_out, n * 4, in[i], inb[i]))
      return SB_ERR_INVALID_ARG;
  if (sbh::overlaps(m_out, n * 4, v_out, n * 4)) return SB_ERR_INVALID_ARG;
  sb::adamw_unpack_kernel<<<(unsigned)((n + 1023) / 1024), 256, 0, sbh::stream_of(stream)>>>(
      n, m, m_top, v, v_top, m_out, v_out);
  return sbh::launch_status();
}
