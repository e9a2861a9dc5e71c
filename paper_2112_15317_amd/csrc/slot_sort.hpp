// slot_sort.hpp -- slots sorted by a small whole number, stable: ids of tokens
// (the embedding's gradient), experts of routed tokens.
//
// A radix sort from the lowest digit up, digits of up to 10 bits, so that experts
// take one pass and vocabularies two.  A pass counts each tile's digits, then every
// block finds where its tile's share of each digit starts (from all counts: at
// most 64 tiles) and moves its slots there in order.  Among the 64 slots of a wave the rank of a
// slot among its equals comes from ballots of the digit's bits: any skew of the
// ids costs the same.  No atomic decides an order, so results are the same in
// every run.  Up to kSortSmall slots one block does all passes in one launch.
#pragma once

#include "sb_internal.hpp"

namespace sb {

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kSortRounds = 4;                             // slots a thread has at once
constexpr int kSortStep = kSortThreads * kSortRounds;      // slots a block ranks at once
constexpr int kSortBins = 1024;
constexpr int kSortTiles = 64;
constexpr int kSortSmall = 8192;

// What is sorted: the keys are ids - first; ids outside [first, first + keys) have
// the key `keys` and come last.
struct SortIn {
  const int32_t* ids;
  int first;
  uint32_t keys;
  int n;
  int bits;                    // of the largest key
  int passes, digit;           // digit: bits of a pass
  int tile, tiles;             // slots of a tile
};

// One pass; in: NULL for the first (ids, slots in their order).
struct SortPass {
  const uint2* in;             // key, slot
  uint2* out;                  // NULL: place instead (the last pass may)
  int32_t* place;              // of each slot, -1 for the last key
  int32_t* offsets;            // [keys + 1], or NULL (one pass only)
  uint32_t* counts;            // [tiles][bins]
  int shift;
};

// Zeros that other blocks of a launch write beside the sort.
struct Fill {
  float* p;
  size_t n;
};

struct SortShared {
  u16 count[kSortWaves][kSortBins];   // of a step, then where a wave's share starts in it
  uint32_t base[kSortBins];           // where the next slot of a digit goes
  uint32_t wave_sum[kSortWaves];
};

inline SortIn sort_plan(const int32_t* ids, int first, int keys, int n) {
  SortIn s{};
  s.ids = ids;
  s.first = first;
  s.keys = (uint32_t)keys;
  s.n = n;
  s.bits = 1;
  while ((s.keys >> s.bits) != 0) ++s.bits;
  s.passes = cdiv(s.bits, 10);
  s.digit = cdiv(s.bits, s.passes);
  s.tiles = n <= kSortSmall ? 1 : n <= kSortStep * kSortTiles ? cdiv(n, kSortStep) : kSortTiles;
  s.tile = n <= kSortSmall ? kSortSmall
                           : (int)round_up((size_t)cdiv(n, s.tiles), (size_t)kSortStep);
  if (n > kSortSmall) s.tiles = cdiv(n, s.tile);
  return s;
}
inline size_t sort_count_bytes(const SortIn& s) {
  return s.tiles > 1 ? (size_t)s.tiles * sizeof(uint32_t) << s.digit : 0;
}

__device__ __forceinline__ uint2 sort_slot(const SortIn& s, const uint2* in, int i) {
  if (in) return in[i];
  const int id = s.ids[i];
  const uint32_t key = (uint32_t)id - (uint32_t)s.first;
  return uint2{id >= s.first && key < s.keys ? key : s.keys, (uint32_t)i};
}

// Counts of the digits of slots i0 .. i1 - 1 into h.base (zero before).
__device__ __forceinline__ void sort_count(const SortIn& s, const SortPass& p, int i0, int i1,
                                           SortShared& h) {
  const uint32_t mask = (1u << s.digit) - 1;
  for (int i = i0 + threadIdx.x; i < i1; i += kSortThreads)
    atomicAdd(&h.base[sort_slot(s, p.in, i).x >> p.shift & mask], 1u);
}

// The sum of v over the threads before this one.
__device__ __forceinline__ uint32_t sort_before(uint32_t v, SortShared& h) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t incl = v;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const uint32_t t = __shfl_up(incl, o, 64);
    if (lane >= o) incl += t;
  }
  if (lane == 63) h.wave_sum[wave] = incl;
  __syncthreads();
  uint32_t start = 0;
  for (int w = 0; w < wave; ++w) start += h.wave_sum[w];
  __syncthreads();
  return start + incl - v;
}

// Slots i0 .. i1 - 1 to their places, from h.base on for each digit.
__device__ __forceinline__ void sort_move(const SortIn& s, const SortPass& p, int i0, int i1,
                                          SortShared& h) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t bins = 1u << s.digit;
  for (int at = i0; at < i1; at += kSortStep) {
    for (uint32_t q = threadIdx.x; q < kSortWaves * bins; q += kSortThreads)
      h.count[q >> s.digit][q & (bins - 1)] = 0;
    __syncthreads();
    uint2 v[kSortRounds];
    uint32_t d[kSortRounds], rank[kSortRounds];
    bool live[kSortRounds];
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
      const int i = at + wave * (64 * kSortRounds) + r * 64 + lane;
      live[r] = i < i1;
      v[r] = live[r] ? sort_slot(s, p.in, i) : uint2{0, 0};
      d[r] = v[r].x >> p.shift & (bins - 1);
    }
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
      uint64_t same = __ballot(live[r]);
      for (int b = 0; b < s.digit; ++b) {
        const bool one = (d[r] >> b & 1) != 0;
        const uint64_t ones = __ballot(one);
        same &= one ? ones : ~ones;
      }
      const uint32_t before = __popcll(same & ((1ull << lane) - 1));
      const uint32_t old = live[r] ? h.count[wave][d[r]] : 0;
      rank[r] = old + before;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (live[r] && before == 0) h.count[wave][d[r]] = (u16)(old + __popcll(same));
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    uint32_t total = 0;
    if (threadIdx.x < bins) {
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t c = h.count[w][threadIdx.x];
        h.count[w][threadIdx.x] = (u16)total;
        total += c;
      }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
      if (!live[r]) continue;
      const uint32_t to = h.base[d[r]] + h.count[wave][d[r]] + rank[r];
      if (p.out) p.out[to] = v[r];
      else p.place[v[r].y] = v[r].x < s.keys ? (int32_t)to : -1;
    }
    __syncthreads();
    if (threadIdx.x < bins) h.base[threadIdx.x] += total;
    __syncthreads();
  }
}

// Zeros over blocks `block` of `blocks`, 16 bytes a lane at any multiple of 4.
__device__ __forceinline__ void fill_zero(const Fill& f, size_t block, size_t blocks) {
  typedef f4 f4_at4 __attribute__((aligned(4)));
  const size_t quads = f.n / 4, step = blocks * blockDim.x;
  const f4 zero = f4{0.f, 0.f, 0.f, 0.f};
  for (size_t q = block * blockDim.x + threadIdx.x; q < quads; q += step)
    *reinterpret_cast<f4_at4*>(f.p + q * 4) = zero;
  if (block == 0 && threadIdx.x < f.n % 4) f.p[quads * 4 + threadIdx.x] = 0.f;
}

// All passes of up to kSortSmall slots, in block 0; between the passes the slots lie
// in `a` and `b` in turn.
__device__ __forceinline__ void sort_small(const SortIn& s, uint2* a, uint2* b,
                                           const SortPass& last, SortShared& h) {
  const uint32_t bins = 1u << s.digit;
  const uint2* in = nullptr;
  for (int pass = 0; pass < s.passes; ++pass) {
    SortPass p = last;
    p.in = in;
    p.shift = pass * s.digit;
    p.out = pass + 1 == s.passes && last.place ? nullptr : pass % 2 ? b : a;
    if (threadIdx.x < bins) h.base[threadIdx.x] = 0;
    __syncthreads();
    sort_count(s, p, 0, s.n, h);
    __syncthreads();
    const uint32_t c = threadIdx.x < bins ? h.base[threadIdx.x] : 0;
    const uint32_t start = sort_before(c, h);
    if (threadIdx.x < bins) h.base[threadIdx.x] = start;
    if (p.offsets && threadIdx.x <= s.keys) p.offsets[threadIdx.x] = (int32_t)start;
    __syncthreads();
    sort_move(s, p, 0, s.n, h);
    in = p.out;
    __threadfence_block();
    __syncthreads();
  }
}

}  // namespace sb

namespace sbh {

// The sort's launches: the slots' places (and offsets, one pass only) where `place` is
// given, else keys and slots in order, in the buffer that is returned (a or b, n
// entries each).  counts: sort_count_bytes.  The first launch writes `fill` beside.
const uint2* sort_slots(const sb::SortIn& s, int32_t* place, int32_t* offsets, uint2* a, uint2* b,
                        uint32_t* counts, const sb::Fill& fill, hipStream_t stream);

}  // namespace sbh
