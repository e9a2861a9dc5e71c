// slot_sort.hpp -- slots sorted by a small whole number, stable: ids of tokens
// (the embedding's gradient), experts of routed tokens.
//
// Up to kSortSmall slots one launch finds each slot's place by counting: with key and slot
// in one 32-bit number no two are equal, and a slot's place is how many are smaller.  A
// block has 16 to 64 slots (so that some 256 blocks have them all), and its 16 waves share out
// the numbers that they are compared with: two instructions for 64 pairs.  (A radix sort by
// one block took 17 us for 4099 slots of 14 bits, alone on its CU.)
//
// More slots go through a radix sort from the lowest digit up, digits of up to 10 bits, so
// that experts take one pass and vocabularies two.  They are cut into at most 64 tiles: a
// launch counts each tile's digits, the next finds where each tile's share of a digit
// starts (from all counts) and moves the slots there.  Among the 64 slots of a wave the
// rank of a slot among its equals comes from ballots of the digit's bits: any skew of
// the ids costs the same.  No atomic decides an order: results are the same in every run.
#pragma once

#include "rows.hpp"

namespace sb {

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kSortRounds = 4;                             // slots a thread has at once
constexpr int kSortStep = kSortThreads * kSortRounds;      // slots a block ranks at once
constexpr int kSortBins = 1024;
constexpr int kSortTiles = 64;
// Slots up to which pairs are counted, with digits to sort by in two passes and more, and in
// one: 16384 ids of 15 bits take 21 us that way, the four launches 21 and what lies between
// them; 8192 slots of 8 experts 11, the two launches 7.8, 5331 slots 6.6.
constexpr int kSortSmall = 16384, kSortSmallOnePass = 6144;

// What is sorted: the keys are ids - first; ids outside [first, first + keys) have
// the key `keys` and come last.
struct SortIn {
  const int32_t* ids;
  int first;
  uint32_t keys;
  int n;
  int bits, slot_bits;         // of the largest key, of the largest slot
  int passes, digit;           // digit: bits of a pass
  int tile, tiles;             // slots of a tile; 0 tiles: counted in one launch
};

// One pass over tiles; in: NULL for the first (ids, slots in their order).
struct SortPass {
  const uint2* in;             // key, slot
  uint2* out;                  // NULL: place instead (the last pass may)
  int32_t* place;              // of each slot, -1 for the last key
  int32_t* offsets;            // [keys + 1], or NULL (one pass only)
  uint32_t* counts;            // [tiles][bins]
  int shift;
};

// Zeros that other blocks write beside the sort in one launch.
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
  s.bits = s.slot_bits = 1;
  while ((s.keys >> s.bits) != 0) ++s.bits;
  while ((n >> s.slot_bits) != 0) ++s.slot_bits;
  s.passes = cdiv(s.bits, 10);
  s.digit = cdiv(s.bits, s.passes);
  if (n <= (s.passes > 1 ? kSortSmall : kSortSmallOnePass) && s.bits + s.slot_bits <= 32) return s;
  s.tiles = n <= kSortStep * kSortTiles ? cdiv(n, kSortStep) : kSortTiles;
  s.tile = (int)round_up((size_t)cdiv(n, s.tiles), (size_t)kSortStep);
  s.tiles = cdiv(n, s.tile);
  return s;
}
inline size_t sort_count_bytes(const SortIn& s) {
  return (size_t)s.tiles * sizeof(uint32_t) << s.digit;
}
__device__ __forceinline__ uint32_t sort_key(const SortIn& s, int id) {
  const uint32_t key = (uint32_t)id - (uint32_t)s.first;
  return id >= s.first && key < s.keys ? key : s.keys;
}
// Slots at, at + step, ...; past the end the last one.  All loads are on their way at once.
template <int R>
__device__ __forceinline__ void sort_load(const SortIn& s, const uint2* in, int at, int step,
                                          int end, uint2* v) {
  if (in) {
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = in[min(at + r * step, end - 1)];
    return;
  }
  int id[R];
#pragma unroll
  for (int r = 0; r < R; ++r) id[r] = s.ids[min(at + r * step, end - 1)];
#pragma unroll
  for (int r = 0; r < R; ++r)
    v[r] = uint2{sort_key(s, id[r]), (uint32_t)min(at + r * step, end - 1)};
}

// Counts of the digits of slots i0 .. i1 - 1 into h.base (zero before).
__device__ __forceinline__ void sort_count(const SortIn& s, const SortPass& p, int i0, int i1,
                                           SortShared& h) {
  const uint32_t mask = (1u << s.digit) - 1;
  for (int at = i0 + threadIdx.x; at < i1; at += kSortStep) {
    uint2 v[kSortRounds];
    sort_load<kSortRounds>(s, p.in, at, kSortThreads, i1, v);
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
      if (at + r * kSortThreads < i1) atomicAdd(&h.base[v[r].x >> p.shift & mask], 1u);
  }
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

// For each round: the wave's lanes that are live and have this lane's digit.
__device__ __forceinline__ void sort_same(const uint32_t* d, const bool* live, int bits,
                                          uint64_t* same) {
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) same[r] = __ballot(live[r]);
#pragma unroll 1
  for (int b = 0; b < bits; ++b) {
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {         // (side by side: one after another waits)
      const uint32_t one = d[r] >> b & 1;
      const uint64_t ones = __ballot(one != 0);
      const uint32_t zero = one - 1;                // all bits where this lane's is 0
      const uint32_t lo = (uint32_t)same[r] & ((uint32_t)ones ^ zero);
      const uint32_t hi = (uint32_t)(same[r] >> 32) & ((uint32_t)(ones >> 32) ^ zero);
      same[r] = (uint64_t)hi << 32 | lo;
    }
  }
}
// The slot's rank among the wave's slots with its digit: those of this round before it, and
// those counted in `count` (where its own are added).
__device__ __forceinline__ uint32_t sort_rank(u16* count, uint32_t d, bool live, uint64_t same,
                                              int lane) {
  const uint32_t before = __popcll(same & ((1ull << lane) - 1));
  const uint32_t old = live ? count[d] : 0;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  if (live && before == 0) count[d] = (u16)(old + __popcll(same));
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  return old + before;
}

// Each wave's counts of a digit become where its share starts among the block's; their
// sum.  For threads below the number of digits.
__device__ __forceinline__ uint32_t sort_share(SortShared& h) {
  uint32_t c[kSortWaves], total = 0;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) c[w] = h.count[w][threadIdx.x];
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) {
    h.count[w][threadIdx.x] = (u16)total;
    total += c[w];
  }
  return total;
}

__device__ __forceinline__ void sort_clear(SortShared& h, int digit) {
  uint32_t* words = reinterpret_cast<uint32_t*>(h.count);
  const uint32_t half = 1u << (digit - 1);             // words of a wave's counts
  for (uint32_t q = threadIdx.x; q < kSortWaves * half; q += kSortThreads)
    words[(q >> (digit - 1)) * (kSortBins / 2) + (q & (half - 1))] = 0;
}

// Slots i0 .. i1 - 1 to their places, from h.base on for each digit.
__device__ __forceinline__ void sort_move(const SortIn& s, const SortPass& p, int i0, int i1,
                                          SortShared& h) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t bins = 1u << s.digit;
  for (int at = i0; at < i1; at += kSortStep) {
    uint2 v[kSortRounds];
    uint32_t rank[kSortRounds];
    bool live[kSortRounds];
    const int first = at + wave * (64 * kSortRounds) + lane;
    sort_load<kSortRounds>(s, p.in, first, 64, i1, v);
    sort_clear(h, s.digit);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) live[r] = first + r * 64 < i1;
    uint32_t d[kSortRounds];
    uint64_t same[kSortRounds];
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) d[r] = v[r].x >> p.shift & (bins - 1);
    sort_same(d, live, s.digit, same);
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
      rank[r] = sort_rank(h.count[wave], d[r], live[r], same[r], lane);
    __syncthreads();
    uint32_t total = 0;
    if (threadIdx.x < bins) total = sort_share(h);
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

// Places of 2 I slots among up to 1024 R, by counting: of slots block * 2 I .., and behind
// the slots, with `offsets`, of the first slot that each key could have.  A wave's numbers lie
// in LDS; 64 / I lanes have the same two slots and every (64 / I)-th four of the numbers.
template <int I, int R>
__device__ __forceinline__ void sort_by_count(const SortIn& s, int32_t* place, int32_t* offsets,
                                              uint2* out, int block, u4 (*numbers)[16 * R],
                                              uint32_t (*share)[2][64]) {
  constexpr int PARTS = 64 / I;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int rounds = (s.n + kSortThreads - 1) / kSortThreads;     // at most R
  uint32_t mine[2], key[2], below[2] = {0, 0};
  int q[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) q[h] = block * 2 * I + h * I + lane % I;
  uint32_t all[R];
  int id[2] = {0, 0};
  if (s.n > 0) {
    uint2 v[R];
#pragma unroll
    for (int h = 0; h < 2; ++h) id[h] = s.ids[min(q[h], s.n - 1)];
    sort_load<R>(s, nullptr, wave * rounds * 64 + lane, 64, s.n, v);
#pragma unroll
    for (int r = 0; r < R; ++r) all[r] = v[r].x << s.slot_bits | v[r].y;
  }
#pragma unroll
  for (int r = 0; r < R; ++r)                       // past the end: smaller than none
    if ((wave * rounds + r) * 64 + lane >= s.n) all[r] = ~0u;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    key[h] = q[h] < s.n ? sort_key(s, id[h]) : min((uint32_t)(q[h] - s.n), s.keys);
    mine[h] = key[h] << s.slot_bits | (q[h] < s.n ? q[h] : 0);
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (r < rounds) reinterpret_cast<uint32_t*>(numbers[wave])[r * 64 + lane] = all[r];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll 4
  for (int j = lane / I; j < 16 * rounds; j += PARTS) {
    const u4 k = numbers[wave][j];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) below[h] += k[e] < mine[h] ? 1 : 0;
  }
  share[wave][0][lane] = below[0];
  share[wave][1][lane] = below[1];
  __syncthreads();
  if (wave > 1 || lane >= I) return;
  uint32_t to = 0;                                  // wave h joins its slots
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w)
#pragma unroll
    for (int p = 0; p < PARTS; ++p) to += share[w][wave][p * I + lane];
  const int at = wave ? q[1] : q[0];
  const uint32_t its = wave ? key[1] : key[0];
  if (at < s.n) {
    if (place) place[at] = its < s.keys ? (int32_t)to : -1;
    else out[to] = uint2{its, (uint32_t)at};
  } else if (offsets && (uint32_t)(at - s.n) <= s.keys) {
    offsets[at - s.n] = (int32_t)to;
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

}  // namespace sb

namespace sbh {

// The sort's launches: the slots' places (and offsets, one pass only) where `place` is
// given, else keys and slots in order, in the buffer that is returned (a or b, n
// entries each; b where there are tiles and several passes).  counts: sort_count_bytes.
// Without tiles the launch has more blocks, which write `fill`; with tiles there is none.
const uint2* sort_slots(const sb::SortIn& s, int32_t* place, int32_t* offsets, uint2* a, uint2* b,
                        uint32_t* counts, const sb::Fill& fill, hipStream_t stream);

}  // namespace sbh
