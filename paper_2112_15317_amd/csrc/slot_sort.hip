// slot_sort.hip -- the launches of slot_sort.hpp.
#include "slot_sort.hpp"

namespace sb {

constexpr int kFillBlocks = 512;       // two a CU of the size that the sort has

// Loads and the launch bound it for few slots, pairs for many: 32 slots of 8 experts 2.8 us, 4096
// ids 4.8 (8 to 9 beside 37 MB of zeros), 5331 slots of 11 experts 6.6, 16384 ids 21.
template <int I, int R>
__global__ __launch_bounds__(kSortThreads) void slot_sort_small(SortIn s, int32_t* place,
                                                                int32_t* offsets, uint2* out,
                                                                int blocks, Fill fill) {
  __shared__ u4 numbers[kSortWaves][16 * R];
  __shared__ uint32_t share[kSortWaves][2][64];
  if ((int)blockIdx.x < blocks)
    sort_by_count<I, R>(s, place, offsets, out, blockIdx.x, numbers, share);
  else
    fill_zero(fill, blockIdx.x - blocks, gridDim.x - blocks);
}

// counts[tile][digit] of one pass.  2.4 to 5 us for 8192 to 262144 slots, loads and launch.
__global__ __launch_bounds__(kSortThreads) void slot_sort_count(SortIn s, SortPass p) {
  __shared__ SortShared h;
  const int tile = blockIdx.x;
  const uint32_t bins = 1u << s.digit;
  if (threadIdx.x < bins) h.base[threadIdx.x] = 0;
  __syncthreads();
  sort_count(s, p, tile * s.tile, min(s.n, (tile + 1) * s.tile), h);
  __syncthreads();
  if (threadIdx.x < bins) p.counts[((size_t)tile << s.digit) + threadIdx.x] = h.base[threadIdx.x];
}

// 5.2 us for 16384 slots of 8 experts, 8 for 65536 ids (9 bits) and 262144 slots: the chain of
// counts, keys, ranks and stores.
__global__ __launch_bounds__(kSortThreads) void slot_sort_move(SortIn s, SortPass p) {
  __shared__ SortShared h;
  const int tile = blockIdx.x;
  const uint32_t bins = 1u << s.digit;
  uint32_t all = 0, before = 0;
  if (threadIdx.x < bins) {
#pragma unroll 16
    for (int t = 0; t < s.tiles; ++t) {
      const uint32_t c = p.counts[((size_t)t << s.digit) + threadIdx.x];
      all += c;
      before += t < tile ? c : 0;
    }
  }
  const uint32_t start = sort_before(all, h);
  if (threadIdx.x < bins) h.base[threadIdx.x] = start + before;
  if (tile == 0 && p.offsets && threadIdx.x <= s.keys) p.offsets[threadIdx.x] = (int32_t)start;
  __syncthreads();
  sort_move(s, p, tile * s.tile, min(s.n, (tile + 1) * s.tile), h);
}

}  // namespace sb

namespace sbh {

const uint2* sort_slots(const sb::SortIn& s, int32_t* place, int32_t* offsets, uint2* a, uint2* b,
                        uint32_t* counts, const sb::Fill& fill, hipStream_t stream) {
  constexpr size_t per = 4 * sb::kSortThreads;
  if (s.tiles == 0) {
    const size_t want = (fill.n + per - 1) / per;
    const int queries = s.n + (offsets ? (int)s.keys + 1 : 0);
    const int fills = want < (size_t)sb::kFillBlocks ? (int)want : sb::kFillBlocks;
    if (queries + fills == 0) return a;
    auto launch = [&](auto slots, auto r) {
      constexpr int I = decltype(slots)::value, R = decltype(r)::value;
      const int sorts = sb::cdiv(queries, 2 * I);
      sb::slot_sort_small<I, R><<<sorts + fills, sb::kSortThreads, 0, stream>>>(
          s, place, offsets, a, sorts, fill);
    };
    using std::integral_constant;
    if (s.n <= 1024) launch(integral_constant<int, 8>(), integral_constant<int, 1>());
    else if (s.n <= 4096) launch(integral_constant<int, 8>(), integral_constant<int, 4>());
    else if (s.n <= 8192) launch(integral_constant<int, 16>(), integral_constant<int, 8>());
    else launch(integral_constant<int, 32>(), integral_constant<int, 16>());
    return a;
  }
  sb::SortPass p{};
  p.place = place;
  p.offsets = offsets;
  p.counts = counts;
  for (int pass = 0; pass < s.passes; ++pass) {
    p.in = p.out;
    p.out = pass + 1 == s.passes && place ? nullptr : pass % 2 ? b : a;
    p.shift = pass * s.digit;
    sb::slot_sort_count<<<s.tiles, sb::kSortThreads, 0, stream>>>(s, p);
    sb::slot_sort_move<<<s.tiles, sb::kSortThreads, 0, stream>>>(s, p);
  }
  return p.out;
}

}  // namespace sbh
