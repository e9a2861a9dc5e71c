// slot_sort.hip -- the launches of slot_sort.hpp.
#include "slot_sort.hpp"

namespace sb {

constexpr int kFillBlocks = 512;       // two a CU of the size that the sort has

__global__ __launch_bounds__(kSortThreads) void slot_sort_small(SortIn s, uint2* a, uint2* b,
                                                                SortPass last, Fill fill) {
  __shared__ SortShared h;
  if (blockIdx.x == 0) sort_small(s, a, b, last, h);
  else fill_zero(fill, blockIdx.x - 1, gridDim.x - 1);
}

// counts[tile][digit] of one pass.
__global__ __launch_bounds__(kSortThreads) void slot_sort_count(SortIn s, SortPass p, Fill fill) {
  __shared__ SortShared h;
  const int tile = blockIdx.x;
  if (tile >= s.tiles) {
    fill_zero(fill, tile - s.tiles, gridDim.x - s.tiles);
    return;
  }
  const uint32_t bins = 1u << s.digit;
  if (threadIdx.x < bins) h.base[threadIdx.x] = 0;
  __syncthreads();
  sort_count(s, p, tile * s.tile, min(s.n, (tile + 1) * s.tile), h);
  __syncthreads();
  if (threadIdx.x < bins) p.counts[((size_t)tile << s.digit) + threadIdx.x] = h.base[threadIdx.x];
}

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
  const size_t quads = fill.n / 4 + 1;
  const int fills = fill.n == 0 ? 0
                    : (int)(quads < (size_t)sb::kFillBlocks * sb::kSortThreads
                                ? (quads + sb::kSortThreads - 1) / sb::kSortThreads
                                : (size_t)sb::kFillBlocks);
  sb::SortPass p{};
  p.place = place;
  p.offsets = offsets;
  p.counts = counts;
  if (s.tiles <= 1) {
    sb::slot_sort_small<<<1 + fills, sb::kSortThreads, 0, stream>>>(s, a, b, p, fill);
    return (s.passes - 1) % 2 ? b : a;
  }
  for (int pass = 0; pass < s.passes; ++pass) {
    p.in = p.out;
    p.out = pass + 1 == s.passes && place ? nullptr : pass % 2 ? b : a;
    p.shift = pass * s.digit;
    sb::slot_sort_count<<<s.tiles + (pass == 0 ? fills : 0), sb::kSortThreads, 0, stream>>>(s, p,
                                                                                            fill);
    sb::slot_sort_move<<<s.tiles, sb::kSortThreads, 0, stream>>>(s, p);
  }
  return p.out;
}

}  // namespace sbh
