// embed.hip -- rows of a vocabulary shard's table for token ids, and the table's
// gradient.
//
// y[i] = scale * table[ids[i] - first], zero for ids of other shards and padding;
// dtable[v] = scale * sum of dy[i] over ids[i] = first + v.
//
// Both move rows and compute next to nothing: HBM bounds them.
//
// The gradient sorts the tokens by id (slot_sort.hpp), so that each row of the table
// is summed by one lane group in the tokens' order: no atomics, the same result in
// every run.  Words in use are few and some of them are in every sentence, so the
// work is split by sorted tokens, not by rows of the table: a group takes 8 to 64
// tokens in a row; an id's tokens that go past a group's end leave partial sums
// (fp32, at most two a group), which a last launch joins in order.  Rows are zeroed beside
// a sort of one launch (the first 48 MB, which the sort of 4099 ids does not wait for), and
// beside the sums those of the others that have no token: 65536 tokens of a table of 131072 x
// 2048 name a quarter of its rows, and zeroing these too would be a sixth of all traffic.
//
// Up to kFewTokens tokens it is one launch without a sort: a block has a token's columns,
// compares its id with all others, and where it is the first with that id sums all of them.
#include "rows.hpp"
#include "slot_sort.hpp"

#include <algorithm>
#include <cmath>

namespace sb {

// A lane group has up to U pieces a lane of a token's row.  HBM bounds it: 65536 rows of 2048
// bf16 from a table of 131072 (411 MB) in 71 to 89 us, 4.6 to 5.8 TB/s where a copy of 4 GiB
// reaches 4.7; 8 rows take the 2 us of a launch.
template <typename T, int U>
__global__ __launch_bounds__(256) void embed_fwd_kernel(RowPlan rp, int n, int first, int vocab,
                                                        int width, int ldy, float scale,
                                                        const T* __restrict__ table,
                                                        const int32_t* __restrict__ ids,
                                                        T* __restrict__ y) {
  constexpr int N = Piece<T>::N;
  const size_t group = ((size_t)blockIdx.x * 256 + threadIdx.x) >> rp.shift;
  const int lane = threadIdx.x & ((1 << rp.shift) - 1);
  const size_t i = group / (unsigned)rp.segs;
  if (i >= (size_t)n) return;
  const int c0 = (int)(group - i * rp.segs) * (U << rp.shift) + lane;
  const int id = ids[i];
  const bool inside = id >= first && (uint32_t)(id - first) < (uint32_t)vocab;
  const T* src = table + (size_t)(inside ? id - first : 0) * width;
  T* dst = y + i * (size_t)ldy;
  Piece<T> p[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + (u << rp.shift);
    p[u].raw = u4{0, 0, 0, 0};
    if (inside && c < rp.pieces) p[u].load(src + (size_t)c * N, width - c * N, width);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + (u << rp.shift);
    if (c >= rp.pieces) continue;
    if (inside) p[u].settle(width - c * N, width);
    if (inside && scale != 1.f) {
      float v[N];
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = p[u].get(e) * scale;
      p[u].set(v);
    }
    p[u].store(dst + (size_t)c * N, width - c * N);
  }
}

struct EmbedBwd {
  RowPlan rp;
  const uint2* slots;          // key, token, sorted; key `vocab`: not the shard's
  int n, vocab, width, ldy;
  int run, runs;               // sorted tokens of a group; groups along them
  int sum_blocks;
  int absent0;                 // first of the rows that are zeroed beside the sums
  float scale;
  int accumulate;
  float* dtable;
  float* part;                 // [runs][2][width]: of an id that began before, of one that goes on
};

// Where keys of at least `key` start among the slots from lo on: 64 probes at a time, one
// wave.
__device__ __forceinline__ int slot_from(const EmbedBwd& b, uint32_t key, int lo, int lane) {
  int hi = b.n;                                     // somewhere in lo .. hi
  while (lo < hi) {
    const int step = (hi - lo + 63) / 64, j = lo + lane * step;
    const int below = __popcll(__ballot(j < hi && b.slots[j].x < key));
    if (below == 0) return lo;
    const int last = lo + (below - 1) * step;       // below the key
    hi = min(hi, last + step);
    lo = last + 1;
  }
  return lo;
}

// A bit for each of the kAbsent rows that a lane's `at` names, over the wave.  (Sixteen: a
// wave with 64 rows of 741 held up a launch of 8 us for 26.)
constexpr int kAbsent = 16;
__device__ __forceinline__ uint32_t all_bits(uint32_t bits) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) bits |= __shfl_xor((int)bits, o, 64);
  return bits;
}
__device__ __forceinline__ uint32_t named_rows(uint32_t at) {
  return all_bits(at < kAbsent ? 1u << at : 0);
}

// Zeros in those of the kAbsent rows from v0 on that are not named; one wave.
__device__ __forceinline__ void zero_rows(const EmbedBwd& b, int v0, uint32_t named, int lane) {
  const int rows = min(b.vocab - v0, kAbsent), pieces = cdiv(b.width, 4);
  const int shift = pieces >= 64 ? 6 : 32 - __clz((pieces - 1) | 1);    // lanes of a row
  for (int at = lane >> shift; at < rows; at += 64 >> shift) {
    if (named >> at & 1) continue;
    for (int c = lane & ((1 << shift) - 1); c < pieces; c += 1 << shift) {
      Piece<float> p;
      p.raw = u4{0, 0, 0, 0};
      p.store(b.dtable + (size_t)(v0 + at) * b.width + c * 4, b.width - c * 4);
    }
  }
}

__device__ __forceinline__ void fill_absent(const EmbedBwd& b, int v0, int lane) {
  const int rows = min(b.vocab - v0, kAbsent);
  uint32_t named = 0;
  for (int j = slot_from(b, v0, 0, lane); j < b.n;) {
    const uint32_t key = j + lane < b.n ? b.slots[j + lane].x : ~0u;
    named |= named_rows(key - v0);
    const uint32_t first = __shfl((int)key, 0, 64), last = __shfl((int)key, 63, 64);
    if (last - v0 >= (uint32_t)rows) break;
    j = first == last ? slot_from(b, first + 1, j + 64, lane) : j + 64;
  }
  zero_rows(b, v0, named, lane);
}

// N columns of a row of the gradient from their sum.
template <int N>
__device__ __forceinline__ void give_row(const EmbedBwd& b, float* out, int left,
                                         const float* acc) {
#pragma unroll
  for (int q = 0; q < N; q += 4) {
    Piece<float> o;
    if (b.accumulate && left > q) {
      o.load(out + q, left - q, b.width);
      o.settle(left - q, b.width);
    }
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      v[e] = b.accumulate ? fmaf(acc[q + e], b.scale, o.get(e)) : acc[q + e] * b.scale;
    o.set(v);
    o.store(out + q, left - q);
  }
}

// Few tokens, up to 64 H: a block has a token's columns, the blocks behind those rows to zero.
// Every wave compares the token's id with all; where it is the first with that id, the waves
// take the others by sixteens in turn, eight rows on their way at once, and the first adds up.
// Latency bounds it; added to a table of 32000 x 2048, 128 tokens of bf16 take 3.2 us, as many of
// one id 7.4.  256 tokens of 741 columns of bf16 4.0 us where their ids differ, 15 where they are
// one; 257, by sorting in three launches, 15 and 13.  With a table of 12501 rows written whole 10
// and 18.5, and 17 and 17.  (512 added at once take 5.6 and 26, by sorting 17 and 19.)
constexpr int kFewTokens = 256;
template <typename T, int H>
__global__ __launch_bounds__(256) void embed_few_kernel(EmbedBwd b, int first, int segs,
                                                        const int32_t* __restrict__ ids,
                                                        const T* __restrict__ dy) {
  constexpr int N = Piece<T>::N, AHEAD = 8;
  __shared__ f4 quarter[3][N / 4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int units = b.n * segs;
  int id[H];
  uint32_t key[H];
#pragma unroll
  for (int h = 0; h < H; ++h) id[h] = b.n > 0 ? ids[min(h * 64 + lane, b.n - 1)] : -1;
#pragma unroll
  for (int h = 0; h < H; ++h) {
    const bool inside = id[h] >= first && (uint32_t)(id[h] - first) < (uint32_t)b.vocab;
    key[h] = inside && h * 64 + lane < b.n ? id[h] - first : ~0u;
  }
  if ((int64_t)blockIdx.x >= units) {
    const int64_t v0 = (((int64_t)blockIdx.x - units) * 4 + wave) * kAbsent;
    if (v0 >= b.vocab) return;
    uint32_t named = 0;
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const uint32_t at = key[h] - (uint32_t)v0;
      named |= at < kAbsent ? 1u << at : 0;
    }
    zero_rows(b, (int)v0, all_bits(named), lane);
    return;
  }
  const int i = blockIdx.x / segs, c = (int)(blockIdx.x - i * segs) * 64 + lane;
  const int left = b.width - c * N;
  uint32_t own = 0;
#pragma unroll
  for (int h = 0; h < H; ++h) own = i >> 6 == h ? key[h] : own;
  const uint32_t mine = __builtin_amdgcn_readlane(own, i & 63);
  if (mine == ~0u) return;
  uint64_t same[H];
  int head = 0, others = -1;                        // (the block's waves all find the same)
  bool found = false;
#pragma unroll
  for (int h = 0; h < H; ++h) {
    same[h] = __ballot(key[h] == mine);
    if (!found && same[h]) head = h * 64 + __ffsll((unsigned long long)same[h]) - 1;
    found = found || same[h] != 0;
    others += __popcll(same[h]);
  }
  if (head != i || (others == 0 && wave)) return;
  float acc[N];
#pragma unroll
  for (int e = 0; e < N; ++e) acc[e] = 0.f;
#pragma unroll
  for (int h = 0; h < H; ++h) {
    uint64_t left_over = others ? same[h] & 0xffffull << 16 * wave : same[h];
    while (left_over) {
      Piece<T> p[AHEAD];
      int j[AHEAD];
#pragma unroll
      for (int a = 0; a < AHEAD; ++a) {
        j[a] = left_over ? h * 64 + __ffsll((unsigned long long)left_over) - 1 : -1;
        left_over &= left_over - 1;
      }
#pragma unroll
      for (int a = 0; a < AHEAD; ++a) {
        p[a].raw = u4{0, 0, 0, 0};
        if (j[a] >= 0 && left > 0) p[a].load(dy + (size_t)j[a] * b.ldy + (size_t)c * N, left, b.width);
      }
#pragma unroll
      for (int a = 0; a < AHEAD; ++a)
        if (j[a] >= 0) {
          p[a].settle(left, b.width);
#pragma unroll
          for (int e = 0; e < N; ++e) acc[e] += p[a].get(e);
        }
    }
  }
  if (others) {
    if (wave)
#pragma unroll
      for (int q = 0; q < N / 4; ++q)
        quarter[wave - 1][q][lane] =
            f4{acc[q * 4], acc[q * 4 + 1], acc[q * 4 + 2], acc[q * 4 + 3]};
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 0; w < 3; ++w)
#pragma unroll
      for (int e = 0; e < N; ++e) acc[e] += quarter[w][e / 4][lane][e % 4];
  }
  if (left > 0) give_row<N>(b, b.dtable + (size_t)mine * b.width + (size_t)c * N, left, acc);
}

// Sums of one group's tokens, N columns a lane, eight rows on their way at once; the blocks
// behind these zero rows.  HBM bounds it: 65536 tokens x 2048 bf16 and the zeros of a table
// of 131072 (1.34 GB) in 260 us, 5.2 TB/s; groups of 8 to 64 tokens take the same time and
// leave the fewer partial sums the longer they are.
template <typename T>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedBwd b, const T* __restrict__ dy) {
  constexpr int N = Piece<T>::N, AHEAD = 8;
  if (blockIdx.x >= (unsigned)b.sum_blocks) {
    const int64_t v0 =
        b.absent0 + ((int64_t)(blockIdx.x - b.sum_blocks) * 4 + (threadIdx.x >> 6)) * kAbsent;
    if (v0 < b.vocab) fill_absent(b, (int)v0, threadIdx.x & 63);
    return;
  }
  const size_t group = ((size_t)blockIdx.x * 256 + threadIdx.x) >> b.rp.shift;
  const int lane = threadIdx.x & ((1 << b.rp.shift) - 1);
  const size_t g = group / (unsigned)b.rp.segs;
  if (g >= (size_t)b.runs) return;
  const int c = (int)(group - g * b.rp.segs) * (1 << b.rp.shift) + lane;
  const int left = b.width - c * N;
  const int j0 = (int)g * b.run, j1 = min(b.n, j0 + b.run);
  const uint32_t none = (uint32_t)b.vocab;
  // The key before the group's first and the one behind its last.
  uint32_t key = j0 > 0 ? b.slots[j0 - 1].x : ~0u;
  const uint32_t behind = j1 < b.n ? b.slots[j1].x : ~0u;
  bool head = j0 > 0 && b.slots[j0].x == key;       // the sum began before this group
  float acc[N];
#pragma unroll
  for (int e = 0; e < N; ++e) acc[e] = 0.f;
  uint2 s[AHEAD], ahead[AHEAD];
#pragma unroll
  for (int a = 0; a < AHEAD; ++a) ahead[a] = b.slots[min(j0 + a, j1 - 1)];
  key = ahead[0].x;
  for (int j = j0; j < j1; j += AHEAD) {
    Piece<T> p[AHEAD];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) s[a] = ahead[a];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) ahead[a] = b.slots[min(j + AHEAD + a, j1 - 1)];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      p[a].raw = u4{0, 0, 0, 0};
      if (j + a < j1 && s[a].x != none && left > 0)
        p[a].load(dy + (size_t)s[a].y * b.ldy + (size_t)c * N, left, b.width);
    }
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      if (j + a >= j1 || key == none) break;
      p[a].settle(left, b.width);
#pragma unroll
      for (int e = 0; e < N; ++e) acc[e] += p[a].get(e);
      const bool last = j + a + 1 >= j1;
      const uint32_t next = last ? behind : a + 1 < AHEAD ? s[(a + 1) % AHEAD].x : ahead[0].x;
      if (next == key && !last) continue;
      const bool on = next == key;                  // goes on in the next group
      if (!head && !on) {
        give_row<N>(b, b.dtable + (size_t)key * b.width + (size_t)c * N, left, acc);
      } else {
        float* out = b.part + ((size_t)g * 2 + (head ? 0 : 1)) * b.width + (size_t)c * N;
#pragma unroll
        for (int q = 0; q < N; q += 4) {
          Piece<float> o;
          o.set(acc + q);
          o.store(out + q, left - q);
        }
      }
#pragma unroll
      for (int e = 0; e < N; ++e) acc[e] = 0.f;
      head = false;
      key = next;
    }
  }
}

// Joins the partial sums of an id whose tokens began in group g and go on behind it: a
// block has 256 columns, each of its waves a quarter of the partial sums.  Latency bounds it:
// 4 us for 4099 tokens, 13 for 65536, most of whose blocks find nothing to join.
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedBwd b) {
  __shared__ f4 quarter[3][64];
  const int g = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int j0 = g * b.run, j1 = j0 + b.run;        // a group lies behind
  const uint32_t key = b.slots[j1 - 1].x, first = b.slots[j0].x;
  const uint32_t before = g > 0 ? b.slots[j0 - 1].x : ~0u;
  if (key == (uint32_t)b.vocab || b.slots[j1].x != key) return;
  if (first == key && before == key) return;        // it began in an earlier group
  int end = g + 1;                                  // behind the last group that begins with it
  for (;;) {
    const int64_t j = (int64_t)(end + lane) * b.run;
    const uint64_t other = ~__ballot(j < b.n && b.slots[j].x == key);
    if (other) {
      end += __ffsll((unsigned long long)other) - 1;
      break;
    }
    end += 64;
  }
  const int c = (blockIdx.y * 64 + lane) * 4, left = b.width - c;
  const int each = (end - g - 1 + 3) / 4;
  const int h0 = g + 1 + wave * each, h1 = min(end, h0 + each);
  f4 v = f4{0.f, 0.f, 0.f, 0.f};
  if (left > 0) {
#pragma unroll 8
    for (int h = h0; h < h1; ++h) {
      Piece<float> p;
      p.load(b.part + (size_t)h * 2 * b.width + c, left, b.width);
      p.settle(left, b.width);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += p.get(e);
    }
  }
  if (wave) quarter[wave - 1][lane] = v;
  __syncthreads();
  if (wave || left <= 0) return;
  Piece<float> p;
  p.load(b.part + ((size_t)g * 2 + 1) * b.width + c, left, b.width);
  float* o = b.dtable + (size_t)key * b.width + c;
  Piece<float> old;
  if (b.accumulate) {
    old.load(o, left, b.width);
    old.settle(left, b.width);
  }
  p.settle(left, b.width);
  float sum[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    sum[e] = p.get(e) + v[e];
#pragma unroll
    for (int q = 0; q < 3; ++q) sum[e] += quarter[q][lane][e];
    sum[e] = b.accumulate ? fmaf(sum[e], b.scale, old.get(e)) : sum[e] * b.scale;
  }
  p.set(sum);
  p.store(o, left);
}

}  // namespace sb

namespace {

constexpr size_t kBesideBytes = (size_t)48 << 20;       // zeroed beside a sort of one launch

// Sorted tokens of a lane group: long ones leave few partial sums, short ones fill the chip.
int embed_run(const sb::RowPlan& rp, int n) {
  int run = 8;
  while (run < 64 && (int64_t)(n / (2 * run)) * rp.segs << rp.shift >= 256 * 1024) run *= 2;
  return run;
}

struct EmbedSpace {
  size_t a, b, counts, part, bytes;
};

sb::RowPlan embed_rows(const sb_embed_desc* d) {
  return sb::row_plan<1>(d->width, 16 / (int)sbh::dsize(d->dtype));
}

// Stretches of a row that a wave has each, and whether the gradient is one launch.
int few_segs(const sb_embed_desc* d) {
  return sb::cdiv(d->width, 64 * 16 / (int)sbh::dsize(d->dtype));
}
bool embed_few(const sb_embed_desc* d) {
  return d->tokens <= sb::kFewTokens && (int64_t)d->tokens * few_segs(d) <= 1 << 20;
}

EmbedSpace embed_space(const sb_embed_desc* d) {
  const sb::SortIn s = sb::sort_plan(nullptr, d->first, d->vocab, d->tokens);
  const int run = embed_run(embed_rows(d), d->tokens);
  EmbedSpace e{};
  if (embed_few(d)) return e;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += sb::round_up(bytes, 256);
    return here;
  };
  e.a = take((size_t)d->tokens * 8);
  e.b = take(s.tiles && s.passes > 1 ? (size_t)d->tokens * 8 : 0);
  e.counts = take(sb::sort_count_bytes(s));
  e.part = take(d->tokens > run ? (size_t)sb::cdiv(d->tokens, run) * 2 * d->width * 4 : 0);
  e.bytes = at;
  return e;
}

constexpr int kFwdUnits = 2;           // pieces of a row that a lane has at once

sb_status embed_check(const sb_embed_desc* d) {
  if (!d || d->tokens < 0 || d->vocab < 1 || d->width < 1 || d->first < 0 || d->ldy < d->width)
    return SB_ERR_INVALID_ARG;
  if (d->dtype != SB_F32 && d->dtype != SB_BF16) return SB_ERR_INVALID_ARG;
  if (!std::isfinite(d->scale) || d->first > INT32_MAX - d->vocab) return SB_ERR_INVALID_ARG;
  if (d->tokens >= 1 << 30 || d->width >= 1 << 23 || d->vocab >= 1 << 29) return SB_ERR_UNSUPPORTED;
  // The forward has the most lanes: the gradient's sums have at least 8 tokens a group, and the
  // rows that it zeroes are four lanes each.
  const sb::RowPlan rp = sb::row_plan<kFwdUnits>(d->width, 16 / (int)sbh::dsize(d->dtype));
  return sb::row_lanes(rp, d->tokens) < sb::kLaunchLanes - 256 ? SB_OK : SB_ERR_UNSUPPORTED;
}

size_t embed_out_bytes(const sb_embed_desc* d) {
  return d->tokens ? ((size_t)(d->tokens - 1) * d->ldy + d->width) * sbh::dsize(d->dtype) : 0;
}

template <typename T>
sb_status embed_fwd(const sb_embed_desc* d, const T* table, const int32_t* ids, T* y,
                    hipStream_t stream) {
  constexpr int U = kFwdUnits;
  const sb::RowPlan rp = sb::row_plan<U>(d->width, sb::Piece<T>::N);
  const size_t blocks = (sb::row_lanes(rp, d->tokens) + 255) / 256;
  sb::embed_fwd_kernel<T, U><<<(unsigned)blocks, 256, 0, stream>>>(
      rp, d->tokens, d->first, d->vocab, d->width, d->ldy, d->scale, table, ids, y);
  return sbh::launch_status();
}

}  // namespace

extern "C" size_t sb_embed_workspace_bytes(const sb_embed_desc* d) {
  if (embed_check(d) != SB_OK) return (size_t)-1;
  return embed_space(d).bytes;
}

extern "C" sb_status sb_embed_fwd(const sb_embed_desc* d, const void* table, const int32_t* ids,
                                  void* y, void* stream) {
  const sb_status s = embed_check(d);
  if (s != SB_OK) return s;
  if (d->tokens == 0) return SB_OK;
  if (!table || !ids || !y) return SB_ERR_INVALID_ARG;
  const size_t e = sbh::dsize(d->dtype), yb = embed_out_bytes(d);
  if ((((uintptr_t)table | (uintptr_t)y) & (e - 1)) || ((uintptr_t)ids & 3))
    return SB_ERR_INVALID_ARG;
  if (sbh::overlaps(y, yb, table, (size_t)d->vocab * d->width * e) ||
      sbh::overlaps(y, yb, ids, (size_t)d->tokens * 4))
    return SB_ERR_INVALID_ARG;
  if (d->dtype == SB_BF16)
    return embed_fwd(d, (const sb::u16*)table, ids, (sb::u16*)y, sbh::stream_of(stream));
  return embed_fwd(d, (const float*)table, ids, (float*)y, sbh::stream_of(stream));
}

extern "C" sb_status sb_embed_bwd(const sb_embed_desc* d, const int32_t* ids, const void* dy,
                                  float* dtable, int accumulate, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  sb_status s = embed_check(d);
  if (s != SB_OK) return s;
  if (!dtable || (accumulate != 0 && accumulate != 1)) return SB_ERR_INVALID_ARG;
  if (d->tokens > 0 && (!ids || !dy)) return SB_ERR_INVALID_ARG;
  const size_t e = sbh::dsize(d->dtype), table = (size_t)d->vocab * d->width;
  if (((uintptr_t)dy & (e - 1)) || (((uintptr_t)ids | (uintptr_t)dtable) & 3) ||
      ((uintptr_t)workspace & 15))
    return SB_ERR_INVALID_ARG;
  const EmbedSpace at = embed_space(d);
  const size_t dyb = embed_out_bytes(d), ib = (size_t)d->tokens * 4;
  if (sbh::overlaps(dtable, table * 4, dy, dyb) || sbh::overlaps(dtable, table * 4, ids, ib) ||
      sbh::overlaps(workspace, at.bytes, dtable, table * 4) ||
      sbh::overlaps(workspace, at.bytes, dy, dyb) || sbh::overlaps(workspace, at.bytes, ids, ib))
    return SB_ERR_INVALID_ARG;
  if (at.bytes && (!workspace || workspace_bytes < at.bytes)) return SB_ERR_WORKSPACE;
  if (d->tokens == 0 && accumulate) return SB_OK;
  char* ws = (char*)workspace;
  hipStream_t st = sbh::stream_of(stream);
  const sb::SortIn in = sb::sort_plan(ids, d->first, d->vocab, d->tokens);
  sb::EmbedBwd b{};
  b.rp = embed_rows(d);
  b.n = d->tokens;
  b.vocab = d->vocab;
  b.width = d->width;
  b.ldy = d->ldy;
  b.run = embed_run(b.rp, d->tokens);
  b.runs = sb::cdiv(d->tokens, b.run);
  b.scale = d->scale;
  b.accumulate = accumulate;
  b.dtable = dtable;
  b.part = (float*)(ws + at.part);
  if (embed_few(d)) {
    const int segs = few_segs(d);
    const size_t zeros = accumulate ? 0 : ((size_t)d->vocab + sb::kAbsent - 1) / sb::kAbsent;
    const unsigned blocks = (unsigned)((size_t)d->tokens * segs + (zeros + 3) / 4);
    if (blocks == 0) return SB_OK;
    auto launch = [&](auto t, auto h) {
      using T = decltype(t);
      sb::embed_few_kernel<T, decltype(h)::value>
          <<<blocks, 256, 0, st>>>(b, d->first, segs, ids, (const T*)dy);
    };
    auto for_type = [&](auto h) {
      if (d->dtype == SB_BF16) launch(sb::u16(), h);
      else launch(float(), h);
    };
    if (d->tokens <= 128) for_type(std::integral_constant<int, 2>());
    else for_type(std::integral_constant<int, 4>());
    return sbh::launch_status();
  }
  const size_t sums = (sb::row_lanes(b.rp, b.runs) + 255) / 256;
  const int beside = accumulate || in.tiles
                         ? 0
                         : (int)std::min<size_t>(d->vocab, kBesideBytes / ((size_t)d->width * 4));
  b.absent0 = beside;
  const size_t absent = accumulate ? 0 : (size_t)(d->vocab - beside);
  const size_t blocks = sums + (absent + 4 * sb::kAbsent - 1) / (4 * sb::kAbsent);
  b.sum_blocks = (int)sums;
  b.slots = sbh::sort_slots(in, nullptr, nullptr, (uint2*)(ws + at.a), (uint2*)(ws + at.b),
                            (uint32_t*)(ws + at.counts),
                            sb::Fill{dtable, (size_t)beside * d->width}, st);
  s = sbh::launch_status();
  if (s != SB_OK) return s;
  if (d->dtype == SB_BF16)
    sb::embed_sum_kernel<sb::u16><<<(unsigned)blocks, 256, 0, st>>>(b, (const sb::u16*)dy);
  else
    sb::embed_sum_kernel<float><<<(unsigned)blocks, 256, 0, st>>>(b, (const float*)dy);
  if (b.runs > 1) {
    const dim3 grid((unsigned)(b.runs - 1), (unsigned)sb::cdiv(d->width, 256));
    sb::embed_join_kernel<<<grid, 256, 0, st>>>(b);
  }
  return sbh::launch_status();
}
