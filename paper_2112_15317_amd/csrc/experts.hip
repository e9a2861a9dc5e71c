// experts.hip -- tokens' rows laid out by expert and brought back with weights.
//
// Slot (t, j) is token t's j-th choice of an expert.  The slots are sorted by
// expert, stable (slot_sort.hpp), and place[t][j] is the row that slot has among
// them; -1 where its expert is not one of this worker's.
//
//   xs[place[t][j]] = x[t]
//   y[t]            = add[t] + sum_j w[t][j] ys[place[t][j]]
//   dys[place]      = w[t][j] dy[t],   dw[t][j] = <dy[t], ys[place]>
//
// HBM bounds all of them.  Going by tokens a row of x or dy is read once for all
// its experts, and the rows of a token are summed by one lane group in the order of j:
// no atomics.  Sorted rows are written past the caches (a nontemporal store): 8192 tokens
// of 2 experts x 2048 bf16 112 -> 86 us over all launches, 32768 of 8 1197 -> 1123.
#include "rows.hpp"
#include "slot_sort.hpp"

#include <cmath>

namespace sb {

struct ExpertRows {
  RowPlan rp;
  int n, top, width, ldx, ldr;
  uint32_t rows;               // n * top: a place past it is none
};

// 32768 tokens of 8 experts x 2048 bf16 (1.21 GB) in 239 us, 5.1 TB/s.
template <typename T, int U>
__global__ __launch_bounds__(256) void expert_gather_kernel(ExpertRows b, const T* __restrict__ x,
                                                            const int32_t* __restrict__ place,
                                                            T* __restrict__ xs) {
  constexpr int N = Piece<T>::N;
  const size_t group = ((size_t)blockIdx.x * 256 + threadIdx.x) >> b.rp.shift;
  const int lane = threadIdx.x & ((1 << b.rp.shift) - 1);
  const size_t t = group / (unsigned)b.rp.segs;
  if (t >= (size_t)b.n) return;
  const int c0 = (int)(group - t * b.rp.segs) * (U << b.rp.shift) + lane;
  Piece<T> p[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + (u << b.rp.shift);
    if (c < b.rp.pieces) p[u].load(x + t * (size_t)b.ldx + (size_t)c * N, b.width - c * N, b.width);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) p[u].settle(b.width - (c0 + (u << b.rp.shift)) * N, b.width);
  for (int j = 0; j < b.top; ++j) {
    const uint32_t to = (uint32_t)place[t * b.top + j];
    if (to >= b.rows) continue;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + (u << b.rp.shift);
      if (c < b.rp.pieces)
        p[u].template store<true>(xs + to * (size_t)b.ldr + (size_t)c * N, b.width - c * N);
    }
  }
}

// Four experts' rows on their way at once.  The same rows (1.21 GB) in 209 us, 5.8 TB/s.
template <typename T, int U, bool FAR>
__global__ __launch_bounds__(256) void expert_combine_kernel(ExpertRows b,
                                                             const T* __restrict__ ys,
                                                             const int32_t* __restrict__ place,
                                                             const float* __restrict__ weights,
                                                             const T* add, T* y) {
  constexpr int N = Piece<T>::N, AHEAD = 4;           // rows on their way at once
  const size_t group = ((size_t)blockIdx.x * 256 + threadIdx.x) >> b.rp.shift;
  const int lane = threadIdx.x & ((1 << b.rp.shift) - 1);
  const size_t t = group / (unsigned)b.rp.segs;
  if (t >= (size_t)b.n) return;
  const int c0 = (int)(group - t * b.rp.segs) * (U << b.rp.shift) + lane;
  float acc[U][N];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + (u << b.rp.shift);
    Piece<T> p;
    p.raw = u4{0, 0, 0, 0};
    if (add && c < b.rp.pieces) {
      p.load(add + t * (size_t)b.ldx + (size_t)c * N, b.width - c * N, b.width);
      p.settle(b.width - c * N, b.width);
    }
#pragma unroll
    for (int e = 0; e < N; ++e) acc[u][e] = p.get(e);
  }
  for (int j0 = 0; j0 < b.top; j0 += AHEAD) {
    uint32_t from[AHEAD];
    float w[AHEAD];
    Piece<T> p[AHEAD][U];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const bool there = j0 + j < b.top;
      from[j] = there ? (uint32_t)place[t * b.top + j0 + j] : ~0u;
      w[j] = there && weights ? weights[t * b.top + j0 + j] : 1.f;
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + (u << b.rp.shift);
        if (from[j] < b.rows && c < b.rp.pieces)
          p[j][u].template load<FAR>(ys + from[j] * (size_t)b.ldr + (size_t)c * N, b.width - c * N,
                                     b.width);
      }
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (from[j] >= b.rows) continue;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        p[j][u].settle(b.width - (c0 + (u << b.rp.shift)) * N, b.width);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[u][e] = fmaf(w[j], p[j][u].get(e), acc[u][e]);
      }
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + (u << b.rp.shift);
    if (c >= b.rp.pieces) continue;
    Piece<T> p;
    p.set(acc[u]);
    p.template store<true>(y + t * (size_t)b.ldx + (size_t)c * N, b.width - c * N);
  }
}

// A group has a whole row of dy, kept in registers where it has at most U pieces a lane, and
// two experts' rows on their way at once.  The same rows (2.28 GB) in 455 us, 5.0 TB/s; one to
// eight rows at once and one to four pieces a lane are within 4 % of each other there.
template <typename T, int U>
__global__ __launch_bounds__(256) void expert_combine_bwd_kernel(
    ExpertRows b, const T* __restrict__ dy, const T* __restrict__ ys,
    const int32_t* __restrict__ place, const float* __restrict__ weights, T* __restrict__ dys,
    float* __restrict__ dweights) {
  constexpr int N = Piece<T>::N, AHEAD = 2;           // rows on their way at once
  const size_t t = ((size_t)blockIdx.x * 256 + threadIdx.x) >> b.rp.shift;
  const int lane = threadIdx.x & ((1 << b.rp.shift) - 1);
  if (t >= (size_t)b.n) return;
  const T* from = dy + t * (size_t)b.ldx;
  Piece<T> g[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = lane + (u << b.rp.shift);
    g[u].raw = u4{0, 0, 0, 0};
    if (c < b.rp.pieces) g[u].load(from + (size_t)c * N, b.width - c * N, b.width);
  }
  if (b.rp.segs == 1) {
#pragma unroll
    for (int u = 0; u < U; ++u) g[u].settle(b.width - (lane + (u << b.rp.shift)) * N, b.width);
  }
  for (int j0 = 0; j0 < b.top; j0 += AHEAD) {
    uint32_t row[AHEAD];
    float w[AHEAD], dot[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const bool there = j0 + j < b.top;
      row[j] = there ? (uint32_t)place[t * b.top + j0 + j] : ~0u;
      w[j] = there && weights ? weights[t * b.top + j0 + j] : 1.f;
      dot[j] = 0.f;
    }
    for (int s = 0; s < b.rp.segs; ++s) {
      Piece<T> o[AHEAD][U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = lane + ((s * U + u) << b.rp.shift), left = b.width - c * N;
        if (c >= b.rp.pieces) continue;
        if (b.rp.segs > 1) g[u].load(from + (size_t)c * N, left, b.width);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
          if (dweights && row[j] < b.rows)
            o[j][u].load(ys + row[j] * (size_t)b.ldr + (size_t)c * N, left, b.width);
      }
      if (b.rp.segs > 1) {
#pragma unroll
        for (int u = 0; u < U; ++u)
          g[u].settle(b.width - (lane + ((s * U + u) << b.rp.shift)) * N, b.width);
      }
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        if (row[j] >= b.rows) continue;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int c = lane + ((s * U + u) << b.rp.shift);
          if (c >= b.rp.pieces) continue;
          if (dweights) o[j][u].settle(b.width - c * N, b.width);
          float v[N];
#pragma unroll
          for (int e = 0; e < N; ++e) {
            if (dweights) dot[j] = fmaf(g[u].get(e), o[j][u].get(e), dot[j]);
            v[e] = g[u].get(e) * w[j];
          }
          o[j][u].set(v);
          o[j][u].template store<true>(dys + row[j] * (size_t)b.ldr + (size_t)c * N,
                                       b.width - c * N);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (!dweights || j0 + j >= b.top) continue;
      for (int o = 1; o < 1 << b.rp.shift; o *= 2) dot[j] += __shfl_xor(dot[j], o, 64);
      if (lane == 0) dweights[t * b.top + j0 + j] = dot[j];
    }
  }
}

}  // namespace sb

namespace {

constexpr int kUnits = 2, kBwdUnits = 4;      // pieces of a row that a lane has at once

sb_status expert_check(const sb_expert_desc* d) {
  if (!d || d->tokens < 0 || d->top < 1 || d->experts < 1 || d->first < 0 || d->width < 1 ||
      d->ldx < d->width || d->ldr < d->width)
    return SB_ERR_INVALID_ARG;
  if (d->dtype != SB_F32 && d->dtype != SB_BF16) return SB_ERR_INVALID_ARG;
  if (d->experts > SB_MAX_EXPERTS || d->first > INT32_MAX - d->experts) return SB_ERR_INVALID_ARG;
  if ((int64_t)d->tokens * d->top >= 1 << 30 || d->width >= 1 << 24) return SB_ERR_UNSUPPORTED;
  const sb::RowPlan rp = sb::row_plan<kUnits>(d->width, 16 / (int)sbh::dsize(d->dtype));
  return sb::row_lanes(rp, d->tokens) < sb::kLaunchLanes - 256 ? SB_OK : SB_ERR_UNSUPPORTED;
}

size_t token_bytes(const sb_expert_desc* d) {
  return d->tokens ? ((size_t)(d->tokens - 1) * d->ldx + d->width) * sbh::dsize(d->dtype) : 0;
}
size_t row_bytes(const sb_expert_desc* d) {
  const size_t rows = (size_t)d->tokens * d->top;
  return rows ? ((rows - 1) * d->ldr + d->width) * sbh::dsize(d->dtype) : 0;
}
size_t slot_bytes(const sb_expert_desc* d) { return (size_t)d->tokens * d->top * 4; }

bool off(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

struct Span {
  const void* p;
  size_t bytes;
};
// Whether one of the outputs meets an input or another output.
bool meets(const Span* outs, int n_out, const Span* ins, int n_in) {
  for (int i = 0; i < n_out; ++i) {
    for (int j = 0; j < n_in; ++j)
      if (sbh::overlaps(outs[i].p, outs[i].bytes, ins[j].p, ins[j].bytes)) return true;
    for (int j = 0; j < i; ++j)
      if (sbh::overlaps(outs[i].p, outs[i].bytes, outs[j].p, outs[j].bytes)) return true;
  }
  return false;
}

template <int U>
sb::ExpertRows expert_rows(const sb_expert_desc* d) {
  sb::ExpertRows b;
  b.rp = sb::row_plan<U>(d->width, 16 / (int)sbh::dsize(d->dtype));
  b.n = d->tokens;
  b.top = d->top;
  b.width = d->width;
  b.ldx = d->ldx;
  b.ldr = d->ldr;
  b.rows = (uint32_t)d->tokens * (uint32_t)d->top;
  return b;
}

// Blocks of `rows` rows' groups; a group of the backward has all stretches of its row.
unsigned blocks_of(const sb::RowPlan& rp, size_t rows, bool whole = false) {
  return (unsigned)(((whole ? rows << rp.shift : sb::row_lanes(rp, rows)) + 255) / 256);
}

// Rows of more than the last cache holds are read past the caches by the combining kernel:
// 1 GB in 209 us, 225 as other loads; 67 MB that lie there take 18.1 and 16.9.
constexpr size_t kFarBytes = (size_t)256 << 20;

}  // namespace

extern "C" size_t sb_expert_workspace_bytes(const sb_expert_desc* d) {
  if (expert_check(d) != SB_OK) return (size_t)-1;
  return sb::round_up(
      sb::sort_count_bytes(sb::sort_plan(nullptr, d->first, d->experts, d->tokens * d->top)), 256);
}

extern "C" sb_status sb_expert_sort(const sb_expert_desc* d, const int32_t* ids, int32_t* place,
                                    int32_t* offsets, void* workspace, size_t workspace_bytes,
                                    void* stream) {
  const sb_status s = expert_check(d);
  if (s != SB_OK) return s;
  if (!offsets || (d->tokens > 0 && (!ids || !place))) return SB_ERR_INVALID_ARG;
  if (off(ids, 4) || off(place, 4) || off(offsets, 4) || off(workspace, 16))
    return SB_ERR_INVALID_ARG;
  const size_t need = sb_expert_workspace_bytes(d);
  const Span in{ids, slot_bytes(d)};
  const Span out[3] = {{place, slot_bytes(d)}, {offsets, ((size_t)d->experts + 1) * 4},
                       {workspace, need}};
  if (meets(out, 3, &in, 1)) return SB_ERR_INVALID_ARG;
  if (need && (!workspace || workspace_bytes < need)) return SB_ERR_WORKSPACE;
  const sb::SortIn p = sb::sort_plan(ids, d->first, d->experts, d->tokens * d->top);
  // (A batch without tokens has no places: any address stands for them.)
  sbh::sort_slots(p, place ? place : offsets, offsets, nullptr, nullptr, (uint32_t*)workspace,
                  sb::Fill{nullptr, 0}, sbh::stream_of(stream));
  return sbh::launch_status();
}

extern "C" sb_status sb_expert_gather(const sb_expert_desc* d, const void* x, const int32_t* place,
                                      void* xs, void* stream) {
  const sb_status s = expert_check(d);
  if (s != SB_OK) return s;
  if (d->tokens == 0) return SB_OK;
  const size_t e = sbh::dsize(d->dtype);
  if (!x || !place || !xs || off(x, e) || off(xs, e) || off(place, 4)) return SB_ERR_INVALID_ARG;
  const Span in[2] = {{x, token_bytes(d)}, {place, slot_bytes(d)}};
  const Span out{xs, row_bytes(d)};
  if (meets(&out, 1, in, 2)) return SB_ERR_INVALID_ARG;
  const sb::ExpertRows b = expert_rows<kUnits>(d);
  const unsigned blocks = blocks_of(b.rp, d->tokens);
  hipStream_t st = sbh::stream_of(stream);
  if (d->dtype == SB_BF16)
    sb::expert_gather_kernel<sb::u16, kUnits><<<blocks, 256, 0, st>>>(b, (const sb::u16*)x, place,
                                                                      (sb::u16*)xs);
  else
    sb::expert_gather_kernel<float, kUnits><<<blocks, 256, 0, st>>>(b, (const float*)x, place,
                                                                    (float*)xs);
  return sbh::launch_status();
}

extern "C" sb_status sb_expert_combine(const sb_expert_desc* d, const void* ys,
                                       const int32_t* place, const float* weights,
                                       const void* add, void* y, void* stream) {
  const sb_status s = expert_check(d);
  if (s != SB_OK) return s;
  if (d->tokens == 0) return SB_OK;
  const size_t e = sbh::dsize(d->dtype);
  if (!ys || !place || !y || off(ys, e) || off(y, e) || off(add, e) || off(place, 4) ||
      off(weights, 4))
    return SB_ERR_INVALID_ARG;
  const Span in[4] = {{ys, row_bytes(d)}, {place, slot_bytes(d)}, {weights, slot_bytes(d)},
                      {add == y ? nullptr : add, token_bytes(d)}};
  const Span out{y, token_bytes(d)};
  if (meets(&out, 1, in, 4)) return SB_ERR_INVALID_ARG;
  const sb::ExpertRows b = expert_rows<kUnits>(d);
  const unsigned blocks = blocks_of(b.rp, d->tokens);
  hipStream_t st = sbh::stream_of(stream);
  const bool far = row_bytes(d) >= kFarBytes;
  auto launch = [&](auto e, auto f) {
    using T = decltype(e);
    sb::expert_combine_kernel<T, kUnits, decltype(f)::value><<<blocks, 256, 0, st>>>(
        b, (const T*)ys, place, weights, (const T*)add, (T*)y);
  };
  if (d->dtype == SB_BF16) {
    if (far) launch(sb::u16(), std::true_type());
    else launch(sb::u16(), std::false_type());
  } else {
    if (far) launch(float(), std::true_type());
    else launch(float(), std::false_type());
  }
  return sbh::launch_status();
}

extern "C" sb_status sb_expert_combine_bwd(const sb_expert_desc* d, const void* dy, const void* ys,
                                           const int32_t* place, const float* weights, void* dys,
                                           float* dweights, void* stream) {
  const sb_status s = expert_check(d);
  if (s != SB_OK) return s;
  if (d->tokens == 0) return SB_OK;
  const size_t e = sbh::dsize(d->dtype);
  if (!dy || !place || !dys || (dweights && !ys) || off(dy, e) || off(ys, e) || off(dys, e) ||
      off(place, 4) || off(weights, 4) || off(dweights, 4))
    return SB_ERR_INVALID_ARG;
  const Span in[4] = {{dy, token_bytes(d)}, {ys, row_bytes(d)}, {place, slot_bytes(d)},
                      {weights, slot_bytes(d)}};
  const Span out[2] = {{dys, row_bytes(d)}, {dweights, slot_bytes(d)}};
  if (meets(out, 2, in, 4)) return SB_ERR_INVALID_ARG;
  const sb::ExpertRows b = expert_rows<kBwdUnits>(d);
  const unsigned blocks = blocks_of(b.rp, d->tokens, true);
  hipStream_t st = sbh::stream_of(stream);
  if (d->dtype == SB_BF16)
    sb::expert_combine_bwd_kernel<sb::u16, kBwdUnits><<<blocks, 256, 0, st>>>(
        b, (const sb::u16*)dy, (const sb::u16*)ys, place, weights, (sb::u16*)dys, dweights);
  else
    sb::expert_combine_bwd_kernel<float, kBwdUnits><<<blocks, 256, 0, st>>>(
        b, (const float*)dy, (const float*)ys, place, weights, (float*)dys, dweights);
  return sbh::launch_status();
}
