// rows.hpp -- rows of a matrix in 16-byte pieces at any address, for kernels
// that move whole rows (embedding, expert rows).
//
// gfx950's vector loads and stores take any address that is a multiple of the
// element's size, so rows of odd widths and strides are moved 16 bytes at a
// time too.  What lies behind a row's last whole piece is read with the row's last 16 bytes
// and written one by one.  (Read one by one each row held up its wave: 131072 rows of 2047
// bf16 combined by experts in 158 us and not 110, their gradients in 334 and not 282.)
#pragma once

#include "sb_internal.hpp"

namespace sb {

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef u4 u4_at2 __attribute__((aligned(2)));
typedef u4 u4_at4 __attribute__((aligned(4)));

// 16 bytes of a row: N elements, held as they lie in memory.
template <typename T> struct Piece;

template <> struct Piece<float> {
  static constexpr int N = 4;
  u4 raw;
  // The piece at p, where `left` > 0 elements of a row of `width` are left; settle() has to
  // follow, behind all loads that are to be on their way at once.  (One load for both kinds
  // of lanes, its address moved back at the end, took 478 us where this takes 462: gradients
  // of 262144 rows of 2048 bf16.)
  template <bool FAR = false>
  __device__ __forceinline__ void load(const float* p, int left, int width) {
    if (left >= N) {
      if constexpr (FAR) raw = __builtin_nontemporal_load(reinterpret_cast<const u4_at4*>(p));
      else raw = *reinterpret_cast<const u4_at4*>(p);
    } else if (width >= N) {
      raw = *reinterpret_cast<const u4_at4*>(p + left - N);
    } else {
      raw = u4{0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e < left) raw[e] = __float_as_uint(p[e]);
    }
  }
  // Past the row's end: `fill`.
  __device__ __forceinline__ void settle(int left, int width, uint32_t fill = 0) {
    if (width < N || width % N == 0) return;      // the whole wave
    if (left < N) {
      const int k = N - left;
      if (k & 1) raw = u4{raw[1], raw[2], raw[3], fill};
      if (k & 2) raw = u4{raw[2], raw[3], fill, fill};
    }
  }
  // FAR: read or written once, not to be kept in the caches.
  template <bool FAR = false>
  __device__ __forceinline__ void store(float* p, int left) const {
    if (left >= N) {
      if constexpr (FAR) __builtin_nontemporal_store(raw, reinterpret_cast<u4_at4*>(p));
      else *reinterpret_cast<u4_at4*>(p) = raw;
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e < left) p[e] = __uint_as_float(raw[e]);
    }
  }
  __device__ __forceinline__ float get(int e) const { return __uint_as_float(raw[e]); }
  __device__ __forceinline__ void set(const float* v) {
#pragma unroll
    for (int e = 0; e < N; ++e) raw[e] = __float_as_uint(v[e]);
  }
};

template <> struct Piece<u16> {
  static constexpr int N = 8;
  u4 raw;
  template <bool FAR = false>
  __device__ __forceinline__ void load(const u16* p, int left, int width) {
    if (left >= N) {
      if constexpr (FAR) raw = __builtin_nontemporal_load(reinterpret_cast<const u4_at2*>(p));
      else raw = *reinterpret_cast<const u4_at2*>(p);
    } else if (width >= N) {
      raw = *reinterpret_cast<const u4_at2*>(p + left - N);
    } else {
      raw = u4{0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e < left) raw[e / 2] |= (uint32_t)p[e] << (e % 2 * 16);
    }
  }
  __device__ __forceinline__ void settle(int left, int width, uint32_t fill = 0) {
    if (width < N || width % N == 0) return;      // the whole wave
    if (left < N) {
      const int k = N - left;
      if (k & 1)
        raw = u4{raw[0] >> 16 | raw[1] << 16, raw[1] >> 16 | raw[2] << 16,
                 raw[2] >> 16 | raw[3] << 16, raw[3] >> 16 | fill << 16};
      if (k & 2) raw = u4{raw[1], raw[2], raw[3], fill};
      if (k & 4) raw = u4{raw[2], raw[3], fill, fill};
    }
  }
  template <bool FAR = false>
  __device__ __forceinline__ void store(u16* p, int left) const {
    if (left >= N) {
      if constexpr (FAR) __builtin_nontemporal_store(raw, reinterpret_cast<u4_at2*>(p));
      else *reinterpret_cast<u4_at2*>(p) = raw;
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e < left) p[e] = (u16)(raw[e / 2] >> (e % 2 * 16));
    }
  }
  __device__ __forceinline__ float get(int e) const {
    return __uint_as_float(e % 2 ? raw[e / 2] & 0xffff0000u : raw[e / 2] << 16);
  }
  __device__ __forceinline__ void set(const float* v) {   // rounds to nearest, ties to even
#pragma unroll
    for (int e = 0; e < N; e += 2) raw[e / 2] = f32x2_to_bf16x2(v[e], v[e + 1]);
  }
};

// A row's pieces are spread over a group of G = 1 << shift lanes (8 to 64: the
// smallest that holds the row in one go, so narrow rows share a wave), U pieces a
// lane; a wider row is `segs` such stretches.
struct RowPlan {
  int shift;                   // lanes of a group
  int pieces;                  // of a row
  int segs;                    // stretches of a row, each a group's work
};

template <int U>
inline RowPlan row_plan(int width, int n_per_piece) {
  RowPlan p;
  p.pieces = cdiv(width, n_per_piece);
  p.shift = 3;
  while (p.shift < 6 && (1 << p.shift) < p.pieces) ++p.shift;
  p.segs = cdiv(p.pieces, U << p.shift);
  return p;
}

// Lanes of `rows` rows' groups.  A launch has fewer than 2^32 (kLaunchLanes).
constexpr size_t kLaunchLanes = (size_t)1 << 32;
inline size_t row_lanes(const RowPlan& p, size_t rows) { return rows * p.segs << p.shift; }

}  // namespace sb
