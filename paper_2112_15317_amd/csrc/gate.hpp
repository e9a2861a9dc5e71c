// gate.hpp -- the gate of the gated FC shard: activations and their derivatives.
#pragma once

#include "sb_internal.hpp"

namespace sb {

// The activation and its derivative, in fp32.
__device__ __forceinline__ void gate_act(int act, float a, float& f, float& df) {
  switch (act) {
    case SB_ACT_SIGMOID: {
      f = 1.f / (1.f + expf(-a));
      df = f * (1.f - f);
      break;
    }
    case SB_ACT_SILU: {
      const float p = 1.f / (1.f + expf(-a));
      f = a * p;
      df = p * (1.f + a * (1.f - p));
      break;
    }
    case SB_ACT_GELU: {
      const float c = 0.5f + 0.5f * erff(a * 0.70710678118654752f);
      f = a * c;
      df = c + a * expf(-0.5f * a * a) * 0.39894228040143268f;
      break;
    }
    case SB_ACT_GELU_TANH: {
      const float r = 0.79788456080286536f;
      const float t = tanhf(r * (a + 0.044715f * a * a * a));
      f = 0.5f * a * (1.f + t);
      // (t is +-1 from |a| = 6 on: within the bound a * a is finite, and 0 times it 0.)
      const float b = fminf(fmaxf(a, -1e4f), 1e4f);
      df = 0.5f * (1.f + t) + 0.5f * b * (1.f - t * t) * r * (1.f + 0.134145f * b * b);
      break;
    }
    default:
      f = a > 0.f ? a : 0.f;
      df = a > 0.f ? 1.f : 0.f;
  }
}

// Four outputs of a row, columns n .. n + 3 (those below N): both projections go to
// pre (this row's a; u is `plane` elements behind) where it is kept, act(a) u to y
// (this row's).
template <class E>
__device__ __forceinline__ void gate_store(int act, f4 a, f4 u, int n, int N, float* pre, size_t plane,
                                           E* y) {
  const bool whole = n + 4 <= N;
  f4 o;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float f, df;
    gate_act(act, a[e], f, df);
    o[e] = f * u[e];
  }
  if (pre) {
    if (whole && (((uintptr_t)(pre + n) | plane * 4) & 15) == 0) {
      *reinterpret_cast<f4*>(pre + n) = a;
      *reinterpret_cast<f4*>(pre + plane + n) = u;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < N) {
          pre[n + e] = a[e];
          pre[plane + n + e] = u[e];
        }
    }
  }
  if (whole && ((uintptr_t)(y + n) & (4 * sizeof(E) - 1)) == 0) {
    Elem<E>::store4(y + n, o);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < N) Elem<E>::store(y, n + e, o[e]);
  }
}

}  // namespace sb
