// The activations of gated layers, act(g) = g sigmoid(k(g)): see gated_kernels.cuh.
#pragma once
#include <cuda_runtime.h>

namespace kdkl {

constexpr int kActSilu = 0, kActGelu = 1;

// sigmoid(k(g)) and k'(g)
template <int ACT>
__device__ __forceinline__ float gate_sigmoid(float g, float& slope) {
  float k = g;
  slope = 1.f;
  if (ACT == kActGelu) {
    constexpr float c = 1.5957691216057308f;          // 2 sqrt(2 / pi)
    const float g2 = g * g;
    k = c * g * fmaf(0.044715f, g2, 1.f);
    slope = c * fmaf(3.f * 0.044715f, g2, 1.f);
  }
  // from exp(-|k|), so that the quotient stays in [1, 2] and the far negative side keeps its relative accuracy
  const float e = __expf(-fabsf(k));
  return __fdividef(k >= 0.f ? 1.f : e, 1.f + e);
}

// sigmoid(k(g)) and act'(g) = s + g s (1 - s) k'(g)
struct GateAct { float sigmoid, slope; };
template <int ACT>
__device__ __forceinline__ GateAct gate_act(float g) {
  GateAct r;
  float k1;
  r.sigmoid = gate_sigmoid<ACT>(g, k1);
  const float t = r.sigmoid * (1.f - r.sigmoid);       // 0 where the sigmoid has saturated, however large k' is
  r.slope = t == 0.f ? r.sigmoid : fmaf(g * t, k1, r.sigmoid);
  return r;
}

}  // namespace kdkl
