// The gated activation of a feed-forward block, h = act(g) u, whose backward pass reads g and u from 8-bit records.
//
//   act(g) = g s,  s = sigmoid(k(g));   silu: k = g,   gelu (tanh form): k = 2 sqrt(2 / pi) (g + 0.044715 g^3)
//   act'(g) = s + g s (1 - s) k'(g)
//   backward: dgate = dh u act'(g), dup = dh act(g), both at the values the records stand for
//
// Element-wise, so bound by memory: forward reads 4 bytes a value and writes 2 (+ 33/32 per record), backward reads
// 2 + 66/32 and writes 4. The records leave in the pass that computes h, from registers. 32768 x 7168 bf16, int8 records,
// one B200, in a loop over inputs beyond the L2: forward 340 us (5.6 TB/s), backward 318 us (5.95 TB/s), a pass of both 657;
// without records forward 207 us (6.8 TB/s: two thirds of it reads, of which a plain sum of two tensors does 7.1, a copy 6.6).
// What the records add to the forward pass is the encoding: about 70 instructions per eight values. Element by element (odd
// widths) 16384 x 7167 takes 1119 and 851 us.
#pragma once
#include "act8.cuh"

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

template <typename T, int ACT, int FMT /* -1: nothing is kept */, bool VEC>
__global__ void __launch_bounds__(256)
gated_forward_kernel(const T* gate, const T* up, long long ld, long long rows, int F,
                     T* __restrict__ h, long long ld_h, ActRecord rec_gate, ActRecord rec_up, ActRecord rec_h) {
  const long long cpitch = act_codes_pitch(F), spitch = act_scale_pitch(F);
  const int c = first_column<VEC>(blockIdx.x * blockDim.x + threadIdx.x);
  grid_dependents_launch();
  grid_dependency_wait();
  for (long long t = blockIdx.y; t < rows; t += gridDim.y) {
    float g[8], u[8], o[8];
    load8<T, VEC>(gate + t * ld, c, F, g);
    load8<T, VEC>(up + t * ld, c, F, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float slope;
      o[i] = g[i] * gate_sigmoid<ACT>(g[i], slope) * u[i];
    }
    const Raw8<T> raw = f32_to_raw<T>(o);
    store_raw8<T, VEC>(h + t * ld_h, c, F, raw);
    if constexpr (FMT >= 0) {
      record_write8<FMT, VEC>(rec_gate, t, cpitch, spitch, c, g);
      record_write8<FMT, VEC>(rec_up, t, cpitch, spitch, c, u);
      if (rec_h.codes != nullptr) {                    // what a record of h, as it was returned, would hold
        raw_to_f32(raw, o);
        record_write8<FMT, VEC>(rec_h, t, cpitch, spitch, c, o);
      }
    }
  }
}

template <typename T, int ACT, int FMT, bool VEC>
__global__ void __launch_bounds__(256)
gated_backward_kernel(ActRecord rec_gate, ActRecord rec_up, const T* dh, long long ld_dh, long long rows,
                      int F, T* __restrict__ dgate, T* __restrict__ dup, long long ld) {
  const long long cpitch = act_codes_pitch(F), spitch = act_scale_pitch(F);
  const int c = first_column<VEC>(blockIdx.x * blockDim.x + threadIdx.x);
  grid_dependents_launch();
  grid_dependency_wait();
  if (c >= F) return;
  for (long long t = blockIdx.y; t < rows; t += gridDim.y) {
    float g[8], u[8], d[8], dg[8], du[8];
    if constexpr (VEC) {                               // c < F: both records' words at once
      uint2 codes_g, codes_u;
      uint32_t byte_g, byte_u;
      record_fetch8(rec_gate, t, cpitch, spitch, c, codes_g, byte_g);
      record_fetch8(rec_up, t, cpitch, spitch, c, codes_u, byte_u);
      load8<T, VEC>(dh + t * ld_dh, c, F, d);
      act_values<FMT>(codes_g, byte_g, g);
      act_values<FMT>(codes_u, byte_u, u);
    } else {
      record_read8<FMT, VEC>(rec_gate, t, cpitch, spitch, c, g);
      record_read8<FMT, VEC>(rec_up, t, cpitch, spitch, c, u);
      load8<T, VEC>(dh + t * ld_dh, c, F, d);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float slope;
      const float s = gate_sigmoid<ACT>(g[i], slope);
      const float t1 = s * (1.f - s);                  // 0 where the sigmoid has saturated, however large k' is
      const float a1 = t1 == 0.f ? s : fmaf(g[i] * t1, slope, s);
      dg[i] = d[i] * u[i] * a1;
      du[i] = d[i] * g[i] * s;
    }
    store_raw8<T, VEC>(dgate + t * ld, c, F, f32_to_raw<T>(dg));
    store_raw8<T, VEC>(dup + t * ld, c, F, f32_to_raw<T>(du));
  }
}

}  // namespace kdkl
