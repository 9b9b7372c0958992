// The gated linear layer for a few tokens, h = act(x Wg^T) (x Wu^T): the weights are read once and nothing else is of any
// size, so the tensor cores, whose tiles hold 256 tokens, would only add their latencies. A warp takes one feature: its
// lanes read the feature's gate row and up row side by side, eight columns at a time, and multiply them with the tokens'
// values, which a block keeps in shared memory; 2 sums a token and lane in fp32, joined by shuffles.
#pragma once
#include "act8.cuh"
#include "gated_math.cuh"

namespace kdkl {

constexpr int kGatedRowsTokens = 8, kGatedRowsWarps = 8;

template <int TOKENS, int ACT>
__global__ void __launch_bounds__(32 * kGatedRowsWarps)
gated_rows_kernel(const __nv_bfloat16* x, long long ld_x, const __nv_bfloat16* weight, int T, int H, int F, __nv_bfloat16* h,
                  long long ld_h, int* status) {
  extern __shared__ uint4 gated_x[];                       // [TOKENS][H / 8]
  const int lane = threadIdx.x & 31, f = blockIdx.x * kGatedRowsWarps + (threadIdx.x >> 5), words = H / 8;
  grid_dependents_launch();
  grid_dependency_wait();
  const uint4* wg = reinterpret_cast<const uint4*>(weight + (long long)f * H);
  const uint4* wu = reinterpret_cast<const uint4*>(weight + ((long long)F + f) * H);
  constexpr int U = 4;                                     // words of each row on their way at once, the first before anything else
  uint4 a[U], b[U];
  auto ask = [&](int i0) {
#pragma unroll
    for (int k = 0; k < U; ++k)
      if (f < F && i0 + 32 * k < words) { a[k] = wg[i0 + 32 * k]; b[k] = wu[i0 + 32 * k]; }
  };
  ask(lane);
  for (int i = threadIdx.x; i < TOKENS * words; i += blockDim.x) {
    const int t = i / words;
    gated_x[i] = t < T ? *reinterpret_cast<const uint4*>(x + t * ld_x + 8 * (i - t * words)) : make_uint4(0u, 0u, 0u, 0u);
  }
  if (blockIdx.x == 0 && threadIdx.x < 2) status[threadIdx.x] = 0;     // nothing here can fail
  __syncthreads();
  if (f >= F) return;
  float2 g[TOKENS], u[TOKENS];
#pragma unroll
  for (int t = 0; t < TOKENS; ++t) g[t] = u[t] = make_float2(0.f, 0.f);
  for (int i0 = lane; i0 < words; i0 += 32 * U) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int i = i0 + 32 * k;
      if (i >= words) break;
      float p[8], q[8];
      words_to_f32(a[k], p, __nv_bfloat16());
      words_to_f32(b[k], q, __nv_bfloat16());
#pragma unroll
      for (int t = 0; t < TOKENS; ++t) {
        float v[8];
        words_to_f32(gated_x[t * words + i], v, __nv_bfloat16());
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 xv = make_float2(v[2 * j], v[2 * j + 1]);
          g[t] = fma2(make_float2(p[2 * j], p[2 * j + 1]), xv, g[t]);
          u[t] = fma2(make_float2(q[2 * j], q[2 * j + 1]), xv, u[t]);
        }
      }
    }
    ask(i0 + 32 * U);
  }
#pragma unroll
  for (int t = 0; t < TOKENS; ++t) {
    float gate = g[t].x + g[t].y, up = u[t].x + u[t].y;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      gate += __shfl_xor_sync(0xffffffffu, gate, o);
      up += __shfl_xor_sync(0xffffffffu, up, o);
    }
    if (lane == 0 && t < T) {
      float slope;
      h[t * ld_h + f] = __float2bfloat16_rn(gate * gate_sigmoid<ACT>(gate, slope) * up);
    }
  }
}

}  // namespace kdkl
