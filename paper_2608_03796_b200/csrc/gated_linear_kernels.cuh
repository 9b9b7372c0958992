// The gated linear layer for one token (or two), h = act(x Wg^T) (x Wu^T): the weights are read once and nothing else is of
// any size, so the tensor cores would only add their latencies. A warp takes one feature: its lanes read the feature's
// gate row and up row side by side, eight columns at a time, and multiply them with the tokens' values, which stay in
// the first cache; 2 sums a token and lane in fp32, joined by shuffles. Blocks are small and registers few, so that all
// features of a layer of usual width are at work at once. U words of each row are on their way at once: 2, or 8 where there are
// fewer than 24 features an SM. One token, weights from memory: 2048 x 5632 9.0 us (U = 8: 11.0), 4096 x 14336 38.2 us
// (6.1 TB/s), 1000 x 2600 3.1 us (U = 2: 4.1). Two tokens 14.7, 48 and 4.8 us: multiplications, from there on
// gated_few_kernels.cuh is faster (12.1, 40 and 5.9 for three) but for small weights.
#pragma once
#include "act8.cuh"
#include "gated_math.cuh"

namespace kdkl {

constexpr int kGatedRowsWarps = 4;

template <int TOKENS, int ACT, int U>
__global__ void __launch_bounds__(32 * kGatedRowsWarps, U == 2 && TOKENS == 1 ? 12 : U == 2 ? 8 : 5)
gated_rows_kernel(const __nv_bfloat16* x, long long ld_x, const __nv_bfloat16* weight, int T, int H, int F, __nv_bfloat16* h,
                  long long ld_h, int* status) {
  const int lane = threadIdx.x & 31, f = blockIdx.x * kGatedRowsWarps + (threadIdx.x >> 5), words = H / 8;
  grid_dependents_launch();
  grid_dependency_wait();
  if (blockIdx.x == 0 && threadIdx.x < 2) status[threadIdx.x] = 0;     // nothing here can fail
  if (f >= F) return;
  const uint4* wg = reinterpret_cast<const uint4*>(weight + (long long)f * H);
  const uint4* wu = reinterpret_cast<const uint4*>(weight + ((long long)F + f) * H);
  float2 g[TOKENS], u[TOKENS];
#pragma unroll
  for (int t = 0; t < TOKENS; ++t) g[t] = u[t] = make_float2(0.f, 0.f);
  for (int i0 = lane; i0 < words; i0 += 32 * U) {
    uint4 a[U], b[U];
#pragma unroll
    for (int k = 0; k < U; ++k)
      if (i0 + 32 * k < words) { a[k] = wg[i0 + 32 * k]; b[k] = wu[i0 + 32 * k]; }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int i = i0 + 32 * k;
      if (i >= words) break;
      float p[8], q[8];
      words_to_f32(a[k], p, __nv_bfloat16());
      words_to_f32(b[k], q, __nv_bfloat16());
#pragma unroll
      for (int t = 0; t < TOKENS; ++t) {
        if (t >= T) break;                                 // (the same for all)
        float v[8];
        words_to_f32(*reinterpret_cast<const uint4*>(x + t * ld_x + 8 * i), v, __nv_bfloat16());
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 xv = make_float2(v[2 * j], v[2 * j + 1]);
          g[t] = fma2(make_float2(p[2 * j], p[2 * j + 1]), xv, g[t]);
          u[t] = fma2(make_float2(q[2 * j], q[2 * j + 1]), xv, u[t]);
        }
      }
    }
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
