// Weight gradient of a linear layer whose input was kept in an 8-bit record:
//   dW[n, h] (= or +=) sum_t dY[t, n] x~[t, h],  x~ = what the record stands for.
#pragma once
#include "act8.cuh"

namespace kdkl {

struct DweightParams {
  const __nv_bfloat16* dy; long long ld_dy;
  ActRecord rec;
  long long T; int N, H;
  void* out; int type; int accumulate;
};

template <int FMT>
__global__ void __launch_bounds__(256)
act8_dweight_simple_kernel(const DweightParams p) {
  __shared__ float a[16][64], b[16][64 + 4];
  const long long cpitch = act_codes_pitch(p.H), spitch = act_scale_pitch(p.H);
  const int n0 = blockIdx.y * 64, h0 = blockIdx.x * 64;
  const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
  float acc[4][4] = {};
  for (long long t0 = 0; t0 < p.T; t0 += 16) {
    for (int i = threadIdx.x; i < 16 * 64; i += 256) {
      const long long t = t0 + i / 64;
      const int n = n0 + i % 64;
      a[i / 64][i % 64] = (t < p.T && n < p.N) ? __bfloat162float(p.dy[t * p.ld_dy + n]) : 0.f;
    }
    if (threadIdx.x < 128) {
      const long long t = t0 + threadIdx.x / 8;
      const int c = h0 + (threadIdx.x % 8) * 8;
      float f[8] = {};
      if (t < p.T && c < cpitch) record_read8<FMT>(p.rec, t, cpitch, spitch, c, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) b[threadIdx.x / 8][(threadIdx.x % 8) * 8 + j] = f[j];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(a[k][ty * 4 + i], b[k][tx * 4 + j], acc[i][j]);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + ty * 4 + i, h = h0 + tx * 4 + j;
      if (n >= p.N || h >= p.H) continue;
      const long long at = (long long)n * p.H + h;
      if (p.type == 1) {
        float* o = reinterpret_cast<float*>(p.out);
        o[at] = p.accumulate ? o[at] + acc[i][j] : acc[i][j];
      } else {
        __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(p.out);
        o[at] = __float2bfloat16_rn(p.accumulate ? __bfloat162float(o[at]) + acc[i][j] : acc[i][j]);
      }
    }
}

}  // namespace kdkl
