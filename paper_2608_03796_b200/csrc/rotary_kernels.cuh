// Rotary positions: the first R of a head's D columns are R / 2 pairs, and pair i of a token at position n is turned by the
// angle 2 pi n f_i (f_i in turns a position) and multiplied by one factor m:
//   (a, b) -> m (a cos - b sin, b cos + a sin)
// A pair is columns (i, i + R / 2) or (2 i, 2 i + 1). The backward pass is the same with the angle negated.
//
// The angle: n f_i in fp64, less the nearest whole number, then sine and cosine of pi times an fp32 number in [-1, 1].
// In fp32 the product alone would be off by 2^-24 of itself, a hundredth of a turn at position 10^6. A block takes a few
// tokens, forms their R / 2 pairs of numbers once in shared memory and uses them for all heads, so that the fp64 work is
// one in (heads D / (R / 2)) values. What remains is one read and one write of every value: bound by memory.
#pragma once
#include "act8.cuh"

namespace kdkl {

struct RotaryTensor {
  const void* x; long long x_token, x_head;      // strides in elements
  void* y;       long long y_token, y_head;
  int heads;
};
struct RotaryParams {
  RotaryTensor t[2];                             // the second may have no heads
  const void* positions; int wide_positions;     // int32 or int64 [T]
  const double* turns;                           // [R / 2]
  float magnitude, sign;
  long long T;
  int D, R, tokens_per_block;
  unsigned long long by_items, by_heads;         // see rotary_quotient
};

// i / d for i < 2^25 and d <= 2^13 by 2^40 / d, rounded up: i times what the rounding adds is below 2^38 (d = 1: 0 stands for it).
// For neighbours that are paired, where a thread's item is half as long: 32768 tokens, 40 heads of 128 columns of bf16 114 us, by
// plain divisions 124; for halves the plain ones, which take fewer registers, are faster: 105 against 109.
__host__ __device__ constexpr unsigned long long rotary_reciprocal(int d) { return d == 1 ? 0ull : (1ull << 40) / d + 1; }
__device__ __forceinline__ int rotary_quotient(int i, unsigned long long by) { return by == 0 ? i : (int)((unsigned long long)i * by >> 40); }

template <typename T, int N, bool ALIGNED> __device__ __forceinline__ void rotary_load(const T* p, float (&f)[N]) {
  if constexpr (ALIGNED && sizeof(T) * N == 16) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    const T* e = reinterpret_cast<const T*>(&v);
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = to_f32(e[i]);
  } else if constexpr (ALIGNED && sizeof(T) * N == 8) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    const T* e = reinterpret_cast<const T*>(&v);
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = to_f32(e[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = to_f32(p[i]);
  }
}
template <typename T, int N, bool ALIGNED> __device__ __forceinline__ void rotary_store(T* p, const float (&f)[N]) {
  T e[N];
#pragma unroll
  for (int i = 0; i < N; ++i) e[i] = from_f32<T>(f[i]);
  if constexpr (ALIGNED && sizeof(T) * N == 16) {
    uint4 v;
    memcpy(&v, e, 16);
    *reinterpret_cast<uint4*>(p) = v;
  } else if constexpr (ALIGNED && sizeof(T) * N == 8) {
    uint2 v;
    memcpy(&v, e, 8);
    *reinterpret_cast<uint2*>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = e[i];
  }
}

// M neighbours of the table, two in a word where they start on one
template <int M, bool ALIGNED> __device__ __forceinline__ void rotary_angles(const float2* table, float2 (&cs)[M]) {
  if constexpr (ALIGNED && M % 2 == 0) {
#pragma unroll
    for (int i = 0; i < M; i += 2) {
      const float4 v = *reinterpret_cast<const float4*>(table + i);
      cs[i] = make_float2(v.x, v.y); cs[i + 1] = make_float2(v.z, v.w);
    }
  } else {
#pragma unroll
    for (int i = 0; i < M; ++i) cs[i] = table[i];
  }
}

// N columns at a time (of each half, where the halves are paired). ALIGNED: N columns are an aligned word of 8 or 16 bytes.
template <typename T, bool HALF, int N, bool ALIGNED>
__global__ void __launch_bounds__(256)
rotary_kernel(const RotaryParams p) {
  extern __shared__ __align__(16) float2 table[];                        // [tokens][R / 2]: (cos, sin)
  const int pairs = p.R / 2;
  const long long t0 = (long long)blockIdx.x * p.tokens_per_block;
  const int tokens = (int)(p.T - t0 < p.tokens_per_block ? p.T - t0 : p.tokens_per_block);
  grid_dependents_launch();
  grid_dependency_wait();
  for (int i = threadIdx.x; i < tokens * pairs; i += blockDim.x) {
    const int k = i / pairs;
    const long long n = p.wide_positions ? reinterpret_cast<const long long*>(p.positions)[t0 + k]
                                         : reinterpret_cast<const int*>(p.positions)[t0 + k];
    const double turns = (double)n * p.turns[i - k * pairs];
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    table[i] = make_float2(c * p.magnitude, s * p.magnitude * p.sign);
  }
  __syncthreads();
  const int heads = p.t[0].heads + p.t[1].heads;
  const int turned = HALF ? pairs / N : p.R / N;           // items of a head that are turned; the others are copied
  const int items = turned + (p.D - p.R) / N;
  const int all = tokens * heads * items;                  // at most 4 x 8192 x 1024
  for (int i = threadIdx.x; i < all; i += blockDim.x) {
    const int th = HALF ? i / items : rotary_quotient(i, p.by_items), item = i - th * items;
    const int k = HALF ? th / heads : rotary_quotient(th, p.by_heads);
    int head = th - k * heads;
    const RotaryTensor& r = head < p.t[0].heads ? p.t[0] : p.t[1];
    if (head >= p.t[0].heads) head -= p.t[0].heads;
    const T* x = reinterpret_cast<const T*>(r.x) + (t0 + k) * r.x_token + head * r.x_head;
    T* y = reinterpret_cast<T*>(r.y) + (t0 + k) * r.y_token + head * r.y_head;
    float a[N];
    if (item >= turned) {
      const int c = p.R + (item - turned) * N;
      rotary_load<T, N, ALIGNED>(x + c, a);
      rotary_store<T, N, ALIGNED>(y + c, a);
    } else if (HALF) {
      float b[N], u[N], v[N];
      const int c = item * N;
      rotary_load<T, N, ALIGNED>(x + c, a);
      rotary_load<T, N, ALIGNED>(x + pairs + c, b);
      float2 cs[N];
      rotary_angles<N, ALIGNED>(table + k * pairs + c, cs);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        u[j] = a[j] * cs[j].x - b[j] * cs[j].y;
        v[j] = b[j] * cs[j].x + a[j] * cs[j].y;
      }
      rotary_store<T, N, ALIGNED>(y + c, u);
      rotary_store<T, N, ALIGNED>(y + pairs + c, v);
    } else {
      float u[N];
      const int c = item * N;
      rotary_load<T, N, ALIGNED>(x + c, a);
      float2 cs[N / 2 > 0 ? N / 2 : 1];
      rotary_angles<(N / 2 > 0 ? N / 2 : 1), ALIGNED>(table + k * pairs + c / 2, cs);
#pragma unroll
      for (int j = 0; j < N; j += 2) {
        u[j] = a[j] * cs[j / 2].x - a[j + 1] * cs[j / 2].y;
        u[j + 1] = a[j + 1] * cs[j / 2].x + a[j] * cs[j / 2].y;
      }
      rotary_store<T, N, ALIGNED>(y + c, u);
    }
  }
}

}  // namespace kdkl
