// Layer norm, forward and backward, with the gradients of its weight and bias.
//
//   mu = mean(x), rho = 1 / sqrt(mean((x - mu)^2) + eps), xh = (x - mu) rho, y = xh w + b
//   dx = rho (dy w - mean(dy w) - xh mean(dy w xh)),  dw = sum_t dy xh,  db = sum_t dy
//
// The variance is taken around the mean of the values in registers, never as a difference of two sums: a warp takes the
// mean of its own columns and the squares around it, and the warps' (sum, squares) pairs are joined exactly,
//   sum (x - mu)^2 = sum_i [ q_i + n_i (mu_i - mu)^2 ],
// so that a row costs one barrier (fp32 rows, and those in whole words: two). Everything is computed in fp32 and rounded once.
//
// A sum of 2880 equal fp32 numbers is rounded on the way, and their mean is then not the number: off by the last bit or two,
// of which a rho of 1 / sqrt(eps) makes hundredths. So the mean m of fp32 rows is corrected by the mean of the values less m,
// which are exact where they lie near m:
//   r = sum (x - m), mu = fl(m + r / H), s = mu - m (exact),  sum (x - mu)^2 = sum (x - m)^2 - s (2 r - H s)
// Equal values of 16 bits have exact sums up to 2^13 columns (11 bits times the count; bf16 2^16): such rows do without, which
// is 6 % of a wide bf16 row's time (8192 x 16384: 252 us).
// It costs fp32 rows of a block nothing (32768 x 4096 196 us), of a warp 7 % (65536 x 512 50.6 us), wider ones 5 % (8192 x
// 16384 337 us).
//
// Bound by memory: 4 bytes a value forward and 6 backward (bf16). 32768 x 4096, one B200: forward 88 us (6.1 TB/s), backward
// 131 (6.1 TB/s), its column sums 6 behind it; 1021 x 2880 4.3 and 13 us with the sums. With int8 records of x and y 254 and 139
// (floors 126 and 105: encoding takes about 70 instructions per eight values and record). Element by element (odd widths) 16384 x
// 4095 bf16 152 and 150 (floors 42 and 62), with records 403 and 276.
//
// Three shapes, by width: rows of at most 512 columns belong to a warp (no barrier); up to 8192 columns a block has the
// row in registers, eight columns a thread; wider rows are read again from the caches for the second look at them.
// In the first two the backward pass keeps the columns' sums of dw and db in registers over all rows of a warp or block
// and leaves one partial row each, which a second kernel adds in a fixed order; of wider rows they are taken by a kernel
// of their own that goes down the columns.
#pragma once
#include <type_traits>

#include "act8.cuh"

namespace kdkl {

constexpr int kLnWarpCols = 512, kLnBlockCols = 8192;
constexpr int kLnWarpThreads = 256, kLnWideThreads = 1024;

struct LnParams {
  const void* x;  long long ld_x;
  const void* weight; const void* bias; int weight_type;
  void* y;                       // contiguous
  float* mean; float* rho;       // [T]; forward: out or null
  ActRecord x_record, y_record;  // codes null: none
  int format;
  const void* dy; long long ld_dy;
  void* dx;
  float* part;                   // [parts][2][H]
  long long T; int H;
  float eps;
};

__device__ __forceinline__ float ln_warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// eight values of the weight or bias, of a type known at run time (uniform)
template <bool VEC>
__device__ __forceinline__ void load8_typed(const void* p, int type, int c, int H, float (&f)[8]) {
  if (type == 0) load8<__nv_bfloat16, VEC>(reinterpret_cast<const __nv_bfloat16*>(p), c, H, f);
  else if (type == 1) load8<float, VEC>(reinterpret_cast<const float*>(p), c, H, f);
  else load8<__half, VEC>(reinterpret_cast<const __half*>(p), c, H, f);
}
template <bool VEC>
__device__ __forceinline__ void load_affine(const LnParams& p, int c, float (&w)[8], float (&b)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) { w[i] = 1.f; b[i] = 0.f; }
  if (p.weight != nullptr) load8_typed<VEC>(p.weight, p.weight_type, c, p.H, w);
  if (p.bias != nullptr) load8_typed<VEC>(p.bias, p.weight_type, c, p.H, b);
}
template <bool VEC> __device__ __forceinline__ int columns_of(int c, int H) {      // how many of a thread's eight exist
  int n = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) n += column<VEC>(c, i) < H ? 1 : 0;
  return n;
}

// (sum, squares around its own mean) of the warps of a block -> mean and squares of the row, known to every thread.
// slots: [2][32] pairs and [32] counts in shared memory; `par` alternates from row to row, which spares a second barrier.
struct LnJoin { float mean, squares; };
// The corrected mean, and the squares around it, from r and q = sum (x - m)^2 (see above).
__device__ __forceinline__ LnJoin ln_corrected(float m, float r, float q, float H) {
  LnJoin j;
  j.mean = m + r / H;
  const float s = j.mean - m;
  const float left = q - s * (2.f * r - H * s);
  j.squares = left < 0.f ? 0.f : left;                     // (a NaN stays one)
  return j;
}
__device__ __forceinline__ LnJoin ln_join(float2 (*slots)[32], const float* counts, int par, int warps, float s, float q, float H) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (lane == 0) slots[par][warp] = make_float2(s, q);
  __syncthreads();
  const bool has = lane < warps;
  const float2 v = has ? slots[par][lane] : make_float2(0.f, 0.f);
  const float n = has ? counts[lane] : 0.f;
  LnJoin r;
  r.mean = ln_warp_sum(v.x) / H;         // a division: an exact sum of equal values has the value for its mean
  const float off = n > 0.f ? v.x / n - r.mean : 0.f;
  r.squares = ln_warp_sum(fmaf(n * off, off, v.y));
  return r;
}
__device__ __forceinline__ float2 ln_join2(float2 (*slots)[32], int par, int warps, float a, float b) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (lane == 0) slots[par][warp] = make_float2(a, b);
  __syncthreads();
  const float2 v = lane < warps ? slots[par][lane] : make_float2(0.f, 0.f);
  return make_float2(ln_warp_sum(v.x), ln_warp_sum(v.y));
}

// WARP: G groups of eight columns a lane, a row a warp; otherwise one group a thread, a row a block.
template <typename X, typename Y, int G, bool WARP, bool VEC>
__global__ void __launch_bounds__(WARP ? kLnWarpThreads : 1024)
layer_norm_forward_kernel(const LnParams p) {
  __shared__ float2 slots[2][32];
  __shared__ float counts[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int tpr = WARP ? 32 : blockDim.x, me = WARP ? lane : threadIdx.x, warps = blockDim.x >> 5;
  const long long first = WARP ? (long long)blockIdx.x * warps + warp : blockIdx.x;
  const long long step = WARP ? (long long)gridDim.x * warps : gridDim.x;
  const long long cpitch = act_codes_pitch(p.H), spitch = act_scale_pitch(p.H);
  const float inv_H = 1.f / (float)p.H;
  int c[G], have = 0;
#pragma unroll
  for (int g = 0; g < G; ++g) { c[g] = first_column<VEC>(me + g * tpr); have += columns_of<VEC>(c[g], p.H); }
  const float n_warp = ln_warp_sum((float)have);
  if (!WARP && lane == 0) counts[warp] = n_warp;
  grid_dependents_launch();
  grid_dependency_wait();
  float w[G][8], b[G][8];
#pragma unroll
  for (int g = 0; g < G; ++g) load_affine<VEC>(p, c[g], w[g], b[g]);
  int par = 0;
  Raw8<X> raw[G];
  const X* x = reinterpret_cast<const X*>(p.x);
#pragma unroll
  for (int g = 0; g < G; ++g)
    if (first < p.T) raw[g] = load_raw8<X, VEC>(x + first * p.ld_x, c[g], p.H);
  for (long long t = first; t < p.T; t += step, par ^= 1) {
    float f[G][8], s = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      raw_to_f32(raw[g], f[g]);
#pragma unroll
      for (int i = 0; i < 8; ++i) s += f[g][i];
    }
    if (t + step < p.T) {                                  // the next row is on its way while this one is worked on
#pragma unroll
      for (int g = 0; g < G; ++g) raw[g] = load_raw8<X, VEC>(x + (t + step) * p.ld_x, c[g], p.H);
    }
    constexpr bool kCorrect = sizeof(X) == 4;
    s = ln_warp_sum(s);
    if (kCorrect && !WARP) s = ln_join2(slots, 0, warps, s, 0.f).x;          // (then `mine` is the row's mean)
    const float n = kCorrect && !WARP ? (float)p.H : n_warp;
    const float mine = n > 0.f ? s / n : 0.f;
    float q = 0.f, r = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = (VEC ? c[g] : column<VEC>(c[g], i)) < p.H ? f[g][i] - mine : 0.f;
        q = fmaf(d, d, q);
        if (kCorrect) r += d;
      }
    q = ln_warp_sum(q);
    LnJoin j = {mine, q};
    if (kCorrect) {
      r = ln_warp_sum(r);
      if (!WARP) { const float2 sums = ln_join2(slots, 1, warps, r, q); r = sums.x; q = sums.y; }
      j = ln_corrected(mine, r, q, (float)p.H);
    } else if (!WARP) {
      j = ln_join(slots, counts, par, warps, s, q, (float)p.H);
    }
    const float mean = j.mean, squares = j.squares;
    const float rho = 1.f / sqrtf(fmaf(squares, inv_H, p.eps));
    if (me == 0 && p.mean != nullptr) { p.mean[t] = mean; p.rho[t] = rho; }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = fmaf((f[g][i] - mean) * rho, w[g][i], b[g][i]);
      const Raw8<Y> out = f32_to_raw<Y>(y);
      store_raw8<Y, VEC>(reinterpret_cast<Y*>(p.y) + t * p.H, c[g], p.H, out);
      if (p.x_record.codes != nullptr) record_write8<VEC>(p.format, p.x_record, t, cpitch, spitch, c[g], f[g]);
      if (p.y_record.codes != nullptr) {                   // of y as it is returned
        raw_to_f32(out, y);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (column<VEC>(c[g], i) >= p.H) y[i] = 0.f;     // padding codes are zeros
        record_write8<VEC>(p.format, p.y_record, t, cpitch, spitch, c[g], y);
      }
    }
  }
}

// ------------------------------------------------------------------ rows of a block, in whole words
// The shape most rows take: a block has a row, a thread two groups of eight columns. A thread's words of the next rows are on
// their way into places of its own in shared memory (cp.async), kLnAhead rows ahead: no barrier but the one of the sums, and
// enough bytes in flight to fill the memory's latency (8 KB rows, two or three blocks an SM: 50 to 100 KB). Two
// values an instruction. What is in the loop beside the arithmetic decides: with 64-bit row counters, a test a column group
// and true divisions the same kernels took 125 and 178 us where they take 88 and 131 now.
constexpr int kLnAhead = 3, kLnRowsThreads = 512;
template <int BYTES> __device__ __forceinline__ void cp_async(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
  if (BYTES == 32) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + 16), "l"(reinterpret_cast<const char*>(from) + 16) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
template <typename T> __device__ __forceinline__ void shared_pairs(uint32_t at, float2 (&f)[4]) {
  Raw8<T> r;
  r.v = ld_shared_v4(at);
  if constexpr (sizeof(T) == 4) r.w = ld_shared_v4(at + 16);
  float v[8];
  raw_to_f32(r, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = make_float2(v[2 * i], v[2 * i + 1]);
}
template <typename T> __device__ __forceinline__ Raw8<T> pairs_to_raw(const float2 (&f)[4]) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = f[i].x; v[2 * i + 1] = f[i].y; }
  return f32_to_raw<T>(v);
}
__device__ __forceinline__ void affine_pairs(const void* p, int type, int c, int H, float fill, float2 (&f)[4]) {
  float v[8];
  if (p != nullptr) load8_typed<true>(p, type, c, H, v);
  else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c < H ? fill : 0.f;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = make_float2(v[2 * i], v[2 * i + 1]);
}

// Sums over a block, known to every thread: a warp's go to its slot, and behind the barrier every thread adds up the slots,
// eight at a time in whole words, in their order. Slots of absent warps stay zeros (ln_slots_clear). Two joins that
// follow one another use different slots, which spares a second barrier.
struct __align__(16) LnSlots { float2 two[32]; float one[32]; };
__device__ __forceinline__ void ln_slots_clear(LnSlots& s) {
  if (threadIdx.x < 32) { s.two[threadIdx.x] = both(0.f); s.one[threadIdx.x] = 0.f; }
}
__device__ __forceinline__ float2 low2(const float4& v) { return make_float2(v.x, v.y); }
__device__ __forceinline__ float2 high2(const float4& v) { return make_float2(v.z, v.w); }
__device__ __forceinline__ float ln_block_sum(LnSlots& s, int warps, float v) {
  v = ln_warp_sum(v);
  if ((threadIdx.x & 31) == 0) s.one[threadIdx.x >> 5] = v;
  __syncthreads();
  const float4* q = reinterpret_cast<const float4*>(s.one);
  float2 t = add2(add2(low2(q[0]), high2(q[0])), add2(low2(q[1]), high2(q[1])));
  for (int i = 8; i < warps; i += 8, q += 2) t = add2(t, add2(add2(low2(q[2]), high2(q[2])), add2(low2(q[3]), high2(q[3]))));
  return t.x + t.y;
}
__device__ __forceinline__ float2 ln_block_sum2(LnSlots& s, int warps, float a, float b) {
  a = ln_warp_sum(a); b = ln_warp_sum(b);
  if ((threadIdx.x & 31) == 0) s.two[threadIdx.x >> 5] = make_float2(a, b);
  __syncthreads();
  const float4* q = reinterpret_cast<const float4*>(s.two);
  float2 t = both(0.f);
  for (int i = 0; i < warps; i += 8, q += 4)
    t = add2(t, add2(add2(add2(low2(q[0]), high2(q[0])), add2(low2(q[1]), high2(q[1]))), add2(add2(low2(q[2]), high2(q[2])), add2(low2(q[3]), high2(q[3])))));
  return t;
}
// s / n with n's reciprocal at hand: the remainder of the first guess is exact, so n times a number is divided without an error
__device__ __forceinline__ float ln_quotient(float s, float n, float inv_n) {
  const float m = s * inv_n;
  return fmaf(fmaf(-m, n, s), inv_n, m);
}

// FULL: every thread's columns exist (H = 16 x threads); otherwise the places of those that do not hold zeros throughout.
template <typename X, typename Y, bool REC, bool FULL>
__global__ void __launch_bounds__(kLnRowsThreads)
layer_norm_forward_rows_kernel(const LnParams p) {
  extern __shared__ uint4 ln_smem[];
  __shared__ LnSlots first, second;
  constexpr int XB = 8 * sizeof(X);
  const int warps = blockDim.x >> 5, far = 8 * blockDim.x, T = (int)p.T;
  const long long cpitch = act_codes_pitch(p.H), spitch = act_scale_pitch(p.H);
  const float H = (float)p.H, inv_H = 1.f / H;
  const int c = 8 * (int)threadIdx.x;                      // and c + far
  const bool in[2] = {FULL || c < p.H, FULL || c + far < p.H};
  const uint32_t mine = smem_u32(ln_smem) + threadIdx.x * XB, group = blockDim.x * XB;
  ln_slots_clear(first); ln_slots_clear(second);
#pragma unroll
  for (int i = 0; i < 2 * kLnAhead; ++i)
    if (!in[i & 1]) {
#pragma unroll
      for (int k = 0; k < XB; k += 16) st_shared_v4(mine + i * group + k, 0u, 0u, 0u, 0u);
    }
  __syncthreads();
  const X* next = reinterpret_cast<const X*>(p.x) + blockIdx.x * p.ld_x + c;
  const long long step = gridDim.x * p.ld_x, out_step = (long long)gridDim.x * p.H;
  int asked = blockIdx.x;
  auto ask = [&](int stage) {
    if (asked < T) {
      if (in[0]) cp_async<XB>(mine + 2 * stage * group, next);
      if (in[1]) cp_async<XB>(mine + (2 * stage + 1) * group, next + far);
    }
    cp_async_commit();
    next += step; asked += gridDim.x;
  };
  grid_dependents_launch();
  grid_dependency_wait();
#pragma unroll
  for (int s = 0; s < kLnAhead; ++s) ask(s);
  float2 w[2][4], b[2][4];
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    affine_pairs(p.weight, p.weight_type, c + g * far, p.H, 1.f, w[g]);
    affine_pairs(p.bias, p.weight_type, c + g * far, p.H, 0.f, b[g]);
  }
  Y* out = reinterpret_cast<Y*>(p.y) + (long long)blockIdx.x * p.H;
  int stage = 0;
  for (int t = blockIdx.x; t < T; t += gridDim.x, out += out_step) {
    cp_async_wait<kLnAhead - 1>();
    float2 f[2][4], sum = both(0.f), squares = both(0.f);
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      shared_pairs<X>(mine + (2 * stage + g) * group, f[g]);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum = add2(sum, f[g][i]);
    }
    ask(stage);                                            // (into places that this thread alone has just read)
    if (++stage == kLnAhead) stage = 0;
    constexpr bool kCorrect = sizeof(X) == 4;
    float mean = ln_quotient(ln_block_sum(first, warps, sum.x + sum.y), H, inv_H), squared;
    float2 rest = both(0.f);
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const float2 off = both(in[g] ? -mean : 0.f);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[g][i] = add2(f[g][i], off);
        squares = fma2(f[g][i], f[g][i], squares);
        if (kCorrect) rest = add2(rest, f[g][i]);
      }
    }
    if constexpr (kCorrect) {
      const float2 sums = ln_block_sum2(second, warps, rest.x + rest.y, squares.x + squares.y);
      const LnJoin j = ln_corrected(mean, sums.x, sums.y, H);
      squared = j.squares;
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const float2 off = both(in[g] ? mean - j.mean : 0.f);
#pragma unroll
        for (int i = 0; i < 4; ++i) f[g][i] = add2(f[g][i], off);
      }
      mean = j.mean;
    } else {
      squared = ln_block_sum(second, warps, squares.x + squares.y);
    }
    // (off by two units at most, where the other shapes' root and division take one: these lie between a row's barrier and its
    // stores, 4.7 against 4.3 us for 1021 x 2880 bf16, 92.5 against 91 for 32768 x 4096)
    const float rho = rsqrtf(fmaf(squared, inv_H, p.eps));
    if (threadIdx.x == 0 && p.mean != nullptr) { p.mean[t] = mean; p.rho[t] = rho; }
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int at = c + g * far;
      float2 y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = fma2(mul2(f[g][i], both(rho)), w[g][i], b[g][i]);
      const Raw8<Y> raw = pairs_to_raw<Y>(y);
      if (in[g]) store_raw8<Y, true>(out, at, at + 1, raw);
      if (REC) {
        float v[8];
        if (p.x_record.codes != nullptr) {                 // x once more, from where it came
          load8<X, true>(reinterpret_cast<const X*>(p.x) + t * p.ld_x, at, p.H, v);
          record_write8<true>(p.format, p.x_record, t, cpitch, spitch, at, v);
        }
        if (p.y_record.codes != nullptr) {                 // of y as it is returned; padding codes are zeros
          raw_to_f32(raw, v);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = in[g] ? v[i] : 0.f;
          record_write8<true>(p.format, p.y_record, t, cpitch, spitch, at, v);
        }
      }
    }
  }
  cp_async_wait<0>();
}

template <typename X, typename Y, int FMT /* -1: from x itself */, bool FULL>
__global__ void __launch_bounds__(kLnRowsThreads)
layer_norm_backward_rows_kernel(const LnParams p) {
  extern __shared__ uint4 ln_smem[];
  __shared__ LnSlots even, odd;
  constexpr bool REC = FMT >= 0;
  constexpr int XB = REC ? 0 : 8 * sizeof(X), YB = 8 * sizeof(Y);
  const int warps = blockDim.x >> 5, far = 8 * blockDim.x, T = (int)p.T;
  const long long cpitch = act_codes_pitch(p.H), spitch = act_scale_pitch(p.H);
  const float inv_H = 1.f / (float)p.H;
  const int c = 8 * (int)threadIdx.x;
  const bool in[2] = {FULL || c < p.H, FULL || c + far < p.H};
  const uint32_t base = smem_u32(ln_smem), group = blockDim.x * (XB + YB);
  const uint32_t my_x = base + threadIdx.x * XB, my_y = base + blockDim.x * XB + threadIdx.x * YB;
  ln_slots_clear(even); ln_slots_clear(odd);
#pragma unroll
  for (int i = 0; i < 2 * kLnAhead; ++i)
    if (!in[i & 1]) {
#pragma unroll
      for (int k = 0; k < XB; k += 16) st_shared_v4(my_x + i * group + k, 0u, 0u, 0u, 0u);
#pragma unroll
      for (int k = 0; k < YB; k += 16) st_shared_v4(my_y + i * group + k, 0u, 0u, 0u, 0u);
    }
  __syncthreads();
  const X* next_x = reinterpret_cast<const X*>(p.x) + blockIdx.x * p.ld_x + c;
  const Y* next_y = reinterpret_cast<const Y*>(p.dy) + blockIdx.x * p.ld_dy + c;
  const long long step_x = gridDim.x * p.ld_x, step_y = gridDim.x * p.ld_dy, out_step = (long long)gridDim.x * p.H;
  int asked = blockIdx.x;
  auto ask = [&](int stage) {
    if (asked < T) {
#pragma unroll
      for (int g = 0; g < 2; ++g)
        if (in[g]) {
          if constexpr (!REC) cp_async<XB>(my_x + (2 * stage + g) * group, next_x + g * far);
          cp_async<YB>(my_y + (2 * stage + g) * group, next_y + g * far);
        }
    }
    cp_async_commit();
    if constexpr (!REC) next_x += step_x;
    next_y += step_y; asked += gridDim.x;
  };
  // the small things of the next row in registers
  uint2 codes[2] = {make_uint2(0u, 0u), make_uint2(0u, 0u)};
  uint32_t bytes[2] = {1u, 1u};
  float mean = 0.f, rho = 0.f;
  auto ahead = [&](int t) {
    if (t < T) {
      mean = p.mean[t]; rho = p.rho[t];
      if (REC) {
#pragma unroll
        for (int g = 0; g < 2; ++g)
          if (in[g]) record_fetch8(p.x_record, t, cpitch, spitch, c + g * far, codes[g], bytes[g]);
      }
    }
  };
  grid_dependents_launch();
  grid_dependency_wait();
#pragma unroll
  for (int s = 0; s < kLnAhead; ++s) ask(s);
  ahead(blockIdx.x);
  float2 w[2][4], aw[2][4], ab[2][4];
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    affine_pairs(p.weight, p.weight_type, c + g * far, p.H, 1.f, w[g]);
#pragma unroll
    for (int i = 0; i < 4; ++i) aw[g][i] = ab[g][i] = both(0.f);
  }
  X* out = reinterpret_cast<X*>(p.dx) + (long long)blockIdx.x * p.H;
  int stage = 0;
  bool second = false;
  for (int t = blockIdx.x; t < T; t += gridDim.x, out += out_step) {
    const float2 off = both(-mean), r = both(rho);
    float2 xh[2][4], d[2][4], s1 = both(0.f), s2 = both(0.f);
    if constexpr (REC) {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        float v[8];
        act_values<REC ? FMT : 0>(codes[g], bytes[g], v);
#pragma unroll
        for (int i = 0; i < 4; ++i) xh[g][i] = make_float2(v[2 * i], v[2 * i + 1]);
      }
    }
    cp_async_wait<kLnAhead - 1>();
    ahead(t + gridDim.x);
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      if constexpr (!REC) shared_pairs<X>(my_x + (2 * stage + g) * group, xh[g]);
      shared_pairs<Y>(my_y + (2 * stage + g) * group, d[g]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        xh[g][i] = mul2(add2(xh[g][i], off), r);
        aw[g][i] = fma2(d[g][i], xh[g][i], aw[g][i]);
        ab[g][i] = add2(ab[g][i], d[g][i]);
        d[g][i] = mul2(d[g][i], w[g][i]);
        s1 = add2(s1, d[g][i]);
        s2 = fma2(d[g][i], xh[g][i], s2);
      }
    }
    ask(stage);
    if (++stage == kLnAhead) stage = 0;
    const float2 sums = ln_block_sum2(second ? odd : even, warps, s1.x + s1.y, s2.x + s2.y);
    second = !second;
    const float2 a = both(-sums.x * inv_H), b = both(-sums.y * inv_H);
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int at = c + g * far;
#pragma unroll
      for (int i = 0; i < 4; ++i) d[g][i] = mul2(add2(d[g][i], fma2(xh[g][i], b, a)), r);
      if (in[g]) store_raw8<X, true>(out, at, at + 1, pairs_to_raw<X>(d[g]));
    }
  }
  cp_async_wait<0>();
  if (p.part == nullptr) return;
  float* part = p.part + (long long)blockIdx.x * 2 * p.H + c;
#pragma unroll
  for (int g = 0; g < 2; ++g)
    if (in[g]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        *reinterpret_cast<float2*>(part + g * far + 2 * i) = aw[g][i];
        *reinterpret_cast<float2*>(part + p.H + g * far + 2 * i) = ab[g][i];
      }
    }
}

// Rows wider than a block's registers: three looks at the row, the second and third from the caches.
template <typename X, typename Y, bool VEC>
__global__ void __launch_bounds__(kLnWideThreads)
layer_norm_forward_wide_kernel(const LnParams p) {
  __shared__ float2 slots[2][32];
  const int warps = blockDim.x >> 5, cols = blockDim.x * 8;
  const long long cpitch = act_codes_pitch(p.H), spitch = act_scale_pitch(p.H);
  const float inv_H = 1.f / (float)p.H;
  const int c0 = first_column<VEC>(threadIdx.x);
  const bool correct = !std::is_same_v<X, __nv_bfloat16> || p.H > 1 << 16;
  grid_dependents_launch();
  grid_dependency_wait();
  for (long long t = blockIdx.x; t < p.T; t += gridDim.x) {
    const X* row = reinterpret_cast<const X*>(p.x) + t * p.ld_x;
    float f[8], s = 0.f, q = 0.f;
    for (int base = 0; base < p.H; base += cols) {
      load8<X, VEC>(row, base + c0, p.H, f);
#pragma unroll
      for (int i = 0; i < 8; ++i) s += f[i];
    }
    const float first = ln_join2(slots, 0, warps, ln_warp_sum(s), 0.f).x / (float)p.H;
    float r = 0.f;
    auto look = [&](auto with) {
      for (int base = 0; base < p.H; base += cols) {
        load8<X, VEC>(row, base + c0, p.H, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float d = column<VEC>(base + c0, i) < p.H ? f[i] - first : 0.f;
          q = fmaf(d, d, q);
          if (decltype(with)::value) r += d;
        }
      }
    };
    LnJoin j = {first, 0.f};
    if (correct) {
      look(std::true_type());
      const float2 sums = ln_join2(slots, 1, warps, ln_warp_sum(r), ln_warp_sum(q));
      j = ln_corrected(first, sums.x, sums.y, (float)p.H);
    } else {
      look(std::false_type());
      j.squares = ln_join2(slots, 1, warps, ln_warp_sum(q), 0.f).x;
    }
    const float mean = j.mean, rho = 1.f / sqrtf(fmaf(j.squares, inv_H, p.eps));
    if (threadIdx.x == 0 && p.mean != nullptr) { p.mean[t] = mean; p.rho[t] = rho; }
    for (int base = 0; base < p.H; base += cols) {         // the same trips for every thread: records are a warp's work
      const int c = base + c0;
      float w[8], b[8], y[8];
      load8<X, VEC>(row, c, p.H, f);
      load_affine<VEC>(p, c, w, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = fmaf((f[i] - mean) * rho, w[i], b[i]);
      const Raw8<Y> out = f32_to_raw<Y>(y);
      store_raw8<Y, VEC>(reinterpret_cast<Y*>(p.y) + t * p.H, c, p.H, out);
      if (p.x_record.codes != nullptr) record_write8<VEC>(p.format, p.x_record, t, cpitch, spitch, c, f);
      if (p.y_record.codes != nullptr) {
        raw_to_f32(out, y);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (column<VEC>(c, i) >= p.H) y[i] = 0.f;
        record_write8<VEC>(p.format, p.y_record, t, cpitch, spitch, c, y);
      }
    }
  }
}

// x of the backward pass: the tensor, or what its record stands for
template <typename X, bool REC, bool VEC>
__device__ __forceinline__ void ln_x8(const LnParams& p, long long t, long long cpitch, long long spitch, int c, float (&f)[8]) {
  if (REC) record_read8<VEC>(p.format, p.x_record, t, cpitch, spitch, c, f);
  else load8<X, VEC>(reinterpret_cast<const X*>(p.x) + t * p.ld_x, c, p.H, f);
}

template <typename X, typename Y, int G, bool WARP, bool REC, bool VEC>
__global__ void __launch_bounds__(WARP ? kLnWarpThreads : 1024)
layer_norm_backward_kernel(const LnParams p) {
  __shared__ float2 slots[2][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int tpr = WARP ? 32 : blockDim.x, me = WARP ? lane : threadIdx.x, warps = blockDim.x >> 5;
  const long long first = WARP ? (long long)blockIdx.x * warps + warp : blockIdx.x;
  const long long step = WARP ? (long long)gridDim.x * warps : gridDim.x;
  const long long cpitch = act_codes_pitch(p.H), spitch = act_scale_pitch(p.H);
  const float inv_H = 1.f / (float)p.H;
  int c[G];
#pragma unroll
  for (int g = 0; g < G; ++g) c[g] = first_column<VEC>(me + g * tpr);
  grid_dependents_launch();
  grid_dependency_wait();
  float w[G][8], aw[G][8], ab[G][8];
#pragma unroll
  for (int g = 0; g < G; ++g) {
#pragma unroll
    for (int i = 0; i < 8; ++i) { w[g][i] = 1.f; aw[g][i] = 0.f; ab[g][i] = 0.f; }
    if (p.weight != nullptr) load8_typed<VEC>(p.weight, p.weight_type, c[g], p.H, w[g]);
  }
  int par = 0;
  for (long long t = first; t < p.T; t += step, par ^= 1) {
    const float mean = p.mean[t], rho = p.rho[t];
    float xh[G][8], d[G][8], s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      ln_x8<X, REC, VEC>(p, t, cpitch, spitch, c[g], xh[g]);
      load8<Y, VEC>(reinterpret_cast<const Y*>(p.dy) + t * p.ld_dy, c[g], p.H, d[g]);   // 0 past the row's end
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        xh[g][i] = (xh[g][i] - mean) * rho;
        aw[g][i] = fmaf(d[g][i], xh[g][i], aw[g][i]);
        ab[g][i] += d[g][i];
        d[g][i] *= w[g][i];
        s1 += d[g][i];
        s2 = fmaf(d[g][i], xh[g][i], s2);
      }
    }
    s1 = ln_warp_sum(s1); s2 = ln_warp_sum(s2);
    if (!WARP) { const float2 s = ln_join2(slots, par, warps, s1, s2); s1 = s.x; s2 = s.y; }
    s1 *= inv_H; s2 *= inv_H;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = rho * (d[g][i] - fmaf(xh[g][i], s2, s1));
      store_raw8<X, VEC>(reinterpret_cast<X*>(p.dx) + t * p.H, c[g], p.H, f32_to_raw<X>(o));
    }
  }
  if (p.part != nullptr) {
    const long long slot = WARP ? (long long)blockIdx.x * warps + warp : blockIdx.x;
    float* part = p.part + slot * 2 * p.H;
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int col = column<VEC>(c[g], i);
        if (col < p.H) { part[col] = aw[g][i]; part[p.H + col] = ab[g][i]; }
      }
  }
}

template <typename X, typename Y, bool REC, bool VEC>
__global__ void __launch_bounds__(kLnWideThreads)
layer_norm_backward_wide_kernel(const LnParams p) {
  __shared__ float2 slots[2][32];
  const int warps = blockDim.x >> 5, cols = blockDim.x * 8;
  const long long cpitch = act_codes_pitch(p.H), spitch = act_scale_pitch(p.H);
  const float inv_H = 1.f / (float)p.H;
  const int c0 = first_column<VEC>(threadIdx.x);
  grid_dependents_launch();
  grid_dependency_wait();
  int par = 0;
  for (long long t = blockIdx.x; t < p.T; t += gridDim.x, par ^= 1) {
    const float mean = p.mean[t], rho = p.rho[t];
    const Y* dy = reinterpret_cast<const Y*>(p.dy) + t * p.ld_dy;
    float x[8], d[8], w[8], s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 1.f;
    for (int base = 0; base < p.H; base += cols) {
      const int c = base + c0;
      ln_x8<X, REC, VEC>(p, t, cpitch, spitch, c, x);
      load8<Y, VEC>(dy, c, p.H, d);
      if (p.weight != nullptr) load8_typed<VEC>(p.weight, p.weight_type, c, p.H, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float e = d[i] * w[i];
        s1 += e;
        s2 = fmaf(e, (x[i] - mean) * rho, s2);
      }
    }
    const float2 s = ln_join2(slots, par, warps, ln_warp_sum(s1), ln_warp_sum(s2));
    s1 = s.x * inv_H; s2 = s.y * inv_H;
    for (int base = 0; base < p.H; base += cols) {
      const int c = base + c0;
      ln_x8<X, REC, VEC>(p, t, cpitch, spitch, c, x);
      load8<Y, VEC>(dy, c, p.H, d);
      if (p.weight != nullptr) load8_typed<VEC>(p.weight, p.weight_type, c, p.H, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) d[i] = rho * (d[i] * w[i] - fmaf((x[i] - mean) * rho, s2, s1));
      store_raw8<X, VEC>(reinterpret_cast<X*>(p.dx) + t * p.H, c, p.H, f32_to_raw<X>(d));
    }
  }
}

// Column sums of wide rows: a block has 2048 columns (256 threads) of the rows blockIdx.y, + gridDim.y, ...
template <typename X, typename Y, bool REC, bool VEC>
__global__ void __launch_bounds__(256)
layer_norm_columns_kernel(const LnParams p) {
  const long long cpitch = act_codes_pitch(p.H), spitch = act_scale_pitch(p.H);
  const int c = blockIdx.x * 2048 + first_column<VEC>(threadIdx.x);
  float aw[8], ab[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) aw[i] = ab[i] = 0.f;
  grid_dependents_launch();
  grid_dependency_wait();
  for (long long t = blockIdx.y; t < p.T; t += gridDim.y) {
    float x[8], d[8];
    const float mean = p.mean[t], rho = p.rho[t];
    ln_x8<X, REC, VEC>(p, t, cpitch, spitch, c, x);
    load8<Y, VEC>(reinterpret_cast<const Y*>(p.dy) + t * p.ld_dy, c, p.H, d);
#pragma unroll
    for (int i = 0; i < 8; ++i) { aw[i] = fmaf(d[i], (x[i] - mean) * rho, aw[i]); ab[i] += d[i]; }
  }
  float* part = p.part + (long long)blockIdx.y * 2 * p.H;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int col = column<VEC>(c, i);
    if (col < p.H) { part[col] = aw[i]; part[p.H + col] = ab[i]; }
  }
}

// dw and db from the partial rows, in a fixed order: 32 columns a block, 32 warps share the rows.
__global__ void __launch_bounds__(1024)
layer_norm_reduce_kernel(const float* part, long long parts, int H, void* dweight, void* dbias, int type) {
  __shared__ float sums[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, which = blockIdx.y;
  const int col = blockIdx.x * 32 + lane;
  grid_dependents_launch();
  grid_dependency_wait();
  float s = 0.f;
  if (col < H) {
#pragma unroll 4
    for (long long r = warp; r < parts; r += 32) s += part[(r * 2 + which) * H + col];
  }
  sums[warp][lane] = s;
  __syncthreads();
  if (warp != 0) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) s += sums[i][lane];
  void* out = which == 0 ? dweight : dbias;
  if (col >= H || out == nullptr) return;
  if (type == 0) reinterpret_cast<__nv_bfloat16*>(out)[col] = __float2bfloat16_rn(s);
  else if (type == 1) reinterpret_cast<float*>(out)[col] = s;
  else reinterpret_cast<__half*>(out)[col] = __float2half_rn(s);
}

}  // namespace kdkl
