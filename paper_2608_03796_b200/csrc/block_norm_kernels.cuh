// The join between two blocks of a student: norm of a block's output, gate, residual sum, norm for the next block.
//
//   n = b rho1 (w1 + o),  rho1 = 1 / sqrt(mean b^2 + eps)         post norm (absent: n = b)
//   x = beta r + alpha gate n                                     gate: none, per channel or per token
//   y = x rho2 (w2 + o),  rho2 = 1 / sqrt(mean x^2 + eps)         pre norm of the next block (absent: no y)
//
// Backward, from dy and the residual stream's gradient dx, with b^ = b rho1 and x^ = x rho2 of what was kept:
//   d  = dx + rho2 (gy - x^ c2),   gy = dy (w2 + o),   c2 = mean(gy x^)
//   dr = beta d,   dw2 = sum_t dy x^
//   db = rho1 (k d - b^ c1),       k = alpha gate (w1 + o),   c1 = mean(k d b^);       dw1 = sum_t alpha gate d b^
//   dgate = sum alpha d b^ (w1 + o), over the tokens (channel gate) or over the row (token gate)
// c1 needs d and so c2, but mean(k d b^) = mean(k b^ (dx + rho2 gy)) - c2 rho2 mean(k b^ x^): all sums of a row come
// from one reduction over its values, and nothing is read twice.
//
// Bound by memory: forward 8 bytes a value (+ 33/32 per record), backward 12 (10.06 from records). One block per row
// and a stride over the rows; a thread keeps the same columns throughout, so the column sums dw1, dw2 and dgate stay
// in its registers until the end, leave as one partial row per block, and a second kernel adds the partial rows in a
// fixed order: bitwise reproducible.
//
// Two kernels each way. The *_rows kernels take rows that are whole words; rows wider than a block's 8192 columns are
// shared by a cluster, whose blocks leave their sums in one another's shared memory. The next rows travel to shared memory
// (cp.async, places that only their own thread touches, so no barrier) while a row is worked on, what depends on the
// column alone is formed once, and two values go through an instruction. The *_any kernels take everything else: odd
// widths and addresses.
// 32768 x 4096 bf16, one B200, in a loop over inputs beyond the L2: forward 180 us (6.0 TB/s), leaving int8 records 255 us
// (5.3 TB/s); backward with its column sums 297 us (5.4 TB/s), from int8 records 291 us (4.6 TB/s). The backward kernel holds
// 128 registers a thread, so 16 warps an SM, and its reduction shows: a form that took 298 us took 255 with it left out (and
// a wrong result). 8192 x 16384, two blocks a row: forward 366, backward 402 us; with int8 records 434 and 570.
// The any kernels: 16384 x 4095 without records forward 175, backward 556 us, with int8 records 599 and 995. Above 4096 columns
// their arrays do not fit the 64 registers that 1024 threads have, and go to memory: 16384 x 4097 takes 6765 and 9850 us.
#pragma once
#include "act8.cuh"
#include "sm100_prims.cuh"

namespace kdkl {

constexpr int kGateNone = 0, kGateChannel = 1, kGateToken = 2;

// Weights and gates come in one of three types; the type is uniform over a launch.
struct AnyVec { const void* p; int type; };              // type: 0 bf16, 1 fp32, 2 fp16
__device__ __forceinline__ float any_at(const AnyVec& v, long long i) {
  if (v.type == 1) return reinterpret_cast<const float*>(v.p)[i];
  if (v.type == 0) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(v.p)[i]);
  return __half2float(reinterpret_cast<const __half*>(v.p)[i]);
}
// one element as bits, and what they stand for: apart, so that nothing waits for the load before its value is used
__device__ __forceinline__ uint32_t any_bits(const AnyVec& v, long long i) {
  return v.type == 1 ? reinterpret_cast<const uint32_t*>(v.p)[i] : reinterpret_cast<const uint16_t*>(v.p)[i];
}
__device__ __forceinline__ float any_value(uint32_t bits, int type) {
  if (type == 1) return __uint_as_float(bits);
  if (type == 0) return __uint_as_float(bits << 16);
  return __half2float(__ushort_as_half((unsigned short)bits));
}
template <bool VEC>
__device__ __forceinline__ void any_load8(const AnyVec& v, int c, int width, float (&f)[8]) {
  if (VEC) {
    if (v.type == 1) load8<float, true>(reinterpret_cast<const float*>(v.p), c, width, f);
    else if (v.type == 0) load8<__nv_bfloat16, true>(reinterpret_cast<const __nv_bfloat16*>(v.p), c, width, f);
    else load8<__half, true>(reinterpret_cast<const __half*>(v.p), c, width, f);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = column<VEC>(c, i) < width ? any_at(v, column<VEC>(c, i)) : 0.f;
  }
}
__device__ __forceinline__ void any_store(void* p, int type, long long i, float x) {
  if (type == 1) reinterpret_cast<float*>(p)[i] = x;
  else if (type == 0) reinterpret_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(x);
  else reinterpret_cast<__half*>(p)[i] = __float2half_rn(x);
}

// Sums of N values over the block, the same in every thread. `sm` holds N * 32 floats. One barrier a call is enough as
// long as no two calls in a row use the same buffer: a warp cannot write a buffer again before it has passed the
// barrier of the call in between, which every warp reaches only after it has read that buffer.
template <int N, int THREADS>
__device__ __forceinline__ void block_sums(float (&x)[N], float* sm) {
  constexpr int WARPS = THREADS / 32;
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int o = 16; o; o >>= 1) x[k] += __shfl_xor_sync(0xffffffffu, x[k], o);
  if (WARPS == 1) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (lane == 0)
#pragma unroll
    for (int k = 0; k < N; ++k) sm[k * 32 + warp] = x[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) {
    float s = lane < WARPS ? sm[k * 32 + lane] : 0.f;
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    x[k] = s;
  }
}

// The same where the number of threads is known at run time only (whole warps, at most 16), over the C blocks of a
// cluster that share a row: after the barrier every thread reads and adds the warps' values itself, which is quicker than
// five more dependent shuffles. `sm` holds 16 floats a sum and block, 16-byte aligned, in every block; those of warps that
// do not exist stay 0 (clear_sums).
template <int C> __device__ __forceinline__ void row_barrier() {
  if (C == 1) __syncthreads(); else cluster_sync_all();
}
template <int C>
__device__ __forceinline__ void clear_sums(float* sm, int n) {
  for (int i = threadIdx.x; i < n; i += blockDim.x) sm[i] = 0.f;
  row_barrier<C>();
}
template <int C>
__device__ __forceinline__ void leave_sum(float* at, float x) {             // at this place in every block of the cluster
  if (C == 1) { *at = x; return; }
#pragma unroll
  for (int q = 0; q < C; ++q)
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(map_to_cta(smem_u32(at), q)), "f"(x) : "memory");
}
template <int C>
__device__ __forceinline__ float sum_of_warps(const float* sm) {
  float s = 0.f;
#pragma unroll
  for (int q = 0; q < C; ++q) {
    const float4* p = reinterpret_cast<const float4*>(sm + 16 * q);
    const float4 a = p[0], b = p[1];
    s += ((a.x + a.y) + (a.z + a.w)) + ((b.x + b.y) + (b.z + b.w));
    if (blockDim.x > 256) {
      const float4 c = p[2], d = p[3];
      s += ((c.x + c.y) + (c.z + c.w)) + ((d.x + d.y) + (d.z + d.w));
    }
  }
  return s;
}
template <int C>
__device__ __forceinline__ float block_sum(float x, float* sm, int rank) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if (C == 1 && blockDim.x == 32) return x;
  if ((threadIdx.x & 31) == 0) leave_sum<C>(sm + 16 * rank + (threadIdx.x >> 5), x);
  row_barrier<C>();
  return sum_of_warps<C>(sm);
}
// Three sums at once: the first two steps of the butterfly also sort the sums by lane (lane 0: the first, 16: the
// second, 8: the third), so that the rest reduces one value instead of three.
template <int C>
__device__ __forceinline__ void block_sums3(float (&x)[3], float* sm, int rank) {
  const int lane = threadIdx.x & 31;
  const bool up = lane & 16, mid = lane & 8;
  float k = up ? x[1] : x[0];
  k += __shfl_xor_sync(0xffffffffu, up ? x[0] : x[1], 16);
  const float third = x[2] + __shfl_xor_sync(0xffffffffu, x[2], 16);
  const float give = mid ? k : third;
  k = (mid ? third : k) + __shfl_xor_sync(0xffffffffu, give, 8);
#pragma unroll
  for (int o = 4; o; o >>= 1) k += __shfl_xor_sync(0xffffffffu, k, o);
  if (C == 1 && blockDim.x == 32) {
    x[0] = __shfl_sync(0xffffffffu, k, 0); x[1] = __shfl_sync(0xffffffffu, k, 16); x[2] = __shfl_sync(0xffffffffu, k, 8);
    return;
  }
  if ((lane & 7) == 0 && lane != 24) leave_sum<C>(sm + (mid ? 32 : up ? 16 : 0) * C + 16 * rank + (threadIdx.x >> 5), k);
  row_barrier<C>();
#pragma unroll
  for (int i = 0; i < 3; ++i) x[i] = sum_of_warps<C>(sm + 16 * C * i);
}

struct NormForward {
  const void* residual; long long ld_residual;
  const void* branch; long long ld_branch;
  AnyVec post, pre, gate;               // p == nullptr: absent
  void* y; void* sum;                   // [T, H]; y only with a pre norm
  float* rho_post; float* rho_pre;      // [T] each, or nullptr
  ActRecord rec_branch, rec_sum, rec_y; // REC; codes == nullptr: not kept
  int format;
  long long T; int H;
  int gate_kind;
  float eps, offset, alpha, beta;
};

template <typename A, typename R, bool REC, int THREADS, int NV>
__global__ void __launch_bounds__(THREADS)
block_norm_forward_any_kernel(const NormForward p) {
  __shared__ float sm[4][32];           // post and pre, alternating by row (see block_sums)
  int parity = 0;
  const int H = p.H;
  const long long cpitch = act_codes_pitch(H), spitch = act_scale_pitch(H);
  const float inv_h = 1.f / (float)H;
  grid_dependents_launch();
  grid_dependency_wait();
  float k[NV][8], w2[NV][8];            // alpha (w1 + o) gate_c;  w2 + o
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = first_column<false>(threadIdx.x + i * THREADS);
    float w[8], g[8];
    if (p.post.p != nullptr) any_load8<false>(p.post, c, H, w);
    if (p.gate_kind == kGateChannel) any_load8<false>(p.gate, c, H, g);
    if (p.pre.p != nullptr) any_load8<false>(p.pre, c, H, w2[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      k[i][j] = p.alpha;
      if (p.post.p != nullptr) k[i][j] *= w[j] + p.offset;
      if (p.gate_kind == kGateChannel) k[i][j] *= g[j];
      w2[i][j] = p.pre.p != nullptr ? w2[i][j] + p.offset : 0.f;
    }
  }
  for (long long t = blockIdx.x; t < p.T; t += gridDim.x, parity ^= 2) {
    const A* brow = reinterpret_cast<const A*>(p.branch) + t * p.ld_branch;
    const R* rrow = reinterpret_cast<const R*>(p.residual) + t * p.ld_residual;
    float b[NV][8], x[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = first_column<false>(threadIdx.x + i * THREADS);
      load8<A, false>(brow, c, H, b[i]);
      load8<R, false>(rrow, c, H, x[i]);
      if constexpr (REC) {
        if (p.rec_branch.codes != nullptr) record_write8<false>(p.format, p.rec_branch, t, cpitch, spitch, c, b[i]);
      }
    }
    float rho1 = 1.f;
    if (p.post.p != nullptr) {
      float s[1] = {0.f};
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) s[0] = fmaf(b[i][j], b[i][j], s[0]);
      block_sums<1, THREADS>(s, sm[parity]);
      rho1 = 1.f / sqrtf(fmaf(s[0], inv_h, p.eps));
    }
    float scale = rho1;
    if (p.gate_kind == kGateToken) scale *= any_at(p.gate, t);
    float s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[i][j] = fmaf(scale * k[i][j], b[i][j], p.beta * x[i][j]);
        s[0] = fmaf(x[i][j], x[i][j], s[0]);
      }
    float rho2 = 1.f;
    if (p.pre.p != nullptr) {
      block_sums<1, THREADS>(s, sm[parity + 1]);
      rho2 = 1.f / sqrtf(fmaf(s[0], inv_h, p.eps));
    }
    if (threadIdx.x == 0) {
      if (p.rho_post != nullptr) p.rho_post[t] = rho1;
      if (p.rho_pre != nullptr) p.rho_pre[t] = rho2;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = first_column<false>(threadIdx.x + i * THREADS);
      const Raw8<R> raw = f32_to_raw<R>(x[i]);
      store_raw8<R, false>(reinterpret_cast<R*>(p.sum) + t * H, c, H, raw);
      if constexpr (REC) {
        if (p.rec_sum.codes != nullptr) {             // what a record of the returned sum would hold
          float v[8];
          raw_to_f32(raw, v);
          record_write8<false>(p.format, p.rec_sum, t, cpitch, spitch, c, v);
        }
      }
      if (p.pre.p != nullptr) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[i][j] *= rho2 * w2[i][j];
        const Raw8<A> yr = f32_to_raw<A>(x[i]);
        store_raw8<A, false>(reinterpret_cast<A*>(p.y) + t * H, c, H, yr);
        if constexpr (REC) {
          if (p.rec_y.codes != nullptr) {
            float v[8];
            raw_to_f32(yr, v);
            record_write8<false>(p.format, p.rec_y, t, cpitch, spitch, c, v);
          }
        }
      }
    }
  }
}

struct NormBackward {
  const void* dsum; long long ld_dsum;  // gradient of x from the residual stream, or nullptr (0)
  const void* dy; long long ld_dy;      // gradient of y, or nullptr (no pre norm)
  const void* sum; long long ld_sum;    // what was kept of x ...
  const void* branch; long long ld_branch;   // ... and of b, where it is not in a record
  ActRecord rec_sum, rec_branch;        // REC
  int format;
  AnyVec post, pre, gate;
  const float* rho_post; const float* rho_pre;
  void* dresidual; void* dbranch;       // [T, H]
  void* dgate_token; int gate_type;     // token gate: [T]
  float* partial;                       // [gridDim.x, 3, Hp]: dw1, dw2, dgate (channel)
  long long T; int H;
  int gate_kind;
  float offset, alpha, beta;
};

// With Q = gate_c (w1 + o), sigma = alpha rho1 gate_t, u = dy rho2 and x, b as kept (not normalised):
//   e = dx + u (w2 + o),  c2 = rho2 mean(u x (w2 + o)),  d = e - rho2 c2 x
//   A = sum_t sigma d b     (per column; dw1 = gate_c A, dgate_c = (w1 + o) A),   dw2 = sum_t u x
//   db = sigma Q d - rho1^2 c1 b
// so a column needs one sum for the gate and the post weight together.
template <typename A, typename R, bool REC, int THREADS, int NV>
__global__ void __launch_bounds__(THREADS)
block_norm_backward_any_kernel(const NormBackward p) {
  __shared__ float sm[2][3 * 32];
  const int H = p.H;
  const long long cpitch = act_codes_pitch(H), spitch = act_scale_pitch(H);
  const float inv_h = 1.f / (float)H;
  const bool has_post = p.post.p != nullptr, has_pre = p.pre.p != nullptr;
  const bool channel = p.gate_kind == kGateChannel, token = p.gate_kind == kGateToken;
  float q[NV][8], w2[NV][8], sum_a[NV][8], sum_w[NV][8];     
  grid_dependents_launch();
  grid_dependency_wait();
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = first_column<false>(threadIdx.x + i * THREADS);
    float g[8];
    if (has_post) any_load8<false>(p.post, c, H, q[i]);
    if (channel) any_load8<false>(p.gate, c, H, g);
    if (has_pre) any_load8<false>(p.pre, c, H, w2[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      q[i][j] = has_post ? q[i][j] + p.offset : 1.f;
      if (channel) q[i][j] *= g[j];
      w2[i][j] = has_pre ? w2[i][j] + p.offset : 0.f;
      sum_a[i][j] = sum_w[i][j] = 0.f;
    }
  }
  int parity = 0;
  for (long long t = blockIdx.x; t < p.T; t += gridDim.x, parity ^= 1) {
    const float rho1 = has_post ? p.rho_post[t] : 1.f, rho2 = has_pre ? p.rho_pre[t] : 1.f;
    const float gate_t = token ? any_at(p.gate, t) : 1.f;
    float e[NV][8], b[NV][8], x[NV][8];
    float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = first_column<false>(threadIdx.x + i * THREADS);
      if constexpr (REC) {
        record_read8<false>(p.format, p.rec_branch, t, cpitch, spitch, c, b[i]);
        if (has_pre) record_read8<false>(p.format, p.rec_sum, t, cpitch, spitch, c, x[i]);
      } else {
        load8<A, false>(reinterpret_cast<const A*>(p.branch) + t * p.ld_branch, c, H, b[i]);
        if (has_pre) load8<R, false>(reinterpret_cast<const R*>(p.sum) + t * p.ld_sum, c, H, x[i]);
      }
      float dy[8];
      if (p.dsum != nullptr) load8<R, false>(reinterpret_cast<const R*>(p.dsum) + t * p.ld_dsum, c, H, e[i]);
      if (has_pre) load8<A, false>(reinterpret_cast<const A*>(p.dy) + t * p.ld_dy, c, H, dy);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (p.dsum == nullptr) e[i][j] = 0.f;
        if (has_pre) {
          const float u = dy[j] * rho2, ux = u * x[i][j];
          sum_w[i][j] += ux;
          s[0] = fmaf(ux, w2[i][j], s[0]);
          e[i][j] = fmaf(u, w2[i][j], e[i][j]);
        } else {
          x[i][j] = 0.f;
        }
        const float qb = q[i][j] * b[i][j];
        s[1] = fmaf(qb, e[i][j], s[1]);
        s[2] = fmaf(qb, x[i][j], s[2]);
      }
    }
    block_sums<3, THREADS>(s, sm[parity]);
    const float k2 = rho2 * rho2 * s[0] * inv_h, dot = rho1 * p.alpha * (s[1] - k2 * s[2]);
    if (token && threadIdx.x == 0) any_store(p.dgate_token, p.gate_type, t, dot);
    const float sigma = p.alpha * rho1 * gate_t, tau = has_post ? -rho1 * rho1 * dot * gate_t * inv_h : 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = first_column<false>(threadIdx.x + i * THREADS);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = fmaf(-k2, x[i][j], e[i][j]), sd = d * sigma;
        sum_a[i][j] = fmaf(sd, b[i][j], sum_a[i][j]);
        e[i][j] = p.beta * d;
        b[i][j] = fmaf(q[i][j], sd, tau * b[i][j]);
      }
      store_raw8<R, false>(reinterpret_cast<R*>(p.dresidual) + t * H, c, H, f32_to_raw<R>(e[i]));
      store_raw8<A, false>(reinterpret_cast<A*>(p.dbranch) + t * H, c, H, f32_to_raw<A>(b[i]));
    }
  }
  float* out = p.partial + (long long)blockIdx.x * 3 * cpitch;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = first_column<false>(threadIdx.x + i * THREADS);
    if (c >= H) continue;
    float w[8], g[8], v[8];
    if (has_post) any_load8<false>(p.post, c, H, w);
    if (channel) any_load8<false>(p.gate, c, H, g);
    if (has_pre) store_raw8<float, false>(out + cpitch, c, (int)cpitch, f32_to_raw<float>(sum_w[i]));
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = channel ? sum_a[i][j] * g[j] : sum_a[i][j];
    if (has_post) store_raw8<float, false>(out, c, (int)cpitch, f32_to_raw<float>(v));
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = has_post ? sum_a[i][j] * (w[j] + p.offset) : sum_a[i][j];
    if (channel) store_raw8<float, false>(out + 2 * cpitch, c, (int)cpitch, f32_to_raw<float>(v));
  }
}

// ------------------------------------------------------------------ rows of whole 16-byte words
// A thread has two groups of eight columns: that halves what a row costs per value in sums, factors and addresses
// (with one group a thread both kernels were bound by instructions, 63 and 54 a value).
constexpr int kRowsThreads = 512, kRowsMaxH = 2 * 8 * kRowsThreads;   // kRowsMaxH: columns a block
constexpr int kRowsMaxCluster = 4;      // wider rows are shared by a cluster of 2 or 4 blocks

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async8(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(live ? 8 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Eight values as pairs.
struct V8 { float2 p[4]; };
__device__ __forceinline__ V8 v8_of(const float (&f)[8]) {
  V8 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v.p[i] = make_float2(f[2 * i], f[2 * i + 1]);
  return v;
}
__device__ __forceinline__ void v8_to(const V8& v, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { f[2 * i] = v.p[i].x; f[2 * i + 1] = v.p[i].y; }
}
template <typename T> __device__ __forceinline__ Raw8<T> v8_raw(const V8& v) {
  float f[8];
  v8_to(v, f);
  return f32_to_raw<T>(f);
}
__device__ __forceinline__ V8 v8_any(const AnyVec& a, int c, int H) {
  float f[8];
  any_load8<true>(a, c, H, f);
  return v8_of(f);
}
__device__ __forceinline__ V8 v8_all(float x) {
  V8 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v.p[i] = both(x);
  return v;
}
__device__ __forceinline__ float sum2(float2 a) { return a.x + a.y; }
template <int FMT>
__device__ __forceinline__ void v8_write_record(const ActRecord& r, long long t, long long cpitch, long long spitch,
                                                int c, const V8& v) {
  float f[8];
  v8_to(v, f);
  record_write8<FMT, true>(r, t, cpitch, spitch, c, f);
}

// What the next row brings waits in shared memory, in places that only their own thread touches: per group of eight
// columns and warp one chunk of 32 lanes' places, field after field, so that every address is one of two lane offsets
// plus a constant.
struct Places {
  uint32_t l16, l8;
  __device__ __forceinline__ Places(uint32_t chunk, int lane) : l16(chunk + lane * 16), l8(chunk + lane * 8) {}
};
// A row's values [c, c + 8) of 2 or 4 bytes; 4-byte values take two places 512 bytes apart.
template <typename T, int AT> __device__ __forceinline__ void fetch8(const Places& s, const T* row, int c, bool live) {
  const T* src = row + (uint32_t)(live ? c : 0);
  cp_async16(s.l16 + AT, src, live);
  if constexpr (sizeof(T) == 4) cp_async16(s.l16 + AT + 512, src + 4, live);
}
template <typename T, int AT> __device__ __forceinline__ V8 take8(const Places& s) {
  Raw8<T> r;
  r.v = ld_shared_v4(s.l16 + AT);
  if constexpr (sizeof(T) == 4) r.w = ld_shared_v4(s.l16 + AT + 512);
  float f[8];
  raw_to_f32(r, f);
  return v8_of(f);
}
// Eight codes. (The scale bytes come into registers a row ahead: copies of 4 bytes a lane cost a tenth of the kernel.)
template <int AT> __device__ __forceinline__ void fetch_codes8(const Places& s, const uint8_t* codes, int c, bool live) {
  cp_async8(s.l8 + AT, codes + (uint32_t)(live ? c : 0), live);
}
template <int FMT, int AT> __device__ __forceinline__ V8 take_record8(const Places& s, uint32_t byte) {
  const uint2 codes = ld_shared_v2(s.l8 + AT);
  float f[8];
  act_values<FMT>(codes, byte, f);
  return v8_of(f);
}
// Bytes of a chunk: fields for 32 lanes.
__host__ __device__ constexpr int rows_forward_chunk(int residual_bytes) { return 512 + 256 * residual_bytes; }
__host__ __device__ constexpr int rows_backward_chunk(int residual_bytes, bool rec) {
  return 256 * residual_bytes + 512 + (rec ? 2 * 256 : 512 + 256 * residual_bytes);
}
// Rows of the backward kernel that are worked on or on their way: three, two where the widest block's 32 chunks of three
// would not fit the shared memory (an fp32 residual without records).
__host__ __device__ constexpr int rows_backward_stages(int residual_bytes, bool rec) {
  return 3 * 32 * rows_backward_chunk(residual_bytes, rec) <= 200 * 1024 ? 3 : 2;
}

// FMT -1: no records. FULL: both norms (and, backward, a gradient along the residual stream) are there, which spares the
// loop its questions. C: blocks that share a row (a cluster); block `rank` of them has the columns of its threads' numbers
// threadIdx.x + (2 rank) blockDim.x and threadIdx.x + (2 rank + 1) blockDim.x.
// (Without records at most 96 registers a thread, so that a third block of 192 threads fits an SM: 138 -> 115 us at
// 32768 x 2816. With records the 113 that the compiler takes are quicker: 240 against 258 us at 32768 x 4096.)
template <typename A, typename R, int FMT, bool FULL, int C>
__global__ void __launch_bounds__(FMT < 0 ? 640 : kRowsThreads)
block_norm_forward_rows_kernel(const NormForward p) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ __align__(16) float sm[4][16 * C];
  constexpr int kResidual = 512;        // field offsets: branch, residual
  clear_sums<C>(sm[0], 64 * C);
  const int H = p.H, threads = blockDim.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long cpitch = act_codes_pitch(H), spitch = act_scale_pitch(H);
  const float inv_h = 1.f / (float)H;
  const bool has_post = FULL || p.post.p != nullptr, has_pre = FULL || p.pre.p != nullptr, token = p.gate_kind == kGateToken;
  const int rank = C == 1 ? 0 : (int)cluster_ctarank();
  const long long first = blockIdx.x / C, step = gridDim.x / C;
  const int c[2] = {(int)(threadIdx.x + 2 * rank * threads) * 8, (int)(threadIdx.x + (2 * rank + 1) * threads) * 8};
  const uint32_t chunk = smem_u32(smem) + warp * rows_forward_chunk(sizeof(R));
  const Places at[2] = {Places(chunk, lane), Places(chunk + (threads >> 5) * rows_forward_chunk(sizeof(R)), lane)};
  auto fetch = [&](long long t) {
    const A* b = reinterpret_cast<const A*>(p.branch) + t * p.ld_branch;
    const R* r = reinterpret_cast<const R*>(p.residual) + t * p.ld_residual;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      fetch8<A, 0>(at[i], b, c[i], c[i] < H);
      fetch8<R, kResidual>(at[i], r, c[i], c[i] < H);
    }
  };
  grid_dependents_launch();
  grid_dependency_wait();
  fetch(first);
  V8 k[2], w2[2];                       // alpha (w1 + o) gate_c;  w2 + o
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    k[i] = w2[i] = v8_all(0.f);
    if (c[i] >= H) continue;
    k[i] = v8_all(p.alpha);
    if (has_post) {
      const V8 w = v8_any(p.post, c[i], H);
#pragma unroll
      for (int j = 0; j < 4; ++j) k[i].p[j] = mul2(k[i].p[j], add2(w.p[j], both(p.offset)));
    }
    if (p.gate_kind == kGateChannel) {
      const V8 g = v8_any(p.gate, c[i], H);
#pragma unroll
      for (int j = 0; j < 4; ++j) k[i].p[j] = mul2(k[i].p[j], g.p[j]);
    }
    if (has_pre) {
      const V8 w = v8_any(p.pre, c[i], H);
#pragma unroll
      for (int j = 0; j < 4; ++j) w2[i].p[j] = add2(w.p[j], both(p.offset));
    }
  }
  int parity = 0;
  uint32_t gate_next = token ? any_bits(p.gate, first) : 0u;
  for (long long t = first; t < p.T; t += step, parity ^= 2) {
    const float gate_t = token ? any_value(gate_next, p.gate.type) : 1.f;
    cp_async_wait_all();
    V8 b[2], x[2];
    float2 acc = both(0.f);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      b[i] = take8<A, 0>(at[i]);
      x[i] = take8<R, kResidual>(at[i]);
#pragma unroll
      for (int j = 0; j < 4; ++j) { acc = fma2(b[i].p[j], b[i].p[j], acc); x[i].p[j] = mul2(x[i].p[j], both(p.beta)); }
    }
    if (t + step < p.T) {               // the row is in registers: its places take the next one
      fetch(t + step);
      if (token) gate_next = any_bits(p.gate, t + step);
    }
    if constexpr (FMT >= 0) {
      if (p.rec_branch.codes != nullptr) {
#pragma unroll
        for (int i = 0; i < 2; ++i) v8_write_record<FMT>(p.rec_branch, t, cpitch, spitch, c[i], b[i]);
      }
    }
    float rho1 = 1.f;
    if (has_post) {
      rho1 = rsqrtf(fmaf(block_sum<C>(sum2(acc), sm[parity], rank), inv_h, p.eps));
    }
    const float2 scale = both(rho1 * gate_t);
    acc = both(0.f);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[i].p[j] = fma2(mul2(k[i].p[j], scale), b[i].p[j], x[i].p[j]);
        acc = fma2(x[i].p[j], x[i].p[j], acc);
      }
    R* sum_row = reinterpret_cast<R*>(p.sum) + t * H;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const Raw8<R> raw = v8_raw<R>(x[i]);
      store_raw8<R, true>(sum_row, c[i], H, raw);
      if constexpr (FMT >= 0) {
        if (p.rec_sum.codes != nullptr) {              // what a record of the returned sum would hold
          float f[8];
          raw_to_f32(raw, f);
          record_write8<FMT, true>(p.rec_sum, t, cpitch, spitch, c[i], f);
        }
      }
    }
    float rho2 = 1.f;
    if (has_pre) {
      rho2 = rsqrtf(fmaf(block_sum<C>(sum2(acc), sm[parity + 1], rank), inv_h, p.eps));
      A* y_row = reinterpret_cast<A*>(p.y) + t * H;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[i].p[j] = mul2(x[i].p[j], mul2(w2[i].p[j], both(rho2)));
        const Raw8<A> raw = v8_raw<A>(x[i]);
        store_raw8<A, true>(y_row, c[i], H, raw);
        if constexpr (FMT >= 0) {
          if (p.rec_y.codes != nullptr) {
            float f[8];
            raw_to_f32(raw, f);
            record_write8<FMT, true>(p.rec_y, t, cpitch, spitch, c[i], f);
          }
        }
      }
    }
    if (threadIdx.x == 0 && rank == 0) {
      if (p.rho_post != nullptr) p.rho_post[t] = rho1;
      if (p.rho_pre != nullptr) p.rho_pre[t] = rho2;
    }
  }
}

template <typename A, typename R, int FMT, bool FULL, int C>
__global__ void __launch_bounds__(kRowsThreads)
block_norm_backward_rows_kernel(const NormBackward p) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ __align__(16) float sm[2][3 * 16 * C];
  clear_sums<C>(sm[0], 96 * C);
  constexpr int kRB = 256 * (int)sizeof(R), kDy = kRB, kBranch = kRB + 512, kSum = kBranch + (FMT >= 0 ? 256 : 512);
  const int H = p.H, threads = blockDim.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long cpitch = act_codes_pitch(H), spitch = act_scale_pitch(H);
  const float inv_h = 1.f / (float)H;
  const bool has_post = FULL || p.post.p != nullptr, has_pre = FULL || p.pre.p != nullptr, token = p.gate_kind == kGateToken;
  const bool has_dx = FULL || p.dsum != nullptr;
  const int rank = C == 1 ? 0 : (int)cluster_ctarank();
  const long long first = blockIdx.x / C, step = gridDim.x / C;
  const int c[2] = {(int)(threadIdx.x + 2 * rank * threads) * 8, (int)(threadIdx.x + (2 * rank + 1) * threads) * 8};
  constexpr int kChunk = rows_backward_chunk(sizeof(R), FMT >= 0);
  const uint32_t chunk = smem_u32(smem) + warp * kChunk;
  const uint32_t stage_bytes = (threads >> 4) * kChunk;
  float rho1_next = 1.f, rho2_next = 1.f;
  uint32_t gate_next = 0u, byte_b[2] = {1u, 1u}, byte_x[2] = {1u, 1u};   // (bytes of columns that do not exist)
  auto places = [&](int i, int stage) { return Places(chunk + stage * stage_bytes + i * (stage_bytes / 2), lane); };
  auto fetch = [&](long long t, int stage) {
    if (t < p.T) {
    const Places at[2] = {places(0, stage), places(1, stage)};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const bool live = c[i] < H;
      if (has_dx) fetch8<R, 0>(at[i], reinterpret_cast<const R*>(p.dsum) + t * p.ld_dsum, c[i], live);
      if (has_pre) fetch8<A, kDy>(at[i], reinterpret_cast<const A*>(p.dy) + t * p.ld_dy, c[i], live);
      if constexpr (FMT >= 0) {
        fetch_codes8<kBranch>(at[i], p.rec_branch.codes + t * cpitch, c[i], live);
        if (has_pre) fetch_codes8<kSum>(at[i], p.rec_sum.codes + t * cpitch, c[i], live);
      } else {
        fetch8<A, kBranch>(at[i], reinterpret_cast<const A*>(p.branch) + t * p.ld_branch, c[i], live);
        if (has_pre) fetch8<R, kSum>(at[i], reinterpret_cast<const R*>(p.sum) + t * p.ld_sum, c[i], live);
      }
    }
    }
    cp_async_commit();
  };
  auto factors = [&](long long t) {
    if (t >= p.T) return;
    if (has_post) rho1_next = p.rho_post[t];
    if (has_pre) rho2_next = p.rho_pre[t];
    if (token) gate_next = any_bits(p.gate, t);
    if constexpr (FMT >= 0) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (c[i] >= H) continue;
        byte_b[i] = ld_global_u8(p.rec_branch.scales + t * spitch + (c[i] >> 5));
        if (has_pre) byte_x[i] = ld_global_u8(p.rec_sum.scales + t * spitch + (c[i] >> 5));
      }
    }
  };
  constexpr int S = rows_backward_stages(sizeof(R), FMT >= 0);
  grid_dependents_launch();
  grid_dependency_wait();
#pragma unroll
  for (int k = 0; k < S - 1; ++k) fetch(first + k * step, k);
  factors(first);
  int stage = 0;
  V8 q[2], w2[2], sum_a[2], sum_w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    q[i] = w2[i] = sum_a[i] = sum_w[i] = v8_all(0.f);
    if (c[i] >= H) continue;
    q[i] = v8_all(1.f);
    if (has_post) {
      const V8 w = v8_any(p.post, c[i], H);
#pragma unroll
      for (int j = 0; j < 4; ++j) q[i].p[j] = add2(w.p[j], both(p.offset));
    }
    if (p.gate_kind == kGateChannel) {
      const V8 g = v8_any(p.gate, c[i], H);
#pragma unroll
      for (int j = 0; j < 4; ++j) q[i].p[j] = mul2(q[i].p[j], g.p[j]);
    }
    if (has_pre) {
      const V8 w = v8_any(p.pre, c[i], H);
#pragma unroll
      for (int j = 0; j < 4; ++j) w2[i].p[j] = add2(w.p[j], both(p.offset));
    }
  }
  int parity = 0;
  for (long long t = first; t < p.T; t += step, parity ^= 1) {
    const float rho1 = rho1_next, rho2 = rho2_next, gate_t = token ? any_value(gate_next, p.gate.type) : 1.f;
    const uint32_t now_b[2] = {byte_b[0], byte_b[1]}, now_x[2] = {byte_x[0], byte_x[1]};
    fetch(t + (S - 1) * step, stage == 0 ? S - 1 : stage - 1);
    factors(t + step);
    cp_async_wait<S - 1>();
    const Places at[2] = {places(0, stage), places(1, stage)};
    stage = stage + 1 == S ? 0 : stage + 1;
    V8 e[2], x[2], b[2];
    float2 a0 = both(0.f), a1 = both(0.f), a2 = both(0.f);   // u x w2';  Q b e;  Q b x
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      e[i] = has_dx ? take8<R, 0>(at[i]) : v8_all(0.f);
      if constexpr (FMT >= 0) b[i] = take_record8<FMT, kBranch>(at[i], now_b[i]);
      else b[i] = take8<A, kBranch>(at[i]);
      if (has_pre) {
        if constexpr (FMT >= 0) x[i] = take_record8<FMT, kSum>(at[i], now_x[i]);
        else x[i] = take8<R, kSum>(at[i]);
        const V8 dy = take8<A, kDy>(at[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 u = mul2(dy.p[j], both(rho2)), ux = mul2(u, x[i].p[j]);
          sum_w[i].p[j] = add2(sum_w[i].p[j], ux);
          a0 = fma2(ux, w2[i].p[j], a0);
          e[i].p[j] = fma2(u, w2[i].p[j], e[i].p[j]);
        }
      } else {
        x[i] = v8_all(0.f);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 qb = mul2(q[i].p[j], b[i].p[j]);
        a1 = fma2(qb, e[i].p[j], a1);
        a2 = fma2(qb, x[i].p[j], a2);
      }
    }
    float s[3] = {sum2(a0), sum2(a1), sum2(a2)};
    block_sums3<C>(s, sm[parity], rank);
    const float k2 = rho2 * rho2 * s[0] * inv_h;             // d = e - k2 x
    const float dot = rho1 * p.alpha * (s[1] - k2 * s[2]);   // sum_h alpha Q b^ d
    if (token && threadIdx.x == 0 && rank == 0) any_store(p.dgate_token, p.gate_type, t, dot);
    const float sigma = p.alpha * rho1 * gate_t;
    const float tau = has_post ? -rho1 * rho1 * dot * gate_t * inv_h : 0.f;
    R* dr_row = reinterpret_cast<R*>(p.dresidual) + t * H;
    A* db_row = reinterpret_cast<A*>(p.dbranch) + t * H;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 d = fma2(x[i].p[j], both(-k2), e[i].p[j]), sd = mul2(d, both(sigma));
        sum_a[i].p[j] = fma2(sd, b[i].p[j], sum_a[i].p[j]);
        e[i].p[j] = mul2(d, both(p.beta));
        b[i].p[j] = fma2(q[i].p[j], sd, mul2(b[i].p[j], both(tau)));
      }
      store_raw8<R, true>(dr_row, c[i], H, v8_raw<R>(e[i]));
      store_raw8<A, true>(db_row, c[i], H, v8_raw<A>(b[i]));
    }
  }
  float* out = p.partial + first * 3 * cpitch;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (c[i] >= H) continue;
    if (has_pre) store_raw8<float, true>(out + cpitch, c[i], (int)cpitch, v8_raw<float>(sum_w[i]));
    if (has_post) {
      V8 v = sum_a[i];
      if (p.gate_kind == kGateChannel) {
        const V8 g = v8_any(p.gate, c[i], H);
#pragma unroll
        for (int j = 0; j < 4; ++j) v.p[j] = mul2(v.p[j], g.p[j]);
      }
      store_raw8<float, true>(out, c[i], (int)cpitch, v8_raw<float>(v));
    }
    if (p.gate_kind == kGateChannel) {
      V8 v = sum_a[i];
      if (has_post) {
        const V8 w = v8_any(p.post, c[i], H);
#pragma unroll
        for (int j = 0; j < 4; ++j) v.p[j] = mul2(v.p[j], add2(w.p[j], both(p.offset)));
      }
      store_raw8<float, true>(out + 2 * cpitch, c[i], (int)cpitch, v8_raw<float>(v));
    }
  }
}

// Column sums of the partial rows, in a fixed order: warp y of a block adds the rows y, y + 32, ... of 32 columns, then
// each warp the 32 partial sums of a column. Starts while the kernel before it drains and waits for it before it reads.
struct NormColumns { void* out[3]; int type[3]; int which[3]; };
__global__ void __launch_bounds__(1024)
block_norm_columns_kernel(const float* partial, int parts, int H, long long cpitch, const NormColumns p) {
  __shared__ float sm[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, q = blockIdx.y;
  grid_dependents_launch();
  grid_dependency_wait();
  float s = 0.f;
  if (blockIdx.x * 32 + lane < H) {
    const float* src = partial + p.which[q] * cpitch + blockIdx.x * 32 + lane;
#pragma unroll 8
    for (int i = warp; i < parts; i += 32) s += __ldcg(src + (long long)i * 3 * cpitch);   // from L2: written just now
  }
  sm[warp][lane] = s;
  __syncthreads();
  s = sm[lane][warp];
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  const int c = blockIdx.x * 32 + warp;
  if (lane == 0 && c < H) any_store(p.out[q], p.type[q], c, s);
}

}  // namespace kdkl
