// The small kernels around the products of the label loss. Per token, with z = W h / tau, y its label, s the smoothing and
// lambda the z term:
//   lse = log sum_v e^z_v,   l = lse - (1 - s) z_y - (s / V) sum_v z_v + lambda lse^2
//   dl/dz_v = (1 + 2 lambda lse) q_v - (1 - s) [v = y] - s / V,   q = softmax(z)
// Three numbers a token carry the gradient into the products: G_v = a q_v - c, less b at the label, with
//   a = w (1 + 2 lambda lse),  b = w (1 - s),  c = w s / V,  w = the token's weight (or its own upstream gradient).
// What all tokens share - upstream gradient / (divisor tau) - is left out of G and multiplies the products in fp32: without
// weights G is then q_v - [v = y], and its largest entry, close to -1, is off by a quarter of the bf16 step at most that
// an arbitrary common factor would cost every token alike. (G is bf16 because the tensor cores take 16-bit operands, as in the
// KL loss: gradients are 1.7e-3 off in norm, their own rounding; with weights, smoothing or a z term 2.3e-3.)
// An ignored token has col = -1, and exact zeros everywhere. All sums go in a fixed order.
// 8192 tokens, V = 131072 (H = 2048, a step of 10.4 ms): join 15 us, the pass over the exponentials 766.
#pragma once
#include <cuda_fp16.h>

#include "aux_state.cuh"
#include "gemm_tcgen05.cuh"

namespace kdkl {

struct LabelParams {
  float tau, smoothing, z_loss;
  int T, H, V;
  long long chunk;
  int mean;                            // 1: the divisor is the number of counted tokens, or denom_device's
  const double* denom_device;
  const float* token_weight;           // [T] or null
  const float* grad;                   // [1] or null (1)
  const float* grad_tokens;            // [T] or null: in place of grad, weight and divisor
  WsHeader* hdr;
  int* col; int* counted;              // [T]
  float* lz2; float* z_label;          // [T]: log2-domain normaliser, raw logit at the label
  float* coefA; float* coefB; float* coefC;
  float* losses;                       // [T]
  float* scale;                        // [1]: upstream gradient / (divisor tau)
  int* arrivals;                       // [1]: blocks of the last chunk's join that are done
  int* tile_counts;                    // [2][ceil(T / 256)]: counted tokens, labels out of range
};

__device__ __forceinline__ double label_divisor(const LabelParams& p, long long counted) {
  if (p.denom_device != nullptr) return *p.denom_device;
  return p.mean ? (double)counted : 1.0;
}
__device__ __forceinline__ void label_coefs(const LabelParams& p, long long t, float lse) {
  const float w = !p.counted[t] ? 0.f : p.grad_tokens != nullptr ? p.grad_tokens[t] : p.token_weight != nullptr ? p.token_weight[t] : 1.f;
  p.coefA[t] = w * fmaf(2.f * p.z_loss, lse, 1.f);
  p.coefB[t] = w * (1.f - p.smoothing);
  p.coefC[t] = w * p.smoothing / (float)p.V;
}
__device__ __forceinline__ void label_scale(const LabelParams& p, long long counted) {        // one thread
  const double d = p.grad_tokens != nullptr ? 1.0 : label_divisor(p, counted), g = p.grad_tokens == nullptr && p.grad != nullptr ? (double)*p.grad : 1.0;
  *p.scale = d > 0.0 ? (float)(g / (d * (double)p.tau)) : 0.f;
}

// Labels to columns, the counted tokens of each row tile (256 tokens) and whether it has any: a block has one tile. Clears the
// status block.
template <typename L>
__global__ void __launch_bounds__(256)
label_prep_kernel(const LabelParams p, const L* labels, long long ignore_index, uint8_t* live) {
  grid_dependents_launch();
  grid_dependency_wait();
  const long long t = (long long)blockIdx.x * 256 + threadIdx.x;
  bool counted = false, bad = false;
  if (t < p.T) {
    const long long y = (long long)labels[t];
    bad = y != ignore_index && (y < 0 || y >= p.V);
    counted = y != ignore_index && !bad;
    p.col[t] = counted ? (int)y : -1;
    p.counted[t] = counted ? 1 : 0;
  }
  const int n = __syncthreads_count(counted), n_bad = __syncthreads_count(bad);
  if (threadIdx.x == 0) {
    live[blockIdx.x] = n > 0 ? 1 : 0;
    p.tile_counts[blockIdx.x] = n;
    p.tile_counts[gridDim.x + blockIdx.x] = n_bad;
  }
  if (blockIdx.x == 0) {
    if (threadIdx.x < 64) reinterpret_cast<int*>(p.hdr)[threadIdx.x] = 0;
    if (threadIdx.x == 64) *p.arrivals = 0;
  }
}

// The number of counted tokens and of labels out of range, from the tiles': a thread's share, and the block's sum of them, which
// thread 0 has.
__device__ __forceinline__ int2 label_count_share(const LabelParams& p) {
  const int tiles = (p.T + 255) / 256;
  int2 n = make_int2(0, 0);
  for (int i = threadIdx.x; i < tiles; i += blockDim.x) { n.x += p.tile_counts[i]; n.y += p.tile_counts[tiles + i]; }
  return n;
}
__device__ __forceinline__ int2 label_count(int2 share) {
  __shared__ int part[2][32];
  int n = share.x, bad = share.y;
  n = __reduce_add_sync(0xffffffffu, n); bad = __reduce_add_sync(0xffffffffu, bad);
  if ((threadIdx.x & 31) == 0) { part[0][threadIdx.x >> 5] = n; part[1][threadIdx.x >> 5] = bad; }
  __syncthreads();
  if (threadIdx.x >= 32) return make_int2(0, 0);
  const bool has = threadIdx.x < blockDim.x / 32;
  n = __reduce_add_sync(0xffffffffu, has ? part[0][threadIdx.x] : 0);
  bad = __reduce_add_sync(0xffffffffu, has ? part[1][threadIdx.x] : 0);
  return make_int2(n, bad);
}

// Joins the partial (max, sum, sum of logits) of a chunk's rows and vocabulary tiles; 32 rows a block, 32 lanes of partials a row.
__global__ void __launch_bounds__(1024)
label_combine_kernel(const LabelParams p, const float* part_m, const float* part_s, const float* part_z, long long stride, int n_tiles,
                     int rows, long long row0, int want_coefs, int last, float* losses_out, float* lse_out, float* loss_out) {
  __shared__ float sm_m[32][33], sm_s[32][33], sm_z[32][33];
  __shared__ double sums[32];
  __shared__ int turn;
  grid_dependents_launch();
  grid_dependency_wait();
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const int r = blockIdx.x * 32 + tx;
  const long long t = row0 + r;
  // what the last block will want for the sum, asked for now
  auto factor = [&](int i) { return p.counted[i] ? (p.token_weight != nullptr ? p.token_weight[i] : 1.f) : 0.f; };
  int2 share = make_int2(0, 0);
  float first_factor = 0.f;
  if (last) {
    share = label_count_share(p);
    if ((int)threadIdx.x < p.T) first_factor = factor(threadIdx.x);
  }
  const bool counted = r < rows && p.counted[t] != 0;      // others' partials may not exist
  float m = -INFINITY, s = 0.f, z = 0.f;
  if (counted) {
    for (int nt = ty; nt < n_tiles; nt += 32) {
      const float pm = part_m[nt * stride + r], mn = fmaxf(m, pm);
      s = s * exp2f(m - mn) + part_s[nt * stride + r] * exp2f(pm - mn);
      m = mn;
      z += part_z[nt * stride + r];
    }
  }
  sm_m[ty][tx] = m; sm_s[ty][tx] = s; sm_z[ty][tx] = z;
  // a warp a row from here on: a lane has one of its 32 partials
  const int row = blockIdx.x * 32 + ty;
  const long long tok = row0 + row;
  const bool counts = row < rows && p.counted[tok] != 0;
  const float z_label = counts ? p.z_label[tok] : 0.f;
  __syncthreads();
  if (row < rows) {
    m = sm_m[tx][ty]; s = sm_s[tx][ty]; z = sm_z[tx][ty];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float om = __shfl_xor_sync(0xffffffffu, m, o), os = __shfl_xor_sync(0xffffffffu, s, o);
      const float mn = fmaxf(m, om);
      // (lanes beyond the tiles have m = -inf and s = 0; both may)
      s = (m > -INFINITY ? s * exp2f(m - mn) : 0.f) + (om > -INFINITY ? os * exp2f(om - mn) : 0.f);
      m = mn;
      z += __shfl_xor_sync(0xffffffffu, z, o);
    }
    if (tx == 0) {
      float loss = 0.f, lse = 0.f, lz2 = 0.f;
      if (counts) {
        lz2 = m + log2f(s);
        lse = lz2 * kLn2;
        const float inv_tau = 1.f / p.tau;
        // taken from the normaliser, so that a confident token's small loss keeps its digits
        loss = (1.f - p.smoothing) * (lse - z_label * inv_tau) + p.smoothing * (lse - z * inv_tau / (float)p.V) + p.z_loss * lse * lse;
        if (!isfinite(loss)) report_error(&p.hdr->status, -11, (int)tok);
      }
      p.lz2[tok] = lz2;
      p.losses[tok] = loss;
      if (losses_out != nullptr) losses_out[tok] = loss;
      if (lse_out != nullptr) lse_out[tok] = lse;
      if (want_coefs) label_coefs(p, tok, lse);
    }
  }
  if (!last) return;
  // The block that is done last adds up the losses, in double and an order of its own; it marks the state as complete.
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();                                       // the block's losses, which the barrier ordered before this
    turn = atomicAdd(p.arrivals, 1);
    __threadfence();
  }
  __syncthreads();
  if (turn != (int)gridDim.x - 1) return;
  double acc = 0.0;
  for (int i = threadIdx.x; i < p.T; i += 1024) {
    const float w = i == (int)threadIdx.x ? first_factor : factor(i);
    if (w != 0.f) acc += (double)__ldcg(p.losses + i) * (double)w;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
  if (tx == 0) sums[ty] = acc;
  const int2 n = label_count(share);                       // (with the barrier that sums needs)
  if (ty != 0) return;
  acc = sums[tx];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
  if (tx == 0) {
    const double d = label_divisor(p, n.x);
    *loss_out = d > 0.0 ? (float)(acc / d) : 0.f;
    p.hdr->n_tokens = n.x; p.hdr->n_bad_idx = n.y;
    if (n.y > 0) atomicCAS(&p.hdr->status, 0, -10);        // KDKL_ERR_INDEX: taken as ignored
    p.hdr->T = p.T; p.hdr->H = p.H; p.hdr->V = p.V; p.hdr->chunk = p.chunk; p.hdr->tau = p.tau; p.hdr->loss_sum = acc;
    __threadfence();
    p.hdr->magic = KDKL_MAGIC;
  }
}

// Before a backward pass of its own: whether the state is this call's, and the tokens' three numbers.
__global__ void __launch_bounds__(256)
label_coef_kernel(const LabelParams p) {
  grid_dependents_launch();
  grid_dependency_wait();
  const WsHeader* h = p.hdr;
  const bool ok = h->magic == KDKL_MAGIC && h->T == p.T && h->H == p.H && h->V == p.V && h->chunk == p.chunk && h->tau == p.tau;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    p.hdr->go = ok ? 1 : 0;
    label_scale(p, h->n_tokens);
    if (!ok) report_error(&p.hdr->status, -9, 0);          // KDKL_ERR_STATE
  }
  const long long t = (long long)blockIdx.x * 256 + threadIdx.x;
  if (ok && t < p.T) label_coefs(p, t, p.lz2[t] * kLn2);
}

// The chunk's exponentials (fp16, each 32 columns with their own power, see EPI_LABEL_E) become G (bf16) in place:
// G = (a 2^(w - lz2)) e - c, less b at the label. 8 rows x 1024 columns a block: 256 factors, one a thread, then 1024 words of
// 8 columns. One read and one write of the buffer: bound by memory. The first block of the first chunk also forms what all tokens
// share, which the products behind it need. 8192 x 131072: 766 us, 5.6 TB/s (0.87 of a copy).
constexpr int kLabelGRows = 8, kLabelGCols = 1024;
__global__ void __launch_bounds__(256)
label_g_kernel(const LabelParams p, uint16_t* G, long long ldg, const float* win_max, long long stride, int rows, long long row0) {
  grid_dependents_launch();
  grid_dependency_wait();
  __shared__ float factor[kLabelGRows][kLabelGCols / 32];
  const int c0 = blockIdx.x * kLabelGCols, r0 = blockIdx.y * kLabelGRows;
  {
    const int r = threadIdx.x % kLabelGRows, w = threadIdx.x / kLabelGRows;
    float f = 0.f;
    if (r0 + r < rows && c0 + 32 * w < p.V) {
      const long long t = row0 + r0 + r;
      if (p.counted[t]) f = p.coefA[t] * exp2f(win_max[(long long)(c0 / 32 + w) * stride + r0 + r] - p.lz2[t]);
    }
    factor[r][w] = f;
  }
  __syncthreads();
  if (row0 == 0 && blockIdx.x == 0 && blockIdx.y == 0) {
    const int2 n = label_count(label_count_share(p));
    if (threadIdx.x == 0) label_scale(p, n.x);
  }
  constexpr int kWords = kLabelGCols / 8, kEach = kLabelGRows * kWords / 256;
  uint4 word[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int at = threadIdx.x + 256 * i, r = at / kWords, c = c0 + 8 * (at % kWords);
    if (r0 + r < rows && c < p.V) word[i] = *reinterpret_cast<const uint4*>(G + (r0 + r) * ldg + c);
  }
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int at = threadIdx.x + 256 * i, r = at / kWords, c = c0 + 8 * (at % kWords);
    if (r0 + r >= rows || c >= p.V) continue;
    const long long t = row0 + r0 + r;
    const int col = p.col[t];
    float f[8];
    if (col >= 0) {
      const float k = factor[r][(at % kWords) / 4], off = p.coefC[t], b = p.coefB[t];
      words_to_f32(word[i], f, __half());
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = fmaf(k, f[j], -off) - (c + j == col ? b : 0.f);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = 0.f;              // whatever an ignored token's logits were
    }
    uint4 o;
    f32_to_words(f, o, __nv_bfloat16());
    *reinterpret_cast<uint4*>(G + (r0 + r) * ldg + c) = o;
  }
}

// A finished gradient times an upstream gradient that came later: the product in fp32, rounded once. A word of 16 bytes a thread;
// bound by memory: 131072 x 2048 bf16 162 us, 6.6 TB/s.
template <typename T>
__global__ void __launch_bounds__(256)
label_rescale_kernel(const uint4* in, const float* factor, uint4* out, long long words) {
  grid_dependents_launch();
  grid_dependency_wait();
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= words) return;
  const float k = *factor;
  uint4 w = in[i];
  if constexpr (sizeof(T) == 4) {
    w = make_uint4(__float_as_uint(k * __uint_as_float(w.x)), __float_as_uint(k * __uint_as_float(w.y)),
                   __float_as_uint(k * __uint_as_float(w.z)), __float_as_uint(k * __uint_as_float(w.w)));
  } else {
    float f[8];
    words_to_f32(w, f, T());
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] *= k;
    f32_to_words(f, w, T());
  }
  out[i] = w;
}

__global__ void __launch_bounds__(256)
label_round_kernel(const float* in, uint2* out, long long n4, const int* go) {
  grid_dependents_launch();
  grid_dependency_wait();
  if (go != nullptr && *go == 0) return;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= n4) return;
  const float4 v = reinterpret_cast<const float4*>(in)[i];
  out[i] = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
}

}  // namespace kdkl
