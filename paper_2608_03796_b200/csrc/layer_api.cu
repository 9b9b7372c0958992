// Host side of the layer norm and of rotary positions. Argument checks and launches; enqueue-only.
#include <math.h>
#include <string.h>

#include "body_host.cuh"
#include "layer_norm_kernels.cuh"
#include "rotary_kernels.cuh"

using namespace kdkl;

// ------------------------------------------------------------------ layer norm
// Partial rows of the weight's gradient: one a warp or block of the row kernels, as many as stay resident.
static bool ln_warp_rows(long long H) { return H <= kLnWarpCols; }
static bool ln_wide(long long H) { return H > kLnBlockCols; }
static int ln_threads(long long H) { return (int)((act_codes_pitch(H) / 8 + 31) / 32 * 32); }
static int ln_rows_threads(long long H) { return (int)((act_codes_pitch(H) / 16 + 31) / 32 * 32); }      // in whole words
static long long ln_blocks(long long T, long long H, int sm_count) {
  if (ln_wide(H)) return T < 2ll * sm_count ? T : 2ll * sm_count;
  if (ln_warp_rows(H)) {
    const long long need = (T + kLnWarpThreads / 32 - 1) / (kLnWarpThreads / 32), most = 3ll * sm_count;
    return need < most ? need : most;
  }
  // as many blocks as an SM holds of the backward rows kernel (up to 128 registers a thread), or of smaller ones a few more
  const long long most = (long long)sm_count * (592 / ln_rows_threads(H));
  return T < most ? T : most;
}
static long long ln_parts(long long T, long long H, int sm_count) {
  const long long blocks = ln_blocks(T, H, sm_count);
  return ln_warp_rows(H) ? blocks * (kLnWarpThreads / 32) : blocks;
}

static int check_ln(const kdkl_layer_norm_args* a, bool backward) {
  if (!a) return KDKL_ERR_NULL;
  if (a->struct_size != (int32_t)sizeof(kdkl_layer_norm_args)) return KDKL_ERR_ARG;
  if (!shape_ok(a->T, a->H)) return KDKL_ERR_SHAPE;
  if (!is_type(a->x_type) || !is_type(a->y_type) || !is_type(a->weight_type)) return KDKL_ERR_ARG;
  if (a->y_type != a->x_type && a->x_type != KDKL_TYPE_F32) return KDKL_ERR_ARG;
  if (a->format != KDKL_ACT8_NONE && !is_format(a->format)) return KDKL_ERR_ARG;
  if (!(a->eps >= 0.f) || isinf(a->eps)) return KDKL_ERR_ARG;
  const int xb = type_bytes(a->x_type), yb = type_bytes(a->y_type), wb = type_bytes(a->weight_type);
  if (((uintptr_t)a->weight | (uintptr_t)a->bias) % wb) return KDKL_ERR_ALIGN;
  const bool records = a->format != KDKL_ACT8_NONE;
  if (records && a->T != 0) {
    if (((uintptr_t)a->x_record | (uintptr_t)a->y_record) & 255) return KDKL_ERR_ALIGN;
    if (a->record_bytes < record_need(a->T, a->H)) return KDKL_ERR_WORKSPACE;
  }
  if (!backward) {
    if (a->T == 0) return KDKL_OK;
    if (!a->x || !a->y || (!a->mean) != (!a->rho)) return KDKL_ERR_NULL;
    if (a->T > 1 && a->ld_x < a->H) return KDKL_ERR_SHAPE;
    if (((uintptr_t)a->x % xb) || ((uintptr_t)a->y % yb) || (((uintptr_t)a->mean | (uintptr_t)a->rho) & 3)) return KDKL_ERR_ALIGN;
    return KDKL_OK;
  }
  if ((a->weight && !a->dweight) || (a->bias && !a->dbias)) return KDKL_ERR_NULL;
  if (((uintptr_t)a->dweight | (uintptr_t)a->dbias) % wb) return KDKL_ERR_ALIGN;
  if (!a->workspace) return KDKL_ERR_NULL;
  if ((uintptr_t)a->workspace & 255) return KDKL_ERR_ALIGN;
  if (a->workspace_bytes < kdkl_layer_norm_workspace_bytes(a->T, a->H)) return KDKL_ERR_WORKSPACE;
  if (a->T == 0) return KDKL_OK;
  if (!a->dy || !a->dx || !a->mean || !a->rho || (records ? !a->x_record : !a->x)) return KDKL_ERR_NULL;
  if (a->T > 1 && ((!records && a->ld_x < a->H) || a->ld_dy < a->H)) return KDKL_ERR_SHAPE;
  if ((!records && (uintptr_t)a->x % xb) || ((uintptr_t)a->dx % xb) || ((uintptr_t)a->dy % yb) ||
      (((uintptr_t)a->mean | (uintptr_t)a->rho) & 3))
    return KDKL_ERR_ALIGN;
  return KDKL_OK;
}
static LnParams ln_params(const kdkl_layer_norm_args* a) {
  LnParams p;
  memset(&p, 0, sizeof(p));
  p.x = a->x; p.ld_x = a->ld_x;
  p.weight = a->weight; p.bias = a->bias; p.weight_type = a->weight_type;
  p.y = a->y; p.mean = a->mean; p.rho = a->rho;
  if (a->format != KDKL_ACT8_NONE) {
    p.x_record = record_at(a->x_record, a->T, a->H);
    p.y_record = record_at(a->y_record, a->T, a->H);
  }
  p.format = a->format;
  p.dy = a->dy; p.ld_dy = a->ld_dy; p.dx = a->dx;
  p.T = a->T; p.H = (int)a->H; p.eps = a->eps;
  return p;
}
static bool ln_vectors_are_words(const kdkl_layer_norm_args* a) {
  return words(a->weight, 0, 1, a->H, a->weight_type) && words(a->bias, 0, 1, a->H, a->weight_type);
}
// A rows kernel with as many blocks as fit on the device at once, at most `most`.
template <auto KERN>
static int launch_ln_rows(const char* name, int threads, int bytes_a_thread, long long most, const LnParams& p, const DeviceInfo& di,
                          cudaStream_t st, int* used) {
  struct Known { bool allowed; int fit[kLnRowsThreads / 32 + 1]; };
  static Known known[kMaxDevices];
  Known none = {};
  Known& k = di.dev >= 0 && di.dev < kMaxDevices ? known[di.dev] : none;
  const int smem = threads * bytes_a_thread;
  if (!k.allowed) {                            // (what the widest rows need, once)
    KDKL_CUDA(cudaFuncSetAttribute(KERN, cudaFuncAttributeMaxDynamicSharedMemorySize, kLnRowsThreads * bytes_a_thread));
    k.allowed = true;
  }
  int fit = k.fit[threads / 32];
  if (fit == 0) {
    KDKL_CUDA(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&fit, KERN, threads, smem));
    if (fit < 1) fit = 1;
    k.fit[threads / 32] = fit;
  }
  const long long held = (long long)di.sm_count * fit;
  const long long grid = most < held ? most : held;
  if (used != nullptr) *used = (int)grid;
  return launch(name, KERN, dim3((unsigned)grid), threads, (size_t)smem, st, p);
}
#define KDKL_LN_TYPES(a, X, Y, ...)                                                                    \
  do {                                                                                                 \
    if ((a)->x_type != KDKL_TYPE_F32) KDKL_BY_TYPE16((a)->x_type, X, { using Y = X; __VA_ARGS__; });   \
    else { using X = float; KDKL_BY_TYPE((a)->y_type, Y, __VA_ARGS__); }                               \
  } while (0)

// ------------------------------------------------------------------ rotary positions
// Columns that a thread takes at a time: as wide an aligned word as rows, heads and halves allow; 0: element by element.
static bool rotary_aligned(const RotaryTensor& r, long long bytes, long long size) {
  return r.heads == 0 || (((uintptr_t)r.x | (uintptr_t)r.y) % bytes == 0 && (r.x_token * size) % bytes == 0 &&
                          (r.x_head * size) % bytes == 0 && (r.y_token * size) % bytes == 0 && (r.y_head * size) % bytes == 0);
}
static int rotary_width(const RotaryParams& p, bool half, int size) {
  for (int bytes = 16; bytes >= 8; bytes /= 2) {
    const int n = bytes / size;
    if ((half ? p.R / 2 : p.R) % n == 0 && (p.D - p.R) % n == 0 && rotary_aligned(p.t[0], bytes, size) &&
        rotary_aligned(p.t[1], bytes, size))
      return n;
  }
  return 0;
}

extern "C" {

size_t kdkl_layer_norm_workspace_bytes(int64_t T, int64_t H) {
  if (!shape_ok(T, H)) return 0;
  const size_t bytes = (size_t)ln_parts(T, H, sm_count_or_default()) * 2 * H * 4;
  return up(bytes < 256 ? 256 : bytes, 256);
}

int kdkl_layer_norm_forward(const kdkl_layer_norm_args* a, void* cuda_stream) {
  g_launches = 0;
  int rc = check_ln(a, false);
  if (rc || a->T == 0) return rc;
  DeviceInfo di;
  if ((rc = need_b200(&di))) return rc;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const LnParams p = ln_params(a);
  const bool vec = words(a->x, a->ld_x, a->T, a->H, a->x_type) && words(a->y, a->H, a->T, a->H, a->y_type) && ln_vectors_are_words(a);
  const unsigned grid = (unsigned)ln_blocks(a->T, a->H, di.sm_count);
  KDKL_LN_TYPES(a, X, Y, KDKL_BY_BOOL(vec, VEC, {
    if (ln_wide(a->H)) {
      rc = launch("layer_norm_forward_wide_kernel", layer_norm_forward_wide_kernel<X, Y, VEC>, dim3(grid), kLnWideThreads, 0, st, p);
    } else if (a->H <= kLnWarpCols / 2) {
      rc = launch("layer_norm_forward_kernel", layer_norm_forward_kernel<X, Y, 1, true, VEC>, dim3(grid), kLnWarpThreads, 0, st, p);
    } else if (ln_warp_rows(a->H)) {
      rc = launch("layer_norm_forward_kernel", layer_norm_forward_kernel<X, Y, 2, true, VEC>, dim3(grid), kLnWarpThreads, 0, st, p);
    } else if constexpr (VEC) {
      const bool rec = p.x_record.codes != nullptr || p.y_record.codes != nullptr;
      KDKL_BY_BOOL(rec, REC, KDKL_BY_BOOL(a->H % 512 == 0, FULL,
        rc = (launch_ln_rows<layer_norm_forward_rows_kernel<X, Y, REC, FULL>>("layer_norm_forward_rows_kernel", ln_rows_threads(a->H),
            2 * kLnAhead * 8 * (int)sizeof(X), a->T, p, di, st, nullptr))));
    } else {
      rc = launch("layer_norm_forward_kernel", layer_norm_forward_kernel<X, Y, 1, false, false>, dim3(grid), ln_threads(a->H), 0, st, p);
    }
  }));
  return rc;
}

int kdkl_layer_norm_backward(const kdkl_layer_norm_args* a, void* cuda_stream) {
  g_launches = 0;
  int rc = check_ln(a, true);
  if (rc) return rc;
  DeviceInfo di;
  if ((rc = need_b200(&di))) return rc;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  LnParams p = ln_params(a);
  const bool rec = a->format != KDKL_ACT8_NONE, sums = a->weight || a->bias;
  // never more partial rows than the workspace was sized for (the count of SMs may be another one there)
  long long blocks = ln_blocks(a->T, a->H, di.sm_count);
  const long long most = ln_blocks(a->T, a->H, sm_count_or_default());
  if (blocks > most) blocks = most;
  p.part = sums ? at<float>(a->workspace, 0) : nullptr;
  const bool vec = a->H % 8 == 0 && (rec || words(a->x, a->ld_x, a->T, a->H, a->x_type)) && words(a->dy, a->ld_dy, a->T, a->H, a->y_type) &&
                   words(a->dx, a->H, a->T, a->H, a->x_type) && words(a->weight, 0, 1, a->H, a->weight_type);
  const dim3 grid((unsigned)blocks);
  if (a->T > 0) {
    KDKL_LN_TYPES(a, X, Y, KDKL_BY_BOOL(vec, VEC, KDKL_BY_BOOL(rec, REC, {
      if (ln_wide(a->H)) {
        rc = launch("layer_norm_backward_wide_kernel", layer_norm_backward_wide_kernel<X, Y, REC, VEC>, grid, kLnWideThreads, 0, st, p);
        if (rc == KDKL_OK && sums)
          rc = launch("layer_norm_columns_kernel", layer_norm_columns_kernel<X, Y, REC, VEC>,
                      dim3((unsigned)((a->H + 2047) / 2048), (unsigned)blocks), 256, 0, st, p);
      } else if (a->H <= kLnWarpCols / 2) {
        rc = launch("layer_norm_backward_kernel", layer_norm_backward_kernel<X, Y, 1, true, REC, VEC>, grid, kLnWarpThreads, 0, st, p);
      } else if (ln_warp_rows(a->H)) {
        rc = launch("layer_norm_backward_kernel", layer_norm_backward_kernel<X, Y, 2, true, REC, VEC>, grid, kLnWarpThreads, 0, st, p);
      } else if constexpr (VEC) {
        int used = 0;
        KDKL_BY_BOOL(a->H % 512 == 0, FULL, {
          if constexpr (REC)
            KDKL_BY_FORMAT(a->format, FMT, rc = (launch_ln_rows<layer_norm_backward_rows_kernel<X, Y, FMT, FULL>>("layer_norm_backward_rows_kernel",
                ln_rows_threads(a->H), 2 * kLnAhead * 8 * (int)sizeof(Y), blocks, p, di, st, &used)));
          else
            rc = (launch_ln_rows<layer_norm_backward_rows_kernel<X, Y, KDKL_ACT8_NONE, FULL>>("layer_norm_backward_rows_kernel", ln_rows_threads(a->H),
                2 * kLnAhead * 8 * (int)(sizeof(X) + sizeof(Y)), blocks, p, di, st, &used));
        });
        blocks = used;
      } else {
        rc = launch("layer_norm_backward_kernel", layer_norm_backward_kernel<X, Y, 1, false, REC, false>, grid, ln_threads(a->H), 0, st, p);
      }
    })));
    if (rc) return rc;
  }
  if (!sums) return KDKL_OK;
  const long long parts = a->T == 0 ? 0 : ln_warp_rows(a->H) ? blocks * (kLnWarpThreads / 32) : blocks;
  return launch("layer_norm_reduce_kernel", layer_norm_reduce_kernel, dim3((unsigned)((a->H + 31) / 32), 2), 1024, 0, st,
                (const float*)at<float>(a->workspace, 0), parts, (int)a->H, a->weight ? a->dweight : nullptr,
                a->bias ? a->dbias : nullptr, (int)a->weight_type);
}

int kdkl_rotary_table(int32_t rotary_dim, double base, int32_t scaling, double factor, double original_length, double* turns,
                      float* magnitude) {
  if (!turns || !magnitude) return KDKL_ERR_NULL;
  if (rotary_dim < 2 || rotary_dim > KDKL_ROTARY_MAX_DIM || rotary_dim % 2) return KDKL_ERR_SHAPE;
  if (!(base > 1.0) || !isfinite(base) || scaling < KDKL_ROTARY_PLAIN || scaling > KDKL_ROTARY_YARN) return KDKL_ERR_ARG;
  if (scaling != KDKL_ROTARY_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return KDKL_ERR_ARG;
  if (scaling == KDKL_ROTARY_YARN && (!(original_length > 0.0) || !isfinite(original_length))) return KDKL_ERR_ARG;
  if (scaling == KDKL_ROTARY_NTK && rotary_dim < 4) return KDKL_ERR_SHAPE;
  const double two_pi = 6.283185307179586476925286766559, R = rotary_dim;
  if (scaling == KDKL_ROTARY_NTK) base *= pow(factor, R / (R - 2.0));
  *magnitude = scaling == KDKL_ROTARY_YARN ? (float)(0.1 * log(factor) + 1.0) : 1.f;
  for (int i = 0; i < rotary_dim / 2; ++i) {
    double f = pow(base, -2.0 * i / R) / two_pi;
    if (scaling == KDKL_ROTARY_LINEAR) f /= factor;
    if (scaling == KDKL_ROTARY_YARN) {
      double keep = (original_length * f - 1.0) / 31.0;        // 1 turn and fewer: stretched; 32 and more: kept
      keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
      f = (1.0 - keep) * f / factor + keep * f;
    }
    turns[i] = f;
  }
  return KDKL_OK;
}

int kdkl_rotary(const kdkl_rotary_args* a, void* cuda_stream) {
  g_launches = 0;
  if (!a) return KDKL_ERR_NULL;
  if (a->struct_size != (int32_t)sizeof(kdkl_rotary_args)) return KDKL_ERR_ARG;
  if (a->T < 0 || a->T > 0x7fffff00ll || a->head_dim < 2 || a->head_dim > KDKL_ROTARY_MAX_DIM || a->head_dim % 2 || a->rotary_dim < 2 ||
      a->rotary_dim > a->head_dim || a->rotary_dim % 2)
    return KDKL_ERR_SHAPE;
  if (a->q_heads < 0 || a->k_heads < 0 || a->q_heads > KDKL_ROTARY_MAX_HEADS || a->k_heads > KDKL_ROTARY_MAX_HEADS) return KDKL_ERR_SHAPE;
  if (!is_type(a->type) || (a->layout != KDKL_ROTARY_HALF && a->layout != KDKL_ROTARY_INTERLEAVED)) return KDKL_ERR_ARG;
  if ((a->inverse != 0 && a->inverse != 1) || (a->wide_positions != 0 && a->wide_positions != 1) || !isfinite(a->magnitude)) return KDKL_ERR_ARG;
  if (a->T == 0 || a->q_heads + a->k_heads == 0) return KDKL_OK;
  if (!a->positions || !a->turns || (a->q_heads && (!a->q || !a->q_out)) || (a->k_heads && (!a->k || !a->k_out))) return KDKL_ERR_NULL;
  const int size = type_bytes(a->type);
  if (((uintptr_t)a->positions % (a->wide_positions ? 8 : 4)) || ((uintptr_t)a->turns & 7)) return KDKL_ERR_ALIGN;
  RotaryParams p;
  memset(&p, 0, sizeof(p));
  p.t[0] = RotaryTensor{a->q, a->q_token, a->q_head, a->q_out, a->q_out_token, a->q_out_head, a->q_heads};
  p.t[1] = RotaryTensor{a->k, a->k_token, a->k_head, a->k_out, a->k_out_token, a->k_out_head, a->k_heads};
  for (const RotaryTensor& r : p.t) {
    if (r.heads == 0) continue;
    if (((uintptr_t)r.x | (uintptr_t)r.y) % size) return KDKL_ERR_ALIGN;
    if (r.x_token < 0 || r.x_head < 0 || r.y_token < 0 || r.y_head < 0) return KDKL_ERR_SHAPE;
    // an output's heads must not overlap, nor its tokens: either the tokens are the outer stride or the heads
    const long long D = a->head_dim;
    const bool head_ok = r.heads == 1 || r.y_head >= D, token_ok = a->T == 1 || r.y_token >= D;
    const bool apart = r.heads == 1 || a->T == 1 || r.y_token >= (r.heads - 1) * r.y_head + D || r.y_head >= (a->T - 1) * r.y_token + D;
    if (!head_ok || !token_ok || !apart) return KDKL_ERR_SHAPE;
  }
  DeviceInfo di;
  int rc = need_b200(&di);
  if (rc) return rc;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  p.positions = a->positions; p.wide_positions = a->wide_positions; p.turns = a->turns;
  p.magnitude = a->magnitude; p.sign = a->inverse ? -1.f : 1.f;
  p.T = a->T; p.D = a->head_dim; p.R = a->rotary_dim;
  // Four tokens a block, fewer where that would leave an SM without its eight blocks. Measured with 40 heads of 128 columns:
  // 32768 tokens 130, 113, 107 and 110 us with 1, 2, 4 and 8; 2047 tokens 10.9, 10.3, 11.5 and 12.4.
  p.tokens_per_block = a->T >= 32ll * di.sm_count ? 4 : a->T >= 8ll * di.sm_count ? 2 : 1;
  const dim3 grid((unsigned)((a->T + p.tokens_per_block - 1) / p.tokens_per_block));
  const size_t smem = (size_t)p.tokens_per_block * (p.R / 2) * sizeof(float2);
  const bool half = a->layout == KDKL_ROTARY_HALF;
  const int n = rotary_width(p, half, size);
  const int by = n > 0 ? n : half ? 1 : 2, items = (half ? p.R / 2 : p.R) / by + (p.D - p.R) / by;
  p.by_items = rotary_reciprocal(items); p.by_heads = rotary_reciprocal(a->q_heads + a->k_heads);
#define KDKL_ROTARY(E, HALF, N, ALIGNED) \
  rc = launch("rotary_kernel", rotary_kernel<E, HALF, N, ALIGNED>, grid, 256, smem, st, p)
  KDKL_BY_BOOL(half, HALF, {
    if (a->type == KDKL_TYPE_F32) {
      if (n == 4) KDKL_ROTARY(float, HALF, 4, true);
      else if (n == 2) KDKL_ROTARY(float, HALF, 2, true);
      else KDKL_ROTARY(float, HALF, (HALF ? 1 : 2), false);
    } else {
      KDKL_BY_TYPE16(a->type, E, {
        if (n == 8) KDKL_ROTARY(E, HALF, 8, true);
        else if (n == 4) KDKL_ROTARY(E, HALF, 4, true);
        else KDKL_ROTARY(E, HALF, (HALF ? 1 : 2), false);
      });
    }
  });
#undef KDKL_ROTARY
  return rc;
}

}  // extern "C"
