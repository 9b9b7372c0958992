// Host side of the block norm: argument checks and launches; enqueue-only.
#include <math.h>
#include <string.h>

#include <type_traits>

#include "block_norm_kernels.cuh"
#include "body_host.cuh"

using namespace kdkl;

// ------------------------------------------------------------------ block norm
static constexpr long long kNormMaxH = 32768;
// Blocks of the *_rows kernels that share a row, and their threads: two groups of eight columns each.
static int rows_cluster(long long H) { return H <= kRowsMaxH ? 1 : H <= 2 * kRowsMaxH ? 2 : 4; }
static int rows_threads(long long H) {
  const long long per = 16 * rows_cluster(H);
  return (int)(((act_codes_pitch(H) + per - 1) / per + 31) / 32 * 32);
}
static_assert(kNormMaxH <= (long long)kRowsMaxCluster * kRowsMaxH, "the widest rows");
// The most blocks of the backward kernels, each of which leaves one partial row: what 1024 threads an SM amount to.
static long long norm_parts(long long T, long long H) {
  const int threads = rows_threads(H);
  const long long most = (long long)sm_count_or_default() * (1024 / threads > 16 ? 16 : 1024 / threads);
  return T < most ? T : most;
}

extern "C" size_t kdkl_block_norm_workspace_bytes(int64_t T, int64_t H) {
  if (!shape_ok(T, H) || H > kNormMaxH) return 0;
  return up((size_t)norm_parts(T, H) * 3 * act_codes_pitch(H) * 4, 256) + 256;
}

static int check_norm(const kdkl_block_norm_args* a, bool backward) {
  if (!a) return KDKL_ERR_NULL;
  if (a->struct_size != (int32_t)sizeof(kdkl_block_norm_args)) return KDKL_ERR_ARG;
  if (!shape_ok(a->T, a->H) || a->H > kNormMaxH) return KDKL_ERR_SHAPE;
  if (a->type != KDKL_TYPE_BF16 && a->type != KDKL_TYPE_F16) return KDKL_ERR_ARG;
  if (a->residual_type != a->type && a->residual_type != KDKL_TYPE_F32) return KDKL_ERR_ARG;
  if (!is_type(a->weight_type) || !is_type(a->gate_type)) return KDKL_ERR_ARG;
  if (a->gate_kind < KDKL_GATE_NONE || a->gate_kind > KDKL_GATE_TOKEN) return KDKL_ERR_ARG;
  if (a->format != KDKL_ACT8_NONE && !is_format(a->format)) return KDKL_ERR_ARG;
  if (!isfinite(a->eps) || a->eps < 0.f || !isfinite(a->weight_offset) || !isfinite(a->branch_scale) ||
      !isfinite(a->residual_scale))
    return KDKL_ERR_ARG;
  if (a->gate_kind != KDKL_GATE_NONE && !a->gate && (a->T != 0 || a->gate_kind == KDKL_GATE_CHANNEL)) return KDKL_ERR_NULL;
  const int tb = type_bytes(a->type), rb = type_bytes(a->residual_type), wb = type_bytes(a->weight_type);
  if ((uintptr_t)a->post_weight % wb || (uintptr_t)a->pre_weight % wb || (uintptr_t)a->gate % type_bytes(a->gate_type))
    return KDKL_ERR_ALIGN;
  if (a->format != KDKL_ACT8_NONE) {
    if ((((uintptr_t)a->branch_record) | ((uintptr_t)a->sum_record) | ((uintptr_t)a->y_record)) & 255) return KDKL_ERR_ALIGN;
    if ((a->branch_record || a->sum_record || a->y_record) && a->record_bytes < record_need(a->T, a->H)) return KDKL_ERR_WORKSPACE;
  }
  if (((uintptr_t)a->rho_post | (uintptr_t)a->rho_pre) & 3) return KDKL_ERR_ALIGN;
  if (!backward) {
    if (a->T == 0) return KDKL_OK;
    if (!a->residual || !a->branch || !a->sum || (a->pre_weight && !a->y)) return KDKL_ERR_NULL;
    if (a->T > 1 && (a->ld_residual < a->H || a->ld_branch < a->H)) return KDKL_ERR_SHAPE;
    if ((uintptr_t)a->residual % rb || (uintptr_t)a->branch % tb || (uintptr_t)a->sum % rb || (uintptr_t)a->y % tb)
      return KDKL_ERR_ALIGN;
    return KDKL_OK;
  }
  const bool has_post = a->post_weight != nullptr, has_pre = a->pre_weight != nullptr;
  if ((has_post && !a->dpost_weight) || (has_pre && !a->dpre_weight) || !a->workspace) return KDKL_ERR_NULL;
  if (a->gate_kind == KDKL_GATE_CHANNEL && !a->dgate) return KDKL_ERR_NULL;
  if ((uintptr_t)a->workspace & 255) return KDKL_ERR_ALIGN;
  if ((uintptr_t)a->dpost_weight % wb || (uintptr_t)a->dpre_weight % wb || (uintptr_t)a->dgate % type_bytes(a->gate_type))
    return KDKL_ERR_ALIGN;
  if (a->workspace_bytes < kdkl_block_norm_workspace_bytes(a->T, a->H)) return KDKL_ERR_WORKSPACE;
  if (a->T == 0) return KDKL_OK;
  if (!a->dresidual || !a->dbranch || (has_pre && !a->dy) || (a->gate_kind == KDKL_GATE_TOKEN && !a->dgate)) return KDKL_ERR_NULL;
  if ((has_post && !a->rho_post) || (has_pre && !a->rho_pre)) return KDKL_ERR_NULL;
  if (a->format != KDKL_ACT8_NONE) {
    if (!a->branch_record || (has_pre && !a->sum_record)) return KDKL_ERR_NULL;
  } else {
    if (!a->branch || (has_pre && !a->sum)) return KDKL_ERR_NULL;
    if (a->T > 1 && a->ld_branch < a->H) return KDKL_ERR_SHAPE;
    if ((uintptr_t)a->branch % tb || (uintptr_t)a->sum % rb) return KDKL_ERR_ALIGN;
  }
  if (a->T > 1 && ((has_pre && a->ld_dy < a->H) || (a->dsum && a->ld_dsum < a->H))) return KDKL_ERR_SHAPE;
  if ((uintptr_t)a->dy % tb || (uintptr_t)a->dsum % rb || (uintptr_t)a->dresidual % rb || (uintptr_t)a->dbranch % tb)
    return KDKL_ERR_ALIGN;
  return KDKL_OK;
}

// Launches a *_rows kernel with as many blocks, or clusters of C, as the device holds at once (at most `most`: one per row,
// one per partial row). The shared memory a kernel may use is an attribute of its copy on the device, set once, to what its
// widest rows take (`smem_widest`) - one value whatever the launch, so that threads that launch it for the first time at the
// same time, at different widths, cannot leave it too small for each other. How many blocks fit an SM is asked once per
// number of warps.
template <auto KERN, int C, typename P>
static int launch_rows(long long most, int threads, int smem, int smem_widest, const P& p, const char* name, const DeviceInfo& di,
                       cudaStream_t st, int* rows) {
  struct Known { bool allowed; int fit[kRowsThreads / 32 + 1]; };
  static Known known[kMaxDevices];
  Known fresh;
  memset(&fresh, 0, sizeof(fresh));
  Known& k = di.dev >= 0 && di.dev < kMaxDevices ? known[di.dev] : fresh;
  if (!k.allowed) {
    KDKL_CUDA(cudaFuncSetAttribute(KERN, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_widest));
    k.allowed = true;
  }
  int fit = k.fit[threads / 32];
  if (fit == 0) {
    KDKL_CUDA(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&fit, KERN, threads, smem));
    if (fit < 1) fit = 1;
    k.fit[threads / 32] = fit;
  }
  const long long held = (long long)di.sm_count * fit / C;
  *rows = (int)(most < held ? most : held);
  return launch_cluster(C, name, KERN, dim3((unsigned)*rows * C, 1, 1), threads, (size_t)smem, st, p);
}

// (rows wider than a block's: without the FULL variants)
#define KDKL_BY_CLUSTER(H, full, C, FULL, ...)                                                                   \
  do {                                                                                                           \
    const int c__ = rows_cluster(H);                                                                             \
    if (c__ == 4) { constexpr int C = 4; constexpr bool FULL = false; __VA_ARGS__; }                             \
    else if (c__ == 2) { constexpr int C = 2; constexpr bool FULL = false; __VA_ARGS__; }                        \
    else { constexpr int C = 1; KDKL_BY_BOOL(full, FULL, __VA_ARGS__); }                                         \
  } while (0)

static bool vectors_are_words(const kdkl_block_norm_args* a) {
  return words(a->post_weight, 0, 1, a->H, a->weight_type) && words(a->pre_weight, 0, 1, a->H, a->weight_type) &&
         (a->gate_kind != KDKL_GATE_CHANNEL || words(a->gate, 0, 1, a->H, a->gate_type));
}

// Threads a row and groups of eight columns a thread of the *_any kernels.
#define KDKL_NORM_SHAPE(H, THREADS, NV, ...)                                              \
  do {                                                                                    \
    if ((H) <= 4096) { constexpr int THREADS = 512, NV = 1; __VA_ARGS__; }                \
    else { constexpr int THREADS = 1024, NV = 4; __VA_ARGS__; }                           \
  } while (0)

extern "C" {

int kdkl_block_norm_forward(const kdkl_block_norm_args* a, void* cuda_stream) {
  g_launches = 0;
  int rc = check_norm(a, false);
  if (rc || a->T == 0) return rc;
  DeviceInfo di;
  if ((rc = need_b200(&di))) return rc;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  NormForward p;
  p.residual = a->residual; p.ld_residual = a->ld_residual;
  p.branch = a->branch; p.ld_branch = a->ld_branch;
  p.post = AnyVec{a->post_weight, a->weight_type}; p.pre = AnyVec{a->pre_weight, a->weight_type};
  p.gate = AnyVec{a->gate, a->gate_type};
  p.y = a->y; p.sum = a->sum; p.rho_post = a->rho_post; p.rho_pre = a->rho_pre;
  p.rec_branch = record_at(a->branch_record, a->T, a->H);
  p.rec_sum = record_at(a->sum_record, a->T, a->H);
  p.rec_y = record_at(a->pre_weight ? a->y_record : nullptr, a->T, a->H);
  p.format = a->format;
  p.T = a->T; p.H = (int)a->H; p.gate_kind = a->gate_kind;
  p.eps = a->eps; p.offset = a->weight_offset; p.alpha = a->branch_scale; p.beta = a->residual_scale;
  const bool vec = words(a->residual, a->ld_residual, a->T, a->H, a->residual_type) &&
                   words(a->branch, a->ld_branch, a->T, a->H, a->type) && words(a->sum, a->H, a->T, a->H, a->residual_type) &&
                   words(a->y, a->H, a->T, a->H, a->type) && vectors_are_words(a);
  const bool any_record = a->format != KDKL_ACT8_NONE && (a->branch_record || a->sum_record || p.rec_y.codes);
  const long long most = (long long)di.sm_count * 8;
  const unsigned grid = (unsigned)(a->T < most ? a->T : most);
  if (vec) {
    const int fmt = any_record ? a->format : KDKL_ACT8_NONE;
    const bool full = a->post_weight && a->pre_weight;
    const int threads = rows_threads(a->H), chunk = rows_forward_chunk(type_bytes(a->residual_type));
    int blocks;
    KDKL_BY_TYPE16(a->type, A, KDKL_BY_BOOL(a->residual_type == KDKL_TYPE_F32, WIDE, KDKL_BY_FORMAT_OR_NONE(fmt, FMT, KDKL_BY_CLUSTER(a->H, full, C, FULL,
      return (launch_rows<block_norm_forward_rows_kernel<A, std::conditional_t<WIDE, float, A>, FMT, FULL, C>, C>(
          a->T, threads, threads / 16 * chunk, kRowsThreads / 16 * chunk, p, "block_norm_forward_rows_kernel", di, st, &blocks))))));
  }
  KDKL_BY_TYPE16(a->type, A, KDKL_BY_BOOL(a->residual_type == KDKL_TYPE_F32, WIDE,
    KDKL_BY_BOOL(any_record, REC, KDKL_NORM_SHAPE(a->H, THREADS, NV,
      rc = (launch("block_norm_forward_any_kernel", block_norm_forward_any_kernel<A, std::conditional_t<WIDE, float, A>, REC, THREADS, NV>,
                   dim3(grid, 1, 1), THREADS, 0, st, p))))));
  return rc;
}

int kdkl_block_norm_backward(const kdkl_block_norm_args* a, void* cuda_stream) {
  g_launches = 0;
  int rc = check_norm(a, true);
  if (rc) return rc;
  DeviceInfo di;
  if ((rc = need_b200(&di))) return rc;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const bool has_post = a->post_weight != nullptr, has_pre = a->pre_weight != nullptr;
  const bool channel = a->gate_kind == KDKL_GATE_CHANNEL;
  int parts = (int)norm_parts(a->T, a->H);
  if (a->T > 0) {
    NormBackward p;
    p.dsum = a->dsum; p.ld_dsum = a->ld_dsum; p.dy = a->dy; p.ld_dy = a->ld_dy;
    p.sum = a->sum; p.ld_sum = a->H; p.branch = a->branch; p.ld_branch = a->ld_branch;
    p.rec_sum = record_at(a->sum_record, a->T, a->H); p.rec_branch = record_at(a->branch_record, a->T, a->H);
    p.format = a->format;
    p.post = AnyVec{a->post_weight, a->weight_type}; p.pre = AnyVec{a->pre_weight, a->weight_type};
    p.gate = AnyVec{a->gate, a->gate_type};
    p.rho_post = a->rho_post; p.rho_pre = a->rho_pre;
    p.dresidual = a->dresidual; p.dbranch = a->dbranch; p.dgate_token = a->dgate; p.gate_type = a->gate_type;
    p.partial = at<float>(a->workspace, 0);
    p.T = a->T; p.H = (int)a->H; p.gate_kind = a->gate_kind;
    p.offset = a->weight_offset; p.alpha = a->branch_scale; p.beta = a->residual_scale;
    const bool kept = a->format != KDKL_ACT8_NONE ||
                      (words(a->branch, a->ld_branch, a->T, a->H, a->type) &&
                       (!has_pre || words(a->sum, a->H, a->T, a->H, a->residual_type)));
    const bool vec = kept && a->H % 8 == 0 && (!has_pre || words(a->dy, a->ld_dy, a->T, a->H, a->type)) &&
                     (!a->dsum || words(a->dsum, a->ld_dsum, a->T, a->H, a->residual_type)) &&
                     words(a->dresidual, a->H, a->T, a->H, a->residual_type) && words(a->dbranch, a->H, a->T, a->H, a->type) &&
                     vectors_are_words(a);
    if (vec) {
      const bool rec = a->format != KDKL_ACT8_NONE, full = has_post && has_pre && a->dsum;
      const int threads = rows_threads(a->H), rb = type_bytes(a->residual_type);
      const int row = rows_backward_stages(rb, rec) * rows_backward_chunk(rb, rec);
      KDKL_BY_TYPE16(a->type, A, KDKL_BY_BOOL(a->residual_type == KDKL_TYPE_F32, WIDE, KDKL_BY_FORMAT_OR_NONE(a->format, FMT, KDKL_BY_CLUSTER(a->H, full, C, FULL,
        rc = (launch_rows<block_norm_backward_rows_kernel<A, std::conditional_t<WIDE, float, A>, FMT, FULL, C>, C>(
            parts, threads, threads / 16 * row, kRowsThreads / 16 * row, p, "block_norm_backward_rows_kernel", di, st, &parts))))));
      if (rc) return rc;
    } else {
      KDKL_BY_TYPE16(a->type, A, KDKL_BY_BOOL(a->residual_type == KDKL_TYPE_F32, WIDE,
        KDKL_BY_BOOL(a->format != KDKL_ACT8_NONE, REC, KDKL_NORM_SHAPE(a->H, THREADS, NV,
          rc = (launch("block_norm_backward_any_kernel",
                       block_norm_backward_any_kernel<A, std::conditional_t<WIDE, float, A>, REC, THREADS, NV>,
                       dim3((unsigned)parts, 1, 1), THREADS, 0, st, p))))));
      if (rc) return rc;
    }
  }
  if (has_post || has_pre || channel) {
    NormColumns c;
    memset(&c, 0, sizeof(c));
    int n = 0;
    auto add = [&](int which, void* out, int type) { c.which[n] = which; c.out[n] = out; c.type[n] = type; ++n; };
    if (has_post) add(0, a->dpost_weight, a->weight_type);
    if (has_pre) add(1, a->dpre_weight, a->weight_type);
    if (channel) add(2, a->dgate, a->gate_type);
    return launch("block_norm_columns_kernel", block_norm_columns_kernel, dim3((unsigned)((a->H + 31) / 32), (unsigned)n, 1),
                  1024, 0, st, at<float>(a->workspace, 0), parts, a->H, act_codes_pitch(a->H), c);
  }
  return KDKL_OK;
}

}  // extern "C"
