// Host side of the gated linear layer. Argument checks and launches; enqueue-only.
#include <string.h>

#include "body_host.cuh"
#include "gated_few_kernels.cuh"
#include "gemm_out.cuh"

using namespace kdkl;

// gate and up of the stacked weight [2 F, H], or dgate and dup inside [T, 2 F]: a [2, rows or features, columns] tensor of boxes
// 64 columns wide.
static int map_halves(CUtensorMap* m, const void* base, uint64_t inner, uint64_t outer, uint64_t pitch_bytes, uint64_t half_bytes,
                      uint32_t box_outer) {
  EncodeTiledFn fn = get_encode_fn();
  if (!fn) { snprintf(g_err, sizeof(g_err), "cuTensorMapEncodeTiled entry point not found"); return KDKL_ERR_CUDA; }
  cuuint64_t dims[3] = {inner, outer, 2}, strides[2] = {pitch_bytes, half_bytes};
  cuuint32_t box[3] = {64, box_outer, 1}, each[3] = {1, 1, 1};
  CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    snprintf(g_err, sizeof(g_err), "cuTensorMapEncodeTiled failed (%d): inner=%llu outer=%llu", (int)r, (unsigned long long)inner,
             (unsigned long long)outer);
    return KDKL_ERR_CUDA;
  }
  return KDKL_OK;
}

// What the backward call needs beside its status: parts of dx, and of the weight gradient (from x itself) or the
// workspace of the one from a record.
struct GatedPlan { OutPlan dx, dw; size_t at, bytes; };
static GatedPlan gated_plan(long long T, long long H, long long F, int dw_type) {
  GatedPlan g;
  const int sms = sm_count_or_default();
  g.dx = out_plan(T, H, 2 * F, sms, false);
  g.dw = out_plan(2 * F, H, T, sms, false);
  g.at = 256;
  size_t most = out_slab_bytes(g.dx, T, H, false);
  // (a bf16 gradient that is added to goes through one part in fp32)
  const size_t dw = out_slab_bytes(g.dw, 2 * F, H, dw_type == KDKL_TYPE_BF16), rec = kdkl_act8_dweight_workspace_bytes(T, 2 * F, H, dw_type);
  if (dw > most) most = dw;
  g.bytes = 256 + most > rec ? 256 + most : rec;
  return g;
}

static bool rows16(const void* p, long long ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0; }

static int check_gated(const kdkl_gated_linear_args* a) {
  if (!a) return KDKL_ERR_NULL;
  if (a->struct_size != (int32_t)sizeof(kdkl_gated_linear_args)) return KDKL_ERR_ARG;
  if (!shape_ok(a->T, a->H) || !shape_ok(a->T, a->F) || a->H % 8 || a->F % 8 || a->F >= (1ll << 29)) return KDKL_ERR_SHAPE;
  if (a->act != KDKL_GATED_SILU && a->act != KDKL_GATED_GELU) return KDKL_ERR_ARG;
  if (a->format != KDKL_ACT8_NONE && !is_format(a->format)) return KDKL_ERR_ARG;
  if (!a->weight || !a->workspace) return KDKL_ERR_NULL;
  if (((uintptr_t)a->weight & 15) || ((uintptr_t)a->workspace & 255)) return KDKL_ERR_ALIGN;
  return KDKL_OK;
}
static int check_kept(const void* record, size_t bytes, int64_t T, int64_t H) {
  if ((uintptr_t)record & 255) return KDKL_ERR_ALIGN;
  return bytes < record_need(T, H) ? KDKL_ERR_WORKSPACE : KDKL_OK;
}

template <int EPI>
static int gated_product(const kdkl_gated_linear_args* a, GemmParams& p, const CUtensorMap& tc, const DeviceInfo& di, cudaStream_t st) {
  CUtensorMap ta, tb;
  int rc;
  const long long ld = a->T > 1 ? a->ld_x : a->H;
  if ((rc = make_tmap_bf16(&ta, a->x, (uint64_t)a->H, (uint64_t)a->T, (uint64_t)ld * 2, BK, BM))) return rc;
  if ((rc = map_halves(&tb, a->weight, (uint64_t)a->H, (uint64_t)a->F, (uint64_t)a->H * 2, (uint64_t)a->F * a->H * 2, kBRows))) return rc;
  p.M = (int)a->T; p.N = (int)a->F; p.K = (int)a->H;
  p.m_tiles = (int)((a->T + kTileM - 1) / kTileM); p.n_tiles = (int)((a->F + kGatedN - 1) / kGatedN);
  p.m_inner = 1; p.m_group = m_group_for(a->H); p.k_splits = 1;
  p.act = a->act; p.format = a->format;
  return launch_gemm<EPI, false, false>(ta, tb, tc, p, di, st, true);
}

// Up to 128 tokens. A cluster of as many CTAs a tile (1, 2 or 4) as bring the SMs to work, while each keeps eight blocks of the
// contraction; one CTA an SM where there are no more CTAs than SMs, else two.
template <int N, int MODE>
static int gated_few_launch(const kdkl_gated_linear_args* a, const CUtensorMap& tw, const CUtensorMap& tx, FewParams p, const DeviceInfo& di,
                            cudaStream_t st) {
  auto kern = gated_few_kernel<N, MODE>;
  constexpr int kMost = 208 * 1024;
  static bool attr_set[kMaxDevices];
  if (di.dev < 0 || di.dev >= kMaxDevices || !attr_set[di.dev]) {
    KDKL_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost));
    if (di.dev >= 0 && di.dev < kMaxDevices) attr_set[di.dev] = true;
  }
  const int tiles = (int)((a->F + kFewFeatures - 1) / kFewFeatures), blocks = (int)((a->H + BK - 1) / BK);
  p.cluster = 1;
  while (p.cluster < 4 && tiles * p.cluster * 10 < di.sm_count * 9 && blocks >= 16 * p.cluster) p.cluster *= 2;
  while (p.cluster > 1 && (blocks + p.cluster - 1) / p.cluster * (p.cluster - 1) >= blocks) p.cluster /= 2;   // (nobody without a block)
  const int room = (tiles * p.cluster <= di.sm_count ? kMost : kMost / 2) - 1024;
  p.stages = room / few_stage_bytes(N);
  if (p.stages > kFewMaxStages) p.stages = kFewMaxStages;
  // (the ring is also where the sums change hands: 512 bytes a token)
  return launch_cluster(p.cluster, "gated_few_kernel", kern, dim3((unsigned)(tiles * p.cluster)), kFewThreads,
                        (size_t)p.stages * few_stage_bytes(N) + 1024, st, tw, tx, p);
}
template <int MODE>
static int gated_few(const kdkl_gated_linear_args* a, const DeviceInfo& di, cudaStream_t st) {
  const int N = a->T <= 16 ? 16 : a->T <= 32 ? 32 : a->T <= 64 ? 64 : 128;
  CUtensorMap tw, tx;
  int rc;
  if ((rc = map_halves(&tw, a->weight, (uint64_t)a->H, (uint64_t)a->F, (uint64_t)a->H * 2, (uint64_t)a->F * a->H * 2, kFewFeatures))) return rc;
  if ((rc = make_tmap_bf16(&tx, a->x, (uint64_t)a->H, (uint64_t)a->T, (uint64_t)(a->T > 1 ? a->ld_x : a->H) * 2, BK, (uint32_t)N))) return rc;
  FewParams p;
  memset(&p, 0, sizeof(p));
  p.T = (int)a->T; p.H = (int)a->H; p.F = (int)a->F; p.act = a->act; p.format = a->format;
  p.status = at<int>(a->workspace, 0);
  if (MODE == kFewBack) {
    p.dh = reinterpret_cast<const __nv_bfloat16*>(a->dh); p.ld_dh = a->ld_dh;
    p.dgate_up = reinterpret_cast<__nv_bfloat16*>(a->dgate_up);
  } else {
    p.h = reinterpret_cast<__nv_bfloat16*>(a->h); p.ld_h = a->ld_h;
  }
  if (MODE == kFewAct8) {
    p.rec_gate = record_at(a->gate_record, a->T, a->F); p.rec_up = record_at(a->up_record, a->T, a->F);
    p.rec_h = record_at(a->h_record, a->T, a->F);
  }
  if (N == 16) return gated_few_launch<16, MODE>(a, tw, tx, p, di, st);
  if (N == 32) return gated_few_launch<32, MODE>(a, tw, tx, p, di, st);
  if (N == 64) return gated_few_launch<64, MODE>(a, tw, tx, p, di, st);
  return gated_few_launch<128, MODE>(a, tw, tx, p, di, st);
}

template <int TOKENS, int U>
static int gated_rows(const kdkl_gated_linear_args* a, cudaStream_t st) {
  int rc = KDKL_OK;
  KDKL_BY_BOOL(a->act == KDKL_GATED_GELU, GELU,
    rc = launch("gated_rows_kernel", gated_rows_kernel<TOKENS, GELU ? kActGelu : kActSilu, U>,
                dim3((unsigned)((a->F + kGatedRowsWarps - 1) / kGatedRowsWarps)), 32 * kGatedRowsWarps, 0, st,
                reinterpret_cast<const __nv_bfloat16*>(a->x), a->ld_x, reinterpret_cast<const __nv_bfloat16*>(a->weight), (int)a->T,
                (int)a->H, (int)a->F, reinterpret_cast<__nv_bfloat16*>(a->h), a->ld_h, at<int>(a->workspace, 0)));
  return rc;
}

extern "C" {

size_t kdkl_gated_linear_workspace_bytes(int64_t T, int64_t H, int64_t F, int32_t dweight_type) {
  if (!shape_ok(T, H) || !shape_ok(T, F) || H % 8 || F % 8 || F >= (1ll << 29) ||
      (dweight_type != KDKL_TYPE_BF16 && dweight_type != KDKL_TYPE_F32))
    return 0;
  return gated_plan(T, H, F, dweight_type).bytes;
}

int kdkl_gated_linear_forward(const kdkl_gated_linear_args* a, void* cuda_stream) {
  g_launches = 0;
  int rc = check_gated(a);
  if (rc) return rc;
  if (a->workspace_bytes < 256) return KDKL_ERR_WORKSPACE;
  if (a->T == 0) return KDKL_OK;
  if (!a->x || !a->h) return KDKL_ERR_NULL;
  if (a->T > 1 && (a->ld_x < a->H || a->ld_h < a->F)) return KDKL_ERR_SHAPE;
  if (!rows16(a->x, a->T > 1 ? a->ld_x : 8) || !rows16(a->h, a->T > 1 ? a->ld_h : 8)) return KDKL_ERR_ALIGN;
  const bool keep = a->format != KDKL_ACT8_NONE;
  if (keep) {
    if (!a->gate_record || !a->up_record) return KDKL_ERR_NULL;
    for (const void* r : {a->gate_record, a->up_record, a->h_record})
      if (r != nullptr && (rc = check_kept(r, a->record_bytes, a->T, a->F))) return rc;
  }
  DeviceInfo di;
  if ((rc = need_b200(&di))) return rc;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  // One token, or two beside small weights, and nothing kept: without tensor cores (figures at the kernel).
  if (!keep && a->T == 1) return a->F < 24ll * di.sm_count ? gated_rows<1, 8>(a, st) : gated_rows<1, 2>(a, st);
  if (!keep && a->T == 2 && a->H * a->F <= (4ll << 20)) return gated_rows<2, 2>(a, st);
  if (a->T <= kFewTokens) return keep ? gated_few<kFewAct8>(a, di, st) : gated_few<kFewForward>(a, di, st);
  KDKL_CUDA(cudaMemsetAsync(a->workspace, 0, 256, st));
  GemmParams p;
  memset(&p, 0, sizeof(p));
  p.status = at<int>(a->workspace, 0);
  CUtensorMap tc;
  if ((rc = make_tmap_out_bf16(&tc, a->h, (uint64_t)a->F, (uint64_t)a->T, (uint64_t)(a->T > 1 ? a->ld_h : a->F)))) return rc;
  if (!keep) return gated_product<EPI_GATED>(a, p, tc, di, st);
  p.rec_gate = record_at(a->gate_record, a->T, a->F);
  p.rec_up = record_at(a->up_record, a->T, a->F);
  p.rec_h = record_at(a->h_record, a->T, a->F);
  return gated_product<EPI_GATED_ACT8>(a, p, tc, di, st);
}

int kdkl_gated_linear_backward(const kdkl_gated_linear_args* a, void* cuda_stream) {
  g_launches = 0;
  int rc = check_gated(a);
  if (rc) return rc;
  if (a->dweight_type != KDKL_TYPE_BF16 && a->dweight_type != KDKL_TYPE_F32) return KDKL_ERR_ARG;
  if (a->accumulate != 0 && a->accumulate != 1) return KDKL_ERR_ARG;
  const bool records = a->format != KDKL_ACT8_NONE;
  if ((uintptr_t)a->dweight & 15) return KDKL_ERR_ALIGN;
  const GatedPlan plan = gated_plan(a->T, a->H, a->F, a->dweight_type);
  if (a->workspace_bytes < plan.bytes) return KDKL_ERR_WORKSPACE;
  const size_t dw_bytes = (size_t)2 * a->F * a->H * type_bytes(a->dweight_type);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  DeviceInfo di;
  if (a->T == 0) {
    if ((rc = need_b200(&di))) return rc;
    KDKL_CUDA(cudaMemsetAsync(a->workspace, 0, 256, st));
    if (a->dweight && !a->accumulate) KDKL_CUDA(cudaMemsetAsync(a->dweight, 0, dw_bytes, st));
    return KDKL_OK;
  }
  if (!a->dh || !a->dgate_up || (!records && !a->x) || (records && (!a->gate_record || !a->up_record || (a->dweight && !a->x_record))))
    return KDKL_ERR_NULL;
  if (a->T > 1 && (a->ld_dh < a->F || (!records && a->ld_x < a->H))) return KDKL_ERR_SHAPE;
  if (!rows16(a->dh, a->T > 1 ? a->ld_dh : 8) || ((uintptr_t)a->dgate_up & 15) || ((uintptr_t)a->dx & 15) ||
      (!records && !rows16(a->x, a->T > 1 ? a->ld_x : 8)))
    return KDKL_ERR_ALIGN;
  if (records) {
    if ((rc = check_kept(a->gate_record, a->record_bytes, a->T, a->F)) || (rc = check_kept(a->up_record, a->record_bytes, a->T, a->F))) return rc;
    if (a->dweight && (rc = check_kept(a->x_record, a->x_record_bytes, a->T, a->H))) return rc;
  }
  if ((rc = need_b200(&di))) return rc;
  __nv_bfloat16* dgu = reinterpret_cast<__nv_bfloat16*>(a->dgate_up);
  if (records || a->T > kFewTokens) KDKL_CUDA(cudaMemsetAsync(a->workspace, 0, 256, st));   // (the kernel for few tokens does)
  if (records) {
    if ((rc = kdkl_gated_act_backward(a->gate_record, a->up_record, a->record_bytes, a->format, a->dh, a->ld_dh, KDKL_TYPE_BF16, a->T, a->F,
                                      a->act, dgu, dgu + a->F, 2 * a->F, cuda_stream)))
      return rc;
  } else if (a->T <= kFewTokens) {
    if ((rc = gated_few<kFewBack>(a, di, st))) return rc;
  } else {
    GemmParams p;
    memset(&p, 0, sizeof(p));
    p.status = at<int>(a->workspace, 0);
    p.dh = reinterpret_cast<const __nv_bfloat16*>(a->dh); p.ld_dh = a->T > 1 ? a->ld_dh : a->F;
    CUtensorMap tc;
    if ((rc = map_halves(&tc, dgu, (uint64_t)a->F, (uint64_t)a->T, (uint64_t)a->F * 4, (uint64_t)a->F * 2, 32))) return rc;
    if ((rc = gated_product<EPI_GATED_BACK>(a, p, tc, di, st))) return rc;
  }
  if (a->dweight && records) {
    const int64_t before = g_launches;
    // (it clears the status block, which the calls before it do not write; those behind it only add to it)
    if ((rc = kdkl_act8_dweight(dgu, 2 * a->F, a->x_record, a->x_record_bytes, a->T, 2 * a->F, a->H, a->format, a->dweight, a->dweight_type,
                                a->accumulate, a->workspace, a->workspace_bytes, cuda_stream)))
      return rc;
    g_launches += before;
  }
  OutGemm o;
  memset(&o, 0, sizeof(o));
  o.status = at<int>(a->workspace, 0);
  o.slab = at<float>(a->workspace, plan.at);
  if (a->dx) {
    o.a = dgu; o.lda = 2 * a->F; o.b = a->weight; o.ldb = a->H;
    o.M = a->T; o.N = a->H; o.K = 2 * a->F;
    o.out = a->dx; o.bf16 = true; o.plan = plan.dx;
    if ((rc = launch_out<false>(o, di, st))) return rc;
  }
  if (a->dweight && !records) {
    o.a = dgu; o.lda = 2 * a->F; o.b = a->x; o.ldb = a->T > 1 ? a->ld_x : a->H;
    o.M = 2 * a->F; o.N = a->H; o.K = a->T;
    o.out = a->dweight; o.bf16 = a->dweight_type == KDKL_TYPE_BF16; o.accumulate = a->accumulate; o.plan = plan.dw;
    if ((rc = launch_out<true>(o, di, st))) return rc;
  }
  return KDKL_OK;
}

}  // extern "C"
