// Host side of the label loss: argument checks, layouts and the launch schedule over chunks of tokens. Enqueue-only.
#include <math.h>
#include <string.h>

#include <type_traits>

#include "body_host.cuh"
#include "gemm_out.cuh"
#include "label_few_kernels.cuh"
#include "label_kernels.cuh"

using namespace kdkl;

// The schedule follows the KL loss (one sweep over the vocabulary a chunk, G of a chunk in bf16, two output products). A chunk
// is up to 8192 tokens by default: as much G as the KL loss keeps for the two chunks of one dW pass.
static long long label_chunk(long long T, long long chunk) {
  long long c = chunk <= 0 ? 8192 : chunk;
  if (c > T) c = T;
  if (c > 256 * MAX_LIVE_M) c = 256 * MAX_LIVE_M;          // (the sweeps' list of row tiles)
  return (long long)up((size_t)(c < 1 ? 1 : c), 256);
}

// What lives from the forward to the backward call: a few numbers a token.
struct LabelState { size_t col, counted, live, lz2, z_label, colread, losses, coefA, coefB, coefC, scale, tile_counts, total; };
static LabelState label_state(long long T) {
  LabelState s;
  size_t at = 256;
  auto take = [&](size_t bytes) { const size_t o = at; at = up(at + bytes, 256); return o; };
  s.col = take(4 * T); s.counted = take(4 * T); s.live = take((T + 255) / 256); s.lz2 = take(4 * T); s.z_label = take(4 * T);
  s.colread = take(4 * T); s.losses = take(4 * T); s.coefA = take(4 * T); s.coefB = take(4 * T); s.coefC = take(4 * T);
  s.scale = take(256);                                     // and the count of arrivals
  s.tile_counts = take(8 * ((T + 255) / 256));
  s.total = at;
  return s;
}

// What a call needs while it runs.
enum { kLabelForward = 0, kLabelBackward = 1, kLabelStep = 2 };
struct LabelLayout {
  long long C, chunks, last, Vpad, n_tiles;
  size_t part_m, part_s, part_z, G, win, slab, dw32, total;
};
static LabelLayout label_layout(long long T, long long H, long long V, long long chunk, int mode, int dw_type) {
  LabelLayout L;
  memset(&L, 0, sizeof(L));
  L.C = label_chunk(T, chunk);
  L.chunks = (T + L.C - 1) / L.C;
  L.last = T - (L.chunks - 1) * L.C;
  L.Vpad = (long long)up((size_t)V, 64);
  L.n_tiles = T <= kLabelFewTokens ? (V + kLabelFewRows - 1) / kLabelFewRows : (V + BN - 1) / BN;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at = up(at + bytes, 256); return o; };
  const bool grads = mode != kLabelForward;
  if (grads) L.G = take((size_t)L.C * L.Vpad * 2);
  const size_t shared = at;
  if (mode != kLabelBackward) {
    L.part_m = take((size_t)L.n_tiles * L.C * 4); L.part_s = take((size_t)L.n_tiles * L.C * 4); L.part_z = take((size_t)L.n_tiles * L.C * 4);
    if (grads) L.win = take((size_t)((V + 31) / 32) * L.C * 4);
  }
  if (grads) {
    const int sms = sm_count_or_default();
    size_t slab = 0;
    for (long long rows : {L.chunks > 1 ? L.C : L.last, L.last}) {
      const size_t a = out_slab_bytes(out_plan(rows, H, V, sms, false), rows, H, false);
      const size_t b = out_slab_bytes(out_plan(V, H, rows, sms, false), V, H, false);
      if (a > slab) slab = a;
      if (b > slab) slab = b;
    }
    // A chunk's products come after the last reader of its partials and maxima, and before the next chunk's sweep: their
    // parts lie in the same place (8192 x 2048 x 131072: 268 MB over 185 MB, beside a G of 2.1 GB).
    L.slab = shared;
    if (at < shared + slab) at = up(shared + slab, 256);
    // a bf16 gradient over several chunks is summed in fp32 and rounded once
    if (L.chunks > 1 && dw_type == KDKL_TYPE_BF16) L.dw32 = take((size_t)V * H * 4);
  }
  L.total = at < 256 ? 256 : at;
  return L;
}

static bool label_shape_ok(long long T, long long H, long long V) {
  return T >= 0 && T < (1ll << 31) - 256 && H >= 8 && H % 8 == 0 && H < (1ll << 30) && V >= 1 && V < (1ll << 31) - 256;
}
static int check_label(const kdkl_label_loss_args* a, int mode) {
  if (!a) return KDKL_ERR_NULL;
  if (a->struct_size != (int32_t)sizeof(kdkl_label_loss_args)) return KDKL_ERR_ARG;
  if (!label_shape_ok(a->T, a->H, a->V)) return KDKL_ERR_SHAPE;
  if (!(a->temperature > 0.f) || isinf(a->temperature) || !(a->label_smoothing >= 0.f && a->label_smoothing <= 1.f) ||
      !isfinite(a->z_loss) || a->chunk < 0)
    return KDKL_ERR_ARG;
  if ((a->label_type != 0 && a->label_type != 1) || (a->reduction != KDKL_LABEL_MEAN && a->reduction != KDKL_LABEL_SUM)) return KDKL_ERR_ARG;
  if (!a->state || !a->workspace) return KDKL_ERR_NULL;
  if (((uintptr_t)a->state & 255) || ((uintptr_t)a->workspace & 255)) return KDKL_ERR_ALIGN;
  if (a->state_bytes < label_state(a->T).total) return KDKL_ERR_WORKSPACE;
  if (((uintptr_t)a->token_weight | (uintptr_t)a->grad | (uintptr_t)a->grad_tokens | (uintptr_t)a->loss | (uintptr_t)a->losses | (uintptr_t)a->lse) & 3) return KDKL_ERR_ALIGN;
  if ((uintptr_t)a->denom_device & 7) return KDKL_ERR_ALIGN;
  if (mode != kLabelForward) {
    if ((a->dhidden_type != KDKL_TYPE_BF16 && a->dhidden_type != KDKL_TYPE_F32) || (a->dweight_type != KDKL_TYPE_BF16 && a->dweight_type != KDKL_TYPE_F32))
      return KDKL_ERR_ARG;
    if ((a->accumulate != 0 && a->accumulate != 1) || (a->accumulate && a->dweight_type != KDKL_TYPE_F32)) return KDKL_ERR_ARG;
    if (a->T > 0 && !a->dweight && !a->dhidden) return KDKL_ERR_NULL;
    if (((uintptr_t)a->dweight & 15) || ((uintptr_t)a->dhidden & 15)) return KDKL_ERR_ALIGN;
  }
  if (a->workspace_bytes < label_layout(a->T, a->H, a->V, a->chunk, mode, a->dweight_type).total) return KDKL_ERR_WORKSPACE;
  if (!a->weight || (a->T > 0 && !a->hidden)) return KDKL_ERR_NULL;
  if (((uintptr_t)a->weight & 15) || ((uintptr_t)a->hidden & 15)) return KDKL_ERR_ALIGN;
  if (mode != kLabelBackward) {
    if (!a->loss || (a->T > 0 && !a->labels)) return KDKL_ERR_NULL;
    if ((uintptr_t)a->labels % (a->label_type ? 8 : 4)) return KDKL_ERR_ALIGN;
  }
  return KDKL_OK;
}

// The sweep for up to 128 tokens: one CTA an SM, as long a ring as its shared memory holds.
template <int N, bool STORE>
static int label_few_launch(const CUtensorMap& tw, const CUtensorMap& tx, LabelFewParams p, const DeviceInfo& di, cudaStream_t st) {
  auto kern = label_few_kernel<N, STORE>;
  constexpr int kMost = 224 * 1024, kTurned = label_few_turned_bytes(N);
  static bool attr_set[kMaxDevices];
  if (di.dev < 0 || di.dev >= kMaxDevices || !attr_set[di.dev]) {
    KDKL_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost));
    if (di.dev >= 0 && di.dev < kMaxDevices) attr_set[di.dev] = true;
  }
  p.stages = (kMost - 1024 - kTurned) / label_few_stage_bytes(N);
  if (p.stages > kLabelFewMaxStages) p.stages = kLabelFewMaxStages;
  return launch("label_few_kernel", kern, dim3((unsigned)(p.tiles < di.sm_count ? p.tiles : di.sm_count)), kLabelFewThreads,
                (size_t)1024 + kTurned + (size_t)p.stages * label_few_stage_bytes(N), st, tw, tx, p);
}
template <bool STORE>
static int label_few(const kdkl_label_loss_args* a, const LabelFewParams& p, const DeviceInfo& di, cudaStream_t st) {
  const int N = p.T <= 16 ? 16 : p.T <= 32 ? 32 : p.T <= 64 ? 64 : 128;
  CUtensorMap tw, tx;
  int rc;
  if ((rc = make_tmap_bf16(&tw, a->weight, (uint64_t)p.H, (uint64_t)p.V, (uint64_t)p.H * 2, BK, kLabelFewRows))) return rc;
  if ((rc = make_tmap_bf16(&tx, a->hidden, (uint64_t)p.H, (uint64_t)p.T, (uint64_t)p.H * 2, BK, (uint32_t)N))) return rc;
  if (N == 16) return label_few_launch<16, STORE>(tw, tx, p, di, st);
  if (N == 32) return label_few_launch<32, STORE>(tw, tx, p, di, st);
  if (N == 64) return label_few_launch<64, STORE>(tw, tx, p, di, st);
  return label_few_launch<128, STORE>(tw, tx, p, di, st);
}

static int label_run(const kdkl_label_loss_args* a, int mode, void* cuda_stream) {
  g_launches = 0;
  int rc = check_label(a, mode);
  if (rc) return rc;
  DeviceInfo di;
  if ((rc = device_info(&di))) return rc;
  if (di.cc_major != 10) return KDKL_ERR_ARCH;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const long long T = a->T, H = a->H, V = a->V;
  const LabelState S = label_state(T);
  const LabelLayout L = label_layout(T, H, V, a->chunk, mode, a->dweight_type);
  const bool sweep = mode != kLabelBackward, grads = mode != kLabelForward;
  LabelParams p;
  memset(&p, 0, sizeof(p));
  p.tau = a->temperature; p.smoothing = a->label_smoothing; p.z_loss = a->z_loss;
  p.T = (int)T; p.H = (int)H; p.V = (int)V; p.chunk = L.C;
  p.mean = a->reduction == KDKL_LABEL_MEAN; p.denom_device = a->denom_device;
  p.token_weight = a->token_weight; p.grad = a->grad; p.grad_tokens = mode == kLabelBackward ? a->grad_tokens : nullptr;
  p.hdr = at<WsHeader>(a->state, 0);
  p.col = at<int>(a->state, S.col); p.counted = at<int>(a->state, S.counted);
  p.lz2 = at<float>(a->state, S.lz2); p.z_label = at<float>(a->state, S.z_label); p.losses = at<float>(a->state, S.losses);
  p.coefA = at<float>(a->state, S.coefA); p.coefB = at<float>(a->state, S.coefB); p.coefC = at<float>(a->state, S.coefC);
  p.scale = at<float>(a->state, S.scale); p.arrivals = at<int>(a->state, S.scale + 128); p.tile_counts = at<int>(a->state, S.tile_counts);
  uint8_t* live = at<uint8_t>(a->state, S.live);
  if (T == 0) {
    if (sweep) KDKL_CUDA(cudaMemsetAsync(a->state, 0, 256, st));
    if (sweep) KDKL_CUDA(cudaMemsetAsync(a->loss, 0, 4, st));
    if (grads && a->dweight && !a->accumulate) KDKL_CUDA(cudaMemsetAsync(a->dweight, 0, (size_t)V * H * (a->dweight_type == KDKL_TYPE_F32 ? 4 : 2), st));
    return KDKL_OK;
  }
  const unsigned by256 = (unsigned)((T + 255) / 256);
  if (sweep) {
    rc = a->label_type == 1 ? launch("label_prep_kernel", label_prep_kernel<long long>, dim3(by256), 256, 0, st, p,
                                     reinterpret_cast<const long long*>(a->labels), a->ignore_index, live)
                            : launch("label_prep_kernel", label_prep_kernel<int>, dim3(by256), 256, 0, st, p,
                                     reinterpret_cast<const int*>(a->labels), a->ignore_index, live);
  } else {
    rc = launch("label_coef_kernel", label_coef_kernel, dim3(by256), 256, 0, st, p);
  }
  if (rc) return rc;
  const int* go = sweep ? nullptr : &p.hdr->go;
  uint16_t* G = grads ? at<uint16_t>(a->workspace, L.G) : nullptr;
  // The sweep's tiles: 256 rows on a pair of SMs, or 128 rows on one where that makes fewer waves (few tokens).
  const long long pairs = di.sm_count / 2, most_rows = L.chunks > 1 ? L.C : L.last, tiles = (V + BN - 1) / BN;
  const bool single = sweep && ((most_rows + BM - 1) / BM * tiles + di.sm_count - 1) / di.sm_count <
                               ((most_rows + kTileM - 1) / kTileM * tiles + pairs - 1) / pairs;
  CUtensorMap tmW, tmH, tmG;
  if ((rc = make_tmap_bf16(&tmW, a->weight, (uint64_t)H, (uint64_t)V, (uint64_t)H * 2, BK, single ? GemmCfg<1>::B_ROWS : kBRows))) return rc;
  for (long long ci = 0; ci < L.chunks; ++ci) {
    const long long s0 = ci * L.C, rows = ci + 1 < L.chunks ? L.C : L.last;
    const __nv_bfloat16* hidden = reinterpret_cast<const __nv_bfloat16*>(a->hidden) + s0 * H;
    const uint8_t* flags = live + s0 / 256;
    if ((rc = make_tmap_bf16(&tmH, hidden, (uint64_t)H, (uint64_t)rows, (uint64_t)H * 2, BK, BM))) return rc;
    tmG = tmH;                                             // (no output in the forward sweep)
    if (grads && (rc = make_tmap_out_bf16(&tmG, G, (uint64_t)V, (uint64_t)rows, (uint64_t)L.Vpad))) return rc;
    GemmParams g;
    memset(&g, 0, sizeof(g));
    g.M = (int)rows; g.N = (int)V; g.K = (int)H;
    g.m_tiles = (int)((rows + kTileM - 1) / kTileM); g.n_tiles = (int)tiles; g.m_inner = 1; g.m_group = m_group_for(H); g.k_splits = 1;
    g.m_live = flags;
    g.status = &p.hdr->status; g.go = go;
    g.scale_log2 = kLog2e / p.tau; g.Ktop = 1;
    g.idx_sorted = p.col + s0; g.nvalid = p.counted + s0;
    g.zg = p.z_label + s0; g.colread = at<int>(a->state, S.colread) + s0;
    g.lz2 = p.lz2 + s0; g.coefA = p.coefA + s0; g.coefB = p.coefB + s0; g.coefC = p.coefC + s0;
    g.row_base = s0;
    if (sweep) {
      g.part_m = at<float>(a->workspace, L.part_m); g.part_s = at<float>(a->workspace, L.part_s); g.part_z = at<float>(a->workspace, L.part_z);
      g.part_stride = L.C;
      if (grads) g.win_max = at<float>(a->workspace, L.win);
      if (T <= kLabelFewTokens) {
        LabelFewParams q;
        memset(&q, 0, sizeof(q));
        q.T = (int)T; q.H = (int)H; q.V = (int)V; q.tiles = (int)L.n_tiles; q.scale_log2 = g.scale_log2; q.col = p.col;
        q.part_m = g.part_m; q.part_s = g.part_s; q.part_z = g.part_z; q.stride = L.C; q.z_label = p.z_label;
        q.E = G; q.ld_e = L.Vpad; q.win_max = g.win_max; q.status = &p.hdr->status;
        rc = grads ? label_few<true>(a, q, di, st) : label_few<false>(a, q, di, st);
      } else if (single) {
        g.m_tiles = (int)((rows + BM - 1) / BM); g.m_group *= 2; g.m_live = nullptr;
        rc = grads ? launch_gemm<EPI_LABEL_E, false, false, false, 1>(tmH, tmW, tmG, g, di, st, true) : launch_gemm<EPI_LSE_SUM, false, false, false, 1>(tmH, tmW, tmG, g, di, st, true);
      } else {
        rc = grads ? launch_gemm<EPI_LABEL_E, false, false>(tmH, tmW, tmG, g, di, st, true) : launch_gemm<EPI_LSE_SUM, false, false>(tmH, tmW, tmG, g, di, st, true);
      }
      if (rc) return rc;
      if ((rc = launch("label_combine_kernel", label_combine_kernel, dim3((unsigned)((rows + 31) / 32)), 1024, 0, st, p, (const float*)g.part_m,
                       (const float*)g.part_s, (const float*)g.part_z, L.C, (int)L.n_tiles, (int)rows, s0, grads ? 1 : 0, ci + 1 == L.chunks ? 1 : 0,
                       a->losses, a->lse, a->loss)))
        return rc;
      if (grads) {
        const dim3 grid((unsigned)((V + kLabelGCols - 1) / kLabelGCols), (unsigned)((rows + kLabelGRows - 1) / kLabelGRows));
        if ((rc = launch("label_g_kernel", label_g_kernel, grid, 256, 0, st, p, G, L.Vpad, (const float*)g.win_max, L.C, (int)rows, s0))) return rc;
      }
    } else if ((rc = launch_gemm<EPI_LABEL_G, false, false>(tmH, tmW, tmG, g, di, st, true))) {
      return rc;
    }
    if (!grads) continue;
    OutGemm o;
    memset(&o, 0, sizeof(o));
    o.status = &p.hdr->status; o.go = go; o.slab = at<float>(a->workspace, L.slab); o.scale = p.scale;
    o.a = G; o.lda = L.Vpad; o.b = a->weight; o.ldb = H;
    o.M = rows; o.N = H; o.K = V;
    o.bf16 = a->dhidden_type == KDKL_TYPE_BF16;
    o.out = at<uint8_t>(a->dhidden, (size_t)s0 * H * (o.bf16 ? 2 : 4));
    o.plan = out_plan(rows, H, V, sm_count_or_default(), false);
    o.m_live = g.m_live;                                   // dead row tiles: zeros
    if (a->dhidden && (rc = launch_out<false>(o, di, st))) return rc;
    if (!a->dweight) continue;
    o.a = G; o.b = hidden;
    o.M = V; o.N = H; o.K = rows;
    o.m_live = nullptr;
    o.k_live = rows <= 32 * kTileM && (rows + BK - 1) / BK <= MAX_LIVE_KB ? flags : nullptr;
    o.plan = out_plan(V, H, rows, sm_count_or_default(), false);
    o.bf16 = a->dweight_type == KDKL_TYPE_BF16 && L.chunks == 1;
    o.out = a->dweight_type == KDKL_TYPE_BF16 && L.chunks > 1 ? at<void>(a->workspace, L.dw32) : a->dweight;
    o.accumulate = ci > 0 || a->accumulate ? 1 : 0;
    if ((rc = launch_out<true>(o, di, st))) return rc;
  }
  if (grads && a->dweight && a->dweight_type == KDKL_TYPE_BF16 && L.chunks > 1) {
    const long long n4 = V * H / 4;
    if ((rc = launch("label_round_kernel", label_round_kernel, dim3((unsigned)((n4 + 255) / 256)), 256, 0, st,
                     (const float*)at<float>(a->workspace, L.dw32), reinterpret_cast<uint2*>(a->dweight), n4, go)))
      return rc;
  }
  return KDKL_OK;
}

extern "C" {

size_t kdkl_label_loss_state_bytes(int64_t T) { return T < 0 || T >= (1ll << 31) - 256 ? 0 : label_state(T).total; }
size_t kdkl_label_loss_workspace_bytes(int64_t T, int64_t H, int64_t V, int64_t chunk, int32_t call, int32_t dweight_type) {
  if (!label_shape_ok(T, H, V) || chunk < 0 || call < KDKL_LABEL_FORWARD || call > KDKL_LABEL_STEP ||
      (dweight_type != KDKL_TYPE_BF16 && dweight_type != KDKL_TYPE_F32))
    return 0;
  return label_layout(T, H, V, chunk, call, dweight_type).total;
}
int kdkl_label_loss_forward(const kdkl_label_loss_args* a, void* cuda_stream) { return label_run(a, kLabelForward, cuda_stream); }
int kdkl_label_loss_backward(const kdkl_label_loss_args* a, void* cuda_stream) { return label_run(a, kLabelBackward, cuda_stream); }
int kdkl_label_loss_step(const kdkl_label_loss_args* a, void* cuda_stream) { return label_run(a, kLabelStep, cuda_stream); }
int kdkl_label_loss_rescale(const void* gradient, int32_t type, int64_t count, const float* factor, void* out, void* cuda_stream) {
  g_launches = 0;
  if (type != KDKL_TYPE_BF16 && type != KDKL_TYPE_F32) return KDKL_ERR_ARG;
  const long long words = count / (type == KDKL_TYPE_F32 ? 4 : 8);
  if (count < 0 || count % 8 || words >= (1ll << 38)) return KDKL_ERR_SHAPE;
  if (!factor || (count > 0 && (!gradient || !out))) return KDKL_ERR_NULL;
  if (((uintptr_t)gradient & 15) || ((uintptr_t)out & 15) || ((uintptr_t)factor & 3)) return KDKL_ERR_ALIGN;
  if (count == 0) return KDKL_OK;
  DeviceInfo di;
  int rc = need_b200(&di);
  if (rc) return rc;
  KDKL_BY_BOOL(type == KDKL_TYPE_F32, F32,
    rc = launch("label_rescale_kernel", label_rescale_kernel<std::conditional_t<F32, float, __nv_bfloat16>>, dim3((unsigned)((words + 255) / 256)), 256,
                0, reinterpret_cast<cudaStream_t>(cuda_stream), reinterpret_cast<const uint4*>(gradient), factor, reinterpret_cast<uint4*>(out), words));
  return rc;
}

}  // extern "C"
