// Host side of the operators of a student's body: 8-bit activation records, gated activation, weight gradient from
// a record. Argument checks and launches; enqueue-only.
#include <math.h>
#include <string.h>

#include "act8.cuh"
#include "act8_dweight.cuh"
#include "gated_kernels.cuh"
#include "body_host.cuh"

using namespace kdkl;

extern "C" {

// ------------------------------------------------------------------ records
size_t kdkl_act8_bytes(int64_t T, int64_t H) {
  if (!shape_ok(T, H)) return 0;
  return up(record_need(T, H), 256);
}

static int check_record(const void* record, size_t bytes, int64_t T, int64_t H, int32_t format) {
  if (!shape_ok(T, H)) return KDKL_ERR_SHAPE;
  if (!is_format(format)) return KDKL_ERR_ARG;
  if ((uintptr_t)record & 255) return KDKL_ERR_ALIGN;
  if (bytes < record_need(T, H)) return KDKL_ERR_WORKSPACE;
  return KDKL_OK;
}

int kdkl_act8_store(const void* x, int32_t type, int64_t ld, int64_t T, int64_t H, int32_t format, void* record,
                    size_t record_bytes, void* cuda_stream) {
  g_launches = 0;
  if (T != 0 && (!x || !record)) return KDKL_ERR_NULL;
  if (!is_type(type)) return KDKL_ERR_ARG;
  int rc = check_record(record, record_bytes, T, H, format);
  if (rc) return rc;
  if (T > 1 && ld < H) return KDKL_ERR_SHAPE;
  if ((uintptr_t)x % type_bytes(type)) return KDKL_ERR_ALIGN;
  if (T == 0) return KDKL_OK;
  DeviceInfo di;
  if ((rc = need_b200(&di))) return rc;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const RowsShape shape = rows_shape(T, H, di, 128);
  const ActRecord rec = record_at(record, T, H);
  KDKL_BY_TYPE(type, E, KDKL_BY_FORMAT(format, FMT, KDKL_BY_BOOL(words(x, ld, T, H, type), VEC,
    rc = (launch("act8_store_kernel", act8_store_kernel<E, FMT, VEC>, shape.grid, shape.threads, 0, st, reinterpret_cast<const E*>(x), ld, T, (int)H, rec)))));
  return rc;
}

int kdkl_act8_load(const void* record, size_t record_bytes, int64_t T, int64_t H, int32_t format, void* out,
                   int32_t type, int64_t ld, void* cuda_stream) {
  g_launches = 0;
  if (T != 0 && (!out || !record)) return KDKL_ERR_NULL;
  if (!is_type(type)) return KDKL_ERR_ARG;
  int rc = check_record(record, record_bytes, T, H, format);
  if (rc) return rc;
  if (T > 1 && ld < H) return KDKL_ERR_SHAPE;
  if ((uintptr_t)out % type_bytes(type)) return KDKL_ERR_ALIGN;
  if (T == 0) return KDKL_OK;
  DeviceInfo di;
  if ((rc = need_b200(&di))) return rc;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const RowsShape shape = rows_shape(T, H, di, 64);
  const ActRecord rec = record_at(record, T, H);
  KDKL_BY_TYPE(type, E, KDKL_BY_FORMAT(format, FMT, KDKL_BY_BOOL(words(out, ld, T, H, type), VEC,
    rc = (launch("act8_load_kernel", act8_load_kernel<E, FMT, VEC>, shape.grid, shape.threads, 0, st, rec, T, (int)H, reinterpret_cast<E*>(out), ld)))));
  return rc;
}

// ------------------------------------------------------------------ gated activation
int kdkl_gated_act_forward(const void* gate, const void* up_, int64_t ld, int32_t type, int64_t T, int64_t F,
                           int32_t act, int32_t format, void* h, int64_t ld_h, void* gate_record, void* up_record,
                           void* h_record, size_t record_bytes, void* cuda_stream) {
  g_launches = 0;
  if (!shape_ok(T, F)) return KDKL_ERR_SHAPE;
  if (type != KDKL_TYPE_BF16 && type != KDKL_TYPE_F16) return KDKL_ERR_ARG;
  if (act != KDKL_GATED_SILU && act != KDKL_GATED_GELU) return KDKL_ERR_ARG;
  if (T != 0 && (!gate || !up_ || !h)) return KDKL_ERR_NULL;
  int rc;
  if (format != KDKL_ACT8_NONE) {
    if (T != 0 && (!gate_record || !up_record)) return KDKL_ERR_NULL;
    if ((rc = check_record(gate_record, record_bytes, T, F, format))) return rc;
    if (((uintptr_t)up_record & 255) || ((uintptr_t)h_record & 255)) return KDKL_ERR_ALIGN;
  }
  if (T > 1 && (ld < F || ld_h < F)) return KDKL_ERR_SHAPE;
  if (((uintptr_t)gate | (uintptr_t)up_ | (uintptr_t)h) & 1) return KDKL_ERR_ALIGN;
  if (T == 0) return KDKL_OK;
  DeviceInfo di;
  if ((rc = need_b200(&di))) return rc;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const RowsShape shape = rows_shape(T, F, di, 128);
  const bool vec = words(gate, ld, T, F, type) && words(up_, ld, T, F, type) && words(h, ld_h, T, F, type);
  KDKL_BY_TYPE16(type, E, KDKL_BY_BOOL(act == KDKL_GATED_GELU, GELU, KDKL_BY_FORMAT_OR_NONE(format, FMT, KDKL_BY_BOOL(vec, VEC,
    rc = (launch("gated_forward_kernel", gated_forward_kernel<E, GELU ? kActGelu : kActSilu, FMT, VEC>, shape.grid, shape.threads, 0, st,
        reinterpret_cast<const E*>(gate), reinterpret_cast<const E*>(up_), ld, T, (int)F, reinterpret_cast<E*>(h), ld_h,
        record_at(gate_record, T, F), record_at(up_record, T, F), record_at(h_record, T, F)))))));
  return rc;
}

int kdkl_gated_act_backward(const void* gate_record, const void* up_record, size_t record_bytes, int32_t format,
                            const void* dh, int64_t ld_dh, int32_t type, int64_t T, int64_t F, int32_t act,
                            void* dgate, void* dup, int64_t ld, void* cuda_stream) {
  g_launches = 0;
  if (type != KDKL_TYPE_BF16 && type != KDKL_TYPE_F16) return KDKL_ERR_ARG;
  if (act != KDKL_GATED_SILU && act != KDKL_GATED_GELU) return KDKL_ERR_ARG;
  if (T != 0 && (!gate_record || !up_record || !dh || !dgate || !dup)) return KDKL_ERR_NULL;
  int rc = check_record(gate_record, record_bytes, T, F, format);
  if (rc) return rc;
  if ((uintptr_t)up_record & 255) return KDKL_ERR_ALIGN;
  if (T > 1 && (ld < F || ld_dh < F)) return KDKL_ERR_SHAPE;
  if (((uintptr_t)dh | (uintptr_t)dgate | (uintptr_t)dup) & 1) return KDKL_ERR_ALIGN;
  if (T == 0) return KDKL_OK;
  DeviceInfo di;
  if ((rc = need_b200(&di))) return rc;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const RowsShape shape = rows_shape(T, F, di, 128);
  const bool vec = words(dh, ld_dh, T, F, type) && words(dgate, ld, T, F, type) && words(dup, ld, T, F, type);
  KDKL_BY_TYPE16(type, E, KDKL_BY_BOOL(act == KDKL_GATED_GELU, GELU, KDKL_BY_FORMAT(format, FMT, KDKL_BY_BOOL(vec, VEC,
    rc = (launch("gated_backward_kernel", gated_backward_kernel<E, GELU ? kActGelu : kActSilu, FMT, VEC>, shape.grid, shape.threads, 0, st,
        record_at(gate_record, T, F), record_at(up_record, T, F), reinterpret_cast<const E*>(dh), ld_dh, T, (int)F,
        reinterpret_cast<E*>(dgate), reinterpret_cast<E*>(dup), ld))))));
  return rc;
}

// ------------------------------------------------------------------ weight gradient from a record
// Rows that tensor maps can describe (16 bytes apart): the tensor-core kernel. Others: the FMA kernel.
static bool dw_mapped(const void* dy, long long ld_dy, long long T, long long N, long long H, const void* out, int type) {
  return words(dy, ld_dy, T, N, KDKL_TYPE_BF16) && words(out, H, N, H, type);
}
// Which tiles are cut, and into how many parts of the contraction: the choice with the least estimated cycles. A block
// of 64 tokens takes a unit 600 cycles, starting a unit and draining its tile about five blocks; the slabs of cut tiles
// one more launch, and being written and read once at about 2600 bytes a cycle. (600 is what the long loop takes; the other
// figures and the bound of 16 parts are estimates. With one or two tiles in all, 16 parts leave most pairs idle:
// 32768 x 256 x 256 takes 24 us, its bytes 4.)
struct DwPlan { int whole, rest, parts; };
static DwPlan dw_plan(long long T, long long N, long long H) {
  const long long tiles = ((N + 255) / 256) * ((H + 255) / 256), kb = (T + 63) / 64;
  const long long pairs = sm_count_or_default() / 2;
  DwPlan best = {(int)tiles, 0, 1};
  double least = (double)((tiles + pairs - 1) / pairs) * (kb + 5) * 600.0;
  const long long rest = tiles % pairs;                    // what whole waves leave over
  for (int parts = 2; rest != 0 && parts <= 16 && kb / parts >= 8; ++parts) {
    const long long waves = (rest * parts + pairs - 1) / pairs;
    const double cost = (double)((tiles / pairs) * (kb + 5) + waves * ((kb + parts - 1) / parts + 5)) * 600.0 + 6000.0 +
                        (double)rest * 65536.0 * (8.0 * parts + 4.0) / 2600.0;
    if (cost < least) { least = cost; best = DwPlan{(int)(tiles - rest), (int)rest, parts}; }
  }
  return best;
}

size_t kdkl_act8_dweight_workspace_bytes(int64_t T, int64_t N, int64_t H, int32_t type) {
  if (!shape_ok(T, H) || !shape_ok(T, N) || (type != KDKL_TYPE_BF16 && type != KDKL_TYPE_F32)) return 0;
  const DwPlan plan = dw_plan(T, N, H);
  return 256 + (size_t)plan.rest * plan.parts * 65536 * 4;
}

}  // extern "C"

template <int FMT, bool F32_OUT>
static int launch_dweight(const CUtensorMap& ty, const CUtensorMap& tc, const CUtensorMap& ts, const CUtensorMap& to,
                          const CUtensorMap& tslab, const DwParams& p, const DeviceInfo& di, cudaStream_t st) {
  auto kern = act8_dweight_kernel<FMT, F32_OUT>;
  static bool attr_set[kMaxDevices];
  if (di.dev < 0 || di.dev >= kMaxDevices || !attr_set[di.dev]) {
    KDKL_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, DwCfg::SMEM_BYTES));
    if (di.dev >= 0 && di.dev < kMaxDevices) attr_set[di.dev] = true;
  }
  const int units = p.whole + p.rest * p.parts, most = di.sm_count / 2;
  return launch("act8_dweight_kernel", kern, dim3(2 * (units < most ? units : most), 1, 1), DwCfg::THREADS,
                DwCfg::SMEM_BYTES, st, ty, tc, ts, to, tslab, p);
}

extern "C" {

int kdkl_act8_dweight(const void* dy, int64_t ld_dy, const void* record, size_t record_bytes, int64_t T, int64_t N,
                      int64_t H, int32_t format, void* dweight, int32_t type, int32_t accumulate, void* workspace,
                      size_t workspace_bytes, void* cuda_stream) {
  g_launches = 0;
  if (!dweight || !workspace || (T != 0 && (!dy || !record))) return KDKL_ERR_NULL;
  if (!shape_ok(T, N)) return KDKL_ERR_SHAPE;
  if (type != KDKL_TYPE_BF16 && type != KDKL_TYPE_F32) return KDKL_ERR_ARG;
  if (accumulate != 0 && accumulate != 1) return KDKL_ERR_ARG;
  int rc = check_record(record, record_bytes, T, H, format);
  if (rc) return rc;
  if (T > 1 && ld_dy < N) return KDKL_ERR_SHAPE;
  if (((uintptr_t)dy & 1) || ((uintptr_t)dweight % type_bytes(type)) || ((uintptr_t)workspace & 255)) return KDKL_ERR_ALIGN;
  if (workspace_bytes < kdkl_act8_dweight_workspace_bytes(T, N, H, type)) return KDKL_ERR_WORKSPACE;
  DeviceInfo di;
  if ((rc = need_b200(&di))) return rc;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const ActRecord rec = record_at(record, T, H);
  int* status = at<int>(workspace, 0);
  if (T == 0 || !dw_mapped(dy, ld_dy, T, N, H, dweight, type)) {
    DweightParams p;
    p.dy = reinterpret_cast<const __nv_bfloat16*>(dy); p.ld_dy = ld_dy;
    p.rec = rec;
    p.T = T; p.N = (int)N; p.H = (int)H;
    p.out = dweight; p.type = type; p.accumulate = accumulate;
    p.status = status;
    const dim3 grid((unsigned)((H + 63) / 64), (unsigned)((N + 63) / 64), 1);
    if (grid.y > 65535) return KDKL_ERR_SHAPE;
    KDKL_BY_FORMAT(format, FMT, rc = (launch("act8_dweight_simple_kernel", act8_dweight_simple_kernel<FMT>, grid, 256, 0, st, p)));
    return rc;
  }
  const DwPlan plan = dw_plan(T, N, H);
  float* slab = at<float>(workspace, 256);
  CUtensorMap ty, tc, ts, to, tslab;
  const long long ld = T > 1 ? ld_dy : N;
  if ((rc = make_tmap_bf16(&ty, dy, (uint64_t)N, (uint64_t)T, (uint64_t)ld * 2, 64, DwCfg::BK))) return rc;
  if ((rc = make_tmap(&tc, CU_TENSOR_MAP_DATA_TYPE_UINT8, rec.codes, (uint64_t)act_codes_pitch(H), (uint64_t)T,
                      (uint64_t)act_codes_pitch(H), 128, DwCfg::RAW_T, CU_TENSOR_MAP_SWIZZLE_NONE)))
    return rc;
  if ((rc = make_tmap(&ts, CU_TENSOR_MAP_DATA_TYPE_UINT8, rec.scales, (uint64_t)act_scale_pitch(H), (uint64_t)T,
                      (uint64_t)act_scale_pitch(H), 16, DwCfg::RAW_T, CU_TENSOR_MAP_SWIZZLE_NONE)))
    return rc;
  if (type == KDKL_TYPE_F32) rc = make_tmap_out_f32(&to, dweight, (uint64_t)H, (uint64_t)N, (uint64_t)H);
  else rc = make_tmap_out_bf16(&to, dweight, (uint64_t)H, (uint64_t)N, (uint64_t)H);
  if (rc) return rc;
  tslab = to;
  if (plan.rest > 0 && (rc = make_tmap_out_f32(&tslab, slab, 256, (uint64_t)plan.rest * plan.parts * 256, 256))) return rc;
  DwParams p;
  p.T = T; p.N = (int)N; p.H = (int)H;
  p.h_tiles = (int)((H + 255) / 256);
  p.whole = plan.whole; p.rest = plan.rest; p.parts = plan.parts;
  p.accumulate = accumulate;
  p.out = reinterpret_cast<const __nv_bfloat16*>(dweight);
  p.status = status;
  KDKL_BY_FORMAT(format, FMT, KDKL_BY_BOOL(type == KDKL_TYPE_F32, F32_OUT,
    rc = (launch_dweight<FMT, F32_OUT>(ty, tc, ts, to, tslab, p, di, st))));
  if (rc || plan.rest == 0) return rc;
  return launch("act8_dweight_join_kernel", act8_dweight_join_kernel, dim3((unsigned)plan.rest * 32, 1, 1), 256, 0, st, slab,
                plan.whole, plan.parts, p.h_tiles, N, H, dweight, type, accumulate);
}

}  // extern "C"
