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
  const ActRecord rec = record_at(record, T, H);
  KDKL_BY_TYPE(type, E, KDKL_BY_FORMAT(format, FMT, KDKL_BY_BOOL(words(x, ld, T, H, type), VEC,
    (act8_store_kernel<E, FMT, VEC><<<rows_grid(T, H, di), 256, 0, st>>>(reinterpret_cast<const E*>(x), ld, T, (int)H, rec)))));
  KDKL_LAUNCHED("act8_store_kernel");
  return KDKL_OK;
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
  const ActRecord rec = record_at(record, T, H);
  KDKL_BY_TYPE(type, E, KDKL_BY_FORMAT(format, FMT, KDKL_BY_BOOL(words(out, ld, T, H, type), VEC,
    (act8_load_kernel<E, FMT, VEC><<<rows_grid(T, H, di), 256, 0, st>>>(rec, T, (int)H, reinterpret_cast<E*>(out), ld)))));
  KDKL_LAUNCHED("act8_load_kernel");
  return KDKL_OK;
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
  const bool vec = words(gate, ld, T, F, type) && words(up_, ld, T, F, type) && words(h, ld_h, T, F, type);
  KDKL_BY_TYPE16(type, E, KDKL_BY_BOOL(act == KDKL_GATED_GELU, GELU, KDKL_BY_FORMAT_OR_NONE(format, FMT, KDKL_BY_BOOL(vec, VEC,
    (gated_forward_kernel<E, GELU ? kActGelu : kActSilu, FMT, VEC><<<rows_grid(T, F, di), 256, 0, st>>>(
        reinterpret_cast<const E*>(gate), reinterpret_cast<const E*>(up_), ld, T, (int)F, reinterpret_cast<E*>(h), ld_h,
        record_at(gate_record, T, F), record_at(up_record, T, F), record_at(h_record, T, F)))))));
  KDKL_LAUNCHED("gated_forward_kernel");
  return KDKL_OK;
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
  const bool vec = words(dh, ld_dh, T, F, type) && words(dgate, ld, T, F, type) && words(dup, ld, T, F, type);
  KDKL_BY_TYPE16(type, E, KDKL_BY_BOOL(act == KDKL_GATED_GELU, GELU, KDKL_BY_FORMAT(format, FMT, KDKL_BY_BOOL(vec, VEC,
    (gated_backward_kernel<E, GELU ? kActGelu : kActSilu, FMT, VEC><<<rows_grid(T, F, di), 256, 0, st>>>(
        record_at(gate_record, T, F), record_at(up_record, T, F), reinterpret_cast<const E*>(dh), ld_dh, T, (int)F,
        reinterpret_cast<E*>(dgate), reinterpret_cast<E*>(dup), ld))))));
  KDKL_LAUNCHED("gated_backward_kernel");
  return KDKL_OK;
}

// ------------------------------------------------------------------ weight gradient from a record
size_t kdkl_act8_dweight_workspace_bytes(int64_t T, int64_t N, int64_t H, int32_t type) {
  if (!shape_ok(T, H) || !shape_ok(T, N) || (type != KDKL_TYPE_BF16 && type != KDKL_TYPE_F32)) return 0;
  return 256;
}

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
  KDKL_CUDA(cudaMemsetAsync(workspace, 0, 256, st));
  DweightParams p;
  p.dy = reinterpret_cast<const __nv_bfloat16*>(dy); p.ld_dy = ld_dy;
  p.rec = record_at(record, T, H);
  p.T = T; p.N = (int)N; p.H = (int)H;
  p.out = dweight; p.type = type; p.accumulate = accumulate;
  const dim3 grid((unsigned)((H + 63) / 64), (unsigned)((N + 63) / 64), 1);
  if (grid.y > 65535) return KDKL_ERR_SHAPE;
  KDKL_BY_FORMAT(format, FMT, (act8_dweight_simple_kernel<FMT><<<grid, 256, 0, st>>>(p)));
  KDKL_LAUNCHED("act8_dweight_simple_kernel");
  return KDKL_OK;
}

}  // extern "C"
