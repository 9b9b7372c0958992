// Host helpers that the library's translation units share: the last error's text and the launch count of a thread,
// tensor-map encoding, what is known about the current device.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <stdio.h>

#include "../../include/kdkl.h"

namespace kdkl {

inline thread_local char g_err[512] = "";
inline thread_local int64_t g_launches = 0;

inline int cuda_fail(const char* what, cudaError_t e) {
  snprintf(g_err, sizeof(g_err), "%s: %s", what, cudaGetErrorString(e));
  return KDKL_ERR_CUDA;
}
#define KDKL_CUDA(call)                                   \
  do {                                                    \
    cudaError_t e__ = (call);                             \
    if (e__ != cudaSuccess) return cuda_fail(#call, e__); \
  } while (0)
#define KDKL_LAUNCHED(name)                               \
  do {                                                    \
    cudaError_t e__ = cudaGetLastError();                 \
    if (e__ != cudaSuccess) return cuda_fail(name, e__);  \
    ++g_launches;                                         \
  } while (0)

inline size_t up(size_t x, size_t a) { return (x + a - 1) / a * a; }
template <typename Tp>
inline Tp* at(void* ws, size_t off) { return reinterpret_cast<Tp*>(reinterpret_cast<uint8_t*>(ws) + off); }

// ------------------------------------------------------------------ tensor maps
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn get_encode_fn() {
  static EncodeTiledFn fn = nullptr;
  if (fn) return fn;
  void* p = nullptr;
  cudaDriverEntryPointQueryResult qres;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qres) != cudaSuccess ||
      qres != cudaDriverEntryPointSuccess)
    return nullptr;
  fn = reinterpret_cast<EncodeTiledFn>(p);
  return fn;
}

// 2-D bf16 tensor, `inner` contiguous elements per row, `outer` rows of `pitch_bytes`;
// boxes of box_inner x box_outer written to shared memory with the 128-byte swizzle unless another is given;
// out-of-bounds elements read as zero.
inline int make_tmap(CUtensorMap* m, CUtensorMapDataType dtype, const void* base, uint64_t inner, uint64_t outer,
                     uint64_t pitch_bytes, uint32_t box_inner, uint32_t box_outer,
                     CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B) {
  EncodeTiledFn fn = get_encode_fn();
  if (!fn) { snprintf(g_err, sizeof(g_err), "cuTensorMapEncodeTiled entry point not found"); return KDKL_ERR_CUDA; }
  cuuint64_t dims[2] = {inner, outer};
  cuuint64_t strides[1] = {pitch_bytes};
  cuuint32_t box[2] = {box_inner, box_outer};
  cuuint32_t estr[2] = {1, 1};
  CUresult r = fn(m, dtype, 2, const_cast<void*>(base), dims, strides, box, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    snprintf(g_err, sizeof(g_err), "cuTensorMapEncodeTiled failed (%d): inner=%llu outer=%llu pitch=%llu box=%ux%u",
             (int)r, (unsigned long long)inner, (unsigned long long)outer, (unsigned long long)pitch_bytes, box_inner,
             box_outer);
    return KDKL_ERR_CUDA;
  }
  return KDKL_OK;
}

inline int make_tmap_bf16(CUtensorMap* m, const void* base, uint64_t inner, uint64_t outer, uint64_t pitch_bytes,
                          uint32_t box_inner, uint32_t box_outer) {
  return make_tmap(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, base, inner, outer, pitch_bytes, box_inner, box_outer);
}
// Output maps: the epilogue stores boxes of 32 rows x 128 bytes (32 fp32 or 64 bf16 columns).
inline int make_tmap_out_f32(CUtensorMap* m, void* base, uint64_t cols, uint64_t rows, uint64_t ld_elems) {
  return make_tmap(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, base, cols, rows, ld_elems * 4, 32, 32);
}
inline int make_tmap_out_bf16(CUtensorMap* m, void* base, uint64_t cols, uint64_t rows, uint64_t ld_elems) {
  return make_tmap(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, base, cols, rows, ld_elems * 2, 64, 32);
}

// What the library has learnt about each device, asked once per device and process (a benign race: two
// threads asking at the same time store the same values).
constexpr int kMaxDevices = 64;
struct DeviceInfo { int dev; int sm_count; int cc_major; };
struct DeviceCache { bool known; int sm_count; int cc_major; };
inline DeviceCache g_devices[kMaxDevices];
inline int device_info(DeviceInfo* di) {
  int dev = 0;
  KDKL_CUDA(cudaGetDevice(&dev));
  di->dev = dev;
  if (dev >= 0 && dev < kMaxDevices && g_devices[dev].known) {
    di->sm_count = g_devices[dev].sm_count; di->cc_major = g_devices[dev].cc_major;
    return KDKL_OK;
  }
  KDKL_CUDA(cudaDeviceGetAttribute(&di->sm_count, cudaDevAttrMultiProcessorCount, dev));
  KDKL_CUDA(cudaDeviceGetAttribute(&di->cc_major, cudaDevAttrComputeCapabilityMajor, dev));
  if (dev >= 0 && dev < kMaxDevices) {
    g_devices[dev].sm_count = di->sm_count; g_devices[dev].cc_major = di->cc_major; g_devices[dev].known = true;
  }
  return KDKL_OK;
}

// SM count of the current device for sizing decisions that are also taken where there may be no device
// (kdkl_workspace_bytes on a build machine): a B200's 148 then.
inline int sm_count_or_default() {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return 148; }
  if (dev >= 0 && dev < kMaxDevices && g_devices[dev].known) return g_devices[dev].sm_count;
  DeviceInfo di;
  if (device_info(&di) != KDKL_OK || di.sm_count < 2) { cudaGetLastError(); return 148; }
  return di.sm_count;
}

}  // namespace kdkl
