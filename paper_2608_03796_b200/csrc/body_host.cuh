// Argument checks and dispatch that the host sides of the student-body operators share.
#pragma once
#include <string.h>

#include "act8.cuh"
#include "host_common.cuh"

namespace kdkl {

inline bool is_type(int type) { return type >= KDKL_TYPE_BF16 && type <= KDKL_TYPE_F16; }
inline bool is_format(int f) { return f == KDKL_ACT8_INT8 || f == KDKL_ACT8_E4M3; }
inline int type_bytes(int type) { return type == KDKL_TYPE_F32 ? 4 : 2; }
inline size_t record_need(long long T, long long H) {
  return (size_t)(act_scales_at(T, H) + T * act_scale_pitch(H));
}
inline ActRecord record_at(const void* record, long long T, long long H) {
  ActRecord r;
  r.codes = reinterpret_cast<uint8_t*>(const_cast<void*>(record));
  r.scales = record == nullptr ? nullptr : r.codes + act_scales_at(T, H);
  return r;
}
// Rows whose groups of eight values are aligned words (16 bytes, 32 of fp32): start, distance and width.
inline bool words(const void* p, long long ld, long long T, long long H, int type) {
  const int word = 8 * type_bytes(type);
  return (uintptr_t)p % word == 0 && (T <= 1 || (ld * type_bytes(type)) % word == 0) && H % 8 == 0;
}
inline bool shape_ok(long long T, long long H) {
  return T >= 0 && T <= 0x7fffff00ll && H >= 1 && H < (1ll << 30);
}
inline int need_b200(DeviceInfo* di) {
  int rc = device_info(di);
  if (rc) return rc;
  return di->cc_major == 10 ? KDKL_OK : KDKL_ERR_ARCH;
}
// Launch shape of the element-wise kernels: the columns in even shares of at most 2048 a block; in y as many rows as make
// `per_sm` blocks an SM.
struct RowsShape { dim3 grid; int threads; };
inline RowsShape rows_shape(long long T, long long H, const DeviceInfo& di, int per_sm) {
  const long long groups = act_codes_pitch(H) / 8, gx = (groups + 255) / 256;
  long long gy = ((long long)di.sm_count * per_sm + gx - 1) / gx;
  if (gy > T) gy = T;
  if (gy > 65535) gy = 65535;
  RowsShape r;
  r.threads = (int)(((groups + gx - 1) / gx + 31) / 32 * 32);
  r.grid = dim3((unsigned)gx, (unsigned)gy, 1);
  return r;
}

// A launch that may start while the kernel before it on the stream drains (every kernel launched so begins with
// grid_dependency_wait). Measured on one B200: 1 to 2 us less between kernels of 5 to 15 us.
template <typename... P, typename... Q>
inline int launch_cluster(int cluster, const char* name, void (*kern)(P...), dim3 grid, int threads, size_t smem,
                          cudaStream_t st, const Q&... args) {
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  cudaError_t e = cudaLaunchKernelEx(&cfg, kern, P(args)...);
  if (e != cudaSuccess) return cuda_fail(name, e);
  ++g_launches;
  return KDKL_OK;
}
template <typename... P, typename... Q>
inline int launch(const char* name, void (*kern)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, const Q&... args) {
  return launch_cluster(1, name, kern, grid, threads, smem, st, args...);
}

#define KDKL_BY_BOOL(cond, NAME, ...)                                  \
  do {                                                                 \
    if (cond) { constexpr bool NAME = true; __VA_ARGS__; }             \
    else { constexpr bool NAME = false; __VA_ARGS__; }                 \
  } while (0)
#define KDKL_BY_FORMAT(fmt, NAME, ...)                                              \
  do {                                                                              \
    if ((fmt) == KDKL_ACT8_INT8) { constexpr int NAME = kFmtInt8; __VA_ARGS__; }    \
    else { constexpr int NAME = kFmtE4M3; __VA_ARGS__; }                            \
  } while (0)
#define KDKL_BY_FORMAT_OR_NONE(fmt, NAME, ...)                           \
  do {                                                                   \
    if ((fmt) == KDKL_ACT8_NONE) { constexpr int NAME = -1; __VA_ARGS__; } \
    else KDKL_BY_FORMAT(fmt, NAME, __VA_ARGS__);                         \
  } while (0)
#define KDKL_BY_TYPE16(type, NAME, ...)                                          \
  do {                                                                           \
    if ((type) == KDKL_TYPE_BF16) { using NAME = __nv_bfloat16; __VA_ARGS__; }   \
    else { using NAME = __half; __VA_ARGS__; }                                   \
  } while (0)
#define KDKL_BY_TYPE(type, NAME, ...)                              \
  do {                                                             \
    if ((type) == KDKL_TYPE_F32) { using NAME = float; __VA_ARGS__; } \
    else KDKL_BY_TYPE16(type, NAME, __VA_ARGS__);                  \
  } while (0)

}  // namespace kdkl
