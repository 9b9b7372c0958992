// Host side of the bf16 GEMM that the library's translation units share: tile choices, launch, splits of a contraction.
#pragma once
#include <string.h>

#include "gemm_tcgen05.cuh"
#include "host_common.cuh"

namespace kdkl {

// All GEMMs run as CTA pairs (256 x 256 tile per pair, see GemmCfg).
constexpr int kNCTA = 2;
constexpr int kTileM = GemmCfg<kNCTA>::TILE_M;
constexpr int kBRows = GemmCfg<kNCTA>::B_ROWS;             // rows of a K-major B box (also per half of a WIDE tile)
constexpr int kWideN = GemmCfg<kNCTA, true>::TILE_N;
static_assert(GemmCfg<kNCTA, true>::B_ROWS / 2 == kBRows, "a WIDE tile's halves take the narrow tile's B boxes");
// Row tiles per raster group of the two vocabulary sweeps (forward, recompute): as many as keep the group's hidden
// rows within 32 MiB, i.e. resident in either half of the L2 while the weight streams past (4096 tokens at H = 4096).
inline int m_group_for(long long H) {
  const long long rows = (32ll << 20) / (H * 2);
  const long long g = rows / kTileM;
  return (int)(g < 1 ? 1 : g);
}
// The output GEMMs (N = H) use WIDE tiles when rounding H up to whole 512-column tiles wastes at most a
// tenth of the tensor work (H = 4096, 1024, 1000 ...); narrow 256-column tiles otherwise.
inline bool use_wide(long long N) { return ((N + kWideN - 1) / kWideN) * kWideN * 10 <= N * 11; }
inline long long n_tiles_for(long long N, bool wide) { return wide ? (N + kWideN - 1) / kWideN : (N + BN - 1) / BN; }
// early: the launch may be prepared while the kernel before it on the stream drains (see launch_cluster in body_host.cuh; every
// kernel before it has then to leave what it writes complete to grid_dependency_wait, which all do). NCTA = 1 takes a B map whose boxes are 256 rows (GemmCfg<1>::B_ROWS), and counts row tiles of 128.
template <int EPI, bool A_MN, bool B_MN, bool WIDE = false, int NCTA = kNCTA>
inline int launch_gemm(const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& tc, const GemmParams& p,
                       const DeviceInfo& di, cudaStream_t st, bool early = false) {
  auto kern = gemm_tcgen05_kernel<EPI, A_MN, B_MN, NCTA, WIDE>;
  constexpr int smem = GemmCfg<NCTA, WIDE>::SMEM_BYTES;
  static_assert(smem <= 227 * 1024, "shared memory per CTA");
  // The shared-memory limit belongs to the current device's copy of this instantiation: set once per device
  // (a process may drive several), not per launch.
  static bool attr_set[kMaxDevices];
  const int sm_count = di.sm_count;
  if (di.dev < 0 || di.dev >= kMaxDevices || !attr_set[di.dev]) {
    KDKL_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    if (di.dev >= 0 && di.dev < kMaxDevices) attr_set[di.dev] = true;
  }
  // persistent: one worker (a CTA, or a pair of CTAs on neighbouring SMs) per SM (pair), each walking
  // the work units with a stride of the worker count
  const int units = p.m_tiles * p.n_tiles * p.k_splits;
  const int max_workers = sm_count / NCTA;
  const int workers = units < max_workers ? units : max_workers;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3((unsigned)(workers * NCTA), 1, 1);
  cfg.blockDim = dim3(GEMM_THREADS, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = NCTA;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.numAttrs = early ? 2 : 1;
  cudaError_t e = cudaLaunchKernelEx(&cfg, kern, ta, tb, tc, p);
  if (e != cudaSuccess) return cuda_fail("gemm_tcgen05_kernel launch", e);
  KDKL_LAUNCHED("gemm_tcgen05_kernel");
  return KDKL_OK;
}

// How many work units to cut each output tile's contraction into so that the units fill whole
// waves of SMs: the smallest count (<= 4, each unit keeping >= 32 k-blocks) that reaches 95 %
// wave efficiency, else the most efficient one, for the device's count of workers (SMs / CTAs per tile).
inline int choose_k_splits(long long tiles, long long kblocks, int sm_count) {
  const long long sms = (sm_count < kNCTA ? kNCTA : sm_count) / kNCTA;
  int best = 1;
  double best_eff = 0.0;
  for (int sp = 1; sp <= 4; ++sp) {
    if (sp > 1 && kblocks / sp < 32) break;
    const long long units = tiles * sp;
    const double eff = (double)units / (double)(((units + sms - 1) / sms) * sms);
    if (eff > best_eff + 1e-9) { best_eff = eff; best = sp; }
    if (eff >= 0.95) break;
  }
  return best;
}

}  // namespace kdkl
