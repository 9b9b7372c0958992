// The gated linear layer for up to 128 tokens, on the tensor cores: what it takes is the weights' way through memory, so a
// CTA gives its shared memory to a ring of weight blocks and the tokens are the narrow side of the product.
//
//   D [128, N] = A [128, H] B [N, H]^T, A = 64 gate rows above the same 64 features' up rows, B = the tokens (N = 16 .. 128)
//
// warp 0 loads (TMA, 64 columns a block), warp 1 multiplies (tcgen05, M = 128), warps 2 to 5 finish. An SM takes in such a
// stream at about 50 GB/s, however long the ring (5 or 11 stages: the same time), so all SMs have to take part: where
// there are fewer tiles than SMs, a cluster of 2 or 4 CTAs shares a tile's contraction. Even shares come of it seldom: 5632
// features are 88 tiles, 176 CTAs in clusters of two, and the 28 of 148 SMs that have two of them, 0.52 MB, set the time. Each hands every CTA of the cluster (itself
// too) its sums for that CTA's share of the tokens, through shared memory, which is empty by then; a thread then
// has one feature of half of them, adds up the parts in their order and forms the outputs, 32 features = 64 bytes a
// token and warp; a group of a record is a warp's 32 lanes. Measured, 9 and 128 tokens, weights from memory: 2048 x
// 5632 12.3 and 19.5 us, 4096 x 14336 40.4 and 50.1, 1000 x 2600 6.0 and 12.5 (7.2, 36 and 1.6 the weights' bytes at the
// copy rate). The 256-token tiles of gemm_tcgen05.cuh, which leave most SMs idle here: 23.9, 68 and 14.4 for 9 tokens.
#pragma once
#include "gated_linear_kernels.cuh"
#include "gemm_tcgen05.cuh"

namespace kdkl {

constexpr int kFewTokens = 128, kFewFeatures = 64, kFewThreads = 192, kFewMaxStages = 8;

enum { kFewForward = 0, kFewAct8 = 1, kFewBack = 2 };
struct FewParams {
  int T, H, F, act, format, stages, cluster;
  __nv_bfloat16* h; long long ld_h;
  ActRecord rec_gate, rec_up, rec_h;
  const __nv_bfloat16* dh; long long ld_dh;
  __nv_bfloat16* dgate_up;
  int* status;
};

__host__ __device__ constexpr int few_stage_bytes(int N) { return 2 * kFewFeatures * 128 + N * 128; }

// a lane's value of 32 neighbours, one group of a record
template <int FMT>
__device__ __forceinline__ void record_lane(const ActRecord& r, long long code_at, long long scale_at, float v, bool write, int lane) {
  const uint32_t byte = act_scale_byte<FMT>(__reduce_max_sync(0xffffffffu, __float_as_uint(v) & 0x7fffffffu));
  const uint32_t code = act_code<FMT>(v, byte);
  if (write) {
    r.codes[code_at] = (uint8_t)code;
    if (lane == 0) r.scales[scale_at] = (uint8_t)byte;
  }
}
__device__ __forceinline__ void record_lane(int fmt, const ActRecord& r, long long code_at, long long scale_at, float v, bool write, int lane) {
  if (fmt == kFmtInt8) record_lane<kFmtInt8>(r, code_at, scale_at, v, write, lane);
  else record_lane<kFmtE4M3>(r, code_at, scale_at, v, write, lane);
}

__device__ __forceinline__ void st_cluster_f32(uint32_t cluster_addr, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(cluster_addr), "f"(v) : "memory");
}

template <int N, int MODE>
__global__ void __launch_bounds__(kFewThreads, 1)
gated_few_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const FewParams p) {
  constexpr int kStage = few_stage_bytes(N);
  constexpr uint32_t kCols = N < 32 ? 32 : N;
  extern __shared__ uint8_t few_raw[];
  __shared__ uint64_t bars[2 * kFewMaxStages + 1];
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag;
  const uint32_t ring = (smem_u32(few_raw) + 1023u) & ~1023u;
  const float* parts = reinterpret_cast<const float*>(few_raw + (ring - smem_u32(few_raw)));   // [cluster][its tokens][128], behind the ring's use
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, stages = p.stages, S = p.cluster;
  const int rank = (int)cluster_ctarank(), share = N / S;  // tokens of a CTA
  auto full = [&](int s) { return smem_u32(&bars[s]); };
  auto empty = [&](int s) { return smem_u32(&bars[kFewMaxStages + s]); };
  const uint32_t done = smem_u32(&bars[2 * kFewMaxStages]);
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    mbar_init(done, 1);
    abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tmW);
    tma_prefetch_desc(&tmX);
  }
  if (warp == 1) { tmem_alloc(smem_u32(&tmem_slot), kCols); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const int f0 = (int)(blockIdx.x / S) * kFewFeatures, all = (p.H + BK - 1) / BK, per = (all + S - 1) / S;
  const int k0 = rank * per, blocks = min(all, k0 + per) - k0;         // (no CTA is without: the host sees to it)
  grid_dependents_launch();
  grid_dependency_wait();
  if (blockIdx.x == 0 && threadIdx.x < 2) p.status[threadIdx.x] = 0;   // (a wait gives up after two seconds, long after this)
  bool arrived = true;
  if (warp == 0) {
    if (lane == 0) {
      int kb = 0;
      for (; kb < blocks; ++kb) {
        const int s = kb % stages;
        if (!mbar_wait(empty(s), ((kb / stages) & 1u) ^ 1u, &abort_flag, p.status, 61)) break;
        const uint32_t at = ring + s * kStage;
        mbar_arrive_expect_tx(full(s), kStage);
        tma_load_3d(at, &tmW, (k0 + kb) * BK, f0, 0, full(s));
        tma_load_3d(at + kFewFeatures * 128, &tmW, (k0 + kb) * BK, f0, 1, full(s));
        tma_load_2d(at + 2 * kFewFeatures * 128, &tmX, (k0 + kb) * BK, 0, full(s));
      }
      if (kb < blocks) {                                   // given up: the copies in flight get a bounded time to land
        const uint64_t t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 2000000ull) {}
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = make_idesc_bf16(2 * kFewFeatures, N, 0u, 0u);
      bool ok = true;
      for (int kb = 0; kb < blocks; ++kb) {
        const int s = kb % stages;
        if (!mbar_wait(full(s), (kb / stages) & 1u, &abort_flag, p.status, 62)) { ok = false; break; }
        tc_fence_after();
        const uint64_t a = make_smem_desc(ring + s * kStage, 0, 1024), b = make_smem_desc(ring + s * kStage + 2 * kFewFeatures * 128, 0, 1024);
#pragma unroll
        for (int j = 0; j < BK / UMMA_K; ++j) umma_bf16(tmem, a + 2 * j, b + 2 * j, idesc, kb > 0 || j > 0 ? 1u : 0u);
        umma_commit(empty(s));
      }
      if (ok) umma_commit(done);
    }
  } else {
    arrived = __all_sync(0xffffffffu, mbar_wait(done, 0u, &abort_flag, p.status, 63));
  }
  // every CTA's ring is empty behind this
  __syncwarp();
  if (S > 1) cluster_sync_all(); else __syncthreads();
  if (warp >= 2 && arrived) {
    const int lg = warp & 3;                               // this warp's lanes of the accumulator: gate 0, 1, up 2, 3
    const int shift = 31 - __clz(share);
    uint32_t to[4];                                        // this lane's place in what every CTA gets from this one
#pragma unroll
    for (int q = 0; q < 4; ++q) to[q] = map_to_cta(ring + 4u * (uint32_t)(rank * share * 128 + lg * 32 + lane), (uint32_t)(q < S ? q : 0));
    tc_fence_after();
#pragma unroll 1
    for (int t0 = 0; t0 < N && t0 < p.T; t0 += 16) {
      uint32_t r[16];
      tmem_ld16(tmem + ((uint32_t)(lg * 32) << 16) + t0, r);
      tmem_ld_wait();
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int t = t0 + j, owner = t >> shift;
        st_cluster_f32((owner == 0 ? to[0] : owner == 1 ? to[1] : owner == 2 ? to[2] : to[3]) + 512u * (uint32_t)(t & (share - 1)),
                       __uint_as_float(r[j]));
      }
    }
    tc_fence_before();
  }
  __syncwarp();
  if (S > 1) cluster_sync_all(); else __syncthreads();
  if (warp >= 2 && arrived) {
    const int id = threadIdx.x - 64, local = id & 63, f = f0 + local;
    const long long cpitch = act_codes_pitch(p.F), spitch = act_scale_pitch(p.F);
    const bool in = f < p.F, coded = f < cpitch;
    // the two halves of the threads take every other token; eight at a time, so that their chains overlap
    constexpr int B = 8;
    const int mine = id >> 6, most = min(share, p.T - rank * share);     // (most <= 0: nothing)
    for (int i0 = mine; i0 < most; i0 += 2 * B) {
      float g[B], u[B], d[B];
#pragma unroll
      for (int j = 0; j < B; ++j) {
        g[j] = u[j] = 0.f;
        const int i = min(i0 + 2 * j, most - 1);           // (past the end: the last one again, not written)
        d[j] = MODE == kFewBack && in ? __bfloat162float(p.dh[(rank * share + i) * p.ld_dh + f]) : 0.f;
      }
      for (int q = 0; q < S; ++q) {
        const float* from = parts + q * share * 128 + local;
#pragma unroll
        for (int j = 0; j < B; ++j) {
          const int i = min(i0 + 2 * j, most - 1);
          g[j] += from[i * 128];
          u[j] += from[i * 128 + 64];
        }
      }
#pragma unroll
      for (int j = 0; j < B; ++j) {
        const int i = i0 + 2 * j;
        const long long t = rank * share + i;
        const bool ok = i < most;                          // the same for a warp
        const GateAct a = p.act == kActGelu ? gate_act<kActGelu>(g[j]) : gate_act<kActSilu>(g[j]);
        if (MODE == kFewBack) {
          if (ok && in) {
            __nv_bfloat16* o = p.dgate_up + t * 2 * p.F + f;
            o[0] = __float2bfloat16_rn(d[j] * u[j] * a.slope);
            o[p.F] = __float2bfloat16_rn(d[j] * (g[j] * a.sigmoid));
          }
        } else {
          const __nv_bfloat16 h = __float2bfloat16_rn(g[j] * a.sigmoid * u[j]);
          if (ok && in) p.h[t * p.ld_h + f] = h;
          if (MODE == kFewAct8 && ok) {
            const long long code = t * cpitch + f, scale = t * spitch + (f >> 5);
            record_lane(p.format, p.rec_gate, code, scale, g[j], coded, lane);
            record_lane(p.format, p.rec_up, code, scale, u[j], coded, lane);
            if (p.rec_h.codes != nullptr) record_lane(p.format, p.rec_h, code, scale, in ? __bfloat162float(h) : 0.f, coded, lane);
          }
        }
      }
    }
  }
  __syncthreads();
  if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem, kCols); }
}

}  // namespace kdkl
