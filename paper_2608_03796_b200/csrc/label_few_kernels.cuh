// The label loss's sweep over the vocabulary for up to 128 tokens. What it takes is the weight's way through memory: the
// vocabulary is the wide side of the product, 128 entries a tile, the tokens the narrow one.
//
//   D [128, N] = W-tile [128, H] h [N, H]^T, N = 16 .. 128
//
// One persistent CTA an SM: warp 0 loads (TMA, blocks of 64 columns into a ring that runs on from tile to tile), warp 1 multiplies
// (tcgen05, two accumulators in turn), warps 2 to 5 finish a tile under the next one's loads: a lane has one vocabulary entry, so
// the tile is turned in shared memory, and 128 / N threads take a token: its largest logit, sum of exponentials and sum of logits
// over the tile, the label's logit, and for the one-step call the exponentials in fp16, each 32 entries to their own largest
// (see EPI_LABEL_E, which does the same for more tokens). Evaluation of 16 tokens, weights from memory, all launches of the call:
// 2816 x 32768 46 us, 4096 x 131072 190, 1024 x 20001 23 (28.6, 166 and 6.3 the weights' bytes at the copy rate); by the
// 256-token tiles, which take 129 tokens in 55, 246 and 30 us, as much as there.
#pragma once
#include "gemm_tcgen05.cuh"

namespace kdkl {

constexpr int kLabelFewTokens = 128, kLabelFewRows = 128, kLabelFewThreads = 192, kLabelFewMaxStages = 8;
__host__ __device__ constexpr int label_few_stage_bytes(int N) { return kLabelFewRows * 128 + N * 128; }
// A token's row of the turned tile: entry r at r + r / 16, rows an odd number of words apart, so that neither the lanes that
// write it (one entry each) nor those that read it (one token, or a share of 16 entries, each) crowd on a bank.
constexpr int kLabelFewRowWords = kLabelFewRows + kLabelFewRows / 16 + 1;
__host__ __device__ constexpr int label_few_turned_bytes(int N) { return (N * kLabelFewRowWords * 4 + 1023) / 1024 * 1024; }
__device__ __forceinline__ int label_few_place(int r) { return r + (r >> 4); }
// Whether all four warps' waits ended well: a decision of all 128 threads, as barriers of theirs follow.
__device__ __forceinline__ bool label_few_agree(bool ok) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 q, %1, 0;\n\tbarrier.cta.red.and.pred p, 1, 128, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(r) : "r"(ok ? 1u : 0u) : "memory");
  return r != 0;
}

struct LabelFewParams {
  int T, H, V, tiles, stages;
  float scale_log2;
  const int* col;                      // [T], -1: not counted
  float* part_m; float* part_s; float* part_z; long long stride;       // [tiles, stride]
  float* z_label;                      // [T]
  uint16_t* E; long long ld_e; float* win_max;                         // one-step call; win_max [ceil(V / 32), stride]
  int* status;
};

template <int N, bool STORE>
__global__ void __launch_bounds__(kLabelFewThreads, 1)
label_few_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const LabelFewParams p) {
  constexpr int kStage = label_few_stage_bytes(N), kRow = kLabelFewRowWords;
  constexpr uint32_t kCols = 2 * N;
  extern __shared__ uint8_t few_raw[];
  __shared__ uint64_t bars[2 * kLabelFewMaxStages + 4];
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag;
  const uint32_t turned_at = (smem_u32(few_raw) + 1023u) & ~1023u, ring = turned_at + label_few_turned_bytes(N);
  float* turned = reinterpret_cast<float*>(few_raw + (turned_at - smem_u32(few_raw)));        // [N][137]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, stages = p.stages;
  auto full = [&](int s) { return smem_u32(&bars[s]); };
  auto empty = [&](int s) { return smem_u32(&bars[kLabelFewMaxStages + s]); };
  auto tfull = [&](int a) { return smem_u32(&bars[2 * kLabelFewMaxStages + a]); };
  auto tempty = [&](int a) { return smem_u32(&bars[2 * kLabelFewMaxStages + 2 + a]); };
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(tfull(a), 1); mbar_init(tempty(a), 4); }
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
  const int blocks = (p.H + BK - 1) / BK;
  grid_dependents_launch();
  grid_dependency_wait();
  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      for (int tile = blockIdx.x; tile < p.tiles && ok; tile += gridDim.x) {
        for (int kb = 0; kb < blocks; ++kb, ++it) {
          const uint32_t s = it % stages;
          if (!mbar_wait(empty(s), ((it / stages) & 1u) ^ 1u, &abort_flag, p.status, 71)) { ok = false; break; }
          const uint32_t at = ring + s * kStage;
          mbar_arrive_expect_tx(full(s), kStage);
          tma_load_2d(at, &tmW, kb * BK, tile * kLabelFewRows, full(s));
          tma_load_2d(at + kLabelFewRows * 128, &tmX, kb * BK, 0, full(s));
        }
      }
      if (!ok) {                                           // given up: the copies in flight get a bounded time to land
        const uint64_t t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 2000000ull) {}
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = make_idesc_bf16(kLabelFewRows, N, 0u, 0u);
      uint32_t it = 0, lt = 0;
      bool ok = true;
      for (int tile = blockIdx.x; tile < p.tiles && ok; tile += gridDim.x, ++lt) {
        const uint32_t acc = lt & 1u;
        if (!mbar_wait(tempty(acc), ((lt >> 1) & 1u) ^ 1u, &abort_flag, p.status, 72)) break;
        tc_fence_after();
        for (int kb = 0; kb < blocks; ++kb, ++it) {
          const uint32_t s = it % stages;
          if (!mbar_wait(full(s), (it / stages) & 1u, &abort_flag, p.status, 73)) { ok = false; break; }
          tc_fence_after();
          const uint64_t a = make_smem_desc(ring + s * kStage, 0, 1024), b = make_smem_desc(ring + s * kStage + kLabelFewRows * 128, 0, 1024);
#pragma unroll
          for (int j = 0; j < BK / UMMA_K; ++j) umma_bf16(tmem + acc * N, a + 2 * j, b + 2 * j, idesc, kb > 0 || j > 0 ? 1u : 0u);
          umma_commit(empty(s));
        }
        if (ok) umma_commit(tfull(acc));
      }
    }
  } else {
    const int lg = warp & 3, id = threadIdx.x - 64;
    constexpr int P = 128 / N, R = kLabelFewRows / P;      // threads a token, entries a thread (16, 32, 64 or 128)
    const int token = id / P, part = id % P;
    const bool mine = token < p.T;
    const int col = mine ? p.col[token] : -1;
    uint32_t lt = 0;
    for (int tile = blockIdx.x; tile < p.tiles; tile += gridDim.x, ++lt) {
      const uint32_t acc = lt & 1u;
      const int v0 = tile * kLabelFewRows;
      if (!label_few_agree(mbar_wait(tfull(acc), (lt >> 1) & 1u, &abort_flag, p.status, 74))) break;
      tc_fence_after();
#pragma unroll 1
      for (int t0 = 0; t0 < N && t0 < p.T; t0 += 16) {
        uint32_t r[16];
        tmem_ld16(tmem + ((uint32_t)(lg * 32) << 16) + acc * N + t0, r);
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 16; ++j) turned[(t0 + j) * kRow + label_few_place(lg * 32 + lane)] = __uint_as_float(r[j]);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(tempty(acc));
      asm volatile("bar.sync 1, 128;" ::: "memory");       // the tile is turned
      const float* z = turned + token * kRow + label_few_place(part * R);
      const int first = v0 + part * R, have = mine ? max(0, min(R, p.V - first)) : 0;        // entries of this thread that exist
      float m = -INFINITY, s = 0.f, sum = 0.f;
      constexpr int W = R < 32 ? R : 32;                   // what a thread has of a window
#pragma unroll 1
      for (int w = 0; w < R / W; ++w) {
        const int n = max(0, min(W, have - w * W));
        float v[W], top = -INFINITY, e_sum = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = z[w * (W + W / 16) + label_few_place(i)];          // (past the last entry: zeros)
#pragma unroll
        for (int i = 0; i < W; ++i) {
          top = fmaxf(top, i < n ? v[i] : -INFINITY);
          sum += i < n ? v[i] : 0.f;
        }
        if (R < 32) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));                   // (two threads share a window)
        const float ref = top > -INFINITY ? top * p.scale_log2 : 0.f;
        uint32_t half[W / 2];
#pragma unroll
        for (int i = 0; i < W; i += 2) {
          const float a = i < n ? ex2_approx(fmaf(v[i], p.scale_log2, -ref)) : 0.f;
          const float b = i + 1 < n ? ex2_approx(fmaf(v[i + 1], p.scale_log2, -ref)) : 0.f;
          e_sum += a + b;
          const __half2 h = __floats2half2_rn(a, b);
          half[i / 2] = *reinterpret_cast<const uint32_t*>(&h);
        }
        if (STORE && n > 0) {
          uint16_t* e = p.E + token * p.ld_e + first + w * W;                                 // (rows are whole 64 entries apart)
#pragma unroll
          for (int i = 0; i < W / 8; ++i)
            if (8 * i < n) *reinterpret_cast<uint4*>(e + 8 * i) = make_uint4(half[4 * i], half[4 * i + 1], half[4 * i + 2], half[4 * i + 3]);
          if (R >= 32 || (part & 1) == 0) p.win_max[(long long)((first + w * W) >> 5) * p.stride + token] = ref;
        }
        if (n > 0) {
          const float mn = fmaxf(m, ref);
          s = s * ex2_approx(m - mn) + e_sum * ex2_approx(ref - mn);
          m = mn;
        }
      }
      if (col >= first && col < first + have) p.z_label[token] = z[label_few_place(col - first)];
#pragma unroll
      for (int o = 1; o < P; o <<= 1) {                    // the token's threads are neighbours
        const float om = __shfl_xor_sync(0xffffffffu, m, o), os = __shfl_xor_sync(0xffffffffu, s, o);
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
        const float mn = fmaxf(m, om);
        s = (m > -INFINITY ? s * ex2_approx(m - mn) : 0.f) + (om > -INFINITY ? os * ex2_approx(om - mn) : 0.f);
        m = mn;
      }
      if (mine && part == 0) {
        p.part_m[(long long)tile * p.stride + token] = m;
        p.part_s[(long long)tile * p.stride + token] = s;
        p.part_z[(long long)tile * p.stride + token] = sum;
      }
      asm volatile("bar.sync 1, 128;" ::: "memory");       // nobody reads the turned tile any more
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem, kCols); }
}

}  // namespace kdkl
