// Products that write a gradient, out [M, N] = A B with B stored [K, N]: which tiles, how many parts of the contraction, and
// the launch. A is K-major ([M, K]) or MN-major ([K, M]). The result is bf16 or fp32, written or added to.
#pragma once
#include "body_host.cuh"
#include "gemm_host.cuh"

namespace kdkl {

// out = (part[0] + part[1] + ..., in that order) scale [+ out], rounded once. One thread per four columns.
template <bool BF16>
__global__ void __launch_bounds__(256)
out_join_kernel(const float* part, long long slab, int splits, long long n4, const float* scale, void* out,
                int accumulate, const int* go) {
  grid_dependents_launch();
  grid_dependency_wait();
  if (go != nullptr && *go == 0) return;
  const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= n4) return;
  float4 a = reinterpret_cast<const float4*>(part)[i];
  for (int s = 1; s < splits; ++s) {
    const float4 b = reinterpret_cast<const float4*>(part + s * slab)[i];
    a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
  }
  if (scale != nullptr) { const float r = *scale; a.x *= r; a.y *= r; a.z *= r; a.w *= r; }
  if (BF16) {
    uint2* o = reinterpret_cast<uint2*>(out) + i;
    if (accumulate) {
      const uint2 w = *o;
      a.x += __uint_as_float(w.x << 16); a.y += __uint_as_float(w.x & 0xffff0000u);
      a.z += __uint_as_float(w.y << 16); a.w += __uint_as_float(w.y & 0xffff0000u);
    }
    *o = make_uint2(pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w));
  } else {
    float4* o = reinterpret_cast<float4*>(out) + i;
    if (accumulate) { const float4 w = *o; a.x += w.x; a.y += w.y; a.z += w.z; a.w += w.w; }
    *o = a;
  }
}

// The plan with the least estimated cycles: waves of units, a unit taking its k-blocks (512 cycles of tensor work each by the
// nominal rate, 952 in a WIDE tile, which brings a quarter less operand data a flop) and about six more to start and to
// drain its tile (ten of a WIDE one's, whose stores nothing overlaps); parts of a contraction cost the slabs' way through memory (2600 bytes a cycle) and one more launch.
// Measured (bf16 out; narrow, then WIDE, parts behind the slash): 1021 x 2816 x 14336 83 / 3 and 76 us / 3, 1021 x 2880 x 20000
// 119 / 3 and 103 / 3, 8192 x 4096 x 131072 6823 / 1 and 6667 / 2, 131072 x 2048 x 8192 3390 / 1 and 3280 / 1; the other way
// round 14336 x 2816 x 1021 80 / 1 and 84 / 1, 300 x 2048 x 11264 23 / 4 and 28 / 8, 4096 x 1024 x 4096 30 / 1 and 37 / 2.
struct OutPlan { bool wide; int splits; };
inline OutPlan out_plan(long long M, long long N, long long K, int sm_count, bool joined) {
  const long long workers = sm_count < 2 ? 1 : sm_count / 2, kb = (K + BK - 1) / BK, mt = (M + kTileM - 1) / kTileM;
  OutPlan best = {false, 1};
  double least = 1e300;
  for (int wide = 0; wide <= 1; ++wide) {
    const long long tiles = mt * n_tiles_for(N, wide != 0);
    for (int sp = 1; sp <= 16; ++sp) {
      if (sp > 1 && kb / sp < 8) break;
      if ((kb + sp - 1) / sp * (sp - 1) >= kb) continue;     // the last part would be empty
      const long long waves = (tiles * sp + workers - 1) / workers;
      double cost = (double)waves * ((kb + sp - 1) / sp + (wide ? 10 : 6)) * (wide ? 952.0 : 512.0);
      if (sp > 1 || joined) cost += 4000.0 + (double)M * N * (8.0 * sp + 2.0) / 2600.0;
      if (cost < least) { least = cost; best = OutPlan{wide != 0, sp}; }
    }
  }
  return best;
}
inline size_t out_slab_bytes(const OutPlan& plan, long long M, long long N, bool joined) {
  return plan.splits > 1 || joined ? up((size_t)plan.splits * up((size_t)M, 32) * N * 4, 256) : 0;
}

struct OutGemm {
  const void* a; long long lda;       // elements; a_mn: stored [K, M]
  const void* b; long long ldb;       // [K, N]
  long long M, N, K;
  void* out; bool bf16; int accumulate;
  OutPlan plan;
  float* slab;                        // out_slab_bytes
  int* status;
  const int* go;
  const uint8_t* m_live; const uint8_t* k_live;
  const float* scale;                 // of the product, on the device; or null
};
template <bool A_MN>
inline int launch_out(const OutGemm& o, const DeviceInfo& di, cudaStream_t st) {
  CUtensorMap ta, tb, tc;
  int rc;
  if (A_MN) rc = make_tmap_bf16(&ta, o.a, (uint64_t)o.M, (uint64_t)o.K, (uint64_t)o.lda * 2, 64, BK);
  else      rc = make_tmap_bf16(&ta, o.a, (uint64_t)o.K, (uint64_t)o.M, (uint64_t)o.lda * 2, BK, BM);
  if (rc) return rc;
  if ((rc = make_tmap_bf16(&tb, o.b, (uint64_t)o.N, (uint64_t)o.K, (uint64_t)o.ldb * 2, 64, BK))) return rc;
  const bool joined = o.plan.splits > 1 || (o.bf16 && o.accumulate);
  GemmParams p;
  memset(&p, 0, sizeof(p));
  p.M = (int)o.M; p.N = (int)o.N; p.K = (int)o.K;
  p.m_tiles = (int)((o.M + kTileM - 1) / kTileM); p.n_tiles = (int)n_tiles_for(o.N, o.plan.wide);
  const long long rows = (long long)up((size_t)o.M, 32);   // of a part: output boxes are 32 rows high
  p.k_splits = o.plan.splits; p.split_rows = (int)rows;
  p.status = o.status; p.go = o.go; p.m_live = o.m_live; p.k_live = o.plan.splits == 1 ? o.k_live : nullptr;
  const bool f32 = joined || !o.bf16;
  if (joined) rc = make_tmap_out_f32(&tc, o.slab, (uint64_t)o.N, (uint64_t)(o.plan.splits * rows), (uint64_t)o.N);
  else if (o.bf16) rc = make_tmap_out_bf16(&tc, o.out, (uint64_t)o.N, (uint64_t)o.M, (uint64_t)o.N);
  else { rc = make_tmap_out_f32(&tc, o.out, (uint64_t)o.N, (uint64_t)o.M, (uint64_t)o.N); p.accumulate = o.accumulate; }
  if (rc) return rc;
  p.out_scale = joined ? nullptr : o.scale;                // (of parts, when they are joined)
#define KDKL_OUT(EPI)                                                                 \
  rc = o.plan.wide ? launch_gemm<EPI, A_MN, true, true>(ta, tb, tc, p, di, st, true)  \
                   : launch_gemm<EPI, A_MN, true, false>(ta, tb, tc, p, di, st, true)
  if (p.out_scale != nullptr) {
    if (f32) KDKL_OUT(EPI_STORE_F32_SCALED);
    else KDKL_OUT(EPI_STORE_BF16_SCALED);
  } else {
    if (f32) KDKL_OUT(EPI_STORE_F32);
    else KDKL_OUT(EPI_STORE_BF16);
  }
#undef KDKL_OUT
  if (rc || !joined) return rc;
  const long long n4 = o.M * o.N / 4;
  const unsigned grid = (unsigned)((n4 + 255) / 256);
  KDKL_BY_BOOL(o.bf16, BF16,
    rc = launch("out_join_kernel", out_join_kernel<BF16>, dim3(grid), 256, 0, st, (const float*)o.slab, rows * o.N, o.plan.splits, n4, o.scale,
                o.out, o.accumulate, o.go));
  return rc;
}

}  // namespace kdkl
