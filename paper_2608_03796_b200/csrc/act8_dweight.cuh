// Weight gradient of a linear layer whose input was kept in an 8-bit record:
//   dW[n, h] (= or +=) sum_t dY[t, n] x~[t, h],  x~ = what the record stands for.
//
// A matrix product of 2 T N H flops over operands that fit the L2 in slices: bound by the tensor pipe from a few
// thousand tokens on. act8_dweight_kernel keeps it there by reading the record inside the product: the codes come
// through TMA (half the bytes of bf16), are turned into bf16 by eight warps - exactly, 7 or 4 significant bits times a
// power of two - and written as the swizzled operand tile that tcgen05.mma reads, while the products of earlier blocks
// run. No bf16 copy of the activations ever exists in memory.
//
//   tile 256 (n) x 256 (h) per CTA pair (cta_group::2); a block of the contraction is 64 tokens
//   warp 0       TMA of dY (bf16, contiguous along n: MN-major operand), STAGES deep
//   warps 2, 3   TMA of codes and scale bytes, 32 tokens x 128 columns each, RAW / 2 deep
//   warp 1       tensor memory; the pair leader's lane 0 issues the MMAs
//   warps 4-11   codes -> bf16 operand tile of this CTA's 128 columns
//   warps 12-19  running sums in registers (128 rows x 256 columns a CTA, 128 values a thread)
//
// Why sums in registers: an accumulator in tensor memory truncates at each addition, measured as a relative error of
// 1.1e-9 per token contracted with two bf16 operands (3.8e-5 at 32768 tokens) and 2.4e-10 with codes on one side. It
// therefore only runs over RUN blocks (1024 tokens); then the eight warps add it, rounding to nearest, to the sums they
// hold, while the second accumulator fills. (Runs of 2048 tokens cost 1 % less.)
// Work units: whole tiles as far as they fill whole waves of CTA pairs, then the remaining tiles cut into parts of the
// contraction, so that the last wave is as short as it can be. Parts leave fp32 slabs that act8_dweight_join_kernel adds
// in order: results are reproducible bit for bit.
//
// One B200, 32768 x 4096 x 4096: 780 to 805 us with int8, 800 to 828 us with e4m3 codes (1410 and 1375 TFLOP/s at best; a
// library product of bf16 operands 675 us); back to back, under the power cap, 955 to 985 us against 813. What the gap is: the conversion, done
// once per 256 rows of the result, takes about 135 us of the cap's energy.
#pragma once
#include "act8.cuh"
#include "sm100_prims.cuh"

namespace kdkl {

struct DweightParams {
  const __nv_bfloat16* dy; long long ld_dy;
  ActRecord rec;
  long long T; int N, H;
  void* out; int type; int accumulate;
  int* status;              // 256 bytes, set to zero by the first block
};
__device__ __forceinline__ void clear_status(int* status) {
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < 64) status[threadIdx.x] = 0;
}

// Any alignment and width: rows of dY or of the result that tensor maps cannot describe (not 16 bytes apart).
// 64 x 64 tiles of fp32 FMAs, so 15 to 40 times the tensor-core form's time: 333 x 2817 x 2816 takes 188 us (12 aligned),
// 4096 x 2816 x 2815 2281.

template <int FMT>
__global__ void __launch_bounds__(256)
act8_dweight_simple_kernel(const DweightParams p) {
  __shared__ float a[16][64], b[16][64 + 4];
  const long long cpitch = act_codes_pitch(p.H), spitch = act_scale_pitch(p.H);
  const int n0 = blockIdx.y * 64, h0 = blockIdx.x * 64;
  const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
  grid_dependents_launch();
  grid_dependency_wait();
  clear_status(p.status);
  float acc[4][4] = {};
  for (long long t0 = 0; t0 < p.T; t0 += 16) {
    for (int i = threadIdx.x; i < 16 * 64; i += 256) {
      const long long t = t0 + i / 64;
      const int n = n0 + i % 64;
      a[i / 64][i % 64] = (t < p.T && n < p.N) ? __bfloat162float(p.dy[t * p.ld_dy + n]) : 0.f;
    }
    if (threadIdx.x < 128) {
      const long long t = t0 + threadIdx.x / 8;
      const int c = h0 + (threadIdx.x % 8) * 8;
      float f[8] = {};
      if (t < p.T && c < cpitch) record_read8<FMT, true>(p.rec, t, cpitch, spitch, c, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) b[threadIdx.x / 8][(threadIdx.x % 8) * 8 + j] = f[j];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(a[k][ty * 4 + i], b[k][tx * 4 + j], acc[i][j]);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + ty * 4 + i, h = h0 + tx * 4 + j;
      if (n >= p.N || h >= p.H) continue;
      const long long at = (long long)n * p.H + h;
      if (p.type == 1) {
        float* o = reinterpret_cast<float*>(p.out);
        o[at] = p.accumulate ? o[at] + acc[i][j] : acc[i][j];
      } else {
        __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(p.out);
        o[at] = __float2bfloat16_rn(p.accumulate ? __bfloat162float(o[at]) + acc[i][j] : acc[i][j]);
      }
    }
}

struct DwCfg {
  static constexpr int TILE = 256, BK = 64, STAGES = 4, RUN = 16;
  static constexpr int A_BYTES = 128 * BK * 2, B_BYTES = 128 * BK * 2, STAGE_BYTES = A_BYTES + B_BYTES;
  // codes and scale bytes wait in slots of half a block, each free again as soon as it is in registers
  static constexpr int RAW = 8, RAW_T = BK / 2, CODE_BYTES = 128 * RAW_T, RAW_BYTES = CODE_BYTES + 16 * RAW_T;
  static constexpr int CONVERT_WARPS = 8, SUM_WARPS = 8;
  static constexpr int CONVERT_TEAM = 2, TEAMS = CONVERT_WARPS / CONVERT_TEAM;   // warps a block; blocks in work at once
  static constexpr int THREADS = 128 + 32 * (CONVERT_WARPS + SUM_WARPS);
  static constexpr int BOX_BYTES = 4096;      // 32 rows x 128 bytes of output per summing warp
  static constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + RAW * RAW_BYTES + SUM_WARPS * BOX_BYTES + 1024 + 256;
  // A wait knows a barrier's phase by one bit, so each slot of a ring has to be waited for by one team, in order: a team
  // that came to a slot of another could take the phase before the last for the one it needs.
  static_assert(STAGES % TEAMS == 0 && RAW % (2 * TEAMS) == 0, "a ring slot belongs to one team");
  // registers a thread of each warpgroup: launched with 96, 32 + 2 * 48 + 2 * 176 <= 5 * 96
  static constexpr int REGS_FEED = 32, REGS_CONVERT = 48, REGS_SUM = 176;
};

struct DwParams {
  long long T;
  int N, H;
  int h_tiles;
  int whole;                       // tiles that are one unit each; the first ones
  int rest, parts;                 // tiles that are cut into `parts` units each: [rest, parts] slabs of 256 x 256 fp32
  int accumulate;
  const __nv_bfloat16* out;        // bf16 output: what += adds to
  int* status;
};

// Four bf16 values from four codes, times `scale` (a power of two in both halves). Exact, but for e4m3 values below bf16's
// last subnormal (2^-133 to 2^-135, at the smallest exponent), which round to a multiple of it. e4m3 codes arrive as their
// value times 2^-120, so their scale carries 2^120.
template <int FMT>
__device__ __forceinline__ void codes_to_bf16x4(uint32_t codes, uint32_t scale, uint32_t (&o)[2]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t v;
    if (FMT == kFmtInt8) {
      // 0x43cc: the low 7 bits of a code as the fraction of 128 + low; minus 128, or minus 256 where the sign bit is set
      const uint32_t p = __byte_perm(codes, 0x43434343u, i == 0 ? 0x4140 : 0x4342);
      const uint32_t a = p & 0xff7fff7fu, b = p & 0xff80ff80u;
      asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(v) : "r"(a), "r"(b));
    } else {
      // 0xcc00: sign, then exponent and fraction four places down: the value times 2^-120 (subnormals included)
      const uint32_t p = __byte_perm(codes, 0u, i == 0 ? 0x1404 : 0x3424);
      v = ((p & 0x7f007f00u) >> 4) | (p & 0x80008000u);
    }
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(o[i]) : "r"(v), "r"(scale));
  }
}
// Sixteen codes of one group. Byte 255 (codes 0) becomes an infinite scale: 0 * infinity = NaN.
template <int FMT>
__device__ __forceinline__ void codes_to_bf16x16(const uint4& c, uint32_t byte, uint32_t (&o)[8]) {
  // e4m3: 2^e 2^120 passes the largest bf16 from byte 135 on (values beyond 57344): the factor 2^120 is then split off
  const bool split = FMT == kFmtE4M3 && byte > 134u;
  const uint32_t scale = ((FMT == kFmtE4M3 && !split ? byte + 120u : byte) << 7) * 0x00010001u;
  const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint32_t v[2];
    codes_to_bf16x4<FMT>(w[k], split ? 0x7b807b80u : scale, v);
    o[2 * k] = v[0]; o[2 * k + 1] = v[1];
  }
  if (split) {
#pragma unroll
    for (int k = 0; k < 8; ++k) asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(o[k]) : "r"(o[k]), "r"(scale));
  }
}

template <int FMT, bool F32_OUT>
__global__ void __launch_bounds__(DwCfg::THREADS, 1) __cluster_dims__(2, 1, 1)
act8_dweight_kernel(const __grid_constant__ CUtensorMap tmY, const __grid_constant__ CUtensorMap tmCodes,
                    const __grid_constant__ CUtensorMap tmScales, const __grid_constant__ CUtensorMap tmOut,
                    const __grid_constant__ CUtensorMap tmSlab, const DwParams p) {
  using C = DwCfg;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t raw0 = base + C::STAGES * C::STAGE_BYTES;
  const uint32_t box0 = raw0 + C::RAW * C::RAW_BYTES;
  const uint32_t bar0 = box0 + C::SUM_WARPS * C::BOX_BYTES;
  // Barriers. In the leader: full (the bytes of both CTAs' dY and both CTAs' converting warps: one wait for the thread that
  // issues the products), tempty (both CTAs' summing warps). In each CTA: empty and tfull (committed to both by the
  // leader's MMAs), rfull, rempty.
  // The leader's MMAs read what the peer's warps wrote into the peer's shared memory, and overwrite tensor memory that
  // those have read (completely: tcgen05.wait::ld). So arrivals on full and tempty, and the leader's waits for them, carry
  // the cluster's scope, restricted to shared memory: 780 to 805 us at 32768 x 4096 x 4096 (775 without). A release of everything
  // in every converting warp cost a quarter of the kernel.
  auto full = [&](uint32_t s) { return bar0 + 8u * s; };
  auto empty = [&](uint32_t s) { return bar0 + 8u * (C::STAGES + s); };
  auto rfull = [&](uint32_t s) { return bar0 + 8u * (2 * C::STAGES + s); };
  auto rempty = [&](uint32_t s) { return bar0 + 8u * (2 * C::STAGES + C::RAW + s); };
  auto tfull = [&](uint32_t a) { return bar0 + 8u * (2 * C::STAGES + 2 * C::RAW + a); };
  auto tempty = [&](uint32_t a) { return bar0 + 8u * (2 * C::STAGES + 2 * C::RAW + 2 + a); };
  constexpr int kBars = 2 * C::STAGES + 2 * C::RAW + 4;
  static_assert(8 * kBars + 8 <= 256, "barrier block");
  uint8_t* bar_ptr = base_ptr + (bar0 - base);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar_ptr + 8 * kBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const bool leader = rank == 0u;
  grid_dependents_launch();
  if (threadIdx.x == 0) {
    for (int s = 0; s < C::STAGES; ++s) {
      mbar_init(full(s), 1 + 2 * C::CONVERT_TEAM);
      mbar_init(empty(s), 1);
    }
    for (int s = 0; s < C::RAW; ++s) { mbar_init(rfull(s), 1); mbar_init(rempty(s), C::CONVERT_TEAM); }
    for (int a = 0; a < 2; ++a) { mbar_init(tfull(a), 1); mbar_init(tempty(a), 2 * C::SUM_WARPS); }
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tmY); tma_prefetch_desc(&tmCodes); tma_prefetch_desc(&tmScales); tma_prefetch_desc(&tmOut);
    if (p.rest > 0) tma_prefetch_desc(&tmSlab);
  }
  if (warp == 1) { tmem_alloc_pair(smem_u32(tmem_slot), 512); tmem_relinquish_pair(); }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  grid_dependency_wait();
  clear_status(p.status);

  const int worker = blockIdx.x >> 1, workers = gridDim.x >> 1;
  const int units = p.whole + p.rest * p.parts;
  const int kblocks = (int)((p.T + C::BK - 1) / C::BK), per_part = (kblocks + p.parts - 1) / p.parts;
  struct Unit { int n0, h0, slab, kb0, kb1; };
  auto unit_at = [&](int u) {
    Unit r;
    int tile = u;
    r.slab = -1; r.kb0 = 0; r.kb1 = kblocks;
    if (u >= p.whole) {
      const int part = (u - p.whole) / p.rest, i = (u - p.whole) % p.rest;
      tile = p.whole + i;
      r.slab = i * p.parts + part;
      r.kb0 = part * per_part;
      if (r.kb0 + per_part < kblocks) r.kb1 = r.kb0 + per_part;
    }
    r.n0 = (tile / p.h_tiles) * C::TILE;
    r.h0 = (tile % p.h_tiles) * C::TILE;
    return r;
  };
  bool ok = true;

  if (warp < 4) {
    regs_dec<C::REGS_FEED>();
    // Each of these warps has 512 cycles for a block, and every instruction of its loop counts: all lanes walk the loop,
    // so that addresses and descriptors stay in uniform registers, and one of them issues.
    if (warp == 0) {
      // -------------------------------------------------- dY
      const bool one = elect_one();
      uint32_t it = 0;
      for (int u = worker; u < units; u += workers) {
        const Unit w = unit_at(u);
        const int n = w.n0 + (int)rank * 128;
        for (int kb = w.kb0; kb < w.kb1; ++kb, ++it) {
          const uint32_t s = it % C::STAGES, ph = (it / C::STAGES) & 1u;
          if (!__all_sync(0xffffffffu, mbar_wait(empty(s), ph ^ 1u, abort_flag, p.status, 1))) { ok = false; goto fed; }
          if (one) {
            if (leader) mbar_arrive_expect_tx(full(s), 2 * C::A_BYTES);
            const uint32_t fb = map_to_cta(full(s), 0u), dst = base + s * C::STAGE_BYTES;
            tma_load_2d_pair(dst, &tmY, n, kb * C::BK, fb);
            tma_load_2d_pair(dst + C::BK * 128, &tmY, n + 64, kb * C::BK, fb);
          }
        }
      }
    } else if (warp >= 2) {
      // -------------------------------------------------- codes and scales: one warp for each half of the blocks
      const bool one = elect_one();
      uint32_t it = 0;
      for (int u = worker; u < units; u += workers) {
        const Unit w = unit_at(u);
        const int h = w.h0 + (int)rank * 128;
        for (int kb = w.kb0; kb < w.kb1; ++kb, ++it) {
          const uint32_t s = (2 * it + warp - 2) % C::RAW, ph = (2 * it / C::RAW) & 1u;
          if (!__all_sync(0xffffffffu, mbar_wait(rempty(s), ph ^ 1u, abort_flag, p.status, 2))) { ok = false; goto fed; }
          if (one) {
            mbar_arrive_expect_tx(rfull(s), C::RAW_BYTES);
            const uint32_t dst = raw0 + s * C::RAW_BYTES;
            const int t = kb * C::BK + (warp - 2) * C::RAW_T;
            tma_load_2d(dst, &tmCodes, h, t, rfull(s));
            tma_load_2d(dst + C::CODE_BYTES, &tmScales, (h / 32) & ~15, t, rfull(s));
          }
        }
      }
    } else if (warp == 1 && leader) {
      // -------------------------------------------------- products
      const uint32_t idesc = make_idesc_bf16(C::TILE, C::TILE, 1u, 1u);
      constexpr uint32_t STEP = (16 * 128) >> 4;               // 16 tokens further in an MN-major tile
      const uint64_t a_proto = make_smem_desc(base, C::BK * 128, 1024);
      const uint64_t b_proto = make_smem_desc(base + C::A_BYTES, C::BK * 128, 1024);
      const uint32_t a_hi = (uint32_t)(a_proto >> 32), a_lo0 = (uint32_t)a_proto;
      const uint32_t b_hi = (uint32_t)(b_proto >> 32), b_lo0 = (uint32_t)b_proto;
      auto desc = [](uint32_t lo, uint32_t hi) { return (static_cast<uint64_t>(hi) << 32) | lo; };
      uint32_t s = 0, ph = 0, run = 0;
      const bool one = elect_one();
      for (int u = worker; u < units; u += workers) {
        const Unit w = unit_at(u);
        for (int k0 = w.kb0; k0 < w.kb1; k0 += C::RUN, ++run) {
          const uint32_t acc = run & 1u, aph = (run >> 1) & 1u;
          if (!__all_sync(0xffffffffu, mbar_wait<true>(tempty(acc), aph ^ 1u, abort_flag, p.status, 3))) goto fed;
          const uint32_t d = tmem + acc * C::TILE;
          uint32_t add = 0u;
          for (int n = (w.kb1 - k0 < C::RUN ? w.kb1 - k0 : C::RUN); n > 0; --n) {
            if (!__all_sync(0xffffffffu, mbar_wait<true>(full(s), ph, abort_flag, p.status, 4))) goto fed;
            tc_fence_after();
            const uint32_t at = s * (C::STAGE_BYTES >> 4);
            if (one) {
#pragma unroll
              for (int j = 0; j < C::BK / 16; ++j) {
                umma_bf16_pair(d, desc(a_lo0 + at + j * STEP, a_hi), desc(b_lo0 + at + j * STEP, b_hi), idesc, add);
                add = 1u;
              }
              umma_commit_pair(empty(s));
            }
            add = 1u;
            s = s + 1 == C::STAGES ? 0u : s + 1;
            ph ^= s == 0u ? 1u : 0u;
          }
          if (one) umma_commit_pair(tfull(acc));
        }
      }
    }
  fed:
    if (warp != 1 && lane == 0 && !ok) {        // aborted: copies in flight get a bounded time to land
      const uint64_t t0 = globaltimer_ns();
      while (globaltimer_ns() - t0 < 2000000ull) {}
    }
  } else if (warp < 4 + C::CONVERT_WARPS) {
    regs_dec<C::REGS_CONVERT>();
    // ---------------------------------------------------- codes -> bf16
    // A block is converted by a team of warps, successive blocks by successive teams, so that their waits overlap.
    // A thread takes 16 columns of a token at a time: eight lanes read the 128 code bytes of a token and write two
    // 128-byte lines of the operand tile, one per 64 columns (chunk c of line t sits at c ^ (t & 7)). The lanes of the
    // second line write their odd chunk first, so that eight lanes always meet all 32 banks once.
    const int team = (warp - 4) / C::CONVERT_TEAM, member = (warp - 4) % C::CONVERT_TEAM;
    const int q = lane & 7;                                    // columns 16 q .. 16 q + 15
    constexpr int T_STEP = 4 * C::CONVERT_TEAM, ITEMS = C::RAW_T / T_STEP;
    static_assert(T_STEP % 8 == 0, "t & 7 is the same for all items of a thread");
    const int t0 = member * 4 + (lane >> 3);
    const uint32_t line = (uint32_t)(q >> 2) * (C::BK * 128) + t0 * 128;
    const int odd = q >> 2;                                    // which of its two chunks a thread writes first
    const uint32_t dst0 = line + ((((q & 3) * 2 + odd) ^ (t0 & 7)) << 4), dst1 = line + ((((q & 3) * 2 + 1 - odd) ^ (t0 & 7)) << 4);
    uint32_t it = 0;
    for (int u = worker; u < units && ok; u += workers) {
      const Unit w = unit_at(u);
      const uint32_t src = raw0 + t0 * 128 + q * 16;
      const uint32_t src_scale = raw0 + C::CODE_BYTES + t0 * 16 + (((w.h0 + (int)rank * 128) / 32) & 15) + (q >> 1);
      for (int kb = w.kb0; kb < w.kb1; ++kb, ++it) {
        if ((int)(it % C::TEAMS) != team) continue;
        const uint32_t s = it % C::STAGES, ph = (it / C::STAGES) & 1u;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const uint32_t r = (2 * it + half) % C::RAW, rph = ((2 * it + half) / C::RAW) & 1u;
          bool here = mbar_wait(rfull(r), rph, abort_flag, p.status, 6);
          uint4 codes[ITEMS];
          uint32_t bytes[ITEMS];
          const uint32_t from = src + r * C::RAW_BYTES, from_scale = src_scale + r * C::RAW_BYTES;
#pragma unroll
          for (int j = 0; j < ITEMS; ++j) {
            codes[j] = ld_shared_v4(from + T_STEP * 128 * j);
            bytes[j] = ld_shared_u8(from_scale + T_STEP * 16 * j);
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(rempty(r));
          if (half == 0) here = here && mbar_wait(empty(s), ph ^ 1u, abort_flag, p.status, 7);
          ok = ok && __all_sync(0xffffffffu, here);
          if (!ok) break;
          const uint32_t tile = base + s * C::STAGE_BYTES + C::A_BYTES + half * (C::RAW_T * 128);
#pragma unroll
          for (int j = 0; j < ITEMS; ++j) {
            const uint4 c = codes[j];
            uint32_t o[8];
            codes_to_bf16x16<FMT>(odd ? make_uint4(c.z, c.w, c.x, c.y) : c, bytes[j], o);
            const uint32_t at = tile + T_STEP * 128 * j;
            st_shared_v4(at + dst0, o[0], o[1], o[2], o[3]);
            st_shared_v4(at + dst1, o[4], o[5], o[6], o[7]);
          }
        }
        if (!ok) break;
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive_pair(map_to_cta(full(s), 0u));
      }
    }
  } else {
    regs_inc<C::REGS_SUM>();
    // ---------------------------------------------------- sums and output
    const int sw = warp - 4 - C::CONVERT_WARPS;
    const int lg = warp & 3;                                   // tensor memory lanes this warp may read
    const int col_half = (sw >> 2) * 128;
    const uint32_t box = box0 + sw * C::BOX_BYTES;
    float sum[128];
    uint32_t run = 0;
    for (int u = worker; u < units && ok; u += workers) {
      const Unit w = unit_at(u);
#pragma unroll
      for (int j = 0; j < 128; ++j) sum[j] = 0.f;              // (a part may be empty)
      for (int k0 = w.kb0; k0 < w.kb1; k0 += C::RUN, ++run) {
        const uint32_t acc = run & 1u, aph = (run >> 1) & 1u;
        const bool here = mbar_wait(tfull(acc), aph, abort_flag, p.status, 8);
        if (!__all_sync(0xffffffffu, here)) { ok = false; break; }
        tc_fence_after();
        const uint32_t taddr = tmem + (uint32_t(lg * 32) << 16) + acc * C::TILE + col_half;
#pragma unroll
        for (int v = 0; v < 8; ++v) {
          uint32_t r[16];
          tmem_ld16(taddr + v * 16, r);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 16; ++j) sum[v * 16 + j] += __uint_as_float(r[j]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_pair(map_to_cta(tempty(acc), 0u));
      }
      if (!ok) break;
      // Boxes of 32 rows x 128 bytes, to the result or to the unit's slab.
      const int row0 = w.n0 + (int)rank * 128 + lg * 32, col0 = w.h0 + col_half;
      auto send = [&](const CUtensorMap* map, int x, int y, bool add) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (add) tma_reduce_add_2d(map, box, x, y); else tma_store_2d(map, box, x, y);
          bulk_commit();
        }
      };
      const bool to_slab = w.slab >= 0;
      if (F32_OUT || to_slab) {
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          if (row0 < p.N && col0 + b * 32 < p.H) {             // uniform over the warp
            if (lane == 0) bulk_wait_read<0>();
            __syncwarp();
#pragma unroll
            for (int ch = 0; ch < 8; ++ch) {
              uint32_t v[4];                                   // volatile: copies made here do not pile up in registers
#pragma unroll
              for (int j = 0; j < 4; ++j) asm volatile("mov.b32 %0, %1;" : "=r"(v[j]) : "f"(sum[b * 32 + ch * 4 + j]));
              st_shared_v4(box + lane * 128 + ((ch ^ (lane & 7)) << 4), v[0], v[1], v[2], v[3]);
            }
            if (to_slab) send(&tmSlab, col_half + b * 32, w.slab * C::TILE + (int)rank * 128 + lg * 32, false);
            else send(&tmOut, col0 + b * 32, row0, p.accumulate != 0);
          }
        }
      } else {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          if (row0 < p.N && col0 + b * 64 < p.H) {
            if (lane == 0) bulk_wait_read<0>();
            __syncwarp();
#pragma unroll
            for (int ch = 0; ch < 8; ++ch) {
              if (p.accumulate) {                              // += in bf16: the old values first, rounded once after
                const int col = col0 + b * 64 + ch * 8;
                float old[8];
                if (row0 + lane < p.N && col < p.H) {          // H % 8 == 0
                  load8<__nv_bfloat16, true>(p.out + (long long)(row0 + lane) * p.H, col, p.H, old);
#pragma unroll
                  for (int j = 0; j < 8; ++j) sum[b * 64 + ch * 8 + j] += old[j];
                }
              }
              uint32_t v[4];
#pragma unroll
              for (int j = 0; j < 4; ++j)
                asm volatile("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(v[j])
                             : "f"(sum[b * 64 + ch * 8 + 2 * j + 1]), "f"(sum[b * 64 + ch * 8 + 2 * j]));
              st_shared_v4(box + lane * 128 + ((ch ^ (lane & 7)) << 4), v[0], v[1], v[2], v[3]);
            }
            send(&tmOut, col0 + b * 64, row0, false);
          }
        }
      }
    }
    if (lane == 0) bulk_wait_all();
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                                          // neither CTA leaves while the other may reach its barriers
  tc_fence_after();
  if (warp == 1) tmem_dealloc_pair(tmem, 512);
}

// The tiles that were cut: out (= or +=) slab 0 + slab 1 + ... in that order, rounded once. One block per 8 rows of a
// tile, 32 threads a row. H % 8 == 0. Starts while the products drain and waits for them before it reads.
__global__ void __launch_bounds__(256)
act8_dweight_join_kernel(const float* slabs, int whole, int parts, int h_tiles, int N, int H,
                         void* out, int type, int accumulate) {
  const int i = blockIdx.x >> 5, r = (blockIdx.x & 31) * 8 + (threadIdx.x >> 5), c = (threadIdx.x & 31) * 8;
  const int tile = whole + i, row = (tile / h_tiles) * 256 + r, col = (tile % h_tiles) * 256 + c;
  const float* src = slabs + ((long long)i * parts * 256 + r) * 256 + c;
  grid_dependents_launch();
  grid_dependency_wait();
  if (row >= N || col >= H) return;
  float f[8] = {};
  for (int q = 0; q < parts; ++q) {          // (from L2: the lines were written while this kernel was starting)
    const float4 a = __ldcg(reinterpret_cast<const float4*>(src + (long long)q * 65536));
    const float4 b = __ldcg(reinterpret_cast<const float4*>(src + (long long)q * 65536) + 1);
    f[0] += a.x; f[1] += a.y; f[2] += a.z; f[3] += a.w; f[4] += b.x; f[5] += b.y; f[6] += b.z; f[7] += b.w;
  }
  const long long at = (long long)row * H + col;
  if (type == 1) {
    float* o = reinterpret_cast<float*>(out) + at;
    if (accumulate) {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] += o[j];
    }
    store_raw8<float, true>(o, 0, 8, f32_to_raw<float>(f));
  } else {
    __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(out) + at;
    if (accumulate) {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] += __bfloat162float(o[j]);
    }
    store_raw8<__nv_bfloat16, true>(o, 0, 8, f32_to_raw<__nv_bfloat16>(f));
  }
}

}  // namespace kdkl
