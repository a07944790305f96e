// The 4-bit matrix product C = act(A B^T + bias), A and B in e2m1 with a
// power-of-two scale per block of 32 along the contraction.  The tensor cores
// apply the scales themselves (kind::mxf4), so a tile is one fp32 accumulator
// in TMEM over the whole contraction.  Large products run on CTA pairs
// (k_fp4_pair), the others on single CTAs that may split the contraction
// (k_fp4_split).
//
// A ring stage is 256 contraction indices: one 128-byte swizzled row of packed
// e2m1 pairs per operand row, and two scale tiles (512 bytes: 128 rows x 4
// blocks of 32) per 128 operand rows, which one thread copies on to TMEM ahead
// of the stage's four MMAs (K = 64).  Each ring stage has TMEM columns of its own
// for them, so that the copies wait for nothing but the stage (with columns for
// two stages in turn each MMA waited for the one before the last to be
// reported: 1 x 8192 x 8192 9.7 us, 4096 x 8192 x 8192 77).
//
// Every mbarrier wait is bounded; one that runs out latches DEVERR_TIMEOUT in
// the call's status word, stops the other roles, and the CTA lets its
// copies and MMAs land before it frees TMEM and exits.
#include <algorithm>
#include <cmath>

#include "ff_api_internal.h"
#include "ff_fp4.h"
#include "ff_ptx.cuh"

namespace ff {
namespace {

constexpr int KS = 256;             // contraction indices per ring stage
constexpr int KB = KS / 2;          // bytes of an operand row per ring stage
constexpr int BM = 128;             // rows of an accumulator: the TMEM lanes
constexpr int SF = 2 * kFp4ScaleTile;  // bytes of a stage's scales for 128 operand rows
constexpr int SFC = 8;              // TMEM columns they take
constexpr int SF_BOX = SF / 4;      // and the words a copy's box has of them
constexpr int EPI = 8;              // epilogue warps
constexpr int THREADS = 64 + 32 * EPI;
static_assert(KB % 16 == 0 && SF % 16 == 0, "every tiled copy starts a multiple of 16 bytes into its row");

__device__ __forceinline__ void latch(int* err, volatile int* abort_flag) {
  *abort_flag = 1;
  atomicOr(err, DEVERR_TIMEOUT);
}
__device__ __forceinline__ float finish(float v, int relu) { return relu && v < 0.f ? 0.f : v; }  // keeps NaN
__device__ __forceinline__ void pause_1ms() {  // MMAs and copies issued before an abort land in bounded time
  const uint64_t t0 = ptx::globaltimer();
  while (ptx::globaltimer() - t0 < 1000000ull) {
  }
}

struct Args {
  int P, Q, K;               // rows of the operand on the TMEM lanes (P) and on the columns (Q)
  const float* bias;
  int relu, out_bf16, swap;  // swap: the lanes are C's columns (P = N, Q = M)
  void* c;
  long long ldc;
  int* err;
  int ntp, ntq;              // tiles
};

// MMAs of K = 64 in stage `s` of a contraction of K indices.
__device__ __forceinline__ int steps_of(int K, int s) { return min(KS / 64, (K - s * KS + 63) / 64); }

// ------------------------------------------------------- large products
constexpr int LSTAGING = 32 * 128;  // per epilogue warp: a block of 32 rows x 128 bytes of C

// CTA pairs (cta_group::2) on 256 x LN tiles: each CTA loads 128 rows of A and
// half of B's LN columns per stage, the scales of its rows and those of all LN
// columns (LN = 256: 35 KB for 8.4 MMAC a CTA), and holds 128 x LN of the accumulator:
// half of its TMEM, the rest of which cannot hold a second one beside the
// scales.  So the epilogue warps first read all of it into registers (128
// columns each), hand it back, and convert and store under the next tile's
// MMAs.  Persistent: the copies run ahead over the tiles.  Warps: 0 producer,
// 1 MMAs (the even CTA's), 2..9 epilogue.
//
// Bound by the MMAs: 4096 x 8192 x 8192, bf16 C 76 us, 7.2 PFLOP/s, 0.93 of four times the
// measured bf16 burst rate.  With a short contraction by the stores, since the
// epilogue warps hold a tile about 2 us (4096 x 8192 x 600, bf16 C: 22 us).
//
// LN columns a tile: 128 where tiles of 256 would leave pairs without one (their
// MMAs read A twice as often for their operations; 1846 x 1127 x 5259: 10.8 us for 13.5).
template <int LN>
struct LCfg {
  static constexpr int STAGES = LN == 256 ? 5 : 7;  // (256: 4, and two staging blocks a warp: 87 us for 77 at 4096 x 8192 x 8192)
  static constexpr int A = BM * KB, B = LN / 2 * KB;  // bytes of a stage's operands
  static constexpr int SB = LN / 128;                 // scale tiles' rows of B's columns
  static constexpr int STAGE = A + B + SF + SB * SF;
  static constexpr int CPW = LN / 2;                  // columns per epilogue warp
  static constexpr uint32_t SCOLS = SFC + SB * SFC;   // TMEM columns of a stage's scales
  static_assert(LN + STAGES * SCOLS <= 512, "the accumulator and the stages' scales");
  static_assert(STAGE % 1024 == 0, "swizzled tiles start on 1024 bytes");
  static constexpr int SMEM = 1024 + STAGES * STAGE + EPI * LSTAGING + EPI * CPW * 4 + 512;
  static_assert(SMEM > 113 * 1024 && SMEM <= 227 * 1024, "one GEMM CTA per SM, so that no TMEM allocation waits on another's");
};

// Tile t of the raster: groups of 8 row tiles, columns outermost within a
// group, so that the tiles in flight share operand panels in L2.
__device__ __forceinline__ void tile_of(int t, int ntp, int ntq, int& tp, int& tq) {
  constexpr int GROUP = 8;
  const int per = GROUP * ntq, g = t / per, in = t - g * per;
  const int rows = min(GROUP, ntp - g * GROUP);
  tp = g * GROUP + in % rows;
  tq = in / rows;
}

// A warp writes a staged block of 32 rows x 128 bytes (16-byte units swizzled
// by the row) to C, `rows` and `left` of its rows and columns being there, the
// lanes along a row.
template <typename U>
__device__ __forceinline__ void rows_out(uint32_t from, U* c, long long ldc, int rows, int left, int lane) {
  constexpr int J = 128 / 32 / (int)sizeof(U);
  c += lane;
#pragma unroll
  for (int r0 = 0; r0 < 32; r0 += 8) {
    uint32_t v[8][J];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int byte = (lane + 32 * j) * (int)sizeof(U);
        const uint32_t at = from + (r0 + i) * 128 + (((byte >> 4) ^ i) << 4) + (byte & 15);
        if constexpr (sizeof(U) == 4)
          asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v[i][j]) : "r"(at));
        else
          asm volatile("{\n\t.reg .u16 h;\n\tld.shared.u16 h, [%1];\n\tcvt.u32.u16 %0, h;\n\t}" : "=r"(v[i][j]) : "r"(at));
      }
    if (rows >= 32 && left >= 32 * J) {
#pragma unroll
      for (int i = 0; i < 8; ++i, c += ldc)
#pragma unroll
        for (int j = 0; j < J; ++j) c[32 * j] = (U)v[i][j];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i, c += ldc)
#pragma unroll
        for (int j = 0; j < J; ++j)
          if (r0 + i < rows && lane + 32 * j < left) c[32 * j] = (U)v[i][j];
    }
  }
}

// TMA_C: C's rows are 16-byte aligned and go out by TMA.  BF16: C's type.
template <int LN, bool TMA_C, bool BF16>
__global__ void __launch_bounds__(THREADS, 1)
    k_fp4_pair(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
               const __grid_constant__ CUtensorMap tmSA, const __grid_constant__ CUtensorMap tmSB,
               const __grid_constant__ CUtensorMap tmC, Args g) {
  using C = LCfg<LN>;
  constexpr int LSTAGES = C::STAGES, LSTAGE = C::STAGE, LA = C::A, LB = C::B, LCPW = C::CPW;
  constexpr uint32_t LSFC = C::SCOLS;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_s = ptx::smem_u32(smem_raw);
  uint8_t* smem = smem_raw + ((1024u - (raw_s & 1023u)) & 1023u);
  uint8_t* staging = smem + LSTAGES * LSTAGE;
  float* sbias = reinterpret_cast<float*>(staging + EPI * LSTAGING);  // [epilogue warp][LCPW]
  uint64_t* full = reinterpret_cast<uint64_t*>(sbias + EPI * LCPW);
  uint64_t* empty = full + LSTAGES;
  uint64_t* tfull = empty + LSTAGES;   // a tile's products are done
  uint64_t* tempty = tfull + 1;        // both CTAs have read them
  uint32_t* tslot = reinterpret_cast<uint32_t*>(tempty + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tslot + 1);
  volatile int* never_set = reinterpret_cast<volatile int*>(tslot + 2);
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const uint32_t crank = ptx::cluster_ctarank();
  const bool lead = crank == 0;
  const int nkb = (g.K + KS - 1) / KS;
  const int ntiles = g.ntp * g.ntq;
  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < LSTAGES; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    ptx::mbar_init(tfull, 1);
    ptx::mbar_init(tempty, 2 * EPI);
    *abort_flag = 0;
    *never_set = 0;
    ptx::fence_mbar_init();
    ptx::prefetch_tmap(&tmA);
    ptx::prefetch_tmap(&tmB);
    ptx::prefetch_tmap(&tmSA);
    ptx::prefetch_tmap(&tmSB);
    ptx::prefetch_tmap(&tmC);
  }
  if (warp == 1) {
    ptx::tmem_alloc_pair(tslot, 512);
    ptx::tmem_relinquish_pair();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::cluster_sync();
  ptx::tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tslot, 0);
  ptx::griddep_wait();

  if (warp == 0) {
    if (lane == 0) {
      const uint32_t full0 = ptx::mapa_shared(ptx::smem_u32(&full[0]), 0);
      int it = 0;
      for (int t = pair; t < ntiles && !*abort_flag; t += npairs) {
        int tp, tq;
        tile_of(t, g.ntp, g.ntq, tp, tq);
        const int ar = tp * 2 * BM + (int)crank * BM, br = tq * LN + (int)crank * (LN / 2);
        for (int kb = 0; kb < nkb; ++kb, ++it) {
          const int s = it % LSTAGES;
          if (!ptx::mbar_wait(&empty[s], (((uint32_t)(it / LSTAGES)) & 1u) ^ 1u, kWaitTimeoutNs, abort_flag)) {
            latch(g.err, abort_flag);
            break;
          }
          if (lead) ptx::mbar_arrive_expect_tx(&full[s], 2 * LSTAGE);
          uint8_t* a = smem + s * LSTAGE;
          const uint32_t bar = full0 + 8u * (uint32_t)s;
          ptx::tma_load_2d_pair(a, &tmA, bar, kb * KB, ar);
          ptx::tma_load_2d_pair(a + LA, &tmB, bar, kb * KB, br);
          ptx::tma_load_2d_pair(a + LA + LB, &tmSA, bar, kb * SF_BOX, tp * 2 + (int)crank);
          ptx::tma_load_2d_pair(a + LA + LB + SF, &tmSB, bar, kb * SF_BOX, tq * C::SB);
        }
      }
      if (!*abort_flag) {
        // the last stages' commits arrive here before the CTA goes away
        for (int k = it; k < it + LSTAGES; ++k)
          if (!ptx::mbar_wait(&empty[k % LSTAGES], (((uint32_t)(k / LSTAGES)) & 1u) ^ 1u, kWaitTimeoutNs, abort_flag)) {
            latch(g.err, abort_flag);
            break;
          }
      }
      if (*abort_flag) {
        // Copies issued earlier land before the shared memory goes away: on
        // this CTA's own barriers (the pair's even CTA), or in bounded time.
        if (lead) {
          for (int k = it < LSTAGES ? 0 : it - LSTAGES; k < it; ++k)
            ptx::mbar_wait(&full[k % LSTAGES], (uint32_t)(k / LSTAGES) & 1u, 10000000ull, never_set);
        } else {
          pause_1ms();
        }
      }
    }
  } else if (warp == 1) {
    if (lead) {
      // The whole warp walks the loop, so that its variables are uniform, and
      // one lane issues.  Descriptors differ from the first stage's by their
      // address field only (16-byte units).
      constexpr uint32_t idesc[2] = {ptx::idesc_mxf4(2 * BM, LN, 0), ptx::idesc_mxf4(2 * BM, LN, 2)};
      const uint64_t ad0 = ptx::sdesc_sw128(ptx::smem_u32(smem), 16, 1024);
      const uint64_t bd0 = ptx::sdesc_sw128(ptx::smem_u32(smem + LA), 16, 1024);
      const uint64_t sd0 = ptx::sdesc_rows16(ptx::smem_u32(smem + LA + LB));
      const int last_steps = steps_of(g.K, nkb - 1);
      int it = 0;
      uint32_t tile = 0;
      bool live = true;
      for (int t = pair; t < ntiles && live; t += npairs, ++tile) {
        bool ok = ptx::mbar_wait_cluster(tempty, (tile & 1u) ^ 1u, kWaitTimeoutNs, abort_flag);
        for (int kb = 0; kb < nkb; ++kb, ++it) {
          const int s = it % LSTAGES;
          ok = ok && ptx::mbar_wait(&full[s], (uint32_t)(it / LSTAGES) & 1u, kWaitTimeoutNs, abort_flag);
          if (!__all_sync(0xffffffffu, ok)) {
            latch(g.err, abort_flag);
            live = false;
            break;
          }
          ptx::tc_fence_after();
          const uint64_t at = (uint64_t)(s * (LSTAGE >> 4));
          const uint32_t sfa = tmem + LN + (uint32_t)s * LSFC, sfb = sfa + SFC;
          const int steps = kb == nkb - 1 ? last_steps : KS / 64;
          if (ptx::elect_one()) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint64_t from = sd0 + at + h * (kFp4ScaleTile >> 4);
              ptx::tmem_cp_rows16_pair(sfa + 4 * h, from);
#pragma unroll
              for (int r = 0; r < C::SB; ++r)
                ptx::tmem_cp_rows16_pair(sfb + (h * C::SB + r) * 4, from + ((r + 1) * SF >> 4));
            }
#pragma unroll
            for (int k = 0; k < KS / 64; ++k)
              if (k < steps)
                ptx::umma_mxf4_pair(tmem, ad0 + at + 2 * k, bd0 + at + 2 * k, idesc[k & 1], sfa + 4 * (k / 2), sfb + C::SB * 4 * (k / 2),
                                    kb > 0 || k > 0);
            ptx::umma_commit_pair(&empty[s], 3);
            if (kb == nkb - 1) ptx::umma_commit_pair(tfull, 3);
          }
          __syncwarp();
        }
      }
    }
  } else {
    const int q = warp & 3, ew = warp - 2, half = ew >> 2;
    const uint32_t trow = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(half * LCPW);
    const uint32_t te0 = ptx::mapa_shared(ptx::smem_u32(tempty), 0);
    uint8_t* stage = staging + ew * LSTAGING;
    float* bias = sbias + ew * LCPW;
    uint32_t tile = 0;
    for (int t = pair; t < ntiles; t += npairs, ++tile) {
      int tp, tq;
      tile_of(t, g.ntp, g.ntq, tp, tq);
      const int rbase = tp * 2 * BM + (int)crank * BM + q * 32;
      const int cbase = tq * LN + half * LCPW;
      __syncwarp();  // the last tile's bias has been read
#pragma unroll
      for (int e = 0; e < LCPW; e += 32)
        bias[e + lane] = g.bias && cbase + e + lane < g.Q ? __ldg(g.bias + cbase + e + lane) : 0.f;
      const bool ok = ptx::mbar_wait(tfull, tile & 1u, 4 * kWaitTimeoutNs, abort_flag);
      if (!ok) latch(g.err, abort_flag);
      if (!__all_sync(0xffffffffu, ok)) break;
      ptx::tc_fence_after();
      uint32_t acc[LCPW / 32][32];
#pragma unroll
      for (int c = 0; c < LCPW / 32; ++c) ptx::tmem_ld32(trow + c * 32, acc[c]);
#pragma unroll
      for (int c = 0; c < LCPW / 32; ++c) ptx::tmem_ld_wait_for(acc[c]);
      ptx::tc_fence_before();
      __syncwarp();
      // TMEM reads that have completed: nothing to release, only an arrival
      if (lane == 0) ptx::mbar_arrive_at(te0);
      if (t + npairs >= ntiles && threadIdx.x == 64) ptx::griddep_launch_dependents();
      // Store: 128 bytes of each of the warp's 32 rows at a time through the
      // swizzled staging block, by TMA where C's rows are 16-byte aligned (it
      // clips what lies past the matrix, and the warp need not wait for the
      // memory), else by the lanes along a row, eight rows read before the
      // first is written.
      auto block = [&]() {  // the staging block, free again
        if (TMA_C && lane == 0) ptx::bulk_wait_read0();
        __syncwarp();
        return stage;
      };
      auto flush = [&](uint8_t* from, int col0) {  // the staged columns of C from col0 on
        if constexpr (TMA_C) {
          ptx::fence_async_smem();
          __syncwarp();
          if (lane == 0) {
            if (rbase < g.P && col0 < g.Q) ptx::tma_store_2d(&tmC, from, col0, rbase);
            ptx::bulk_commit();
          }
        } else {
          __syncwarp();
          const int rows = g.P - rbase, left = g.Q - col0;
          const long long at = (long long)rbase * g.ldc + col0;
          if constexpr (BF16)
            rows_out(ptx::smem_u32(from), static_cast<uint16_t*>(g.c) + at, g.ldc, rows, left, lane);
          else
            rows_out(ptx::smem_u32(from), static_cast<uint32_t*>(g.c) + at, g.ldc, rows, left, lane);
        }
      };
      // four accumulators with bias and activation
      auto value = [&](int i) {
        const float4 v = *reinterpret_cast<const float4*>(bias + i);
        const uint32_t* r = acc[i / 32] + i % 32;
        return make_float4(finish(__uint_as_float(r[0]) + v.x, g.relu), finish(__uint_as_float(r[1]) + v.y, g.relu),
                           finish(__uint_as_float(r[2]) + v.z, g.relu), finish(__uint_as_float(r[3]) + v.w, g.relu));
      };
      if constexpr (BF16) {
#pragma unroll
        for (int ch = 0; ch < LCPW / 64; ++ch) {
          uint8_t* to = block();
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            const float4 v = value(ch * 64 + u * 8), w = value(ch * 64 + u * 8 + 4);
            const __nv_bfloat162 h[4] = {__floats2bfloat162_rn(v.x, v.y), __floats2bfloat162_rn(v.z, v.w),
                                         __floats2bfloat162_rn(w.x, w.y), __floats2bfloat162_rn(w.z, w.w)};
            *reinterpret_cast<uint4*>(to + lane * 128 + ((u ^ (lane & 7)) << 4)) = *reinterpret_cast<const uint4*>(h);
          }
          flush(to, cbase + ch * 64);
        }
      } else {
#pragma unroll
        for (int ch = 0; ch < LCPW / 32; ++ch) {
          uint8_t* to = block();
#pragma unroll
          for (int u = 0; u < 8; ++u)
            *reinterpret_cast<float4*>(to + lane * 128 + ((u ^ (lane & 7)) << 4)) = value(ch * 32 + u * 4);
          flush(to, cbase + ch * 32);
        }
      }
    }
    if (TMA_C && lane == 0) ptx::bulk_wait_read0();
    __syncwarp();
  }

  ptx::tc_fence_before();
  __syncthreads();
  if (*abort_flag) pause_1ms();  // MMAs issued before the abort finish before TMEM is released
  __syncwarp();
  ptx::cluster_sync();
  ptx::tc_fence_after();
  if (warp == 1) ptx::tmem_dealloc_pair(tmem, 512);
}

// ------------------------------------------------------- small products
// One CTA per 128 x BN tile and slice of the contraction: the CTAs of a
// cluster (1, 2, 4 or 8) share a tile's stages, exchange their partial sums
// through distributed shared memory (each sums its share of the columns, in
// rank order) and store.  With few rows of A its rows go on the MMA's columns
// (swap), so that a single row needs 16 columns and not 128 lanes.  Bound by the
// weights' bytes where they are many (1 x 8192 x 8192: 9.3 us from HBM, 3.8 TB/s, of which
// launch, ring fill, exchange and store are some 4 us), else by these steps' latency
// (1 x 10 x 2000: 3.3 us).  Roles:
//
//   warp 0      TMA producer
//   warp 1      allocates TMEM, one lane copies the scales and issues the MMAs
//   warps 2..9  epilogue: TMEM lane quarter warp % 4, half of the columns each
//
// A tile takes its columns' scales from a whole scale tile of 128, from TMEM
// column (q0 % 128) / 32 of it on, which must be even: BN < 64 serves products of
// one column tile only.
template <int BN>
struct SCfg {
  static constexpr int STAGE = (BM + BN) * KB + 2 * SF;
  static constexpr int STAGES = BN >= 64 ? 8 : 9;
  static constexpr int CPW = BN / 2;
  static constexpr uint32_t ACC = BN < 32 ? 32 : BN;       // TMEM columns of the accumulator
  static constexpr uint32_t TCOLS = 256;
  static_assert(ACC + 2 * SFC * STAGES <= TCOLS, "the accumulator and the stages' scales");
  static constexpr int PITCH = BM + 1;                     // floats per column of the exchange buffer
  static constexpr int SMEM = 1024 + STAGES * STAGE + 512;
  static_assert(SMEM > 113 * 1024 && SMEM <= 227 * 1024, "one GEMM CTA per SM, so that no TMEM allocation waits on another's");
  static_assert(BN * PITCH * 4 <= STAGES * STAGE, "the exchange buffer lies over the ring");
  static_assert(STAGE % 1024 == 0, "swizzled tiles start on 1024 bytes");
};

template <int BN>
__global__ void __launch_bounds__(THREADS, 1)
    k_fp4_split(const __grid_constant__ CUtensorMap tmP, const __grid_constant__ CUtensorMap tmQ,
                const __grid_constant__ CUtensorMap tmSP, const __grid_constant__ CUtensorMap tmSQ, Args g, int ks_log) {
  using C = SCfg<BN>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_s = ptx::smem_u32(smem_raw);
  uint8_t* smem = smem_raw + ((1024u - (raw_s & 1023u)) & 1023u);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::STAGES * C::STAGE);
  uint64_t* empty = full + C::STAGES;
  uint64_t* done = empty + C::STAGES;
  uint32_t* tslot = reinterpret_cast<uint32_t*>(done + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tslot + 1);
  volatile int* never_set = reinterpret_cast<volatile int*>(tslot + 2);
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int ks = 1 << ks_log;
  const int rank = (int)(blockIdx.x & (unsigned)(ks - 1));
  const int tile = (int)(blockIdx.x >> ks_log);
  const int p0 = (tile % g.ntp) * BM, q0 = (tile / g.ntp) * BN;
  const int nkb_all = (g.K + KS - 1) / KS;
  const int kb0 = (int)((long long)nkb_all * rank >> ks_log), kb1 = (int)((long long)nkb_all * (rank + 1) >> ks_log);
  const int nkb = kb1 - kb0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::STAGES; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    ptx::mbar_init(done, 1);
    *abort_flag = 0;
    *never_set = 0;
    ptx::fence_mbar_init();
    ptx::prefetch_tmap(&tmP);
    ptx::prefetch_tmap(&tmQ);
    ptx::prefetch_tmap(&tmSP);
    ptx::prefetch_tmap(&tmSQ);
  }
  if (warp == 1) {
    ptx::tmem_alloc(tslot, C::TCOLS);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tslot, 0);
  ptx::griddep_wait();

  const int q = warp & 3, ew = warp - 2, half = ew >> 2;
  float acc[C::CPW];
#pragma unroll
  for (int i = 0; i < C::CPW; ++i) acc[i] = 0.f;

  if (warp == 0) {
    if (lane == 0) {
      int it = 0;
      for (; it < nkb; ++it) {
        const int s = it % C::STAGES;
        if (!ptx::mbar_wait(&empty[s], (((uint32_t)(it / C::STAGES)) & 1u) ^ 1u, kWaitTimeoutNs, abort_flag)) {
          latch(g.err, abort_flag);
          break;
        }
        ptx::mbar_arrive_expect_tx(&full[s], C::STAGE);
        uint8_t* a = smem + s * C::STAGE;
        ptx::tma_load_2d(a, &tmP, &full[s], (kb0 + it) * KB, p0);
        ptx::tma_load_2d(a + BM * KB, &tmQ, &full[s], (kb0 + it) * KB, q0);
        ptx::tma_load_2d(a + (BM + BN) * KB, &tmSP, &full[s], (kb0 + it) * SF_BOX, p0 / 128);
        ptx::tma_load_2d(a + (BM + BN) * KB + SF, &tmSQ, &full[s], (kb0 + it) * SF_BOX, q0 / 128);
      }
      if (*abort_flag)
        for (int k = it < C::STAGES ? 0 : it - C::STAGES; k < it; ++k)
          ptx::mbar_wait(&full[k % C::STAGES], (uint32_t)(k / C::STAGES) & 1u, 10000000ull, never_set);
    }
  } else if (warp == 1) {
    constexpr uint32_t idesc[2] = {ptx::idesc_mxf4(BM, BN, 0), ptx::idesc_mxf4(BM, BN, 2)};
    const uint64_t pd0 = ptx::sdesc_sw128(ptx::smem_u32(smem), 16, 1024);
    const uint64_t qd0 = ptx::sdesc_sw128(ptx::smem_u32(smem + BM * KB), 16, 1024);
    const uint64_t sd0 = ptx::sdesc_rows16(ptx::smem_u32(smem + (BM + BN) * KB));
    const uint32_t qcol = (uint32_t)(q0 % 128) / 32u;
    for (int it = 0; it < nkb; ++it) {
      const int s = it % C::STAGES;
      const bool ok = ptx::mbar_wait(&full[s], (uint32_t)(it / C::STAGES) & 1u, kWaitTimeoutNs, abort_flag);
      if (!__all_sync(0xffffffffu, ok)) {
        latch(g.err, abort_flag);
        break;
      }
      ptx::tc_fence_after();
      const uint64_t at = (uint64_t)(s * (C::STAGE >> 4));
      const uint32_t sfp = tmem + C::ACC + (uint32_t)s * 2 * SFC, sfq = sfp + SFC;
      const int steps = steps_of(g.K, kb0 + it);
      if (ptx::elect_one()) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          ptx::tmem_cp_rows16(sfp + 4 * h, sd0 + at + h * (kFp4ScaleTile >> 4));
          ptx::tmem_cp_rows16(sfq + 4 * h, sd0 + at + (SF >> 4) + h * (kFp4ScaleTile >> 4));
        }
#pragma unroll
        for (int k = 0; k < KS / 64; ++k)
          if (k < steps)
            ptx::umma_mxf4(tmem, pd0 + at + 2 * k, qd0 + at + 2 * k, idesc[k & 1], sfp + 4 * (k / 2), sfq + 4 * (k / 2) + qcol,
                           it > 0 || k > 0);
        ptx::umma_commit(&empty[s]);
        if (it == nkb - 1) ptx::umma_commit(done);
      }
      __syncwarp();
    }
  } else {
    const bool ok = ptx::mbar_wait(done, 0, 2 * kWaitTimeoutNs, abort_flag);
    if (!ok) latch(g.err, abort_flag);
    if (__all_sync(0xffffffffu, ok)) {
      ptx::tc_fence_after();
      constexpr int LD = C::CPW < 16 ? 8 : 16;
      const uint32_t trow = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(half * C::CPW);
#pragma unroll
      for (int c = 0; c < C::CPW; c += LD) {
        uint32_t r[LD];
        if constexpr (LD == 8)
          ptx::tmem_ld8(trow + c, r);
        else
          ptx::tmem_ld16(trow + c, r);
        ptx::tmem_ld_wait_for(r);
#pragma unroll
        for (int i = 0; i < LD; ++i) acc[c + i] = __uint_as_float(r[i]);
      }
    }
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (*abort_flag) pause_1ms();
  __syncwarp();
  ptx::tc_fence_after();
  if (warp == 1) ptx::tmem_dealloc(tmem, C::TCOLS);
  if (threadIdx.x == 64) ptx::griddep_launch_dependents();

  // Exchange: [source rank][column of the owner's share][row], over the ring,
  // which every CTA of the cluster has finished reading.
  if (ks > 1) ptx::cluster_sync();
  const int share = BN >> ks_log;
  float* buf = reinterpret_cast<float*>(smem);
  if (warp >= 2) {
    const uint32_t local = ptx::smem_u32(buf) + (uint32_t)(q * 32 + lane) * 4;
#pragma unroll
    for (int i = 0; i < C::CPW; ++i) {
      const int col = half * C::CPW + i, owner = col / share;
      const uint32_t at = local + (uint32_t)((rank * share + col - owner * share) * C::PITCH) * 4;
      if (owner == rank)
        asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(acc[i]) : "memory");
      else
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(ptx::mapa_shared(at, (uint32_t)owner)), "f"(acc[i])
                     : "memory");
    }
  }
  if (ks > 1)
    ptx::cluster_sync();
  else
    __syncthreads();
  const int qs = q0 + rank * share;
  auto total = [&](int col, int row) {
    float v = buf[col * C::PITCH + row];
    for (int r = 1; r < ks; ++r) v += buf[(r * share + col) * C::PITCH + row];
    return v;
  };
  auto put = [&](long long at, float v) {
    if (g.out_bf16)
      static_cast<bf16*>(g.c)[at] = __float2bfloat16_rn(v);
    else
      static_cast<float*>(g.c)[at] = v;
  };
  if (g.swap) {
    // lanes along the tile's rows: consecutive columns of C
    const int row = threadIdx.x & (BM - 1), n = p0 + row;
    if (threadIdx.x < 2 * BM && n < g.P) {
      const float bias = g.bias ? __ldg(g.bias + n) : 0.f;
      const int cols = min(share, g.Q - qs);
#pragma unroll 4
      for (int col = threadIdx.x >> 7; col < cols; col += 2)
        put((long long)(qs + col) * g.ldc + n, finish(total(col, row) + bias, g.relu));
    }
  } else {
    // lanes along the tile's columns, 32 (or the share) of a row at a time
    const int w = share < 32 ? share : 32, per = 32 / w;
    for (int c0 = lane & (w - 1); c0 < share; c0 += 32) {
      if (qs + c0 >= g.Q) break;
      const float bias = g.bias ? __ldg(g.bias + qs + c0) : 0.f;
#pragma unroll 4
      for (int row = warp * per + lane / w; row < BM; row += THREADS / 32 * per)
        if (p0 + row < g.P) put((long long)(p0 + row) * g.ldc + qs + c0, finish(total(c0, row) + bias, g.relu));
    }
  }
}

// ------------------------------------------------------------------- host
template <typename F, typename... A>
cudaError_t launch(F* kernel, unsigned grid, int threads, int cluster, int smem, cudaStream_t st, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)cluster;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Clusters of a split kernel the GPU holds at once, for 1, 2, 4 and 8 CTAs each.
template <int BN>
int resident_clusters(int dev, int ks_log) {
  struct Counts { int n[4]; };
  static PerDevice<Counts> kept;
  Counts c{};
  const cudaError_t e = kept.get(dev, &c, [](Counts* r) {
    cudaError_t e = allow_smem<k_fp4_split<BN>>(SCfg<BN>::SMEM);
    if (e != cudaSuccess) return e;
    for (int l = 0; l < 4; ++l) {
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3(1u << l);
      cfg.blockDim = dim3(THREADS);
      cfg.dynamicSmemBytes = SCfg<BN>::SMEM;
      cudaLaunchAttribute at[1];
      at[0].id = cudaLaunchAttributeClusterDimension;
      at[0].val.clusterDim.x = 1u << l;
      at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
      cfg.attrs = at;
      cfg.numAttrs = 1;
      e = cudaOccupancyMaxActiveClusters(&r->n[l], k_fp4_split<BN>, &cfg);
      if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
  });
  if (e != cudaSuccess) cudaGetLastError();  // leave no error behind
  return e == cudaSuccess ? c.n[ks_log] : 0;
}
int clusters_of(int dev, int bn, int ks_log) {
  switch (bn) {
    case 16: return resident_clusters<16>(dev, ks_log);
    case 32: return resident_clusters<32>(dev, ks_log);
    default: return resident_clusters<64>(dev, ks_log);
  }
}

// CTA pairs the GPU holds at once.
template <int LN, bool TMA_C, bool BF16>
int resident_pairs(int dev) {
  static PerDevice<int> kept;
  int n = 0;
  const cudaError_t e = kept.get(dev, &n, [](int* pairs) {
    constexpr auto kernel = k_fp4_pair<LN, TMA_C, BF16>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, LCfg<LN>::SMEM);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = LCfg<LN>::SMEM;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaOccupancyMaxActiveClusters(pairs, kernel, &cfg);
  });
  if (e != cudaSuccess) cudaGetLastError();  // leave no error behind: the split kernel runs
  return e == cudaSuccess ? n : 0;
}
template <bool BF16>
int pairs_of(int dev) {
  return std::min(std::min(resident_pairs<256, true, BF16>(dev), resident_pairs<256, false, BF16>(dev)),
                  std::min(resident_pairs<128, true, BF16>(dev), resident_pairs<128, false, BF16>(dev)));
}
template <int LN>
cudaError_t run_pair(const CUtensorMap (&m)[4], const CUtensorMap& c, const Args& g, int pairs, bool tma_c, cudaStream_t st) {
  const unsigned grid = 2u * (unsigned)std::min((long long)pairs, (long long)g.ntp * g.ntq);
  auto* const kernel = g.out_bf16 ? (tma_c ? k_fp4_pair<LN, true, true> : k_fp4_pair<LN, false, true>)
                                  : (tma_c ? k_fp4_pair<LN, true, false> : k_fp4_pair<LN, false, false>);
  return launch(kernel, grid, THREADS, 2, LCfg<LN>::SMEM, st, m[0], m[1], m[2], m[3], c, g);
}

// The shape of a product: tile, orientation and split with the least estimated
// time (us): a wave of tiles takes a time per stage, each wave after the first a
// fixed one, and a split its exchange.  The constants are least-squares readings
// of a sweep of all shapes over 88 sizes from 1 x 10 x 2000 to 4096 x 8192 x 8192, within
// 13 % of them (root mean square); what this picks is within 3 % of the fastest
// shape of a size on average.  Single CTAs on 128 x 128 tiles were never that.
struct Plan {
  int bn;  // columns; 0: no shape fits
  bool swap;
  int ks_log;
  bool pair;
};
Plan plan(int dev, int M, int N, int K, int pairs) {
  const double nkb = cdiv(K, KS);
  Plan best{0, false, 0, false};
  double t = 1e30;
  if (pairs > 0) {
    const double tiles = (double)cdiv(M, 2 * BM) * cdiv(N, 256), narrow = (double)cdiv(M, 2 * BM) * cdiv(N, 128);
    t = 2.9 + std::ceil(tiles / pairs) * (nkb * 0.30 + 2.04);
    best = Plan{256, false, 0, true};
    const double c = 2.9 + std::ceil(narrow / pairs) * (nkb * 0.27 + 1.03);
    if (c < t) {
      t = c;
      best.bn = 128;
    }
  }
  struct Shape { int bn; bool swap; double step, first, wave, split; };
  const Shape shapes[6] = {{16, true, 0.25, 2.4, 4.9, 1.2},  {32, true, 0.24, 2.7, 5.4, 1.5},  {64, true, 0.23, 3.7, 5.2, 1.7},
                           {16, false, 0.27, 2.5, 6.9, 1.1}, {32, false, 0.25, 3.0, 7.7, 1.3}, {64, false, 0.24, 4.7, 5.8, 0.9}};
  for (const Shape& sh : shapes) {
    const int P = sh.swap ? N : M, Q = sh.swap ? M : N;
    if (sh.bn < 64 && Q > sh.bn) continue;
    const double tiles = (double)cdiv(P, BM) * cdiv(Q, sh.bn);
    for (int l = 0; l < 4; ++l) {
      const int room = clusters_of(dev, sh.bn, l);
      if ((1 << l) > nkb || room < 1) break;
      const double waves = std::ceil(tiles / room), per = std::ceil(nkb / (1 << l));
      const double c = sh.first + (l ? sh.split : 0.0) + waves * per * sh.step + (waves - 1) * sh.wave;
      if (c < t) {
        t = c;
        best = Plan{sh.bn, sh.swap, l, false};
      }
    }
  }
  return best;
}

template <int BN>
cudaError_t run_split(const CUtensorMap (&m)[4], const Args& g, int ks_log, cudaStream_t st) {
  const cudaError_t e = allow_smem<k_fp4_split<BN>>(SCfg<BN>::SMEM);
  if (e != cudaSuccess) return e;
  return launch(k_fp4_split<BN>, (unsigned)(g.ntp * g.ntq) << ks_log, THREADS, 1 << ks_log, SCfg<BN>::SMEM, st, m[0], m[1], m[2],
                m[3], g, ks_log);
}

}  // namespace

ff_status fp4_gemm(const Fp4Gemm& f, cudaStream_t st) {
  int dev = 0;
  FF_TRY(cudaGetDevice(&dev), "4-bit matrix product");
  const int pairs = f.out_bf16 ? pairs_of<true>(dev) : pairs_of<false>(dev);
  const Plan pl = plan(dev, f.M, f.N, f.K, pairs);
  if (pl.bn == 0) return FF_ERR_UNSUPPORTED;
  Args g{};
  g.P = pl.swap ? f.N : f.M;
  g.Q = pl.swap ? f.M : f.N;
  g.K = f.K;
  g.bias = f.bias;
  g.relu = f.relu;
  g.out_bf16 = f.out_bf16;
  g.swap = pl.swap;
  g.c = f.c;
  g.ldc = f.ldc;
  g.err = f.status;
  g.ntp = cdiv(g.P, pl.pair ? 2 * BM : BM);
  g.ntq = cdiv(g.Q, pl.bn);
  if ((long long)g.ntp * g.ntq << pl.ks_log > 0x3FFFFFFFll) return FF_ERR_UNSUPPORTED;
  const int ld = fp4_stride(f.K), words = cdiv(f.K, 128) * (kFp4ScaleTile / 4);
  CUtensorMap m[4];
  if (!make_sw128_map(&m[0], pl.swap ? f.b : f.a, 1, ld, g.P, ld, KB, BM) ||
      !make_sw128_map(&m[1], pl.swap ? f.a : f.b, 1, ld, g.Q, ld, KB, pl.pair ? pl.bn / 2 : pl.bn) ||
      !make_plain_map(&m[2], pl.swap ? f.sb : f.sa, 4, words, cdiv(g.P, 128), words, SF_BOX, 1) ||
      !make_plain_map(&m[3], pl.swap ? f.sa : f.sb, 4, words, cdiv(g.Q, 128), words, SF_BOX, pl.pair && pl.bn == 256 ? 2 : 1))
    return FF_ERR_INVALID_ARG;
  const int es = f.out_bf16 ? 2 : 4;
  CUtensorMap c = m[0];
  // whole 16-byte units a row: a row that ends inside one is written to the
  // unit's end, into what lies between the rows
  const bool tma_c = pl.pair && (long long)f.N * es % 16 == 0 && f.ldc <= 0x7FFFFFFFll && f.ldc >= f.N &&
                     make_sw128_map(&c, f.c, es, f.N, f.M, (int)f.ldc, 128 / es, 32);
  auto go = [&]() -> cudaError_t {
    if (pl.pair) return pl.bn == 256 ? run_pair<256>(m, c, g, pairs, tma_c, st) : run_pair<128>(m, c, g, pairs, tma_c, st);
    switch (pl.bn) {
      case 16: return run_split<16>(m, g, pl.ks_log, st);
      case 32: return run_split<32>(m, g, pl.ks_log, st);
      default: return run_split<64>(m, g, pl.ks_log, st);
    }
  };
  FF_LAUNCH(pl.pair ? K_FP4_PAIR : K_FP4_GEMM, 2.0 * f.M * f.N * f.K, st, go(), "4-bit matrix product");
  return FF_OK;
}

}  // namespace ff
