// The 8-bit matrix product C = act(A B^T + bias), A and B in e4m3 with an fp32
// scale per block of 128 along the contraction:
//
//   C[m, n] = sum_kb sa[kb, m] sb[kb, n or n / 128] sum_{k in kb} A[m, k] B[n, k]
//
// The tensor cores cannot apply fp32 scales, so each k-block's product goes to
// a TMEM buffer of its own and the epilogue warps add it, scaled, to fp32
// registers while the MMAs of the next k-block fill another buffer.  A
// k-block is exactly one 128-byte swizzled row of e4m3, so a ring stage is a
// k-block too.
//
//   warp 0      TMA producer
//   warp 1      allocates TMEM, one lane issues tcgen05.mma (K = 32, four per
//               k-block, the first overwriting the buffer)
//   warps 2..9  epilogue: TMEM lane quarter warp % 4, half of the columns each
//
// Every mbarrier wait is bounded; one that runs out latches DEVERR_TIMEOUT in
// the caller's status word, stops the other roles, and the CTA lets its
// copies and MMAs land before it frees TMEM and exits.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ff_api_internal.h"
#include "ff_fp8.h"
#include "ff_ptx.cuh"

namespace ff {
namespace {

constexpr int KB = 128;  // contraction indices (and bytes) per block and per ring stage
constexpr int BM = 128;  // rows of an accumulator: the TMEM lanes
constexpr int EPI = 8;   // epilogue warps
constexpr int THREADS = 64 + 32 * EPI;

__device__ __forceinline__ void latch(int* err, volatile int* abort_flag) {
  *abort_flag = 1;
  if (err) atomicOr(err, DEVERR_TIMEOUT);
}

// One operand's scales: block kb of row i is p[kb * stride + (i >> shift)].
struct Scales {
  const float* p;
  int stride, shift;
};
__device__ __forceinline__ const float* scale_ptr(const Scales& s, int kb, int i) {
  return s.p + (long long)kb * s.stride + (i >> s.shift);
}

// acc += factor * p over CPW columns of this warp's TMEM lanes, p read 8 to
// 32 columns at a time with the next read in flight under the arithmetic.
// COLS: each column has a factor of its own beside the row's, cs[0..CPW) in
// shared memory.
// release() runs once the last columns are in registers.
template <int CPW, bool COLS, typename Release>
__device__ __forceinline__ void promote(float (&acc)[CPW], uint32_t taddr, float row, const float* cs,
                                        Release release) {
  constexpr int LD = CPW < 16 ? 8 : CPW < 128 ? 16 : 32;
  constexpr int NC = CPW / LD;
  uint32_t r[2][LD];
  auto load = [&](int c, uint32_t (&d)[LD]) {
    if constexpr (LD == 8)
      ptx::tmem_ld8(taddr + c * LD, d);
    else if constexpr (LD == 16)
      ptx::tmem_ld16(taddr + c * LD, d);
    else
      ptx::tmem_ld32(taddr + c * LD, d);
  };
  load(0, r[0]);
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    ptx::tmem_ld_wait_for(r[c & 1]);
    if (c + 1 < NC)
      load(c + 1, r[(c + 1) & 1]);
    else
      release();
#pragma unroll
    for (int i = 0; i < LD; i += 4) {
      float f[4] = {row, row, row, row};
      if constexpr (COLS) {
        const float4 v = *reinterpret_cast<const float4*>(cs + c * LD + i);
        f[0] *= v.x;
        f[1] *= v.y;
        f[2] *= v.z;
        f[3] *= v.w;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[c * LD + i + e] = fmaf(f[e], __uint_as_float(r[c & 1][i + e]), acc[c * LD + i + e]);
    }
  }
}

struct Args {
  int P, Q, K;       // rows of the operand on the TMEM lanes (P) and on the columns (Q)
  Scales sp, sq;
  const float* bias;
  int relu, out_bf16, swap;  // swap: the lanes are C's columns (P = N, Q = M)
  void* c;
  long long ldc;
  int* err;
  int ntp, ntq;      // tiles
};

__device__ __forceinline__ float finish(float v, int relu) { return relu && v < 0.f ? 0.f : v; }  // keeps NaN

// ------------------------------------------------------- large products
// CTA pairs (cta_group::2) on 256 x 256 tiles: each CTA loads 128 rows of A
// and half of B's 256 columns per k-block (32 KB for 8.4 MMAC) and promotes its
// own 128 x 256 accumulator.  Persistent: the MMAs of the next tile's first
// k-blocks run under the last promotions and the store of this one.
constexpr int LN = 256;
constexpr int LSTAGES = 5;
constexpr int LSTAGE = (BM + LN / 2) * KB;
constexpr int LCPW = LN / 2;  // columns per epilogue warp
constexpr int LSTAGING = 32 * 128;  // per epilogue warp: 32 rows x 128 bytes of C
constexpr int LSLOTS = 8;           // k-blocks of scales in flight or in use
constexpr int LSLOT = BM + LN;      // the CTA's rows' and the tile's columns' scales
// Three warpgroups: producer, MMA and two scale-loading warps, and two of
// epilogue warps, which take the registers the first gives up: a launch of
// 168 a thread is split 40 / 232 / 232.
constexpr int LTHREADS = 384;
constexpr int LREGS = 168, LREGS_LOW = 40, LREGS_EPI = 232;
static_assert(LREGS_LOW + 2 * LREGS_EPI <= 3 * LREGS, "the split must fit what the launch holds");
constexpr int L_SMEM = 1024 + LSTAGES * LSTAGE + EPI * LSTAGING + LSLOTS * LSLOT * 4 + 512;
static_assert(L_SMEM > 113 * 1024 && L_SMEM <= 227 * 1024, "one GEMM CTA per SM, so that no TMEM allocation waits on another's");

// Tile t of the raster: groups of 8 row tiles, columns outermost within a
// group, so that the tiles in flight share operand panels in L2.
__device__ __forceinline__ void tile_of(int t, int ntp, int ntq, int& tp, int& tq) {
  constexpr int GROUP = 8;
  const int per = GROUP * ntq, g = t / per, in = t - g * per;
  const int rows = min(GROUP, ntp - g * GROUP);
  tp = g * GROUP + in % rows;
  tq = in / rows;
}

template <bool COLS>
__global__ void __launch_bounds__(LTHREADS, 1)
    k_fp8_pair(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, Args g) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_s = ptx::smem_u32(smem_raw);
  uint8_t* smem = smem_raw + ((1024u - (raw_s & 1023u)) & 1023u);
  uint8_t* staging = smem + LSTAGES * LSTAGE;
  float* slots = reinterpret_cast<float*>(staging + EPI * LSTAGING);  // [LSLOTS][LSLOT]
  uint64_t* full = reinterpret_cast<uint64_t*>(slots + LSLOTS * LSLOT);
  uint64_t* empty = full + LSTAGES;
  uint64_t* tfull = empty + LSTAGES;   // [2] a TMEM buffer holds a k-block's product
  uint64_t* tempty = tfull + 2;        // [2] both CTAs have read it
  uint64_t* sfull = tempty + 2;        // [LSLOTS] a slot holds a k-block's scales
  uint64_t* sempty = sfull + LSLOTS;   // [LSLOTS] the epilogue has used them
  uint32_t* tslot = reinterpret_cast<uint32_t*>(sempty + LSLOTS);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tslot + 1);
  volatile int* never_set = reinterpret_cast<volatile int*>(tslot + 2);
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const uint32_t crank = ptx::cluster_ctarank();
  const bool lead = crank == 0;
  const int nkb = (g.K + KB - 1) / KB;
  const int ntiles = g.ntp * g.ntq;
  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < LSTAGES; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      ptx::mbar_init(&tfull[b], 1);
      ptx::mbar_init(&tempty[b], 2 * EPI);
    }
    for (int i = 0; i < LSLOTS; ++i) {
      ptx::mbar_init(&sfull[i], 64);
      ptx::mbar_init(&sempty[i], EPI);
    }
    *abort_flag = 0;
    *never_set = 0;
    ptx::fence_mbar_init();
    ptx::prefetch_tmap(&tmA);
    ptx::prefetch_tmap(&tmB);
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

  if (warp < 4) {
    ptx::regs_dec<LREGS_LOW>();
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
          ptx::tma_load_2d_pair(a, &tmA, full0 + 8u * (uint32_t)s, kb * KB, ar);
          ptx::tma_load_2d_pair(a + BM * KB, &tmB, full0 + 8u * (uint32_t)s, kb * KB, br);
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
          const uint64_t t0 = ptx::globaltimer();
          while (ptx::globaltimer() - t0 < 1000000ull) {
          }
        }
      }
    }
  } else if (warp == 1) {
    if (lead) {
      // Few instructions between the MMAs: this warp shares its scheduler with
      // two epilogue warps, and while it lags the tensor cores stand still.
      // The whole warp walks the loop, so that its variables are uniform, and
      // one lane issues.  Descriptors differ from the first stage's by their
      // address field only (16-byte units).
      constexpr uint32_t idesc = ptx::idesc_e4m3_f32(2 * BM, LN);
      const uint64_t ad0 = ptx::sdesc_sw128(ptx::smem_u32(smem), 16, 1024);
      const uint64_t bd0 = ptx::sdesc_sw128(ptx::smem_u32(smem + BM * KB), 16, 1024);
      const int total = ntiles > pair ? (ntiles - pair + npairs - 1) / npairs * nkb : 0;
      int s = 0;
      uint32_t ph = 0, tph = 1;  // parities of full[s] and tempty[b]
      for (int it = 0; it < total; ++it) {
        const uint32_t b = (uint32_t)it & 1u;
        const bool ok = ptx::mbar_wait(&tempty[b], tph, kWaitTimeoutNs, abort_flag) &&
                        ptx::mbar_wait(&full[s], ph, kWaitTimeoutNs, abort_flag);
        if (!__all_sync(0xffffffffu, ok)) {
          latch(g.err, abort_flag);
          break;
        }
        ptx::tc_fence_after();
        const uint64_t ad = ad0 + (uint64_t)(s * (LSTAGE >> 4)), bd = bd0 + (uint64_t)(s * (LSTAGE >> 4));
        const uint32_t d = tmem + b * LN;
        if (ptx::elect_one()) {
          ptx::umma_f8_pair(d, ad, bd, idesc, 0u);
#pragma unroll
          for (int k = 1; k < KB / 32; ++k) ptx::umma_f8_pair(d, ad + 2 * k, bd + 2 * k, idesc, 1u);
          ptx::umma_commit_pair(&empty[s], 3);
          ptx::umma_commit_pair(&tfull[b], 3);
        }
        __syncwarp();
        tph ^= b;
        if (++s == LSTAGES) {
          s = 0;
          ph ^= 1u;
        }
      }
    }
  } else if (warp < 4) {
    // Scales of the k-blocks to come: this CTA's rows', and the columns' of
    // the tile (COLS) or of its two 128-column halves.
    const int l = (int)threadIdx.x - 64;  // 0 .. 63
    int it = 0;
    for (int t = pair; t < ntiles && !*abort_flag; t += npairs) {
      int tp, tq;
      tile_of(t, g.ntp, g.ntq, tp, tq);
      const int row = tp * 2 * BM + (int)crank * BM + l, col = tq * LN;
      for (int kb = 0; kb < nkb; ++kb, ++it) {
        const int s = it % LSLOTS;
        if (!ptx::mbar_wait(&sempty[s], (((uint32_t)(it / LSLOTS)) & 1u) ^ 1u, kWaitTimeoutNs, abort_flag)) {
          latch(g.err, abort_flag);
          break;
        }
        float* d = slots + s * LSLOT;
        // rows and columns past the matrix hold zeros: any scale will do
        ptx::cp_async4(d + l, scale_ptr(g.sp, kb, min(row, g.P - 1)));
        ptx::cp_async4(d + 64 + l, scale_ptr(g.sp, kb, min(row + 64, g.P - 1)));
        if constexpr (COLS) {
#pragma unroll
          for (int e = 0; e < LN; e += 64)
            ptx::cp_async4(d + BM + e + l, scale_ptr(g.sq, kb, min(col + e + l, g.Q - 1)));
        } else {
          if (l < 2) ptx::cp_async4(d + BM + l, scale_ptr(g.sq, kb, min(col + l * LCPW, g.Q - 1)));
        }
        ptx::cp_async_arrive(&sfull[s]);
      }
    }
    ptx::cp_async_commit();
    ptx::cp_async_wait<0>();
  }
  } else {
    ptx::regs_inc<LREGS_EPI>();
    const int q = warp & 3, ew = warp - 4, half = ew / 4;
    const uint32_t trow = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(half * LCPW);
    const uint32_t te0 = ptx::mapa_shared(ptx::smem_u32(&tempty[0]), 0);
    uint8_t* stage = staging + ew * LSTAGING;
    int it = 0;
    bool live = true;
    for (int t = pair; t < ntiles && live; t += npairs) {
      int tp, tq;
      tile_of(t, g.ntp, g.ntq, tp, tq);
      const int rbase = tp * 2 * BM + (int)crank * BM + q * 32;
      const int cbase = tq * LN + half * LCPW;
      float acc[LCPW];
#pragma unroll
      for (int i = 0; i < LCPW; ++i) acc[i] = 0.f;
      for (int kb = 0; kb < nkb; ++kb, ++it) {
        const int b = it & 1;
        const int sl = it % LSLOTS;
        const float* d = slots + sl * LSLOT;
        bool ok = ptx::mbar_wait(&sfull[sl], (uint32_t)(it / LSLOTS) & 1u, kWaitTimeoutNs, abort_flag);
        float row = d[q * 32 + lane];
        if constexpr (!COLS) row *= d[BM + half];
        ok = ok && ptx::mbar_wait(&tfull[b], (uint32_t)(it >> 1) & 1u, kWaitTimeoutNs, abort_flag);
        if (!ok) latch(g.err, abort_flag);
        if (!__all_sync(0xffffffffu, ok)) {
          live = false;
          break;
        }
        ptx::tc_fence_after();
        promote<LCPW, COLS>(acc, trow + (uint32_t)(b * LN), row, d + BM + half * LCPW, [&]() {
          ptx::tc_fence_before();
          __syncwarp();
          // the arrival orders TMEM reads only (the fence above), so it needs
          // no cluster-wide release of memory
          if (lane == 0) ptx::mbar_arrive_at(te0 + 8u * (uint32_t)b);
        });
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&sempty[sl]);
      }
      if (!live) break;
      if (t + npairs >= ntiles && threadIdx.x == 128) ptx::griddep_launch_dependents();
      // Store: 128 bytes of each of the warp's 32 rows at a time through the
      // swizzled staging block, then whole row segments.
      const int es = g.out_bf16 ? 2 : 4;
      const bool vec = ((reinterpret_cast<uintptr_t>(g.c) | (uintptr_t)(g.ldc * es)) & 15) == 0;
      auto flush = [&](int col0, int cols) {  // staged columns col0 .. col0 + cols of C
        __syncwarp();
        if (vec) {
          const int u = lane & 7, per = 16 / es, col = col0 + u * per;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int rr = i * 4 + (lane >> 3);
            const uint4 w = *reinterpret_cast<const uint4*>(stage + rr * 128 + ((u ^ (rr & 7)) << 4));
            if (rbase + rr >= g.P || col >= g.Q) continue;
            char* dst = static_cast<char*>(g.c) + ((long long)(rbase + rr) * g.ldc + col) * es;
            if (col + per <= g.Q) {
              *reinterpret_cast<uint4*>(dst) = w;
            } else if (es == 2) {
              const uint32_t h[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (col + e < g.Q) reinterpret_cast<uint16_t*>(dst)[e] = (uint16_t)(h[e / 2] >> (16 * (e & 1)));
            } else {
              const uint32_t h[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (col + e < g.Q) reinterpret_cast<uint32_t*>(dst)[e] = h[e];
            }
          }
        } else {
          for (int rr = 0; rr < 32 && rbase + rr < g.P; ++rr)
            for (int j = lane; j < cols && col0 + j < g.Q; j += 32) {
              const int byte = j * es;
              const uint8_t* src = stage + rr * 128 + (((byte >> 4) ^ (rr & 7)) << 4) + (byte & 15);
              const long long at = (long long)(rbase + rr) * g.ldc + col0 + j;
              if (es == 2)
                static_cast<uint16_t*>(g.c)[at] = *reinterpret_cast<const uint16_t*>(src);
              else
                static_cast<uint32_t*>(g.c)[at] = *reinterpret_cast<const uint32_t*>(src);
            }
        }
        __syncwarp();
      };
      auto value = [&](int i, int col) {  // accumulator pair i with bias and activation
        float2 v = make_float2(acc[2 * i], acc[2 * i + 1]);
        if (g.bias) {
          v.x += col < g.Q ? __ldg(g.bias + col) : 0.f;
          v.y += col + 1 < g.Q ? __ldg(g.bias + col + 1) : 0.f;
        }
        return make_float2(finish(v.x, g.relu), finish(v.y, g.relu));
      };
      if (g.out_bf16) {
#pragma unroll
        for (int ch = 0; ch < LCPW / 64; ++ch) {
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int i = ch * 32 + u * 4 + e;
              const float2 v = value(i, cbase + 2 * i);
              const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
              w[e] = *reinterpret_cast<const uint32_t*>(&h);
            }
            *reinterpret_cast<uint4*>(stage + lane * 128 + ((u ^ (lane & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
          }
          flush(cbase + ch * 64, 64);
        }
      } else {
#pragma unroll
        for (int ch = 0; ch < LCPW / 32; ++ch) {
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            const int i = ch * 16 + u * 2;
            const float2 v = value(i, cbase + 2 * i), w = value(i + 1, cbase + 2 * i + 2);
            *reinterpret_cast<float4*>(stage + lane * 128 + ((u ^ (lane & 7)) << 4)) = make_float4(v.x, v.y, w.x, w.y);
          }
          flush(cbase + ch * 32, 32);
        }
      }
    }
  }

  ptx::tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    // MMAs issued before the abort finish before TMEM is released: they read
    // stages that have landed, so a short bounded pause covers them
    const uint64_t t0 = ptx::globaltimer();
    while (ptx::globaltimer() - t0 < 1000000ull) {
    }
  }
  __syncwarp();
  ptx::cluster_sync();
  ptx::tc_fence_after();
  if (warp == 1) ptx::tmem_dealloc_pair(tmem, 512);
}

// ------------------------------------------------------- small products
// One CTA per 128 x BN tile and slice of the contraction: the CTAs of a
// cluster (1, 2, 4 or 8) share a tile's k-blocks, exchange their partial sums
// through distributed shared memory (each sums its share of the columns, in
// rank order) and store.  With few rows of A its rows go on the MMA's columns
// (swap), so that a token needs 16 columns and not 128 lanes.
template <int BN>
struct SCfg {
  static constexpr int STAGE = (BM + BN) * KB;
  static constexpr int STAGES = BN >= 128 ? 6 : BN >= 64 ? 8 : 9;
  static constexpr int CPW = BN / 2;
  static constexpr int BUFS = 2;                          // TMEM buffers (the loops count on two)
  static constexpr uint32_t ACC = BN < 32 ? 32 : BN;      // TMEM columns of a buffer
  static constexpr uint32_t TCOLS = BUFS * ACC;
  static constexpr int PITCH = BM + 1;                    // floats per column of the exchange buffer
  static constexpr int SLOTS = 4;                         // as LSLOTS
  static constexpr int SLOT = 32 + (CPW < 32 ? 32 : CPW);
  static constexpr int SLOT_BYTES = EPI * SLOTS * SLOT * 4;
  static constexpr int SMEM = 1024 + STAGES * STAGE + SLOT_BYTES + 512;
  static_assert(SMEM > 113 * 1024 && SMEM <= 227 * 1024, "one GEMM CTA per SM");
  static_assert(BN * PITCH * 4 <= STAGES * STAGE, "the exchange buffer lies over the ring");
};

template <int BN, bool COLS>
__global__ void __launch_bounds__(THREADS, 1)
    k_fp8_split(const __grid_constant__ CUtensorMap tmP, const __grid_constant__ CUtensorMap tmQ, Args g, int ks_log) {
  using C = SCfg<BN>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_s = ptx::smem_u32(smem_raw);
  uint8_t* smem = smem_raw + ((1024u - (raw_s & 1023u)) & 1023u);
  float* slots = reinterpret_cast<float*>(smem + C::STAGES * C::STAGE);  // [warp][SLOTS][SLOT]
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::STAGES * C::STAGE + C::SLOT_BYTES);
  uint64_t* empty = full + C::STAGES;
  uint64_t* tfull = empty + C::STAGES;
  uint64_t* tempty = tfull + C::BUFS;
  uint32_t* tslot = reinterpret_cast<uint32_t*>(tempty + C::BUFS);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tslot + 1);
  volatile int* never_set = reinterpret_cast<volatile int*>(tslot + 2);
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int ks = 1 << ks_log;
  const int rank = (int)(blockIdx.x & (unsigned)(ks - 1));
  const int tile = (int)(blockIdx.x >> ks_log);
  const int p0 = (tile % g.ntp) * BM, q0 = (tile / g.ntp) * BN;
  const int nkb_all = (g.K + KB - 1) / KB;
  const int kb0 = (int)((long long)nkb_all * rank >> ks_log), kb1 = (int)((long long)nkb_all * (rank + 1) >> ks_log);
  const int nkb = kb1 - kb0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::STAGES; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < C::BUFS; ++b) {
      ptx::mbar_init(&tfull[b], 1);
      ptx::mbar_init(&tempty[b], EPI);
    }
    *abort_flag = 0;
    *never_set = 0;
    ptx::fence_mbar_init();
    ptx::prefetch_tmap(&tmP);
    ptx::prefetch_tmap(&tmQ);
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
      }
      if (*abort_flag)
        for (int k = it < C::STAGES ? 0 : it - C::STAGES; k < it; ++k)
          ptx::mbar_wait(&full[k % C::STAGES], (uint32_t)(k / C::STAGES) & 1u, 10000000ull, never_set);
    }
  } else if (warp == 1) {
    {
      constexpr uint32_t idesc = ptx::idesc_e4m3_f32(BM, BN);
      const uint64_t pd0 = ptx::sdesc_sw128(ptx::smem_u32(smem), 16, 1024);
      const uint64_t qd0 = ptx::sdesc_sw128(ptx::smem_u32(smem + BM * KB), 16, 1024);
      int s = 0;
      uint32_t ph = 0, tph = 1;
      for (int it = 0; it < nkb; ++it) {
        const uint32_t b = (uint32_t)it & 1u;
        const bool ok = ptx::mbar_wait(&tempty[b], tph, kWaitTimeoutNs, abort_flag) &&
                        ptx::mbar_wait(&full[s], ph, kWaitTimeoutNs, abort_flag);
        if (!__all_sync(0xffffffffu, ok)) {
          latch(g.err, abort_flag);
          break;
        }
        ptx::tc_fence_after();
        const uint64_t pd = pd0 + (uint64_t)(s * (C::STAGE >> 4)), qd = qd0 + (uint64_t)(s * (C::STAGE >> 4));
        const uint32_t d = tmem + b * C::ACC;
        if (ptx::elect_one()) {
          ptx::umma_f8(d, pd, qd, idesc, 0u);
#pragma unroll
          for (int k = 1; k < KB / 32; ++k) ptx::umma_f8(d, pd + 2 * k, qd + 2 * k, idesc, 1u);
          ptx::umma_commit(&empty[s]);
          ptx::umma_commit(&tfull[b]);
        }
        __syncwarp();
        tph ^= b;
        if (++s == C::STAGES) {
          s = 0;
          ph ^= 1u;
        }
      }
    }
  } else {
    const uint32_t trow = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(half * C::CPW);
    const int prow = min(p0 + q * 32 + lane, g.P - 1);
    const int cbase = q0 + half * C::CPW;
    float* sl = slots + ew * C::SLOTS * C::SLOT;
    // scales three k-blocks ahead of their use, as in the pair kernel
    auto fetch = [&](int it) {
      if (it < nkb) {
        float* d = sl + (it % C::SLOTS) * C::SLOT;
        ptx::cp_async4(d + lane, scale_ptr(g.sp, kb0 + it, prow));
        if constexpr (COLS) {
#pragma unroll
          for (int e = 0; e < C::CPW; e += 32)
            if (e + lane < C::CPW)
              ptx::cp_async4(d + 32 + e + lane, scale_ptr(g.sq, kb0 + it, min(cbase + e + lane, g.Q - 1)));
        } else {
          ptx::cp_async4(d + 32 + lane, scale_ptr(g.sq, kb0 + it, min(cbase, g.Q - 1)));
        }
      }
      ptx::cp_async_commit();
    };
    for (int i = 0; i < C::SLOTS - 1; ++i) fetch(i);
    for (int it = 0; it < nkb; ++it) {
      const int b = it % C::BUFS;
      ptx::cp_async_wait<C::SLOTS - 2>();
      __syncwarp();
      const float* d = sl + (it % C::SLOTS) * C::SLOT;
      float row = d[lane];
      if constexpr (!COLS) row *= d[32 + lane];
      fetch(it + C::SLOTS - 1);
      const bool ok = ptx::mbar_wait(&tfull[b], (uint32_t)(it / C::BUFS) & 1u, kWaitTimeoutNs, abort_flag);
      if (!ok) latch(g.err, abort_flag);
      if (!__all_sync(0xffffffffu, ok)) break;
      ptx::tc_fence_after();
      promote<C::CPW, COLS>(acc, trow + (uint32_t)b * C::ACC, row, d + 32, [&]() {
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&tempty[b]);
      });
    }
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    const uint64_t t0 = ptx::globaltimer();  // MMAs issued before the abort finish in bounded time
    while (ptx::globaltimer() - t0 < 1000000ull) {
    }
  }
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
  auto total = [&](int col, int row) {
    float v = buf[col * C::PITCH + row];
    for (int r = 1; r < ks; ++r) v += buf[(r * share + col) * C::PITCH + row];
    return v;
  };
  const int qs = q0 + rank * share;
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
      for (int col = threadIdx.x >> 7; col < share && qs + col < g.Q; col += 2)
        put((long long)(qs + col) * g.ldc + n, finish(total(col, row) + bias, g.relu));
    }
  } else {
    for (int i = threadIdx.x; i < BM * share; i += THREADS) {
      const int row = i / share, col = i - row * share;
      if (p0 + row < g.P && qs + col < g.Q)
        put((long long)(p0 + row) * g.ldc + qs + col,
            finish(total(col, row) + (g.bias ? __ldg(g.bias + qs + col) : 0.f), g.relu));
    }
  }
}

// ------------------------------------------------------------------- host
template <typename F>
cudaError_t launch(F* kernel, unsigned grid, int threads, int cluster, int smem, cudaStream_t st, const CUtensorMap& p,
                   const CUtensorMap& q, const Args& g, int ks_log = -1) {
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
  if constexpr (std::is_invocable_v<F, CUtensorMap, CUtensorMap, Args, int>)
    return cudaLaunchKernelEx(&cfg, kernel, p, q, g, ks_log);
  else
    return cudaLaunchKernelEx(&cfg, kernel, p, q, g);
}

// CTA pairs the GPU holds at once (one CTA per SM; an SM without a partner in
// its cluster group stays out); 0 if the pair kernel was not built with the
// registers that its split counts on, and so must not run.
template <bool COLS>
int resident_pairs() {
  static const int n = [] {
    cudaFuncAttributes fa{};
    if (cudaFuncGetAttributes(&fa, k_fp8_pair<COLS>) != cudaSuccess || fa.numRegs != LREGS) return 0;
    if (cudaFuncSetAttribute(k_fp8_pair<COLS>, cudaFuncAttributeMaxDynamicSharedMemorySize, L_SMEM) != cudaSuccess) return 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2);
    cfg.blockDim = dim3(LTHREADS);
    cfg.dynamicSmemBytes = L_SMEM;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    int c = 0;
    if (cudaOccupancyMaxActiveClusters(&c, k_fp8_pair<COLS>, &cfg) != cudaSuccess) {
      cudaGetLastError();
      return 0;
    }
    return c;
  }();
  return n;
}

template <int BN, bool COLS>
cudaError_t split_attr() {
  static const cudaError_t e =
      cudaFuncSetAttribute(k_fp8_split<BN, COLS>, cudaFuncAttributeMaxDynamicSharedMemorySize, SCfg<BN>::SMEM);
  return e;
}
template <int BN, bool COLS>
cudaError_t run_split(const CUtensorMap& p, const CUtensorMap& q, const Args& g, int ks_log, cudaStream_t st) {
  const cudaError_t e = split_attr<BN, COLS>();
  if (e != cudaSuccess) return e;
  return launch(k_fp8_split<BN, COLS>, (unsigned)(g.ntp * g.ntq) << ks_log, THREADS, 1 << ks_log, SCfg<BN>::SMEM, st, p, q, g,
                ks_log);
}

// The shape of a product: tile and split with the least estimated time, in
// clocks.  A CTA spends on a k-block the longest of its MMAs (8192 MAC a
// clock), its operand feed (about 73 bytes a clock) and its share of HBM, and
// a fixed cost per launch wave.
struct Plan {
  int bn;      // 256: the pair kernel
  bool swap;
  int ks_log;
};
Plan plan(int M, int N, int K, int pairs) {
  const double nkb = cdiv(K, KB);
  Plan best{LN, false, 0};
  double t = 1e30;
  if (pairs > 0) {
    const double tiles = (double)cdiv(M, 2 * BM) * cdiv(N, LN);
    t = std::max(1.0, std::ceil(tiles / pairs)) * (nkb * 560 + 1500) + 3000;
  }
  const int sizes[4] = {16, 32, 64, 128};
  for (int swap = 0; swap < 2; ++swap)
    for (int bn : sizes) {
      if (!swap && bn != 128) continue;
      const int P = swap ? N : M, Q = swap ? M : N;
      const double tiles = (double)cdiv(P, BM) * cdiv(Q, bn);
      for (int l = 0; l < 4; ++l) {
        if ((1 << l) > nkb) break;
        const double per = std::ceil(nkb / (1 << l));
        const double ctas = tiles * (1 << l), waves = std::ceil(ctas / 144);  // clusters of 8 do not use every SM
        const double step = std::max(2.0 * bn, (BM + bn) * KB / 73.0);
        const double c = waves * (per * step + 2000) + 3000 + (l ? 800 : 0) + bn * 8.0;
        if (c < t) {
          t = c;
          best = Plan{bn, swap != 0, l};
        }
      }
    }
  return best;
}

}  // namespace

ff_status fp8_gemm(const Fp8Gemm& f, cudaStream_t st) {
  const int ld = fp8_stride(f.K);
  const bool cols = !f.b_tiles;
  const int pairs = cols ? resident_pairs<true>() : resident_pairs<false>();
  const Plan pl = plan(f.M, f.N, f.K, pairs);
  Args g{};
  const Scales sa{f.sa, f.M, 0};
  const Scales sb{f.sb, f.b_tiles ? cdiv(f.N, KB) : f.N, f.b_tiles ? 7 : 0};
  g.P = pl.swap ? f.N : f.M;
  g.Q = pl.swap ? f.M : f.N;
  g.K = f.K;
  g.sp = pl.swap ? sb : sa;
  g.sq = pl.swap ? sa : sb;
  g.bias = f.bias;
  g.relu = f.relu;
  g.out_bf16 = f.out_bf16;
  g.swap = pl.swap;
  g.c = f.c;
  g.ldc = f.ldc;
  g.err = f.status;
  const bool pairk = pl.bn == LN;
  g.ntp = cdiv(g.P, pairk ? 2 * BM : BM);
  g.ntq = cdiv(g.Q, pl.bn);
  if ((long long)g.ntp * g.ntq << pl.ks_log > 0x3FFFFFFFll) return FF_ERR_UNSUPPORTED;
  CUtensorMap p, q;
  if (!make_sw128_map(&p, pl.swap ? f.b : f.a, 1, f.K, g.P, ld, KB, BM) ||
      !make_sw128_map(&q, pl.swap ? f.a : f.b, 1, f.K, g.Q, ld, KB, pairk ? LN / 2 : pl.bn))
    return FF_ERR_INVALID_ARG;
  const double work = 2.0 * f.M * f.N * f.K;
  auto go = [&]() -> cudaError_t {
    if (pairk) {
      const unsigned grid = 2u * (unsigned)std::min((long long)pairs, (long long)g.ntp * g.ntq);
      return cols ? launch(k_fp8_pair<true>, grid, LTHREADS, 2, L_SMEM, st, p, q, g)
                  : launch(k_fp8_pair<false>, grid, LTHREADS, 2, L_SMEM, st, p, q, g);
    }
    const bool c = cols || pl.swap;
    switch (pl.bn) {
      case 16: return run_split<16, true>(p, q, g, pl.ks_log, st);
      case 32: return run_split<32, true>(p, q, g, pl.ks_log, st);
      case 64: return run_split<64, true>(p, q, g, pl.ks_log, st);
      default: return c ? run_split<128, true>(p, q, g, pl.ks_log, st) : run_split<128, false>(p, q, g, pl.ks_log, st);
    }
  };
  FF_LAUNCH(K_FP8_GEMM, work, st, go(), "8-bit matrix product");
  return FF_OK;
}

}  // namespace ff
