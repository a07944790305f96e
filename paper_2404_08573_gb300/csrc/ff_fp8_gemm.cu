// The 8-bit matrix product C = act(A B^T + bias), A and B in e4m3 with an fp32
// scale per block of 128 along the contraction:
//
//   C[m, n] = sum_kb sa[kb, m] sb[kb, n or n / 128] sum_{k in kb} A[m, k] B[n, k]
//
// The tensor cores cannot apply fp32 scales, so each k-block's product goes to
// a TMEM buffer of its own and the epilogue warps add it, scaled, to fp32
// registers while the MMAs of the next k-block fill another buffer.  A
// k-block is exactly one 128-byte swizzled row of e4m3, so a ring stage is a
// k-block too.  Large products run on CTA pairs (k_fp8_pair), the others on
// single CTAs that may split the contraction (k_fp8_split).  The roles of the
// latter:
//
//   warp 0      TMA producer
//   warp 1      allocates TMEM, one lane issues tcgen05.mma (K = 32, four per
//               k-block, the first overwriting the buffer)
//   warps 2..9  epilogue: TMEM lane quarter warp % 4, half of the columns each
//
// Every mbarrier wait is bounded; one that runs out latches DEVERR_TIMEOUT in
// the call's status word, stops the other roles, and the CTA lets its
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
static_assert(KB % 16 == 0, "every tiled copy starts a multiple of KB bytes (C: of 128) into its row");
constexpr int EPI = 8;   // epilogue warps
constexpr int THREADS = 64 + 32 * EPI;

__device__ __forceinline__ void latch(int* err, volatile int* abort_flag) {
  *abort_flag = 1;
  atomicOr(err, DEVERR_TIMEOUT);
}

// One operand's scales: block kb of row i is p[kb * stride + (i >> shift)].
struct Scales {
  const float* p;
  int stride, shift;
};
__device__ __forceinline__ const float* scale_ptr(const Scales& s, int kb, int i) {
  return s.p + (long long)kb * s.stride + (i >> s.shift);
}

// Reads LD of this warp's TMEM columns into registers (asynchronous).
template <int LD>
__device__ __forceinline__ void tmem_read(uint32_t taddr, uint32_t (&r)[LD]) {
  if constexpr (LD == 8)
    ptx::tmem_ld8(taddr, r);
  else if constexpr (LD == 16)
    ptx::tmem_ld16(taddr, r);
  else
    ptx::tmem_ld32(taddr, r);
}

// acc[0..LD) += row * cs[.] * p, on pairs.  COLS: each column has a factor of
// its own, cs in shared memory; else the row's is all.
template <int LD, bool COLS>
__device__ __forceinline__ void scaled_add(float* acc, const uint32_t (&p)[LD], uint64_t row2, const float* cs) {
#pragma unroll
  for (int i = 0; i < LD; i += 4) {
    float* d = acc + i;
    uint64_t f0 = row2, f1 = row2, lo = ptx::pack2(d[0], d[1]), hi = ptx::pack2(d[2], d[3]);
    if constexpr (COLS) {
      const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(cs + i);
      f0 = ptx::mul2(row2, v.x);
      f1 = ptx::mul2(row2, v.y);
    }
    ptx::fma2_to(lo, f0, ptx::pack2(p[i], p[i + 1]));
    ptx::fma2_to(hi, f1, ptx::pack2(p[i + 2], p[i + 3]));
    const float2 x = ptx::unpack2(lo), y = ptx::unpack2(hi);
    d[0] = x.x;
    d[1] = x.y;
    d[2] = y.x;
    d[3] = y.y;
  }
}

// One k-block: acc += scaled product over the CPW columns at TMEM address
// `at`, a chunk's read in flight under the arithmetic of the one before it.
// release() runs once the last columns are in registers.
template <int CPW, bool COLS, typename Release>
__device__ __forceinline__ void promote(float (&acc)[CPW], uint32_t at, float row, const float* cs, Release release) {
  constexpr int LD = CPW < 16 ? 8 : 16;
  constexpr int NC = CPW / LD;
  uint32_t r[2][LD];
  const uint64_t row2 = ptx::pack2(row, row);
  tmem_read<LD>(at, r[0]);
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    ptx::tmem_ld_wait_for(r[c & 1]);
    if (c + 1 < NC)
      tmem_read<LD>(at + (c + 1) * LD, r[(c + 1) & 1]);
    else
      release();
    scaled_add<LD, COLS>(acc + c * LD, r[c & 1], row2, cs + c * LD);
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
// and half of B's 256 columns per k-block (32 KB for 4.2 MMAC) and promotes its
// own 128 x 256 accumulator.  A k-block's MMAs run as two halves of 128
// columns, each with its own TMEM buffers and its own four epilogue warps, so
// that a buffer is handed back after half a k-block's MMAs and the two
// epilogue warps of a scheduler work in turn.  Persistent: the MMAs of the
// next tile's first k-blocks run under the store of this one.
//
// Bound by the MMAs: 4096 x 8192 x 8192 with a scale per 128 x 128 tile of B takes
// 188 us, 2.92 PFLOP/s (0.78 of twice the measured bf16 burst rate, 0.85 of
// twice the sustained one).  With a scale per row of B each value of the
// product takes a second multiplication, and the promotion bounds: 289 us.
constexpr int LN = 256;
constexpr int LSTAGES = 4;
constexpr int LSTAGE = (BM + LN / 2) * KB;
constexpr int LCPW = LN / 2;  // columns per epilogue warp
constexpr int LSTAGING = 2 * 32 * 128;  // per epilogue warp: two blocks of 32 rows x 128 bytes of C
constexpr int LGROUP = 4;           // k-blocks of scales per barrier
constexpr int LGROUPS = 2;          // groups in flight or in use
constexpr int LSLOT = BM + LN;      // a k-block's: the CTA's rows' and the tile's columns' scales
// Three warpgroups: producer, two MMA and a scale-loading warp, and two of
// epilogue warps, which take the registers the first gives up: a launch of
// 168 a thread is split 40 / 232 / 232.
constexpr int LTHREADS = 384;
constexpr int LREGS = 168, LREGS_LOW = 40, LREGS_EPI = 232;
static_assert(LREGS_LOW + 2 * LREGS_EPI <= 3 * LREGS, "the split must fit what the launch holds");
constexpr int L_SMEM = 1024 + LSTAGES * LSTAGE + EPI * LSTAGING + LGROUPS * LGROUP * LSLOT * 4 + EPI * LCPW * 4 + 512;
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

// A warp writes a staged block of 32 rows x 128 bytes (16-byte units swizzled
// by the row) to C, `rows` and `left` of its rows and columns being there.
template <typename U>
__device__ __forceinline__ void rows_out(const uint8_t* from, U* c, long long ldc, int rows, int left, int lane) {
  constexpr int J = 128 / 32 / (int)sizeof(U);
#pragma unroll
  for (int r0 = 0; r0 < 32; r0 += 8) {
    U v[8][J];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int byte = (lane + 32 * j) * (int)sizeof(U);
        v[i][j] = *reinterpret_cast<const U*>(from + (r0 + i) * 128 + (((byte >> 4) ^ i) << 4) + (byte & 15));
      }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < J; ++j)
        if (r0 + i < rows && lane + 32 * j < left) c[(r0 + i) * ldc + lane + 32 * j] = v[i][j];
  }
}

// TMA_C: C's rows are 16-byte aligned and go out by TMA.  BF16: C's type.
// (Kernels of their own: with all four stores' code in one the products were 1
// to 3 % slower.)
template <bool COLS, bool TMA_C, bool BF16>
__global__ void __launch_bounds__(LTHREADS, 1)
    k_fp8_pair(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
               const __grid_constant__ CUtensorMap tmC, Args g) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_s = ptx::smem_u32(smem_raw);
  uint8_t* smem = smem_raw + ((1024u - (raw_s & 1023u)) & 1023u);
  uint8_t* staging = smem + LSTAGES * LSTAGE;
  float* slots = reinterpret_cast<float*>(staging + EPI * LSTAGING);  // [LGROUPS * LGROUP][LSLOT]
  float* sbias = slots + LGROUPS * LGROUP * LSLOT;                    // [epilogue warp][LCPW]
  uint64_t* full = reinterpret_cast<uint64_t*>(sbias + EPI * LCPW);
  uint64_t* empty = full + LSTAGES;
  uint64_t* tfull = empty + LSTAGES;    // [2 * half + buffer] holds a k-block's product
  uint64_t* tempty = tfull + 4;         // [2 * half + buffer] both CTAs have read it
  uint64_t* sfull = tempty + 4;         // [LGROUPS] a group holds its k-blocks' scales
  uint64_t* sempty = sfull + LGROUPS;   // [LGROUPS] the epilogue has used them
  uint32_t* tslot = reinterpret_cast<uint32_t*>(sempty + LGROUPS);
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
      ptx::mbar_init(&empty[s], 2);  // the MMAs of both halves
    }
    for (int b = 0; b < 4; ++b) {
      ptx::mbar_init(&tfull[b], 1);
      ptx::mbar_init(&tempty[b], EPI);  // four warps of each CTA
    }
    for (int i = 0; i < LGROUPS; ++i) {
      ptx::mbar_init(&sfull[i], 32);
      ptx::mbar_init(&sempty[i], EPI);
    }
    *abort_flag = 0;
    *never_set = 0;
    ptx::fence_mbar_init();
    ptx::prefetch_tmap(&tmA);
    ptx::prefetch_tmap(&tmB);
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

  if (warp < 4) {
    ptx::regs_dec<LREGS_LOW>();
  if (warp == 0) {
    if (lane == 0) {
      const uint32_t full0 = ptx::mapa_shared(ptx::smem_u32(&full[0]), 0);
      int it = 0;
      for (int t = pair; t < ntiles && !*abort_flag; t += npairs) {
        int tp, tq;
        tile_of(t, g.ntp, g.ntq, tp, tq);
        const int ar = tp * 2 * BM + (int)crank * BM, br = tq * LN + (int)crank * (LN / 4);
        for (int kb = 0; kb < nkb; ++kb, ++it) {
          const int s = it % LSTAGES;
          if (!ptx::mbar_wait(&empty[s], (((uint32_t)(it / LSTAGES)) & 1u) ^ 1u, kWaitTimeoutNs, abort_flag)) {
            latch(g.err, abort_flag);
            break;
          }
          if (lead) ptx::mbar_arrive_expect_tx(&full[s], 2 * LSTAGE);
          uint8_t* a = smem + s * LSTAGE;
          ptx::tma_load_2d_pair(a, &tmA, full0 + 8u * (uint32_t)s, kb * KB, ar);
          // this CTA's 64 of each half's 128 columns
          ptx::tma_load_2d_pair(a + BM * KB, &tmB, full0 + 8u * (uint32_t)s, kb * KB, br);
          ptx::tma_load_2d_pair(a + BM * KB + LN / 4 * KB, &tmB, full0 + 8u * (uint32_t)s, kb * KB, br + LN / 2);
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
  } else if (warp <= 2) {
    if (lead) {
      // Warp 1 issues the MMAs of the first half of the columns, warp 2 those
      // of the second: a k-block's waits and issues take one warp longer than
      // its MMAs run, since it shares its scheduler with two epilogue warps.
      // The whole warp walks the loop, so that its variables are uniform, and
      // one lane issues.  Descriptors differ from the first stage's by their
      // address field only (16-byte units).
      constexpr uint32_t idesc = ptx::idesc_e4m3_f32(2 * BM, LN / 2);
      const int h = warp - 1;
      const uint64_t ad0 = ptx::sdesc_sw128(ptx::smem_u32(smem), 16, 1024);
      const uint64_t bd0 = ptx::sdesc_sw128(ptx::smem_u32(smem + BM * KB + h * (LN / 4) * KB), 16, 1024);
      const int total = ntiles > pair ? (ntiles - pair + npairs - 1) / npairs * nkb : 0;
      uint64_t *te = &tempty[2 * h], *tf = &tfull[2 * h];
      int s = 0;
      uint32_t ph = 0, tph = 1;  // parities of full[s] and te[b]
      for (int it = 0; it < total; ++it) {
        const uint32_t b = (uint32_t)it & 1u;
        const bool ok = ptx::mbar_wait(&full[s], ph, kWaitTimeoutNs, abort_flag) &&
                        ptx::mbar_wait_cluster(&te[b], tph, kWaitTimeoutNs, abort_flag);
        if (!__all_sync(0xffffffffu, ok)) {
          latch(g.err, abort_flag);
          break;
        }
        ptx::tc_fence_after();
        const uint64_t ad = ad0 + (uint64_t)(s * (LSTAGE >> 4)), bd = bd0 + (uint64_t)(s * (LSTAGE >> 4));
        const uint32_t d = tmem + (uint32_t)h * LN + b * (LN / 2);
        if (ptx::elect_one()) {
          ptx::umma_f8_pair(d, ad, bd, idesc, 0u);
#pragma unroll
          for (int k = 1; k < KB / 32; ++k) ptx::umma_f8_pair(d, ad + 2 * k, bd + 2 * k, idesc, 1u);
          ptx::umma_commit_pair(&tf[b], 3);
          ptx::umma_commit_pair(&empty[s], 3);
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
    const int total = ntiles > pair ? (ntiles - pair + npairs - 1) / npairs * nkb : 0;
    int it = 0;
    for (int t = pair; t < ntiles && !*abort_flag; t += npairs) {
      int tp, tq;
      tile_of(t, g.ntp, g.ntq, tp, tq);
      const int row = tp * 2 * BM + (int)crank * BM, col = tq * LN;
      for (int kb = 0; kb < nkb; ++kb, ++it) {
        const int gr = (it / LGROUP) % LGROUPS;
        if (it % LGROUP == 0 && !ptx::mbar_wait(&sempty[gr], (((uint32_t)(it / (LGROUP * LGROUPS))) & 1u) ^ 1u,
                                                kWaitTimeoutNs, abort_flag)) {
          latch(g.err, abort_flag);
          break;
        }
        float* d = slots + it % (LGROUP * LGROUPS) * LSLOT;
        // rows and columns past the matrix hold zeros: any scale will do
#pragma unroll
        for (int e = lane; e < BM; e += 32) ptx::cp_async4(d + e, scale_ptr(g.sp, kb, min(row + e, g.P - 1)));
        if constexpr (COLS) {
#pragma unroll
          for (int e = lane; e < LN; e += 32) ptx::cp_async4(d + BM + e, scale_ptr(g.sq, kb, min(col + e, g.Q - 1)));
        } else {
          if (lane < 2) ptx::cp_async4(d + BM + lane, scale_ptr(g.sq, kb, min(col + lane * LCPW, g.Q - 1)));
        }
        if (it % LGROUP == LGROUP - 1 || it == total - 1) ptx::cp_async_arrive(&sfull[gr]);
      }
    }
    ptx::cp_async_commit();
    ptx::cp_async_wait<0>();
  }
  } else {
    ptx::regs_inc<LREGS_EPI>();
    const int q = warp & 3, ew = warp - 4, half = ew / 4;
    const uint32_t trow = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(half * LN);
    const uint32_t te0 = ptx::mapa_shared(ptx::smem_u32(&tempty[2 * half]), 0);
    uint8_t* stage = staging + ew * LSTAGING;
    float* bias = sbias + ew * LCPW;
    uint64_t* tf = &tfull[2 * half];
    uint32_t it = 0;
    for (int t = pair; t < ntiles; t += npairs) {
      int tp, tq;
      tile_of(t, g.ntp, g.ntq, tp, tq);
      const int rbase = tp * 2 * BM + (int)crank * BM + q * 32;
      const int cbase = tq * LN + half * LCPW;
      float acc[LCPW];
#pragma unroll
      for (int i = 0; i < LCPW; ++i) acc[i] = 0.f;
      __syncwarp();  // the last tile's bias has been read
#pragma unroll
      for (int e = 0; e < LCPW; e += 32)
        bias[e + lane] = g.bias && cbase + e + lane < g.Q ? __ldg(g.bias + cbase + e + lane) : 0.f;
      // Between a k-block's last read and the next one's first, the tensor
      // cores may be waiting for this warp: the next k-block's scales are read
      // and its barrier is tested before the last chunk's arithmetic, and its
      // first read is issued there if its product is already in.
      constexpr int LD = 32, NC = LCPW / LD;
      static_assert(NC % 2 == 0, "each k-block starts with the same registers");
      uint32_t r[2][LD];
      uint64_t row2 = 0;
      const float* cs = nullptr;
      bool ok = true;
      auto scales = [&](uint32_t j) {  // of k-block j, counted over the tiles
        if (j % LGROUP == 0)
          ok = ptx::mbar_wait(&sfull[(j / LGROUP) % LGROUPS], (j / (LGROUP * LGROUPS)) & 1u, kWaitTimeoutNs, abort_flag);
        const float* d = slots + j % (LGROUP * LGROUPS) * LSLOT;
        float f = d[q * 32 + lane];
        if constexpr (!COLS) f *= d[BM + half];
        row2 = ptx::pack2(f, f);
        cs = d + BM + half * LCPW;
      };
      scales(it);
      bool early = false, live = true;
      for (int kb = 0; kb < nkb; ++kb, ++it) {
        const uint32_t b = it & 1u, at = trow + b * LCPW;
        if (!early) {
          ok = ok && ptx::mbar_wait(&tf[b], (it >> 1) & 1u, kWaitTimeoutNs, abort_flag);
          if (!ok) latch(g.err, abort_flag);
          live = __all_sync(0xffffffffu, ok);
          if (!live) break;
          ptx::tc_fence_after();
          tmem_read<LD>(at, r[0]);
        }
        const uint64_t now2 = row2;
        const float* nowc = cs;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          ptx::tmem_ld_wait_for(r[c & 1]);
          if (c + 1 < NC) {
            tmem_read<LD>(at + (c + 1) * LD, r[(c + 1) & 1]);
          } else {
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) {
              // TMEM reads that have completed (the wait above, and the fence):
              // nothing to release, only an arrival that the issuing CTA sees
              // (a release at cluster scope: 4096 x 8192 x 8192 with its quantizer
              // 461 us in place of 221)
              ptx::mbar_arrive_at(te0 + 8u * b);
              // the scales of the group before this k-block are used up
              if (it % LGROUP == 0 && it > 0) ptx::mbar_arrive(&sempty[(it / LGROUP - 1) % LGROUPS]);
            }
            early = false;
            if (kb + 1 < nkb) {
              scales(it + 1);
              early = __all_sync(0xffffffffu, ok && ptx::mbar_test(&tf[b ^ 1u], ((it + 1) >> 1) & 1u));
              if (early) {
                ptx::tc_fence_after();
                tmem_read<LD>(trow + (b ^ 1u) * LCPW, r[0]);
              }
            }
          }
          scaled_add<LD, COLS>(acc + c * LD, r[c & 1], now2, nowc + c * LD);
        }
      }
      if (!live) break;
      if (t + npairs >= ntiles && threadIdx.x == 128) ptx::griddep_launch_dependents();
      // Store: 128 bytes of each of the warp's 32 rows at a time through the
      // swizzled staging block, by TMA where C's rows are 16-byte aligned (it
      // clips what lies past the matrix, and the warp need not wait for the
      // memory), else by the lanes along a row, eight rows read before the
      // first is written (2023 x 2375 x 368, bf16 C: 10.9 us, 24 one by one,
      // 8.2 for 2376 columns).
      auto block = [&](int ch) {  // staging block of chunk ch, free again
        if (TMA_C && lane == 0) ptx::bulk_wait_read1();
        __syncwarp();
        return stage + (ch & 1) * (LSTAGING / 2);
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
            rows_out(from, static_cast<uint16_t*>(g.c) + at, g.ldc, rows, left, lane);
          else
            rows_out(from, static_cast<uint32_t*>(g.c) + at, g.ldc, rows, left, lane);
        }
      };
      // four accumulators with bias and activation
      auto value = [&](int i) {
        const float4 v = *reinterpret_cast<const float4*>(bias + i);
        return make_float4(finish(acc[i] + v.x, g.relu), finish(acc[i + 1] + v.y, g.relu),
                           finish(acc[i + 2] + v.z, g.relu), finish(acc[i + 3] + v.w, g.relu));
      };
      if constexpr (BF16) {
#pragma unroll
        for (int ch = 0; ch < LCPW / 64; ++ch) {
          uint8_t* to = block(ch);
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
          uint8_t* to = block(ch);
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
// (swap), so that a single row needs 16 columns and not 128 lanes.
//
// Bound by the weights' bytes where they are many (1 x 8192 x 8192: 14.9 us, 4.5
// TB/s), else by latency: launch, ring fill, exchange, store (1 x 2000 x 2000:
// 5.1 us from operands beyond L2, 4.0 from weights in it; 333 x 1999 x 1337: 7.9
// us).
template <int BN>
struct SCfg {
  static constexpr int STAGE = (BM + BN) * KB;
  static constexpr int STAGES = BN >= 128 ? 6 : BN >= 64 ? 8 : 9;
  static constexpr int CPW = BN / 2;
  static constexpr int BUFS = 4;                          // TMEM buffers (a power of 2)
  static constexpr uint32_t ACC = BN < 32 ? 32 : BN;      // TMEM columns of a buffer
  static constexpr uint32_t TCOLS = BUFS * ACC;
  static constexpr int PITCH = BM + 1;                    // floats per column of the exchange buffer
  static constexpr int SLOTS = 4;                         // k-blocks of scales in flight or in use
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
        const uint32_t b = (uint32_t)it % C::BUFS;
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
        tph ^= b == C::BUFS - 1 ? 1u : 0u;
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
    // scales three k-blocks ahead of their use
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
      __syncwarp();  // every lane's copies of this slot, and its use of the slot filled next
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

// CTA pairs the GPU holds at once (one CTA per SM; an SM without a partner in
// its cluster group stays out); 0 if the pair kernel was not built with the
// registers that its split counts on, and so must not run.
template <bool COLS, bool TMA_C, bool BF16>
int resident_pairs(int dev) {
  static PerDevice<int> kept;
  int n = 0;
  const cudaError_t e = kept.get(dev, &n, [](int* pairs) {
    cudaFuncAttributes fa{};
    constexpr auto kernel = k_fp8_pair<COLS, TMA_C, BF16>;
    cudaError_t e = cudaFuncGetAttributes(&fa, kernel);
    if (e != cudaSuccess || fa.numRegs != LREGS) return e;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, L_SMEM);
    if (e != cudaSuccess) return e;
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
    return cudaOccupancyMaxActiveClusters(pairs, kernel, &cfg);
  });
  if (e != cudaSuccess) cudaGetLastError();  // leave no error behind: the split kernel runs
  return e == cudaSuccess ? n : 0;
}

template <int BN, bool COLS>
cudaError_t run_split(const CUtensorMap& p, const CUtensorMap& q, const Args& g, int ks_log, cudaStream_t st) {
  const cudaError_t e = allow_smem<k_fp8_split<BN, COLS>>(SCfg<BN>::SMEM);
  if (e != cudaSuccess) return e;
  return launch(k_fp8_split<BN, COLS>, (unsigned)(g.ntp * g.ntq) << ks_log, THREADS, 1 << ks_log, SCfg<BN>::SMEM, st, p, q, g,
                ks_log);
}

// Clusters of a split kernel the GPU holds at once.
template <int BN, bool COLS>
int resident_clusters(int dev, int ks_log) {
  struct Counts { int n[4]; };
  static PerDevice<Counts> kept;
  Counts c{};
  const cudaError_t e = kept.get(dev, &c, [](Counts* r) {
    cudaError_t e = allow_smem<k_fp8_split<BN, COLS>>(SCfg<BN>::SMEM);
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
      e = cudaOccupancyMaxActiveClusters(&r->n[l], k_fp8_split<BN, COLS>, &cfg);
      if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
  });
  if (e != cudaSuccess) cudaGetLastError();
  return e == cudaSuccess ? c.n[ks_log] : 0;
}
int clusters_of(int dev, int bn, bool each, int ks_log) {
  switch (bn) {
    case 16: return resident_clusters<16, true>(dev, ks_log);
    case 32: return resident_clusters<32, true>(dev, ks_log);
    case 64: return resident_clusters<64, true>(dev, ks_log);
    default: return each ? resident_clusters<128, true>(dev, ks_log) : resident_clusters<128, false>(dev, ks_log);
  }
}

// The shape of a product: tile, orientation and split with the least
// estimated time.  The constants (us) are least-squares readings of a sweep of
// all shapes over 23 sizes from 1 x 2000 x 2000 to 512 x 8192 x 8192: a wave
// of tiles takes a time per k-block and a fixed one (launch, fill, exchange,
// store), and no shape moves its operands faster than about 9 TB/s.
struct Plan {
  int bn;      // 256: the pair kernel
  bool swap;
  int ks_log;
};
Plan plan(int dev, int M, int N, int K, bool cols, int pairs) {
  const double nkb = cdiv(K, KB);
  Plan best{LN, false, 0};
  double t = 1e30;
  if (pairs > 0) {
    const double tiles = (double)cdiv(M, 2 * BM) * cdiv(N, LN);
    t = 3.5 + std::ceil(tiles / pairs) * (nkb * (cols ? 0.62 : 0.38) + 1.0);
  }
  struct Shape { int bn; bool swap; double step, fixed; };
  const Shape shapes[5] = {
      {16, true, 0.24, 2.9}, {32, true, 0.30, 3.2}, {64, true, 0.28, 4.6}, {128, true, 0.42, 6.0},
      {128, false, cols ? 0.42 : 0.31, 7.0}};
  for (const Shape& sh : shapes) {
    const int P = sh.swap ? N : M, Q = sh.swap ? M : N;
    const double tiles = (double)cdiv(P, BM) * cdiv(Q, sh.bn);
    const double moved = tiles * nkb * (BM + sh.bn) * KB / 9e6;
    for (int l = 0; l < 4; ++l) {
      const int room = clusters_of(dev, sh.bn, sh.swap || cols, l);
      if ((1 << l) > nkb || room < 1) break;
      const double waves = std::ceil(tiles / room), per = std::ceil(nkb / (1 << l));
      const double c = sh.fixed + (l ? 0.5 : 0.0) + std::max(moved, waves * per * sh.step + (waves - 1) * sh.fixed);
      if (c < t) {
        t = c;
        best = Plan{sh.bn, sh.swap, l};
      }
    }
  }
  return best;
}

}  // namespace

ff_status fp8_gemm(const Fp8Gemm& f, cudaStream_t st) {
  const int ld = fp8_stride(f.K);
  const bool cols = !f.b_tiles;
  int dev = 0;
  FF_TRY(cudaGetDevice(&dev), "8-bit matrix product");
  auto room = [&](auto c, auto b) {
    return std::min(resident_pairs<c.value, true, b.value>(dev), resident_pairs<c.value, false, b.value>(dev));
  };
  using Y = std::true_type;
  using N = std::false_type;
  const int pairs = cols ? (f.out_bf16 ? room(Y{}, Y{}) : room(Y{}, N{})) : (f.out_bf16 ? room(N{}, Y{}) : room(N{}, N{}));
  const Plan pl = plan(dev, f.M, f.N, f.K, cols, pairs);
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
  if (pairk && pairs < 1) return FF_ERR_UNSUPPORTED;  // no kernel fits this device
  g.ntp = cdiv(g.P, pairk ? 2 * BM : BM);
  g.ntq = cdiv(g.Q, pl.bn);
  if ((long long)g.ntp * g.ntq << pl.ks_log > 0x3FFFFFFFll) return FF_ERR_UNSUPPORTED;
  CUtensorMap p, q;
  if (!make_sw128_map(&p, pl.swap ? f.b : f.a, 1, f.K, g.P, ld, KB, BM) ||
      !make_sw128_map(&q, pl.swap ? f.a : f.b, 1, f.K, g.Q, ld, KB, pairk ? LN / 4 : pl.bn))
    return FF_ERR_INVALID_ARG;
  const int es = f.out_bf16 ? 2 : 4;
  CUtensorMap c = p;
  // whole 16-byte units a row: a row that ends inside one is written to the
  // unit's end, into what lies between the rows
  const bool tma_c = pairk && (long long)f.N * es % 16 == 0 && f.ldc <= 0x7FFFFFFFll && f.ldc >= f.N && make_sw128_map(&c, f.c, es, f.N, f.M, (int)f.ldc, 128 / es, 32);
  const double work = 2.0 * f.M * f.N * f.K;
  auto go = [&]() -> cudaError_t {
    if (pairk) {
      const unsigned grid = 2u * (unsigned)std::min((long long)pairs, (long long)g.ntp * g.ntq);
      auto* kernel =
          f.out_bf16 ? (cols ? (tma_c ? k_fp8_pair<true, true, true> : k_fp8_pair<true, false, true>)
                             : (tma_c ? k_fp8_pair<false, true, true> : k_fp8_pair<false, false, true>))
                     : (cols ? (tma_c ? k_fp8_pair<true, true, false> : k_fp8_pair<true, false, false>)
                             : (tma_c ? k_fp8_pair<false, true, false> : k_fp8_pair<false, false, false>));
      return launch(kernel, grid, LTHREADS, 2, L_SMEM, st, p, q, c, g);
    }
    const bool each = cols || pl.swap;
    switch (pl.bn) {
      case 16: return run_split<16, true>(p, q, g, pl.ks_log, st);
      case 32: return run_split<32, true>(p, q, g, pl.ks_log, st);
      case 64: return run_split<64, true>(p, q, g, pl.ks_log, st);
      default: return each ? run_split<128, true>(p, q, g, pl.ks_log, st) : run_split<128, false>(p, q, g, pl.ks_log, st);
    }
  };
  FF_LAUNCH(pairk ? K_FP8_PAIR : K_FP8_GEMM, work, st, go(), "8-bit matrix product");
  return FF_OK;
}

}  // namespace ff
