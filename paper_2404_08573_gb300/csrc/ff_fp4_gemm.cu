// The 4-bit matrix product C = act(A B^T + bias), A and B in e2m1 with a
// power-of-two scale per block of 32 along the contraction.  The tensor cores
// apply the scales themselves (kind::mxf4), so a tile is one fp32 accumulator
// in TMEM over the whole contraction.
//
// A ring stage is 256 contraction indices: one 128-byte swizzled row of packed
// e2m1 pairs per operand row, and two scale tiles (512 bytes: 128 rows x 4
// blocks of 32) per 128 operand rows, which one thread copies on to TMEM ahead
// of the stage's four MMAs (K = 64).
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

// ------------------------------------------------------- small products
// One CTA per 128 x BN tile and slice of the contraction: the CTAs of a
// cluster (1, 2, 4 or 8) share a tile's stages, exchange their partial sums
// through distributed shared memory (each sums its share of the columns, in
// rank order) and store.  With few rows of A its rows go on the MMA's columns
// (swap), so that a single row needs 16 columns and not 128 lanes.  Roles:
//
//   warp 0      TMA producer
//   warp 1      allocates TMEM, one lane copies the scales and issues the MMAs
//   warps 2..9  epilogue: TMEM lane quarter warp % 4, half of the columns each
//
// A tile of BN < 128 columns takes its scales from a whole scale tile of 128,
// from column (q0 % 128) / 32 of it on, which must be even: BN < 64 serves
// products of one column tile only.
template <int BN>
struct SCfg {
  static constexpr int STAGE = (BM + BN) * KB + 2 * SF;
  static constexpr int STAGES = BN >= 128 ? 6 : BN >= 64 ? 8 : 9;
  static constexpr int CPW = BN / 2;
  static constexpr uint32_t ACC = BN < 32 ? 32 : BN;       // TMEM columns of the accumulator
  static constexpr uint32_t TCOLS = BN >= 128 ? 256 : BN >= 64 ? 128 : 64;
  static_assert(ACC + 4 * SFC <= TCOLS, "the accumulator and two stages' scales");
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
      bool ok = ptx::mbar_wait(&full[s], (uint32_t)(it / C::STAGES) & 1u, kWaitTimeoutNs, abort_flag);
      // two stages' scales fit TMEM: those of the stage before the last have been used
      if (it >= 2)
        ok = ok && ptx::mbar_wait(&empty[(it - 2) % C::STAGES], (uint32_t)((it - 2) / C::STAGES) & 1u, kWaitTimeoutNs, abort_flag);
      if (!__all_sync(0xffffffffu, ok)) {
        latch(g.err, abort_flag);
        break;
      }
      ptx::tc_fence_after();
      const uint64_t at = (uint64_t)(s * (C::STAGE >> 4));
      const uint32_t sfp = tmem + C::ACC + (uint32_t)(it & 1) * 2 * SFC, sfq = sfp + SFC;
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
    case 64: return resident_clusters<64>(dev, ks_log);
    default: return resident_clusters<128>(dev, ks_log);
  }
}

// The shape of a product: tile, orientation and split with the least estimated
// time: a wave of tiles takes a time per stage and a fixed one (launch, fill,
// exchange, store), and no shape moves its operands faster than about 9 TB/s.
struct Plan {
  int bn;  // 0: no shape fits
  bool swap;
  int ks_log;
};
Plan plan(int dev, int M, int N, int K) {
  const double nkb = cdiv(K, KS);
  Plan best{0, false, 0};
  double t = 1e30;
  struct Shape { int bn; bool swap; double step, fixed; };
  const Shape shapes[5] = {{16, true, 0.24, 2.9}, {32, true, 0.28, 3.2}, {64, true, 0.28, 4.6}, {128, true, 0.31, 6.0},
                           {128, false, 0.31, 7.0}};
  for (const Shape& sh : shapes) {
    const int P = sh.swap ? N : M, Q = sh.swap ? M : N;
    if (sh.bn < 64 && Q > sh.bn) continue;
    const double tiles = (double)cdiv(P, BM) * cdiv(Q, sh.bn);
    const double moved = tiles * nkb * (BM + sh.bn) * KB / 9e6;
    for (int l = 0; l < 4; ++l) {
      const int room = clusters_of(dev, sh.bn, l);
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
  const Plan pl = plan(dev, f.M, f.N, f.K);
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
  g.ntp = cdiv(g.P, BM);
  g.ntq = cdiv(g.Q, pl.bn);
  if ((long long)g.ntp * g.ntq << pl.ks_log > 0x3FFFFFFFll) return FF_ERR_UNSUPPORTED;
  const int ld = fp4_stride(f.K), words = cdiv(f.K, 128) * (kFp4ScaleTile / 4);
  CUtensorMap m[4];
  if (!make_sw128_map(&m[0], pl.swap ? f.b : f.a, 1, ld, g.P, ld, KB, BM) ||
      !make_sw128_map(&m[1], pl.swap ? f.a : f.b, 1, ld, g.Q, ld, KB, pl.bn) ||
      !make_plain_map(&m[2], pl.swap ? f.sb : f.sa, 4, words, cdiv(g.P, 128), words, SF_BOX, 1) ||
      !make_plain_map(&m[3], pl.swap ? f.sa : f.sb, 4, words, cdiv(g.Q, 128), words, SF_BOX, 1))
    return FF_ERR_INVALID_ARG;
  auto go = [&]() -> cudaError_t {
    switch (pl.bn) {
      case 16: return run_split<16>(m, g, pl.ks_log, st);
      case 32: return run_split<32>(m, g, pl.ks_log, st);
      case 64: return run_split<64>(m, g, pl.ks_log, st);
      default: return run_split<128>(m, g, pl.ks_log, st);
    }
  };
  FF_LAUNCH(K_FP4_GEMM, 2.0 * f.M * f.N * f.K, st, go(), "4-bit matrix product");
  return FF_OK;
}

}  // namespace ff
