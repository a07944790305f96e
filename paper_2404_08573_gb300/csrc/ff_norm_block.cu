// Group norm, the block path: a slab (one or more whole groups) of one sample is
// held in the shared memory of a thread block, so x (and dy) are read once.
//
// Persistent: a block takes consecutive (slab, sample) units, so gamma, beta
// and the gradient's column sums change with the slab only, and the next
// unit's values are copied (cp.async) under the arithmetic of this one.  A
// thread has one vector column of the slab and every TR-th position, and reads
// only what it copied itself.  Its sums go through shared memory to a few
// lanes per group and back.  Sums of x are held relative to the group's pivot,
// as in ff_norm.cu.
//
// Bound by latency in bf16: a unit costs two barriers around the fold and some
// 450 instructions per thread beside the 14 or so of a value with silu (256 x 49
// x 1024, 32 groups: 21 us with 4 vectors a thread, 16 with 7), and few warps are
// there to cover them.  64 x 784 x 256 (32 groups) takes 17.5 us, 2.9 TB/s, in
// 128 blocks of 16 warps: 24 SMs have none, the others a quarter of their
// warps and issue 52 % of the time.  fp32 moves twice the bytes for the same
// (512 x 196 x 256 in 16 groups: 40 us, 5.1 TB/s, gradient 61 us, 5.0 TB/s; with
// silu, whose exponential is the full one there, 46 and 75 us).  Splitting a slab's
// positions over a cluster of 2 to 8 blocks, with the sums exchanged through
// distributed shared memory, reached larger samples but was slower than the
// column passes there (32 x 4096 x 512: 100 against 72 us), so larger ones take
// those.
#include <algorithm>
#include <cmath>

#include "ff_norm.cuh"

namespace ff {
namespace {

constexpr int kMaxT = 512, kMaxGS = 64;
constexpr int kGradValues = 32;  // values per thread whose du the gradient keeps in registers

struct Geom {
  int T, GS, nv, V;
  int WV, Wg;    // vectors per position of the slab, and of a group
  int TR, M;     // thread rows; threads per group
  int R, r_log;  // lanes that add up a group's threads (a power of 2)
  int lo, rem;   // thread rows below rem have lo + 1 positions, the others lo
  int units, total;  // units per block and in all
  int span;      // gradient: vectors from one stage (x and dy) to the next
  int wide;      // gamma and beta are 16-byte aligned
  float inv;     // 1 / values of a group
  FastDiv by_WV, by_Wg, by_n;
};

struct Place {
  int tc, tr, gl, slot;  // vector column, thread row, group within the slab, place among its threads
  int mine;              // positions of this thread
  bool on;
  __device__ __forceinline__ explicit Place(const Geom& q) {
    tr = (int)q.by_WV.div(threadIdx.x);
    tc = (int)threadIdx.x - tr * q.WV;
    on = tr < q.TR;
    gl = on ? (int)q.by_Wg.div((uint32_t)tc) : 0;
    slot = gl * q.M + tr * q.Wg + (tc - gl * q.Wg);
    mine = on ? q.lo + (tr < q.rem ? 1 : 0) : 0;
  }
};

// Where a thread stands among the units: sample and slab, and how far its
// first position lies from the start of a matrix of row stride ld.  Units
// follow one another sample by sample, slab by slab.
struct Cursor {
  int b, slab;
  __device__ __forceinline__ Cursor(int u, const GnShape& s, const Geom& q) {
    slab = (int)q.by_n.div((uint32_t)u);
    b = u - slab * s.n;
  }
  __device__ __forceinline__ void next(const GnShape& s) {
    if (++b == s.n) {
      b = 0;
      ++slab;
    }
  }
  __device__ __forceinline__ long long offset(const GnShape& s, const Geom& q, const Place& p, long long ld) const {
    return ((long long)b * s.S + p.tr) * ld + slab * q.GS * s.Cg + (p.on ? p.tc * q.V : 0);
  }
};

// Bytes of the groups' totals and of the threads' sums, before the stages.
__host__ __device__ constexpr int head_bytes(int T, int GS) { return (2 * GS * 8 + 2 * T * 8 + 15) & ~15; }

// This thread's positions of a unit, into its own places of a stage:
// vector i at [i T + thread].
template <typename T, int V>
__device__ __forceinline__ void fetch(typename Vec<T, V>::Raw* stage, const T* p, long long step, int mine, int threads) {
  typename Vec<T, V>::Raw* d = stage + threadIdx.x;
  auto copy = [&](int i) {
    if constexpr (sizeof(T) * V == 16)
      ptx::cp_async16(d, p);
    else if constexpr (sizeof(T) * V == 4)
      ptx::cp_async4(d, p);
    else  // two bytes: there is no asynchronous copy
      *d = Vec<T, V>::load(p);
    d += threads;
    p += step;
  };
#pragma unroll 4
  for (int i = 0; i < mine; ++i) copy(i);
}

template <typename T, int V>
__global__ void __launch_bounds__(kMaxT, 2) k_gn_block(GnArgs<T> a, Geom q) {
  using VV = Vec<T, V>;
  using PV = Pairs<V>;
  using Raw = typename VV::Raw;
  extern __shared__ __align__(16) uint8_t smem[];
  const GnShape& s = a.s;
  const Place p(q);
  float2* totals = reinterpret_cast<float2*>(smem);  // [2][GS]
  float2* parts = totals + 2 * q.GS;                 // [2][T]
  Raw* stages = reinterpret_cast<Raw*>(smem + head_bytes(q.T, q.GS));  // [2][nv T]
  const int stage = q.nv * q.T;
  const int u0 = (int)blockIdx.x * q.units, u1 = min(q.total, u0 + q.units);
  ptx::griddep_wait();
  Cursor cur(u0, s, q), ahead = cur;
  const long long xstep = (long long)q.TR * s.ldx, ystep = (long long)q.TR * s.ldy;
  float pivot = 0.f;  // the next unit's group's
  auto start = [&](int u, int k) {
    if (u < u1) {
      fetch<T, V>(stages + k * stage, a.x + ahead.offset(s, q, p, s.ldx), xstep, p.mine, q.T);
      const T* head = a.x + (long long)ahead.b * s.S * s.ldx + (ahead.slab * q.GS + p.gl) * s.Cg;
      float v[1], w[1];
      Vec<T, 1>::unpack(Vec<T, 1>::load(head), v);
      Vec<T, 1>::unpack(Vec<T, 1>::load(head + second_of(s)), w);
      pivot = pivot_of(v[0], w[0]);
      ahead.next(s);
    }
    ptx::cp_async_commit();
  };
  start(u0, 0);
  float ga[V], be[V];
  int slab = -1;
  for (int u = u0; u < u1; ++u, cur.next(s)) {
    const int k = (u - u0) & 1;
    const float P = pivot;
    start(u + 1, k ^ 1);
    if (cur.slab != slab) {
      slab = cur.slab;
      const int c = slab * q.GS * s.Cg + (p.on ? p.tc * V : 0);
      load_params<V>(ga, a.gamma, c, 1.f, q.wide);
      load_params<V>(be, a.beta, c, 0.f, q.wide);
    }
    float2* part = parts + k * q.T;
    ptx::cp_async_wait<1>();
    const Raw* mem = stages + k * stage + threadIdx.x;
    // sums relative to the thread's own first value
    float piv = P;
    if (p.mine > 0) {
      float v[V];
      VV::unpack(mem[0], v);
      piv = v[0];
    }
    const uint64_t npiv = both(-piv);
    uint64_t s1 = 0, s2 = 0;
    const Raw* m = mem;
#pragma unroll 4
    for (int i = 0; i < p.mine; ++i, m += q.T) {
      float v[V];
      uint64_t d[PV::N];
      VV::unpack(*m, v);
      PV::of(v, d);
      if constexpr (V == 1) {
        d[0] = ptx::pack2(v[0] - piv, 0.f);
      } else {
#pragma unroll
        for (int e = 0; e < PV::N; ++e) d[e] = ptx::add2(d[e], npiv);
      }
#pragma unroll
      for (int e = 0; e < PV::N; ++e) {
        s1 = ptx::add2(s1, d[e]);
        s2 = ptx::fma2(d[e], d[e], s2);
      }
    }
    if (p.on) {
      const float2 f1 = ptx::unpack2(s1), f2 = ptx::unpack2(s2);
      const float t1 = f1.x + f1.y, dm = p.mine > 0 ? __fdividef(t1, (float)(p.mine * V)) : 0.f;
      part[p.slot] = make_float2((piv - P) + dm, (f2.x + f2.y) - t1 * dm);
    }
    __syncthreads();
    if ((int)(threadIdx.x & ~31u) < q.GS * q.R) {
      const int gg = (int)(threadIdx.x >> q.r_log), l = (int)(threadIdx.x & (unsigned)(q.R - 1));
      const bool real = gg < q.GS;
      const float2* t = part + gg * q.M;
      // a group's threads in order of their thread rows: the first `many` have one position more
      const int many = q.rem * q.Wg;
      const float chi = (float)((q.lo + 1) * V), clo = (float)(q.lo * V);
      float sum = 0.f, m2 = 0.f;
      for (int j = l; real && j < q.M; j += q.R) sum = fmaf(t[j].x, j < many ? chi : clo, sum);
      for (int o = q.R / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      const float mean = sum * q.inv;
      for (int j = l; real && j < q.M; j += q.R) {
        const float cnt = j < many ? chi : clo, d = t[j].x - mean;
        if (cnt > 0.f) m2 += fmaf(d * d, cnt, t[j].y);
      }
      for (int o = q.R / 2; o > 0; o >>= 1) m2 += __shfl_xor_sync(0xffffffffu, m2, o);
      if (real && l == 0) totals[k * q.GS + gg] = make_float2(mean, rsqrtf(m2 * q.inv + s.eps));
    }
    __syncthreads();
    if (!p.on) continue;
    const float2 tot = totals[k * q.GS + p.gl];
    const float mean = P + tot.x, rstd = tot.y;
    if (a.mean && p.tr == 0 && p.tc == p.gl * q.Wg) {
      const long long at = (long long)cur.b * s.G + cur.slab * q.GS + p.gl;
      a.mean[at] = mean;
      a.rstd[at] = rstd;
    }
    // y = x A + B.  fp32: A = gamma rstd and B = beta with the mean taken off x
    // first (see GradCols in ff_norm.cu).  bf16: B = beta - mean A, rounded
    // once: as far off as the rounding of the mean itself brings y, and far
    // below the output's (with the mean off first 64 x 784 x 256 took 17.9 us
    // in place of 16.6).
    constexpr bool FIRST = sizeof(T) == 4;
    float fa[V], fb[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      fa[e] = ga[e] * rstd;
      fb[e] = FIRST ? be[e] : fmaf(-mean, fa[e], be[e]);
    }
    uint64_t A[PV::N], B[PV::N];
    PV::of(fa, A);
    PV::of(fb, B);
    const uint64_t minus = both(-mean);
    T* y = a.out + cur.offset(s, q, p, s.ldy);
    m = mem;
#pragma unroll 2
    for (int i = 0; i < p.mine; ++i, m += q.T, y += ystep) {
      float v[V];
      uint64_t d[PV::N];
      VV::unpack(*m, v);
      PV::of(v, d);
#pragma unroll
      for (int e = 0; e < PV::N; ++e) d[e] = ptx::fma2(FIRST ? ptx::add2(d[e], minus) : d[e], A[e], B[e]);
      act_pairs<T, V>(d, s.act);
      PV::to(d, v);
      VV::store(y, v);
    }
  }
}

// The gradient.  part_out receives the column sums (du, du h) of each run of
// units of one slab: row (block - first block of the slab).
template <typename T, int V, int NV>
__global__ void __launch_bounds__(kMaxT, 1) k_gn_block_grad(GnArgs<T> a, Geom q, float2* part_out) {
  using VV = Vec<T, V>;
  using PV = Pairs<V>;
  using Raw = typename VV::Raw;
  extern __shared__ __align__(16) uint8_t smem[];
  const GnShape& s = a.s;
  const Place p(q);
  float2* totals = reinterpret_cast<float2*>(smem);  // [2][GS]
  float2* parts = totals + 2 * q.GS;                 // [2][T]
  // [2]: x [nv T], dy [nv T]; or the column sums
  Raw* stages = reinterpret_cast<Raw*>(smem + head_bytes(q.T, q.GS));
  const int stage = q.nv * q.T;
  const int block = (int)blockIdx.x;
  const int u0 = block * q.units, u1 = min(q.total, u0 + q.units);
  ptx::griddep_wait();
  Cursor cur(u0, s, q), ahead = cur;
  const long long xstep = (long long)q.TR * s.ldx, dstep = (long long)q.TR * s.lddy, ostep = (long long)q.TR * s.ldy;
  float nmu = 0.f, nrs = 0.f;
  auto start = [&](int u, int k) {
    if (u < u1) {
      fetch<T, V>(stages + k * q.span, a.x + ahead.offset(s, q, p, s.ldx), xstep, p.mine, q.T);
      fetch<T, V>(stages + k * q.span + stage, a.dy + ahead.offset(s, q, p, s.lddy), dstep, p.mine, q.T);
      const long long at = (long long)ahead.b * s.G + ahead.slab * q.GS + p.gl;
      nmu = __ldg(a.mean + at);
      nrs = __ldg(a.rstd + at);
      ahead.next(s);
    }
    ptx::cp_async_commit();
  };
  start(u0, 0);
  float ga[V], be[V];
  uint64_t G2[PV::N], B2[PV::N], p0[PV::N], p1[PV::N];
#pragma unroll
  for (int e = 0; e < PV::N; ++e) p0[e] = p1[e] = G2[e] = B2[e] = 0;
  int slab = -1;
  // The column sums so far, of slab `of`: over the thread rows in shared
  // memory (the stage that is free), then to their row of part_out.
  auto flush = [&](int of, int k) {
    if (!part_out) return;
    float2* cols = reinterpret_cast<float2*>(stages + k * q.span);  // [V][T]
    float v0[V], v1[V];
    PV::to(p0, v0);
    PV::to(p1, v1);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; ++e) cols[e * q.T + threadIdx.x] = make_float2(v0[e], v1[e]);
    __syncthreads();
    const int first = (int)((long long)of * s.n / q.units);  // block that took the slab's first unit
    float2* to = part_out + (long long)(block - first) * s.C + of * q.GS * s.Cg;
    for (int i = threadIdx.x; i < q.WV * V; i += q.T) {
      const int e = (int)q.by_WV.div((uint32_t)i), tc = i - e * q.WV;
      const float2* col = cols + e * q.T + tc;
      float2 t = col[0];
      for (int r = 1; r < q.TR; ++r) {
        t.x += col[r * q.WV].x;
        t.y += col[r * q.WV].y;
      }
      to[tc * V + e] = t;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < PV::N; ++e) p0[e] = p1[e] = 0;
  };
  for (int u = u0; u < u1; ++u, cur.next(s)) {
    const int k = (u - u0) & 1;
    if (cur.slab != slab) {
      if (slab >= 0) flush(slab, k ^ 1);
      slab = cur.slab;
      const int c = slab * q.GS * s.Cg + (p.on ? p.tc * V : 0);
      load_params<V>(ga, a.gamma, c, 1.f, q.wide);
      load_params<V>(be, a.beta, c, 0.f, q.wide);
      PV::of(ga, G2);
      PV::of(be, B2);
    }
    const float mu = nmu, rs = nrs;
    float2* part = parts + k * q.T;
    start(u + 1, k ^ 1);
    ptx::cp_async_wait<1>();
    const Raw* mx = stages + k * q.span + threadIdx.x;
    const Raw* my = mx + stage;
    // h = (x - mu) rs, the mean taken off first (see GradCols in ff_norm.cu); u = gamma h + beta
    const uint64_t r2 = both(rs), minus = both(-mu);
    uint64_t du[NV][PV::N], q0[PV::N], q1[PV::N];
#pragma unroll
    for (int e = 0; e < PV::N; ++e) q0[e] = q1[e] = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i < p.mine) {
        float x[V], d[V];
        uint64_t hx[PV::N], dd[PV::N];
        VV::unpack(mx[i * q.T], x);
        VV::unpack(my[i * q.T], d);
        PV::of(x, hx);
        PV::of(d, dd);
        uint64_t up[PV::N];
#pragma unroll
        for (int e = 0; e < PV::N; ++e) {
          hx[e] = ptx::mul2(ptx::add2(hx[e], minus), r2);
          up[e] = ptx::fma2(hx[e], G2[e], B2[e]);
        }
        act_grad_pairs<T, V>(dd, up, s.act);
#pragma unroll
        for (int e = 0; e < PV::N; ++e) {
          du[i][e] = dd[e];
          q0[e] = ptx::add2(q0[e], dd[e]);
          q1[e] = ptx::fma2(dd[e], hx[e], q1[e]);
        }
      }
    uint64_t m1 = 0, m2 = 0;
#pragma unroll
    for (int e = 0; e < PV::N; ++e) {
      m1 = ptx::fma2(G2[e], q0[e], m1);
      m2 = ptx::fma2(G2[e], q1[e], m2);
      p0[e] = ptx::add2(p0[e], q0[e]);
      p1[e] = ptx::add2(p1[e], q1[e]);
    }
    if (!a.out) continue;
    if (p.on) {
      const float2 f1 = ptx::unpack2(m1), f2 = ptx::unpack2(m2);
      part[p.slot] = make_float2(f1.x + f1.y, f2.x + f2.y);
    }
    __syncthreads();
    if ((int)(threadIdx.x & ~31u) < q.GS * q.R) {
      const int gg = (int)(threadIdx.x >> q.r_log), l = (int)(threadIdx.x & (unsigned)(q.R - 1));
      const bool real = gg < q.GS;
      const float2* t = part + gg * q.M;
      float2 w = make_float2(0.f, 0.f);
      for (int j = l; real && j < q.M; j += q.R) {
        w.x += t[j].x;
        w.y += t[j].y;
      }
      for (int o = q.R / 2; o > 0; o >>= 1) {
        w.x += __shfl_xor_sync(0xffffffffu, w.x, o);
        w.y += __shfl_xor_sync(0xffffffffu, w.y, o);
      }
      if (real && l == 0) totals[k * q.GS + gg] = w;
    }
    __syncthreads();
    if (!p.on) continue;
    const float2 tot = totals[k * q.GS + p.gl];
    // dx = rs (gamma du - <.> - h <.>) = du (gamma rs) + h c2 + c1
    const uint64_t c1 = both(-rs * tot.x * q.inv), c2 = both(-rs * tot.y * q.inv);
    uint64_t gr[PV::N];
#pragma unroll
    for (int e = 0; e < PV::N; ++e) gr[e] = ptx::mul2(G2[e], r2);
    T* o = a.out + cur.offset(s, q, p, s.ldy);
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i < p.mine) {
        float x[V];
        uint64_t hx[PV::N];
        VV::unpack(mx[i * q.T], x);
        PV::of(x, hx);
#pragma unroll
        for (int e = 0; e < PV::N; ++e)
          hx[e] = ptx::fma2(du[i][e], gr[e], ptx::fma2(ptx::mul2(ptx::add2(hx[e], minus), r2), c2, c1));
        PV::to(hx, x);
        VV::store(o, x);
        o += ostep;
      }
  }
  // all copies have landed and been used; the last unit's stage is not read any more by its own thread,
  // and the other stage is free
  if (slab >= 0) flush(slab, ((u1 - u0 - 1) & 1) ^ 1);
}

template <typename T>
Geom geom_of(const GnArgs<T>& a, int V, const GnBlockPlan& p) {
  const GnShape& s = a.s;
  Geom q;
  q.T = p.T;
  q.GS = p.GS;
  q.nv = p.nv;
  q.V = V;
  q.Wg = s.Cg / V;
  q.WV = q.Wg * q.GS;
  q.TR = q.T / q.WV;
  q.M = q.TR * q.Wg;
  q.lo = s.S / q.TR;
  q.rem = s.S - q.lo * q.TR;
  q.r_log = 5;
  while ((q.GS << q.r_log) > q.T) --q.r_log;
  q.R = 1 << q.r_log;
  q.units = p.units;
  q.span = std::max(2 * q.nv * q.T, (int)(q.T * V * sizeof(float2) / (V * sizeof(T))));
  q.total = s.n * (s.G / q.GS);
  q.wide = ((reinterpret_cast<uintptr_t>(a.gamma) | reinterpret_cast<uintptr_t>(a.beta)) & 15) == 0;
  q.inv = 1.f / ((float)s.S * (float)s.Cg);
  q.by_WV = FastDiv(q.WV);
  q.by_Wg = FastDiv(q.Wg);
  q.by_n = FastDiv(s.n);
  return q;
}

constexpr int kSmem = 227 * 1024;  // of an SM, 1 KB of it reserved per CTA

// Two stages; one of the gradient holds x and dy, or the column sums (V float2 per thread).
int stage_bytes(int T, int nv, int V, int esize, bool grad) {
  const int one = T * nv * V * esize;
  return 2 * (grad ? std::max(2 * one, T * V * 8) : one);
}

template <auto KERNEL, typename... A>
ff_status run(KernelKind kind, double bytes, const Geom& q, const GnBlockPlan& p, int smem, cudaStream_t st,
              const A&... args) {
  FF_TRY(allow_smem<KERNEL>(kSmem), "group norm");
  PdlLaunch l(dim3((unsigned)p.blocks), dim3((unsigned)q.T), st, (size_t)smem);
  FF_LAUNCH(kind, bytes, st, cudaLaunchKernelEx(&l.cfg, KERNEL, args...), "group norm");
  return FF_OK;
}

template <typename T, int V, int NV>
ff_status run_grad(const GnArgs<T>& a, const Geom& q, const GnBlockPlan& p, double bytes, int smem, float2* part,
                   cudaStream_t st) {
  return run<k_gn_block_grad<T, V, NV>>(K_GNORM_GRAD, bytes, q, p, smem, st, a, q, part);
}

template <typename T, int V>
ff_status run_v(const GnArgs<T>& a, const GnBlockPlan& p, bool grad, cudaStream_t st) {
  const Geom q = geom_of(a, V, p);
  const double bytes = (double)a.s.n * a.s.S * a.s.C * sizeof(T);
  const int smem = head_bytes(q.T, q.GS) + stage_bytes(q.T, q.nv, V, sizeof(T), grad);
  if (!grad) return run<k_gn_block<T, V>>(K_GNORM, 2 * bytes, q, p, smem, st, a, q);
  float2* part = a.dgamma ? static_cast<float2*>(a.ws) : nullptr;
  constexpr int N = V == 1 ? 16 : kGradValues / V;  // vectors per thread at most
  const ff_status e = q.nv <= N / 4   ? run_grad<T, V, N / 4>(a, q, p, 3 * bytes, smem, part, st)
                      : q.nv <= N / 2 ? run_grad<T, V, N / 2>(a, q, p, 3 * bytes, smem, part, st)
                                      : run_grad<T, V, N>(a, q, p, 3 * bytes, smem, part, st);
  if (e != FF_OK || !part) return e;
  return gn_param_fold(part, GnFold{0, p.units, a.s.n, q.GS * a.s.Cg}, a.s.C, a.dgamma, a.dbeta, st);
}

}  // namespace

// Threads and slab with the least estimated time (us): the rounds of a block
// at its instructions' time (a warp issues every 6 clocks or so, an SM's all
// together one a clock and scheduler), or the bytes at the rate this path
// reaches with the slab's row segments, whichever is longer.
GnBlockPlan gn_block_plan(const GnShape& s, int V, int esize, bool grad) {
  GnBlockPlan best{};
  best.us = 1e30;
  const double total = (double)s.n * s.S * s.C * esize * (grad ? 3 : 2);
  // du of a thread's values stays in registers: 32 of them, 16 one by one
  const int most = grad ? (V == 1 ? 16 : kGradValues) : 1024;
  for (int GS = 1; GS <= s.G && GS <= kMaxGS; ++GS) {
    if (s.G % GS) continue;
    const long long WV = (long long)GS * (s.Cg / V);
    if (WV > kMaxT) break;
    const double seg = (double)WV * V * esize;
    const double eff = seg >= 128 ? 1.0 : seg >= 64 ? 0.95 : seg >= 32 ? 0.85 : seg / 38;
    for (int T = 128; T <= kMaxT; T *= 2) {
      if (WV > T || GS > T) continue;
      const int TR = T / (int)WV, nv = cdiv(s.S, TR);
      if ((long long)nv * V > most) continue;
      const long long bytes = head_bytes(T, GS) + stage_bytes(T, nv, V, esize, grad);
      if (bytes > kSmem - 1024) continue;
      const int regs = !grad ? 64 : nv * V <= 8 ? 104 : 128;
      const int per_sm = std::max(1, std::min(std::min(2048 / T, 65536 / (T * regs)), (int)(kSmem / (bytes + 1024))));
      const long long units = (long long)s.n * (s.G / GS);
      if (units > 0x3FFFFFFF) continue;
      const long long room = 152ll * per_sm, rounds = (units + room - 1) / room;
      const double warps = per_sm * T / 32.0, issue = std::max(6.0, warps / 4.0) / 1900.0;
      // 2-byte copies are not asynchronous: a value waits for its own (100 x 300
      // x 2000 in 16 groups of 125: 209 us, column passes 75)
      const double round = 0.6 + (grad ? 200 + nv * V * 18 : 450 + nv * V * (V * esize < 4 ? 60 : 12)) * issue;
      const double rate = esize == 4 && seg >= 128 ? (grad ? 4.8e6 : 5.2e6) : (grad ? 2.9e6 : 3.4e6);
      double us = 3.0 + std::max(rounds * round, total / rate / eff);
      // measured beside the estimate: one block of 512 per SM hides less, and
      // 2-byte copies cost still more (100 x 100 x 100 in 4 groups: 17 us)
      if (grad && T == kMaxT) us *= 1.2;
      if (grad && V * esize < 4) us *= 2.5;
      const long long each = grad ? std::min<long long>(rounds, kGradSamples) : rounds;  // (its sums: see kGradSamples)
      if (us < best.us) best = GnBlockPlan{T, GS, nv, (int)((units + each - 1) / each), (int)each, us};
    }
  }
  return best;
}

template <typename T>
ff_status gn_block(const GnArgs<T>& a, int V, const GnBlockPlan& p, bool grad, cudaStream_t st) {
  if constexpr (sizeof(T) == 2) {
    if (V == 8) return run_v<T, 8>(a, p, grad, st);
    if (V == 2) return run_v<T, 2>(a, p, grad, st);
  } else {
    if (V == 4) return run_v<T, 4>(a, p, grad, st);
  }
  return run_v<T, 1>(a, p, grad, st);
}
template ff_status gn_block<bf16>(const GnArgs<bf16>&, int, const GnBlockPlan&, bool, cudaStream_t);
template ff_status gn_block<float>(const GnArgs<float>&, int, const GnBlockPlan&, bool, cudaStream_t);

}  // namespace ff
