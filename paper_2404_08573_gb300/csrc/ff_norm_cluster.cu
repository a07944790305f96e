// Group norm, the cluster path: a slab (one or more whole groups) of one sample
// is held in the shared memory of a CTA, or of a cluster of CTAs that split its
// positions, so x (and dy) are read once, however far apart a group's values
// lie.
//
// Persistent: a cluster takes consecutive (slab, sample) units, so gamma, beta
// and the gradient's column sums change with the slab only, and the next
// unit's values are copied (cp.async) under the arithmetic of this one.  A
// thread has one vector column of the slab and every TR-th position, and reads
// only what it copied itself.  Its sums go through shared memory to a few
// lanes per group, from there (with more than one CTA) to every CTA of the
// cluster through distributed shared memory, and each thread forms its group's
// totals in the same order.  Sums of x are held relative to the group's first
// value, as in ff_norm.cu.  The arithmetic is on pairs: with silu a value
// costs about 9 instructions forward and 12 in the gradient, which keeps it
// under the time of its bytes.  Bound by HBM.
#include <algorithm>
#include <cmath>

#include "ff_norm.cuh"

namespace ff {
namespace {

constexpr int kMaxT = 512, kMaxK = 8, kMaxGS = 64;
constexpr int kGradValues = 32;  // values per thread whose du the gradient keeps in registers

struct Geom {
  int T, GS, K, k_log, nv, V;
  int WV, Wg;    // vectors per position of the slab, and of a group
  int TR, M;     // thread rows; threads per group
  int R, r_log;  // lanes that add up a group's threads (a power of 2)
  int units, total;  // units per cluster and in all
  int span;          // gradient: vectors from one stage (x and dy) to the next
  int wide;      // gamma and beta are 16-byte aligned
  float inv;     // 1 / values of a group
  FastDiv by_WV, by_Wg, by_TR, by_n;
};

struct Place {
  int rank, r0;
  int lo, rem;           // thread rows below rem take lo + 1 of the CTA's positions, the others lo
  int tc, tr, gl, slot;  // vector column, thread row, group within the slab, place among its threads
  int mine;              // positions of this thread
  bool on;
  __device__ __forceinline__ Place(const GnShape& s, const Geom& q) {
    rank = (int)(blockIdx.x & (unsigned)(q.K - 1));
    r0 = (int)((long long)s.S * rank >> q.k_log);
    const int rows = (int)((long long)s.S * (rank + 1) >> q.k_log) - r0;
    lo = (int)q.by_TR.div((uint32_t)rows);
    rem = rows - lo * q.TR;
    tr = (int)q.by_WV.div(threadIdx.x);
    tc = (int)threadIdx.x - tr * q.WV;
    on = tr < q.TR;
    gl = on ? (int)q.by_Wg.div((uint32_t)tc) : 0;
    slot = gl * q.M + tr * q.Wg + (tc - gl * q.Wg);
    mine = on ? lo + (tr < rem ? 1 : 0) : 0;
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
    return ((long long)b * s.S + p.r0 + p.tr) * ld + slab * q.GS * s.Cg + (p.on ? p.tc * q.V : 0);
  }
};

// The groups' totals of each CTA of a cluster, in every CTA of it: sent as
// asynchronous stores that a barrier of the receiver counts (a cluster barrier
// would make every thread wait for its global stores as well).  Two buffers:
// a CTA sends unit u + 2 only after it has everyone's u + 1, which each sends
// after it has read u.
template <typename E>
struct Exchange {
  uint64_t* bar;  // [2]
  E* at;          // [2][K][GS]
  volatile int* never;
  int K, GS;
  __device__ __forceinline__ Exchange(uint8_t* mem, const Geom& q)
      : bar(reinterpret_cast<uint64_t*>(mem)),
        at(reinterpret_cast<E*>(mem + 32)),
        never(reinterpret_cast<volatile int*>(mem + 16)),
        K(q.K),
        GS(q.GS) {
    if (K > 1) {
      if (threadIdx.x == 0) {
        ptx::mbar_init(&bar[0], 1);
        ptx::mbar_init(&bar[1], 1);
        *never = 0;
        ptx::fence_mbar_init();
      }
      __syncwarp();
      ptx::cluster_arrive_relaxed();
    }
  }
  __device__ __forceinline__ E* of(int k, int rank) const { return at + (k * K + rank) * GS; }
  __device__ __forceinline__ void expect(int k) {
    if (K > 1 && threadIdx.x == 0) ptx::mbar_arrive_expect_tx(&bar[k], (uint32_t)(K * GS * sizeof(E)));
    __syncwarp();
  }
  // A group's totals of this CTA, to CTA `to`.
  __device__ __forceinline__ void send(int k, int from, int to, int g, const E& v) {
    if (K == 1)
      of(k, 0)[g] = v;
    else if constexpr (sizeof(E) == 16)
      ptx::st_async4(of(k, from) + g, &bar[k], (uint32_t)to, v);
    else
      ptx::st_async2(of(k, from) + g, &bar[k], (uint32_t)to, v);
  }
  // Everyone's totals of the k-th buffer's n-th use are here; false if they
  // did not come in time.
  __device__ __forceinline__ bool wait(int k, int n) {
    if (K > 1) return ptx::mbar_wait_cluster(&bar[k], (uint32_t)n & 1u, kWaitTimeoutNs, const_cast<int*>(never));
    __syncthreads();
    return true;
  }
};
// Bytes of the exchange and of the threads' sums, before the stages.
__host__ __device__ constexpr int head_bytes(int T, int GS, int K, int esize) {
  return (32 + 2 * K * GS * esize + 2 * T * 8 + 15) & ~15;
}

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
__global__ void __launch_bounds__(kMaxT, 2) k_gn_cluster(GnArgs<T> a, Geom q) {
  using VV = Vec<T, V>;
  using PV = Pairs<V>;
  using Raw = typename VV::Raw;
  extern __shared__ __align__(16) uint8_t smem[];
  const GnShape& s = a.s;
  const Place p(s, q);
  Exchange<float4> xch(smem, q);
  float2* parts = reinterpret_cast<float2*>(smem + 32 + 2 * q.K * q.GS * sizeof(float4));  // [2][T]
  Raw* stages = reinterpret_cast<Raw*>(smem + head_bytes(q.T, q.GS, q.K, sizeof(float4)));  // [2][nv T]
  const int stage = q.nv * q.T;
  const int u0 = (int)(blockIdx.x >> q.k_log) * q.units, u1 = min(q.total, u0 + q.units);
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  Cursor cur(u0, s, q), ahead = cur;
  const long long xstep = (long long)q.TR * s.ldx, ystep = (long long)q.TR * s.ldy;
  float pivot = 0.f;  // the next unit's group's first value
  auto start = [&](int u, int k) {
    if (u < u1) {
      fetch<T, V>(stages + k * stage, a.x + ahead.offset(s, q, p, s.ldx), xstep, p.mine, q.T);
      float v[1];
      Vec<T, 1>::unpack(
          Vec<T, 1>::load(a.x + (long long)ahead.b * s.S * s.ldx + (ahead.slab * q.GS + p.gl) * s.Cg), v);
      pivot = v[0];
      ahead.next(s);
    }
    ptx::cp_async_commit();
  };
  start(u0, 0);
  if (q.K > 1) ptx::cluster_wait();  // every CTA of the cluster runs: its shared memory may be written
  float ga[V], be[V];
  int slab = -1;
  for (int u = u0; u < u1; ++u, cur.next(s)) {
    const int k = (u - u0) & 1;
    const float P = pivot;
    xch.expect(k);
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
      const int many = p.rem * q.Wg;
      const float chi = (float)((p.lo + 1) * V), clo = (float)(p.lo * V);
      const float n = chi * (float)many + clo * (float)(q.M - many);
      float sum = 0.f, m2 = 0.f;
      for (int j = l; real && j < q.M; j += q.R) sum = fmaf(t[j].x, j < many ? chi : clo, sum);
      for (int o = q.R / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      const float mean = __fdividef(sum, n);
      for (int j = l; real && j < q.M; j += q.R) {
        const float cnt = j < many ? chi : clo, d = t[j].x - mean;
        if (cnt > 0.f) m2 += fmaf(d * d, cnt, t[j].y);
      }
      for (int o = q.R / 2; o > 0; o >>= 1) m2 += __shfl_xor_sync(0xffffffffu, m2, o);
      // lane r of the group tells CTA r (R >= K, see the plan)
      if (real && l < q.K) xch.send(k, p.rank, l, gg, make_float4(n, mean, m2, 0.f));
    }
    const bool ok = xch.wait(k, (u - u0) >> 1);
    if (!p.on) continue;
    const float4* tot = xch.of(k, 0) + p.gl;
    float dm = tot[0].y, m2 = tot[0].z;
    if (q.K > 1) {
      float sum = 0.f;
      for (int r = 0; r < q.K; ++r) sum = fmaf(tot[r * q.GS].x, tot[r * q.GS].y, sum);
      dm = sum * q.inv;
      m2 = 0.f;
      for (int r = 0; r < q.K; ++r) {
        const float4 t = tot[r * q.GS];
        m2 += fmaf((t.y - dm) * (t.y - dm), t.x, t.z);
      }
    }
    // (totals that never came leave NaN behind)
    const float mean = ok ? P + dm : __int_as_float(0x7FC00000), rstd = rsqrtf(m2 * q.inv + s.eps);
    if (a.mean && p.rank == 0 && p.tr == 0 && p.tc == p.gl * q.Wg) {
      const long long at = (long long)cur.b * s.G + cur.slab * q.GS + p.gl;
      a.mean[at] = mean;
      a.rstd[at] = rstd;
    }
    float fa[V], fb[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      fa[e] = ga[e] * rstd;
      fb[e] = fmaf(-mean, fa[e], be[e]);
    }
    uint64_t A[PV::N], B[PV::N];
    PV::of(fa, A);
    PV::of(fb, B);
    T* y = a.out + cur.offset(s, q, p, s.ldy);
    m = mem;
#pragma unroll 2
    for (int i = 0; i < p.mine; ++i, m += q.T, y += ystep) {
      float v[V];
      uint64_t d[PV::N];
      VV::unpack(*m, v);
      PV::of(v, d);
#pragma unroll
      for (int e = 0; e < PV::N; ++e) d[e] = ptx::fma2(d[e], A[e], B[e]);
      act_pairs<V>(d, s.act);
      PV::to(d, v);
      VV::store(y, v);
    }
  }
  if (q.K > 1) {  // no CTA leaves while another may still send to it
    ptx::cluster_arrive_relaxed();
    ptx::cluster_wait();
  }
}

// The gradient.  part_out receives the column sums (du, du h) of each run of
// units of one slab: row (cluster - first cluster of the slab) K + rank.
template <typename T, int V, int NV>
__global__ void __launch_bounds__(kMaxT, 1) k_gn_cluster_grad(GnArgs<T> a, Geom q, float2* part_out) {
  using VV = Vec<T, V>;
  using PV = Pairs<V>;
  using Raw = typename VV::Raw;
  extern __shared__ __align__(16) uint8_t smem[];
  const GnShape& s = a.s;
  const Place p(s, q);
  Exchange<float2> xch(smem, q);
  float2* parts = reinterpret_cast<float2*>(smem + 32 + 2 * q.K * q.GS * sizeof(float2));  // [2][T]
  // [2]: x [nv T], dy [nv T]; or the column sums
  Raw* stages = reinterpret_cast<Raw*>(smem + head_bytes(q.T, q.GS, q.K, sizeof(float2)));
  const int stage = q.nv * q.T;
  const int cluster = (int)(blockIdx.x >> q.k_log);
  const int u0 = cluster * q.units, u1 = min(q.total, u0 + q.units);
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
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
  if (q.K > 1) ptx::cluster_wait();
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
    const int first = (int)((long long)of * s.n / q.units);  // cluster that took the slab's first unit
    float2* to = part_out + ((long long)(cluster - first) * q.K + p.rank) * s.C + of * q.GS * s.Cg;
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
    if (a.out) xch.expect(k);
    start(u + 1, k ^ 1);
    ptx::cp_async_wait<1>();
    const Raw* mx = stages + k * q.span + threadIdx.x;
    const Raw* my = mx + stage;
    // h = x rs - mu rs; u = gamma h + beta
    const uint64_t r2 = both(rs), o2 = both(-mu * rs);
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
          hx[e] = ptx::fma2(hx[e], r2, o2);
          up[e] = ptx::fma2(hx[e], G2[e], B2[e]);
        }
        act_grad_pairs<V>(dd, up, s.act);
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
      if (real && l < q.K) xch.send(k, p.rank, l, gg, w);
    }
    const bool ok = xch.wait(k, (u - u0) >> 1);
    if (!p.on) continue;
    float w1 = ok ? 0.f : __int_as_float(0x7FC00000), w2 = w1;
    const float2* tot = xch.of(k, 0) + p.gl;
    for (int r = 0; r < q.K; ++r) {
      w1 += tot[r * q.GS].x;
      w2 += tot[r * q.GS].y;
    }
    // dx = rs (gamma du - <.> - h <.>) = du (gamma rs) + h c2 + c1
    const uint64_t c1 = both(-rs * w1 * q.inv), c2 = both(-rs * w2 * q.inv);
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
          hx[e] = ptx::fma2(du[i][e], gr[e], ptx::fma2(ptx::fma2(hx[e], r2, o2), c2, c1));
        PV::to(hx, x);
        VV::store(o, x);
        o += ostep;
      }
  }
  // all copies have landed and been used; the last unit's stage is not read any more by its own thread,
  // and the other stage is free
  if (slab >= 0) flush(slab, ((u1 - u0 - 1) & 1) ^ 1);
  if (q.K > 1) {
    ptx::cluster_arrive_relaxed();
    ptx::cluster_wait();
  }
}

template <typename T>
Geom geom_of(const GnArgs<T>& a, int V, const GnClusterPlan& p) {
  const GnShape& s = a.s;
  Geom q;
  q.T = p.T;
  q.GS = p.GS;
  q.K = p.K;
  q.nv = p.nv;
  q.V = V;
  q.k_log = 0;
  while ((1 << q.k_log) < q.K) ++q.k_log;
  q.Wg = s.Cg / V;
  q.WV = q.Wg * q.GS;
  q.TR = q.T / q.WV;
  q.M = q.TR * q.Wg;
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
  q.by_TR = FastDiv(q.TR);
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
ff_status run(KernelKind kind, double bytes, const Geom& q, const GnClusterPlan& p, int smem, cudaStream_t st,
              const A&... args) {
  static const cudaError_t attr =
      cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  FF_TRY(attr, "group norm");
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.clusters * q.K));
  cfg.blockDim = dim3((unsigned)q.T);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)q.K;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = q.K > 1 ? 2 : 1;
  FF_LAUNCH(kind, bytes, st, cudaLaunchKernelEx(&cfg, KERNEL, args...), "group norm");
  return FF_OK;
}

template <typename T, int V, int NV>
ff_status run_grad(const GnArgs<T>& a, const Geom& q, const GnClusterPlan& p, double bytes, int smem, float2* part,
                   cudaStream_t st) {
  return run<k_gn_cluster_grad<T, V, NV>>(K_GNORM_GRAD, bytes, q, p, smem, st, a, q, part);
}

template <typename T, int V>
ff_status run_v(const GnArgs<T>& a, const GnClusterPlan& p, bool grad, cudaStream_t st) {
  const Geom q = geom_of(a, V, p);
  const double bytes = (double)a.s.n * a.s.S * a.s.C * sizeof(T);
  const int smem = head_bytes(q.T, q.GS, q.K, grad ? 8 : 16) + stage_bytes(q.T, q.nv, V, sizeof(T), grad);
  if (!grad) return run<k_gn_cluster<T, V>>(K_GNORM, 2 * bytes, q, p, smem, st, a, q);
  float2* part = a.dgamma ? static_cast<float2*>(a.ws) : nullptr;
  constexpr int N = V == 1 ? 16 : kGradValues / V;  // vectors per thread at most
  const ff_status e = q.nv <= N / 4   ? run_grad<T, V, N / 4>(a, q, p, 3 * bytes, smem, part, st)
                      : q.nv <= N / 2 ? run_grad<T, V, N / 2>(a, q, p, 3 * bytes, smem, part, st)
                                      : run_grad<T, V, N>(a, q, p, 3 * bytes, smem, part, st);
  if (e != FF_OK || !part) return e;
  return gn_param_fold(part, GnFold{0, p.units, a.s.n, q.GS * a.s.Cg, q.K}, a.s.C, a.dgamma, a.dbeta, st);
}

}  // namespace

// Threads, slab, cluster and stages with the least estimated time (us): the
// rounds of a cluster at the latency of one (copy, two exchanges, store) or
// the bytes at the rate that the slab's row segments allow, whichever is
// longer.
GnClusterPlan gn_cluster_plan(const GnShape& s, int V, int esize, bool grad) {
  GnClusterPlan best{};
  double t = 1e30;
  const double total = (double)s.n * s.S * s.C * esize * (grad ? 3 : 2);
  // du of a thread's values stays in registers: 32 of them, 16 one by one
  const int most = grad ? (V == 1 ? 16 : kGradValues) : 1 << 20;
  for (int GS = 1; GS <= s.G && GS <= kMaxGS; ++GS) {
    if (s.G % GS) continue;
    const long long WV = (long long)GS * (s.Cg / V);
    if (WV > kMaxT) break;
    const double seg = (double)WV * V * esize;
    const double eff = seg >= 128 ? 1.0 : seg >= 64 ? 0.9 : seg >= 32 ? 0.8 : seg / 40;
    for (int T = 128; T <= kMaxT; T *= 2) {
      if (WV > T) continue;
      const int TR = T / (int)WV;
      for (int K = 1; K <= kMaxK && K <= s.S; K *= 2) {
        if (K * GS > T) continue;  // a lane per group and CTA
        const int nv = cdiv(cdiv(s.S, K), TR);
        if ((long long)nv * V > most) continue;
        if ((long long)nv * V > 1024) continue;
        const long long bytes = head_bytes(T, GS, K, grad ? 8 : 16) + stage_bytes(T, nv, V, esize, grad);
        if (bytes > kSmem) continue;
        const int regs = !grad ? 64 : nv * V <= 8 ? 104 : 128;
        int per_sm = std::min(std::min(2048 / T, 65536 / (T * regs)), (int)(kSmem / (bytes + 1024)));
        per_sm = std::max(1, std::min(per_sm, 32));
        const int sms = K == 8 ? 120 : K == 4 ? 144 : 152;  // clusters do not fill every GPC
        const long long units = (long long)s.n * (s.G / GS);
        if (units > 0x3FFFFFFF) continue;
        const long long room = std::max(1ll, (long long)sms * per_sm / K);
        const long long rounds = (units + room - 1) / room;
        // a value's instructions, at the rate that the SM's warps reach: each
        // issues every 6 clocks or so, all together one a clock and scheduler
        const double warps = per_sm * T / 32.0, issue = std::max(6.0, warps / 4.0) / 1900.0;
        const double lat = 0.6 + (K > 1 ? 0.6 : 0.0) + (200 + nv * V * (grad ? 18 : 12)) * issue;
        const double c = std::max(rounds * lat, total / 6.4e6 / eff * 152.0 / sms) + 2.0;
        if (c < t) {
          t = c;
          best = GnClusterPlan{T, GS, K, nv, per_sm, (int)((units + rounds - 1) / rounds), (int)rounds};
        }
      }
    }
  }
  return best;
}

template <typename T>
ff_status gn_cluster(const GnArgs<T>& a, int V, const GnClusterPlan& p, bool grad, cudaStream_t st) {
  if constexpr (sizeof(T) == 2) {
    if (V == 8) return run_v<T, 8>(a, p, grad, st);
    if (V == 2) return run_v<T, 2>(a, p, grad, st);
  } else {
    if (V == 4) return run_v<T, 4>(a, p, grad, st);
  }
  return run_v<T, 1>(a, p, grad, st);
}
template ff_status gn_cluster<bf16>(const GnArgs<bf16>&, int, const GnClusterPlan&, bool, cudaStream_t);
template ff_status gn_cluster<float>(const GnArgs<float>&, int, const GnClusterPlan&, bool, cudaStream_t);

}  // namespace ff
