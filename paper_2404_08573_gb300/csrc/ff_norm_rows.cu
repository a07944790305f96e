// Group norm, the rows path: groups held in the registers of up to a warp
// (at most 512 values) or, for single positions, of a whole block (at most
// 8192).
//
// A warp (or block) walks over the samples with its groups fixed, so gamma, beta
// and the gradient's sums over the samples stay in registers; the next
// sample's values are loaded under the arithmetic of this one.  Mean and
// centred sum of squares are two passes over registers.  In bf16 neither HBM
// nor the schedulers are full (8192 x 4096 in 32 groups, silu: 40 us, 3.4 TB/s,
// issuing 74 % of the time; gradient 58 us, 63 % with 24 % of the warps): some 30
// instructions a value, and between them the latency of the sums' shuffles.
// fp32 moves twice the bytes for them: 52 us, 5.1 TB/s, and 92 us.  Odd groups
// are read a value at a time (2048 x 2000 in 16 groups of 125, fp32, relu: 11 and
// 15 us).
#include <algorithm>

#include "ff_norm.cuh"

namespace ff {
namespace {

constexpr int kWarps = 8;               // of a block that serves a group per warp or less
constexpr int kMostThreads = 512;       // of a block that serves one group

// Sum over the lanes of a group: 2^k of a warp, or (WIDE) a block.  `tmp` [2 x
// 16] of shared memory; consecutive calls alternate its halves.
template <bool WIDE>
struct Adder {
  float* tmp;
  int lanes, half = 0;
  __device__ __forceinline__ float operator()(float v) {
    if constexpr (WIDE) {
      v = warp_sum(v);
      float* t = tmp + 16 * half;
      half ^= 1;
      if ((threadIdx.x & 31) == 0) t[threadIdx.x >> 5] = v;
      __syncthreads();
      v = 0.f;
      for (int w = 0; w < (int)(blockDim.x >> 5); ++w) v += t[w];
    } else {
      for (int o = lanes / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    }
    return v;
  }
};

// Where a lane's NV vectors of its group lie: on(i) says whether vector i
// exists, ch(i) is its first channel within the group, at(i, ld) its offset
// from the group's first value.  ONE: a single position (rows of an activity),
// where the vectors are evenly spaced and nothing need be kept.
template <int V, int NV, bool ONE>
struct Slots {
  uint32_t have = 0;
  int first, gap;
  int row[ONE ? 1 : NV], col[ONE ? 1 : NV];
  __device__ __forceinline__ Slots(const GnShape& s, int l, int lanes, bool active) : first(l * V), gap(lanes * V) {
    const int per = s.Cg / V, total = s.S * per;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = l + i * lanes;
      if (active && j < total) have |= 1u << i;
      if constexpr (!ONE) {
        row[i] = j / per;
        col[i] = (j - row[i] * per) * V;
      }
    }
  }
  __device__ __forceinline__ bool on(int i) const { return have >> i & 1; }
  __device__ __forceinline__ int ch(int i) const {
    if constexpr (ONE)
      return first + i * gap;
    else
      return col[i];
  }
  __device__ __forceinline__ int at(int i, int ld) const {
    if constexpr (ONE)
      return first + i * gap;
    else
      return row[i] * ld + col[i];
  }
};

// A thread's group and its place in it, and the samples it walks over.
template <bool WIDE>
struct Walk {
  int set, p, l, g, b, step;
  bool active;
  __device__ __forceinline__ Walk(const GnShape& s, const GnRowsPlan& pl) {
    set = (int)blockIdx.x % pl.sets;
    p = (int)blockIdx.x / pl.sets;
    if constexpr (WIDE) {
      l = (int)threadIdx.x;
      g = set;
      b = p;
      step = pl.P;
    } else {
      const int lane = (int)threadIdx.x & 31;
      l = lane & (pl.lanes - 1);
      g = set * (32 / pl.lanes) + lane / pl.lanes;
      b = p * kWarps + (int)(threadIdx.x >> 5);
      step = pl.P * kWarps;
    }
    active = g < s.G;
  }
};

// gamma and beta of a lane's vectors, its values in pairs.
template <int V, int NV, typename S, typename T>
__device__ __forceinline__ void params(uint64_t (&ga)[NV * V / 2], uint64_t (&be)[NV * V / 2], const GnArgs<T>& a,
                                       const S& sl, int c0) {
  float g[NV * V], o[NV * V];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      g[i * V + e] = a.gamma && sl.on(i) ? __ldg(a.gamma + c0 + sl.ch(i) + e) : 1.f;
      o[i * V + e] = a.beta && sl.on(i) ? __ldg(a.beta + c0 + sl.ch(i) + e) : 0.f;
    }
  Pairs<NV * V>::of(g, ga);
  Pairs<NV * V>::of(o, be);
}
template <typename T, int V, int NV>
__device__ __forceinline__ void to_pairs(const typename Vec<T, V>::Raw (&r)[NV], uint64_t (&p)[NV * V / 2]) {
  float f[NV * V];
#pragma unroll
  for (int i = 0; i < NV; ++i) Vec<T, V>::unpack(r[i], reinterpret_cast<float(&)[V]>(f[i * V]));
  Pairs<NV * V>::of(f, p);
}
__device__ __forceinline__ float both_of(uint64_t p) {
  const float2 f = ptx::unpack2(p);
  return f.x + f.y;
}

template <typename T, int V, int NV, bool ONE, bool WIDE>
__global__ void __launch_bounds__(WIDE ? kMostThreads : 32 * kWarps) k_gn_rows(GnArgs<T> a, GnRowsPlan pl) {
  using VV = Vec<T, V>;
  __shared__ float tmp[32];
  const GnShape& s = a.s;
  const Walk<WIDE> w(s, pl);
  const Slots<V, NV, ONE> sl(s, w.l, pl.lanes, w.active);
  Adder<WIDE> add{tmp, pl.lanes};
  const int c0 = w.active ? w.g * s.Cg : 0;
  ptx::griddep_wait();
  constexpr int N = NV * V / 2;
  uint64_t ga[N], be[N];
  params<V, NV>(ga, be, a, sl, c0);
  const float inv = 1.f / ((float)s.S * (float)s.Cg);
  // vectors that do not exist stay zero: the activation is formed on pairs,
  // and a value's partner must not change from call to call
  typename VV::Raw cur[NV] = {}, nxt[NV] = {};
  const int ldx = (int)s.ldx, ldy = (int)s.ldy;  // within a sample (near, see plan_of)
  const long long dx = (long long)w.step * s.S * s.ldx, dy = (long long)w.step * s.S * s.ldy;
  const T* px = a.x + (long long)w.b * s.S * s.ldx + c0;  // the next sample to load
  T* q = a.out + (long long)w.b * s.S * s.ldy + c0;
  auto load = [&](typename VV::Raw(&r)[NV]) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (sl.on(i)) r[i] = VV::load(px + sl.at(i, ldx));
    px += dx;
  };
  // counted down, since the sample after the last could be past 2^31
  if (w.b < s.n) load(cur);
  for (int left = s.n - w.b; left > 0; left -= w.step) {
    const int b = s.n - left;
    if (left > w.step) load(nxt);
    uint64_t d[N], t = 0;
    to_pairs<T, V, NV>(cur, d);
#pragma unroll
    for (int i = 0; i < N; ++i) t = ptx::add2(t, d[i]);  // zero where there is no vector
    const float mean = add(both_of(t)) * inv;
    const uint64_t minus = both(-mean);
    t = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      d[i] = ptx::add2(d[i], minus);
      if constexpr (V == 1) {
        const float2 f = ptx::unpack2(d[i]);
        d[i] = ptx::pack2(sl.on(2 * i) ? f.x : 0.f, sl.on(2 * i + 1) ? f.y : 0.f);
        t = ptx::fma2(d[i], d[i], t);
      } else if (sl.on(2 * i / V)) {
        t = ptx::fma2(d[i], d[i], t);
      }
    }
    const float rstd = rsqrtf(add(both_of(t)) * inv + s.eps);
    const uint64_t r2 = both(rstd);
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] = ptx::fma2(ptx::mul2(d[i], r2), ga[i], be[i]);
    act_pairs<T, NV * V>(d, s.act);
    float y[NV * V];
    Pairs<NV * V>::to(d, y);
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (sl.on(i)) VV::store(q + sl.at(i, ldy), reinterpret_cast<const float(&)[V]>(y[i * V]));
    q += dy;
    if (a.mean && w.active && w.l == 0) {
      a.mean[(long long)b * s.G + w.g] = mean;
      a.rstd[(long long)b * s.G + w.g] = rstd;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) cur[i] = nxt[i];
  }
}

// The gradient; each block's warps share their groups, and leave the sums
// (du, du h) over the block's samples in part[(p S + position) C + channel].
// With 4 values a thread four blocks fit an SM, which the launch counts on
// (2048 x 2000 in 16 groups of 125, fp32: 14.8 us, with three 19.7).
template <typename T, int V, int NV, bool ONE, bool WIDE>
__global__ void __launch_bounds__(WIDE ? kMostThreads : 32 * kWarps, NV * V <= 4 && (ONE || V > 1) ? 4 : 0)
    k_gn_rows_grad(GnArgs<T> a, GnRowsPlan pl, float2* part) {
  using VV = Vec<T, V>;
  __shared__ float2 red[WIDE ? 1 : kWarps][WIDE ? 1 : NV * V][32];
  __shared__ float tmp[32];
  const GnShape& s = a.s;
  const Walk<WIDE> w(s, pl);
  const Slots<V, NV, ONE> sl(s, w.l, pl.lanes, w.active);
  Adder<WIDE> add{tmp, pl.lanes};
  const int c0 = w.active ? w.g * s.Cg : 0;
  ptx::griddep_wait();
  constexpr int N = NV * V / 2;
  uint64_t ga[N], be[N], p0[N], p1[N];
  params<V, NV>(ga, be, a, sl, c0);
#pragma unroll
  for (int i = 0; i < N; ++i) p0[i] = p1[i] = 0;
  const float inv = 1.f / ((float)s.S * (float)s.Cg);
  typename VV::Raw cx[NV] = {}, cy[NV] = {}, nx[NV] = {}, ny[NV] = {};
  const int ldx = (int)s.ldx, lddy = (int)s.lddy, ldo = (int)s.ldy;  // within a sample (near, see plan_of)
  const T* px = a.x + (long long)w.b * s.S * s.ldx + c0;  // the next sample to load
  const T* py = a.dy + (long long)w.b * s.S * s.lddy + c0;
  T* q = a.out + (a.out ? (long long)w.b * s.S * s.ldy + c0 : 0);
  const long long sx = (long long)w.step * s.S * s.ldx, sy = (long long)w.step * s.S * s.lddy,
                  so = (long long)w.step * s.S * s.ldy;
  float mu = 0.f, rs = 0.f, nmu = 0.f, nrs = 0.f;
  auto load = [&](typename VV::Raw(&rx)[NV], typename VV::Raw(&ry)[NV], int b, float& m, float& r) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (sl.on(i)) {
        rx[i] = VV::load(px + sl.at(i, ldx));
        ry[i] = VV::load(py + sl.at(i, lddy));
      }
    px += sx;
    py += sy;
    if (w.active) {
      m = __ldg(a.mean + (long long)b * s.G + w.g);
      r = __ldg(a.rstd + (long long)b * s.G + w.g);
    }
  };
  // counted down, as in the forward pass
  if (w.b < s.n) load(cx, cy, w.b, mu, rs);
  for (int left = s.n - w.b; left > 0; left -= w.step) {
    const int b = s.n - left;
    if (left > w.step) load(nx, ny, b + w.step, nmu, nrs);
    // a vector that does not exist has du = 0
    uint64_t h[N], d[N], t1 = 0, t2 = 0;
    {
      uint64_t u[N];
      const uint64_t minus = both(-mu), r2 = both(rs);
      to_pairs<T, V, NV>(cx, h);
      to_pairs<T, V, NV>(cy, d);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        h[i] = ptx::mul2(ptx::add2(h[i], minus), r2);
        u[i] = ptx::fma2(ga[i], h[i], be[i]);
      }
      act_grad_pairs<T, NV * V>(d, u, s.act);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      p0[i] = ptx::add2(p0[i], d[i]);
      p1[i] = ptx::fma2(d[i], h[i], p1[i]);
      d[i] = ptx::mul2(d[i], ga[i]);
      t1 = ptx::add2(t1, d[i]);
      t2 = ptx::fma2(d[i], h[i], t2);
    }
    if (a.out) {
      const float m1 = add(both_of(t1)) * inv, m2 = add(both_of(t2)) * inv;
      // dx = rs (gamma du - <.> - h <.>)
      const uint64_t r2 = both(rs), c1 = both(-rs * m1), c2 = both(-rs * m2);
      float v[NV * V];
#pragma unroll
      for (int i = 0; i < N; ++i) d[i] = ptx::fma2(d[i], r2, ptx::fma2(h[i], c2, c1));
      Pairs<NV * V>::to(d, v);
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (sl.on(i)) VV::store(q + sl.at(i, ldo), reinterpret_cast<const float(&)[V]>(v[i * V]));
      q += so;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      cx[i] = nx[i];
      cy[i] = ny[i];
    }
    mu = nmu;
    rs = nrs;
  }
  if (!part) return;
  float s0[NV * V], s1[NV * V];
  Pairs<NV * V>::to(p0, s0);
  Pairs<NV * V>::to(p1, s1);
  if constexpr (WIDE) {  // one position, and every thread has its channels alone
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (sl.on(i))
#pragma unroll
        for (int e = 0; e < V; ++e)
          part[(long long)w.p * s.C + c0 + sl.ch(i) + e] = make_float2(s0[i * V + e], s1[i * V + e]);
  } else {
#pragma unroll
    for (int i = 0; i < NV * V; ++i) red[threadIdx.x >> 5][i][threadIdx.x & 31] = make_float2(s0[i], s1[i]);
    __syncthreads();
    const int per = s.Cg / V, total = s.S * per;
    for (int i = threadIdx.x; i < NV * V * 32; i += 32 * kWarps) {
      const int ln = i & 31, k = i >> 5;
      const int j = (ln & (pl.lanes - 1)) + (k / V) * pl.lanes;
      const int gg = w.set * (32 / pl.lanes) + ln / pl.lanes;
      if (gg >= s.G || j >= total) continue;
      float2 t = red[0][k][ln];
#pragma unroll
      for (int v = 1; v < kWarps; ++v) {
        t.x += red[v][k][ln].x;
        t.y += red[v][k][ln].y;
      }
      const int r = j / per, c = (j - r * per) * V + k % V;
      part[((long long)w.p * s.S + r) * s.C + gg * s.Cg + c] = t;
    }
  }
}

template <typename T, int V, int NV, bool ONE, bool WIDE>
ff_status go(const GnArgs<T>& a, const GnRowsPlan& pl, bool grad, cudaStream_t st) {
  const double bytes = (double)a.s.n * a.s.S * a.s.C * sizeof(T);
  PdlLaunch l(dim3((unsigned)(pl.sets * pl.P)), dim3((unsigned)(WIDE ? pl.lanes : 32 * kWarps)), st);
  if (!grad) {
    FF_LAUNCH(K_GNORM, 2 * bytes, st, cudaLaunchKernelEx(&l.cfg, k_gn_rows<T, V, NV, ONE, WIDE>, a, pl),
              "group norm of rows");
    return FF_OK;
  }
  float2* part = a.dgamma ? static_cast<float2*>(a.ws) : nullptr;
  FF_LAUNCH(K_GNORM_GRAD, 3 * bytes, st, cudaLaunchKernelEx(&l.cfg, k_gn_rows_grad<T, V, NV, ONE, WIDE>, a, pl, part),
            "group norm gradient of rows");
  return part ? gn_param_fold(part, GnFold{(long long)pl.P * a.s.S, 0, 0, 0}, a.s.C, a.dgamma, a.dbeta, st) : FF_OK;
}
template <typename T, int V, int NV>
ff_status run(const GnArgs<T>& a, const GnRowsPlan& pl, bool grad, cudaStream_t st) {
  if constexpr (NV * V >= 8)  // a block per group: more than 4 values a thread
    if (pl.lanes > 32) return go<T, V, NV, true, true>(a, pl, grad, st);
  return a.s.S == 1 ? go<T, V, NV, true, false>(a, pl, grad, st) : go<T, V, NV, false, false>(a, pl, grad, st);
}

}  // namespace

// Whether the path takes these groups: 512 values at any number of positions,
// 8192 of a single one.
bool gn_rows_fit(const GnShape& s) { return (long long)s.S * s.Cg <= (s.S == 1 ? 16 * kMostThreads : 512); }

// Lanes per group: from four on as few as leave each 8 values where they come
// in vectors (the sums' shuffles are shared by more of them: 8192 x 4096 in 32
// groups, fp32, 69 us with 4 values each, 48 with 8; 3000 x 3200 in 32 groups,
// bf16, 20 with up to 4, 17 with 8), and 4 values, which a lane has room for
// anyhow, where they do not (5182 x 1120 in 32 groups of 35, bf16, gradient: 28
// us, with one or two each 52; 2048 x 2000 in 16 groups of 125, fp32, gradient:
// 16 us, with 8 each 18).
GnRowsPlan gn_rows_plan(const GnShape& s, int V, bool grad) {
  GnRowsPlan p;
  const int vecs = s.S * s.Cg / V;
  int per = 1;  // groups a block serves side by side
  int rows = 1; // samples a block takes at once
  if (s.S * s.Cg > 512) {
    p.lanes = 64;
    while (p.lanes < kMostThreads && p.lanes * std::max(1, 8 / V) < vecs) p.lanes *= 2;
    p.sets = s.G;
  } else {
    p.lanes = 1;
    const int each = V > 1 ? 8 / V : 4, least = V > 1 ? 4 : 2;  // vectors, lanes
    while (p.lanes < 32 && p.lanes < vecs && (p.lanes < least || p.lanes * each < vecs)) p.lanes *= 2;
    per = 32 / p.lanes;
    p.sets = cdiv(s.G, per);
    rows = kWarps;
  }
  // about 8 blocks of 256 threads per SM; the gradient's partial sums grow
  // with the blocks, so it takes 4, or as many as leave each thread
  // kGradSamples samples
  const int threads = p.lanes > 32 ? p.lanes : 32 * kWarps;
  const long long want = 152ll * (grad ? 4 : 8) * (32 * kWarps) / threads / p.sets;
  p.P = cdiv(s.n, rows);
  const long long least = grad ? cdiv(s.n, rows * kGradSamples) : 1;
  p.P = (int)std::min<long long>(p.P, std::max(want, least));
  return p;
}

template <typename T>
ff_status gn_rows(const GnArgs<T>& a, int V, bool grad, cudaStream_t st) {
  const GnRowsPlan pl = gn_rows_plan(a.s, V, grad);
  const int nv = cdiv(a.s.S * a.s.Cg / V, pl.lanes);  // vectors per lane
  if constexpr (sizeof(T) == 2) {
    if (V == 8) return nv <= 1 ? run<T, 8, 1>(a, pl, grad, st) : run<T, 8, 2>(a, pl, grad, st);
    if (V == 2)
      return nv <= 2   ? run<T, 2, 2>(a, pl, grad, st)
             : nv <= 4 ? run<T, 2, 4>(a, pl, grad, st)
                       : run<T, 2, 8>(a, pl, grad, st);
  } else {
    if (V == 4)
      return nv <= 1   ? run<T, 4, 1>(a, pl, grad, st)
             : nv <= 2 ? run<T, 4, 2>(a, pl, grad, st)
                       : run<T, 4, 4>(a, pl, grad, st);
  }
  return nv <= 4   ? run<T, 1, 4>(a, pl, grad, st)
         : nv <= 8 ? run<T, 1, 8>(a, pl, grad, st)
                   : run<T, 1, 16>(a, pl, grad, st);
}
template ff_status gn_rows<bf16>(const GnArgs<bf16>&, int, bool, cudaStream_t);
template ff_status gn_rows<float>(const GnArgs<float>&, int, bool, cudaStream_t);

}  // namespace ff
