// Group norm, the rows path: groups held in the registers of up to a warp
// (at most 512 values) or, for single positions, of a whole block (at most
// 8192).
//
// A warp (or block) walks over the samples with its groups fixed, so gamma, beta
// and the gradient's sums over the samples stay in registers; the next
// sample's values are loaded under the arithmetic of this one.  Mean and
// centred sum of squares are two passes over registers.  Bound by the
// instructions: with silu a value takes about 12 forward and 25 in the
// gradient, and odd groups are read a value at a time (8192 x 4096 in 32
// groups, bf16, silu: 40 us, 3.4 TB/s, gradient 60 us; 2048 x 2000 in 16 groups
// of 125, fp32, relu: 11 and 19 us).
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

// gamma and beta of a lane's vectors.
template <int V, int NV, typename S, typename T>
__device__ __forceinline__ void params(float (&ga)[NV][V], float (&be)[NV][V], const GnArgs<T>& a, const S& sl, int c0) {
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      ga[i][e] = a.gamma && sl.on(i) ? __ldg(a.gamma + c0 + sl.ch(i) + e) : 1.f;
      be[i][e] = a.beta && sl.on(i) ? __ldg(a.beta + c0 + sl.ch(i) + e) : 0.f;
    }
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
  ptx::griddep_launch_dependents();
  float ga[NV][V], be[NV][V];
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
  int b = w.b;
  if (b < s.n) load(cur);
  for (; b < s.n; b += w.step) {
    if (s.n - b > w.step) load(nxt);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float v[V];
      VV::unpack(cur[i], v);
#pragma unroll
      for (int e = 0; e < V; ++e) sum += v[e];  // zero where there is no vector
    }
    const float mean = add(sum) * inv;
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float v[V];
      VV::unpack(cur[i], v);
      if (sl.on(i))
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float d = v[e] - mean;
          sq = fmaf(d, d, sq);
        }
    }
    const float rstd = rsqrtf(add(sq) * inv + s.eps);
    float y[NV * V];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float v[V];
      VV::unpack(cur[i], v);
#pragma unroll
      for (int e = 0; e < V; ++e) y[i * V + e] = fmaf((v[e] - mean) * rstd, ga[i][e], be[i][e]);
    }
    act_values<NV * V>(y, s.act);
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
template <typename T, int V, int NV, bool ONE, bool WIDE>
__global__ void __launch_bounds__(WIDE ? kMostThreads : 32 * kWarps)
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
  ptx::griddep_launch_dependents();
  float ga[NV][V], be[NV][V], p0[NV][V], p1[NV][V];
  params<V, NV>(ga, be, a, sl, c0);
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) p0[i][e] = p1[i][e] = 0.f;
  const float inv = 1.f / ((float)s.S * (float)s.Cg);
  typename VV::Raw cx[NV] = {}, cy[NV] = {}, nx[NV] = {}, ny[NV] = {};
  const int ldx = (int)s.ldx, lddy = (int)s.lddy, ldo = (int)s.ldy;  // within a sample (near, see plan_of)
  int b = w.b;
  const T* px = a.x + (long long)b * s.S * s.ldx + c0;  // the next sample to load
  const T* py = a.dy + (long long)b * s.S * s.lddy + c0;
  T* q = a.out + (a.out ? (long long)b * s.S * s.ldy + c0 : 0);
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
  if (b < s.n) load(cx, cy, b, mu, rs);
  for (; b < s.n; b += w.step) {
    if (s.n - b > w.step) load(nx, ny, b + w.step, nmu, nrs);
    // a vector that does not exist has h = 0 and du = 0
    float h[NV * V], d[NV * V], m1 = 0.f, m2 = 0.f;
    {
      float u[NV * V];
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        float x[V], t[V];
        VV::unpack(cx[i], x);
        VV::unpack(cy[i], t);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const int j = i * V + e;
          h[j] = sl.on(i) ? (x[e] - mu) * rs : 0.f;
          d[j] = t[e];
          u[j] = fmaf(ga[i][e], h[j], be[i][e]);
        }
      }
      act_grad_values<NV * V>(d, u, s.act);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int j = i * V + e;
        p0[i][e] += d[j];
        p1[i][e] = fmaf(d[j], h[j], p1[i][e]);
        d[j] *= ga[i][e];
        m1 += d[j];
        m2 = fmaf(d[j], h[j], m2);
      }
    if (a.out) {
      m1 = add(m1) * inv;
      m2 = add(m2) * inv;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (sl.on(i)) {
          float v[V];
#pragma unroll
          for (int e = 0; e < V; ++e) v[e] = rs * (d[i * V + e] - m1 - h[i * V + e] * m2);
          VV::store(q + sl.at(i, ldo), v);
        }
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
  if constexpr (WIDE) {  // one position, and every thread has its channels alone
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (sl.on(i))
#pragma unroll
        for (int e = 0; e < V; ++e)
          part[(long long)w.p * s.C + c0 + sl.ch(i) + e] = make_float2(p0[i][e], p1[i][e]);
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) red[threadIdx.x >> 5][i * V + e][threadIdx.x & 31] = make_float2(p0[i][e], p1[i][e]);
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
  if (pl.lanes > 32) return go<T, V, NV, true, true>(a, pl, grad, st);
  return a.s.S == 1 ? go<T, V, NV, true, false>(a, pl, grad, st) : go<T, V, NV, false, false>(a, pl, grad, st);
}

}  // namespace

// Whether the path takes these groups: 512 values at any number of positions,
// 8192 of a single one.
bool gn_rows_fit(const GnShape& s) { return (long long)s.S * s.Cg <= (s.S == 1 ? 16 * kMostThreads : 512); }

// Lanes per group: down to one vector each in narrow groups, up to 16 values
// each in wide ones.
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
    while (p.lanes < 32 && p.lanes < vecs) p.lanes *= 2;
    per = 32 / p.lanes;
    p.sets = cdiv(s.G, per);
    rows = kWarps;
  }
  // about 8 blocks of 256 threads per SM; the gradient's partial sums grow
  // with the blocks, so it takes 4
  const int threads = p.lanes > 32 ? p.lanes : 32 * kWarps;
  const long long want = 152ll * (grad ? 4 : 8) * (32 * kWarps) / threads / p.sets;
  p.P = cdiv(s.n, rows);
  if (p.P > want) p.P = want > 1 ? (int)want : 1;
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
