// Group norm, the rows path: groups of at most 512 values (a row's groups, or a
// few positions), each held in the registers of up to a warp.
//
// A warp walks over the samples with its groups fixed, so gamma, beta and the
// gradient's sums over the samples stay in registers; the next sample's values
// are loaded under the arithmetic of this one.  Mean and centred sum of squares
// are two passes over registers.  Bound by HBM: x (and dy) once in, once out.
#include "ff_norm.cuh"

namespace ff {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

// Sum over the 2^k lanes of a group.
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
  for (int o = lanes / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Where a lane's NV vectors of its group lie: bit i of `on` says whether vector
// i exists, px and py are offsets from the group's first value.
template <int V, int NV>
struct Slots {
  uint32_t on;
  int px[NV], py[NV], ch[NV];
  __device__ __forceinline__ Slots(const GnShape& s, int l, int lanes, bool active, long long ldy) {
    const int per = s.Cg / V, total = s.S * per;
    on = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = l + i * lanes;
      const int r = j / per, c = (j - r * per) * V;
      if (active && j < total) on |= 1u << i;
      ch[i] = c;
      px[i] = (int)(r * s.ldx) + c;
      py[i] = (int)(r * ldy) + c;
    }
  }
};

template <typename T, int V, int NV>
__global__ void __launch_bounds__(kThreads) k_gn_rows(GnArgs<T> a, GnRowsPlan pl) {
  using VV = Vec<T, V>;
  const GnShape& s = a.s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int l = lane & (pl.lanes - 1), set = blockIdx.x % pl.sets;
  const int g = set * (32 / pl.lanes) + lane / pl.lanes;
  const bool active = g < s.G;
  const Slots<V, NV> sl(s, l, pl.lanes, active, s.ldy);
  const int c0 = active ? g * s.Cg : 0;
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  float ga[NV][V], be[NV][V];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      ga[i][e] = a.gamma && (sl.on >> i & 1) ? __ldg(a.gamma + c0 + sl.ch[i] + e) : 1.f;
      be[i][e] = a.beta && (sl.on >> i & 1) ? __ldg(a.beta + c0 + sl.ch[i] + e) : 0.f;
    }
  const float inv = 1.f / ((float)s.S * (float)s.Cg);
  // vectors that do not exist stay zero: the activation is formed on pairs,
  // and a value's partner must not change from call to call
  typename VV::Raw cur[NV] = {}, nxt[NV] = {};
  auto load = [&](typename VV::Raw(&r)[NV], int b) {
    const T* p = a.x + (long long)b * s.S * s.ldx + c0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (sl.on >> i & 1) r[i] = VV::load(p + sl.px[i]);
  };
  const int step = pl.P * kWarps;
  int b = (int)(blockIdx.x / pl.sets) * kWarps + warp;
  if (b < s.n) load(cur, b);
  for (; b < s.n; b += step) {
    if (s.n - b > step) load(nxt, b + step);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float v[V];
      VV::unpack(cur[i], v);
      if (sl.on >> i & 1)
#pragma unroll
        for (int e = 0; e < V; ++e) sum += v[e];
    }
    const float mean = lanes_sum(sum, pl.lanes) * inv;
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float v[V];
      VV::unpack(cur[i], v);
      if (sl.on >> i & 1)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float d = v[e] - mean;
          sq = fmaf(d, d, sq);
        }
    }
    const float rstd = 1.f / sqrtf(lanes_sum(sq, pl.lanes) * inv + s.eps);
    T* q = a.out + (long long)b * s.S * s.ldy + c0;
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
      if (sl.on >> i & 1) VV::store(q + sl.py[i], reinterpret_cast<const float(&)[V]>(y[i * V]));
    if (a.mean && active && l == 0) {
      a.mean[(long long)b * s.G + g] = mean;
      a.rstd[(long long)b * s.G + g] = rstd;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) cur[i] = nxt[i];
  }
}

// The gradient; each block's warps share their groups, and leave the sums
// (du, du h) over the block's samples in part[(p S + position) C + channel].
template <typename T, int V, int NV>
__global__ void __launch_bounds__(kThreads) k_gn_rows_grad(GnArgs<T> a, GnRowsPlan pl, float2* part) {
  using VV = Vec<T, V>;
  __shared__ float2 red[kWarps][NV * V][32];
  const GnShape& s = a.s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int l = lane & (pl.lanes - 1), set = blockIdx.x % pl.sets, p = blockIdx.x / pl.sets;
  const int g = set * (32 / pl.lanes) + lane / pl.lanes;
  const bool active = g < s.G;
  const Slots<V, NV> sl(s, l, pl.lanes, active, s.lddy);
  const int c0 = active ? g * s.Cg : 0;
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  float ga[NV][V], be[NV][V], p0[NV][V], p1[NV][V];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      ga[i][e] = a.gamma && (sl.on >> i & 1) ? __ldg(a.gamma + c0 + sl.ch[i] + e) : 1.f;
      be[i][e] = a.beta && (sl.on >> i & 1) ? __ldg(a.beta + c0 + sl.ch[i] + e) : 0.f;
      p0[i][e] = p1[i][e] = 0.f;
    }
  const float inv = 1.f / ((float)s.S * (float)s.Cg);
  typename VV::Raw cx[NV] = {}, cy[NV] = {}, nx[NV] = {}, ny[NV] = {};
  auto load = [&](typename VV::Raw(&rx)[NV], typename VV::Raw(&ry)[NV], int b) {
    const T* px = a.x + (long long)b * s.S * s.ldx + c0;
    const T* py = a.dy + (long long)b * s.S * s.lddy + c0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (sl.on >> i & 1) {
        rx[i] = VV::load(px + sl.px[i]);
        ry[i] = VV::load(py + sl.py[i]);
      }
  };
  const int step = pl.P * kWarps;
  int b = p * kWarps + warp;
  float mu = 0.f, rs = 0.f, nmu = 0.f, nrs = 0.f;
  auto stats = [&](int b, float& m, float& r) {
    if (active) {
      m = __ldg(a.mean + (long long)b * s.G + g);
      r = __ldg(a.rstd + (long long)b * s.G + g);
    }
  };
  if (b < s.n) {
    load(cx, cy, b);
    stats(b, mu, rs);
  }
  for (; b < s.n; b += step) {
    if (s.n - b > step) {
      load(nx, ny, b + step);
      stats(b + step, nmu, nrs);
    }
    // a vector that does not exist has h = 0 and du = 0
    float h[NV * V], w[NV * V], m1 = 0.f, m2 = 0.f;
    {
      float u[NV * V];
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        float x[V], d[V];
        VV::unpack(cx[i], x);
        VV::unpack(cy[i], d);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const int j = i * V + e;
          const bool on = sl.on >> i & 1;
          h[j] = on ? (x[e] - mu) * rs : 0.f;
          w[j] = on ? d[e] : 0.f;
          u[j] = fmaf(ga[i][e], h[j], be[i][e]);
        }
      }
      act_grad_values<NV * V>(w, u, s.act);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int j = i * V + e;
        p0[i][e] += w[j];
        p1[i][e] = fmaf(w[j], h[j], p1[i][e]);
        w[j] *= ga[i][e];
        m1 += w[j];
        m2 = fmaf(w[j], h[j], m2);
      }
    if (a.out) {
      m1 = lanes_sum(m1, pl.lanes) * inv;
      m2 = lanes_sum(m2, pl.lanes) * inv;
      T* q = a.out + (long long)b * s.S * s.ldy + c0;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (sl.on >> i & 1) {
          float v[V];
#pragma unroll
          for (int e = 0; e < V; ++e) v[e] = rs * (w[i * V + e] - m1 - h[i * V + e] * m2);
          // dx has its own stride: its row of this vector
          const int r = (l + i * pl.lanes) / (s.Cg / V);
          VV::store(q + (long long)r * s.ldy + sl.ch[i], v);
        }
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
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) red[warp][i * V + e][lane] = make_float2(p0[i][e], p1[i][e]);
  __syncthreads();
  const int per = s.Cg / V, total = s.S * per;
  for (int i = threadIdx.x; i < NV * V * 32; i += kThreads) {
    const int ln = i & 31, k = i >> 5;
    const int j = (ln & (pl.lanes - 1)) + (k / V) * pl.lanes;
    const int gg = set * (32 / pl.lanes) + ln / pl.lanes;
    if (gg >= s.G || j >= total) continue;
    float2 t = red[0][k][ln];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) {
      t.x += red[w][k][ln].x;
      t.y += red[w][k][ln].y;
    }
    const int r = j / per, c = (j - r * per) * V + k % V;
    part[((long long)p * s.S + r) * s.C + gg * s.Cg + c] = t;
  }
}

template <typename T, int V, int NV>
ff_status run(const GnArgs<T>& a, const GnRowsPlan& pl, bool grad, cudaStream_t st) {
  const double bytes = (double)a.s.n * a.s.S * a.s.C * sizeof(T);
  PdlLaunch l(dim3((unsigned)(pl.sets * pl.P)), dim3(kThreads), st);
  if (!grad) {
    FF_LAUNCH(K_GNORM, 2 * bytes, st, cudaLaunchKernelEx(&l.cfg, k_gn_rows<T, V, NV>, a, pl), "group norm of rows");
    return FF_OK;
  }
  float2* part = a.dgamma ? static_cast<float2*>(a.ws) : nullptr;
  FF_LAUNCH(K_GNORM_GRAD, 3 * bytes, st, cudaLaunchKernelEx(&l.cfg, k_gn_rows_grad<T, V, NV>, a, pl, part),
            "group norm gradient of rows");
  return part ? gn_param_fold(part, GnFold{(long long)pl.P * a.s.S, 0, 0, 0}, a.s.C, a.dgamma, a.dbeta, st) : FF_OK;
}

}  // namespace

// Lanes per group: enough for 16 values each (wider groups: a warp), so that
// at most kRowsMax / 32 = 16 values are a lane's.
GnRowsPlan gn_rows_plan(const GnShape& s, int V, bool grad) {
  GnRowsPlan p;
  const int vecs = s.S * s.Cg / V;
  p.lanes = 1;
  // small groups spread over lanes down to one vector each
  while (p.lanes < 32 && p.lanes < vecs) p.lanes *= 2;
  p.sets = cdiv(s.G, 32 / p.lanes);
  // about 8 blocks per SM; the gradient's partial sums grow with the blocks,
  // so it takes 4
  const int want = 152 * (grad ? 4 : 8) / p.sets;
  p.P = cdiv(s.n, kWarps);
  if (p.P > want) p.P = want > 1 ? want : 1;
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
