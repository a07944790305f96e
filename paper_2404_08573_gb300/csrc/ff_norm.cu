// Group norm with an activation over channels-last data, and its gradient.
//
//   forward   mean and rstd of each sample's channel group, then
//             y = act(gamma (x - mean) rstd + beta)
//   gradient  du = dy act'(u); dbeta = sum du, dgamma = sum du h;
//             dx = rstd (gamma du - <gamma du> - h <gamma du h>)
//
// Everything a group needs follows from sums over each channel's positions:
// the group's mean and centred sum of squares from the channels' (combined
// by Chan, Golub and LeVeque's update, so no large mean cancels), the two
// averages of the gradient from gamma-weighted channel sums, and dgamma and
// dbeta are those sums added up over the samples.  So the general path is
// column sums over chunks of positions (k_gn_colstats, k_gn_grad_colsums), a
// small fold per group, and an element-wise pass -- whatever the group's
// width, since a 16-byte vector may span groups.
#include <cmath>

#include "ff_api_internal.h"
#include "ff_ptx.cuh"
#include "ff_vec.cuh"

namespace ff {
namespace {

struct GnShape {
  int n, S, C, G, Cg;
  long long ldx, ldy, lddy;  // forward: x -> y; gradient: (dy, x) -> dx with ldy the stride of dx
  float eps;
  int act;
};

__device__ __forceinline__ float act_of(float u, int act) {
  if (act == FF_ACT_RELU) return u < 0.f ? 0.f : u;  // keeps NaN
  if (act == FF_ACT_SILU) return u * __fdividef(1.f, 1.f + __expf(-u));
  return u;
}
// dy act'(u)
__device__ __forceinline__ float act_grad(float dy, float u, int act) {
  if (act == FF_ACT_RELU) return u > 0.f ? dy : 0.f;
  if (act == FF_ACT_SILU) {
    const float p = __fdividef(1.f, 1.f + __expf(-u));
    return dy * (p * fmaf(u, 1.f - p, 1.f));
  }
  return dy;
}

// ------------------------------------------------------------ general path
constexpr int kColThreads = 256;
constexpr int kColVecs = 32;       // at most this many vectors of columns per block
constexpr int kRowsPerThread = 64; // bounds the rounding of a thread's one-pass sums (see k_gn_colstats)

struct ColGeom {
  int CV, TC, TR, ctiles, chunk, chunks;
};
// Blocks of TC vector columns x TR thread rows; `chunk` positions per block,
// enough blocks to fill the GPU several times where the work allows.
ColGeom col_geom(int n, int S, int C, int V) {
  ColGeom g;
  g.CV = C / V;
  g.TC = g.CV < kColVecs ? g.CV : kColVecs;
  g.TR = kColThreads / g.TC;
  g.ctiles = cdiv(g.CV, g.TC);
  const long long want = 152 * 8;
  long long chunks = (want + (long long)n * g.ctiles - 1) / ((long long)n * g.ctiles);
  long long chunk = (S + chunks - 1) / chunks;
  const long long lo = (long long)g.TR * 4, hi = (long long)g.TR * kRowsPerThread;
  chunk = chunk < lo ? lo : chunk > hi ? hi : chunk;
  g.chunk = (int)(chunk < S ? chunk : S);
  g.chunks = cdiv(S, g.chunk);
  return g;
}

template <typename T>
__device__ __forceinline__ float group_pivot(const T* x, const GnShape& s, int b, int g) {
  float v[1];
  Vec<T, 1>::unpack(Vec<T, 1>::load(x + (long long)b * s.S * s.ldx + (long long)g * s.Cg), v);
  return v[0];
}

// Column (mean - P, centred sum of squares) over a chunk of a sample's
// positions, P being the first value of the column's group: what is combined
// later are differences of means, and those keep their bits when the means
// are large beside the spread only if they are held relative to a value
// nearby.  A thread sums x - p and (x - p)^2 with p its own first value: p
// belongs to the data, so it is off the mean by at most the root of the total
// it measures, and over at most 64 rows the difference loses at most 64
// rounding units of that total.
template <typename T, int V>
__global__ void __launch_bounds__(kColThreads) k_gn_colstats(const T* x, GnShape s, ColGeom g, float2* part) {
  __shared__ float2 red[kColThreads * V];
  __shared__ int cnt[kColThreads];
  ptx::griddep_wait();
  const int ct = blockIdx.x % g.ctiles;
  const int rest = blockIdx.x / g.ctiles;
  const int ch = rest % g.chunks, b = rest / g.chunks;
  const int tc = threadIdx.x % g.TC, tr = threadIdx.x / g.TC;
  const int col = ct * g.TC + tc;
  const int r0 = ch * g.chunk, r1 = min(s.S, r0 + g.chunk);
  const bool on = tr < g.TR && col < g.CV;
  float piv[V], P[V], a1[V], a2[V];
#pragma unroll
  for (int e = 0; e < V; ++e) piv[e] = P[e] = a1[e] = a2[e] = 0.f;
  int m = 0;
  if (on) {
    const T* p = x + ((long long)b * s.S) * s.ldx + (long long)col * V;
#pragma unroll
    for (int e = 0; e < V; ++e) P[e] = group_pivot(x, s, b, (col * V + e) / s.Cg);
    if (r0 + tr < r1) Vec<T, V>::unpack(Vec<T, V>::load(p + (long long)(r0 + tr) * s.ldx), piv);
#pragma unroll 4
    for (int r = r0 + tr; r < r1; r += g.TR, ++m) {
      float v[V];
      Vec<T, V>::unpack(Vec<T, V>::load(p + (long long)r * s.ldx), v);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = v[e] - piv[e];
        a1[e] += d;
        a2[e] = fmaf(d, d, a2[e]);
      }
    }
  }
  const float inv = m > 0 ? 1.f / (float)m : 0.f;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const float dm = a1[e] * inv;
    red[threadIdx.x * V + e] = make_float2((piv[e] - P[e]) + dm, a2[e] - a1[e] * dm);
  }
  cnt[threadIdx.x] = m;
  __syncthreads();
  if (on && tr == 0) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      float mean = 0.f, M2 = 0.f, k = 0.f;
      for (int t = 0; t < g.TR; ++t) {
        const int i = t * g.TC + tc;
        if (!cnt[i]) continue;
        const float2 q = red[i * V + e];
        const float kt = (float)cnt[i], d = q.x - mean, kn = k + kt;
        mean = fmaf(d, kt / kn, mean);
        M2 += q.y + d * d * (k * kt / kn);
        k = kn;
      }
      part[((long long)b * g.chunks + ch) * s.C + (long long)col * V + e] = make_float2(mean, M2);
    }
  }
}

__device__ __forceinline__ float block_sum(float v, float* sm) {
  v = warp_sum(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
  __syncthreads();
  float t = 0.f;
  for (int w = 0; w < (int)(blockDim.x >> 5); ++w) t += sm[w];
  return t;
}

// One block per (sample, group): the chunks' column statistics to mean and rstd.
template <typename T>
__global__ void __launch_bounds__(128) k_gn_fold(const T* x, const float2* part, GnShape s, ColGeom g,
                                                 float* mean_out, float* rstd_out) {
  __shared__ float sm[4];
  ptx::griddep_wait();
  const int b = blockIdx.x / s.G, gr = blockIdx.x % s.G;
  const long long cells = (long long)g.chunks * s.Cg;
  const float2* p = part + (long long)b * g.chunks * s.C + gr * s.Cg;
  const float total = (float)s.S * (float)s.Cg;
  float sum = 0.f;
  for (long long i = threadIdx.x; i < cells; i += blockDim.x) {
    const int ch = (int)(i / s.Cg), c = (int)(i % s.Cg);
    const float rows = (float)(min(s.S, (ch + 1) * g.chunk) - ch * g.chunk);
    sum = fmaf(p[(long long)ch * s.C + c].x, rows, sum);
  }
  const float mean = block_sum(sum, sm) / total;
  float M2 = 0.f;
  for (long long i = threadIdx.x; i < cells; i += blockDim.x) {
    const int ch = (int)(i / s.Cg), c = (int)(i % s.Cg);
    const float rows = (float)(min(s.S, (ch + 1) * g.chunk) - ch * g.chunk);
    const float2 q = p[(long long)ch * s.C + c];
    const float d = q.x - mean;
    M2 += fmaf(d * d, rows, q.y);
  }
  const float var = block_sum(M2, sm) / total;
  if (threadIdx.x == 0) {
    mean_out[blockIdx.x] = group_pivot(x, s, b, gr) + mean;
    rstd_out[blockIdx.x] = 1.f / sqrtf(var + s.eps);
  }
}

template <typename T, int V>
__global__ void __launch_bounds__(kColThreads) k_gn_apply(const T* x, GnShape s, ColGeom g, const float* gamma,
                                                          const float* beta, const float* mean, const float* rstd,
                                                          T* y) {
  ptx::griddep_wait();
  const int ct = blockIdx.x % g.ctiles;
  const int rest = blockIdx.x / g.ctiles;
  const int ch = rest % g.chunks, b = rest / g.chunks;
  const int tc = threadIdx.x % g.TC, tr = threadIdx.x / g.TC;
  const int col = ct * g.TC + tc;
  const int r0 = ch * g.chunk, r1 = min(s.S, r0 + g.chunk);
  if (tr >= g.TR || col >= g.CV) return;
  float mu[V], a[V], bt[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const int c = col * V + e, st = b * s.G + c / s.Cg;
    mu[e] = mean[st];
    a[e] = rstd[st] * (gamma ? gamma[c] : 1.f);
    bt[e] = beta ? beta[c] : 0.f;
  }
  const long long row0 = (long long)b * s.S;
#pragma unroll 4
  for (int r = r0 + tr; r < r1; r += g.TR) {
    float v[V];
    Vec<T, V>::unpack(Vec<T, V>::load(x + (row0 + r) * s.ldx + (long long)col * V), v);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = act_of(fmaf(v[e] - mu[e], a[e], bt[e]), s.act);
    Vec<T, V>::store(y + (row0 + r) * s.ldy + (long long)col * V, v);
  }
}

// Column sums (du, du h) over a chunk of a sample's positions.
template <typename T, int V>
__global__ void __launch_bounds__(kColThreads) k_gn_grad_colsums(const T* dy, const T* x, GnShape s, ColGeom g,
                                                                 const float* mean, const float* rstd,
                                                                 const float* gamma, const float* beta,
                                                                 float2* part) {
  __shared__ float2 red[kColThreads * V];
  ptx::griddep_wait();
  const int ct = blockIdx.x % g.ctiles;
  const int rest = blockIdx.x / g.ctiles;
  const int ch = rest % g.chunks, b = rest / g.chunks;
  const int tc = threadIdx.x % g.TC, tr = threadIdx.x / g.TC;
  const int col = ct * g.TC + tc;
  const int r0 = ch * g.chunk, r1 = min(s.S, r0 + g.chunk);
  const bool on = tr < g.TR && col < g.CV;
  float p0[V], p1[V];
#pragma unroll
  for (int e = 0; e < V; ++e) p0[e] = p1[e] = 0.f;
  if (on) {
    float mu[V], rs[V], ga[V], bt[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int c = col * V + e, st = b * s.G + c / s.Cg;
      mu[e] = mean[st];
      rs[e] = rstd[st];
      ga[e] = gamma ? gamma[c] : 1.f;
      bt[e] = beta ? beta[c] : 0.f;
    }
    const long long row0 = (long long)b * s.S;
#pragma unroll 2
    for (int r = r0 + tr; r < r1; r += g.TR) {
      float v[V], d[V];
      Vec<T, V>::unpack(Vec<T, V>::load(x + (row0 + r) * s.ldx + (long long)col * V), v);
      Vec<T, V>::unpack(Vec<T, V>::load(dy + (row0 + r) * s.lddy + (long long)col * V), d);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float h = (v[e] - mu[e]) * rs[e];
        const float du = act_grad(d[e], fmaf(ga[e], h, bt[e]), s.act);
        p0[e] += du;
        p1[e] = fmaf(du, h, p1[e]);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < V; ++e) red[threadIdx.x * V + e] = make_float2(p0[e], p1[e]);
  __syncthreads();
  if (on && tr == 0) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      float2 t = make_float2(0.f, 0.f);
      for (int k = 0; k < g.TR; ++k) {
        const float2 q = red[(k * g.TC + tc) * V + e];
        t.x += q.x;
        t.y += q.y;
      }
      part[((long long)b * g.chunks + ch) * s.C + (long long)col * V + e] = t;
    }
  }
}

// One block per (sample, group): the averages <gamma du> and <gamma du h>.
__global__ void __launch_bounds__(128) k_gn_grad_fold(const float2* part, GnShape s, ColGeom g, const float* gamma,
                                                      float2* avg) {
  __shared__ float sm[4];
  ptx::griddep_wait();
  const int b = blockIdx.x / s.G, gr = blockIdx.x % s.G;
  const long long cells = (long long)g.chunks * s.Cg;
  const float2* p = part + (long long)b * g.chunks * s.C + gr * s.Cg;
  float m1 = 0.f, m2 = 0.f;
  for (long long i = threadIdx.x; i < cells; i += blockDim.x) {
    const int ch = (int)(i / s.Cg), c = (int)(i % s.Cg);
    const float2 q = p[(long long)ch * s.C + c];
    const float ga = gamma ? gamma[gr * s.Cg + c] : 1.f;
    m1 = fmaf(ga, q.x, m1);
    m2 = fmaf(ga, q.y, m2);
  }
  const float total = (float)s.S * (float)s.Cg;
  m1 = block_sum(m1, sm);
  m2 = block_sum(m2, sm);
  if (threadIdx.x == 0) avg[blockIdx.x] = make_float2(m1 / total, m2 / total);
}

// dbeta and dgamma: the partial column sums [rows, C] added up, in an order
// that depends on the sizes only.
constexpr int kFoldCols = 32, kFoldRows = 16;
__global__ void __launch_bounds__(kFoldCols * kFoldRows) k_gn_param_fold(const float2* part, long long rows, int C,
                                                                        float* dgamma, float* dbeta) {
  __shared__ float2 red[kFoldRows][kFoldCols];
  ptx::griddep_wait();
  const int tc = threadIdx.x % kFoldCols, tr = threadIdx.x / kFoldCols;
  const int c = blockIdx.x * kFoldCols + tc;
  float2 t = make_float2(0.f, 0.f);
  if (c < C) {
#pragma unroll 8
    for (long long r = tr; r < rows; r += kFoldRows) {
      const float2 q = part[r * C + c];
      t.x += q.x;
      t.y += q.y;
    }
  }
  red[tr][tc] = t;
  __syncthreads();
  if (tr == 0 && c < C) {
    for (int k = 1; k < kFoldRows; ++k) {
      t.x += red[k][tc].x;
      t.y += red[k][tc].y;
    }
    dbeta[c] = t.x;
    dgamma[c] = t.y;
  }
}

template <typename T, int V>
__global__ void __launch_bounds__(kColThreads) k_gn_grad_apply(const T* dy, const T* x, GnShape s, ColGeom g,
                                                               const float* mean, const float* rstd,
                                                               const float* gamma, const float* beta,
                                                               const float2* avg, T* dx) {
  ptx::griddep_wait();
  const int ct = blockIdx.x % g.ctiles;
  const int rest = blockIdx.x / g.ctiles;
  const int ch = rest % g.chunks, b = rest / g.chunks;
  const int tc = threadIdx.x % g.TC, tr = threadIdx.x / g.TC;
  const int col = ct * g.TC + tc;
  const int r0 = ch * g.chunk, r1 = min(s.S, r0 + g.chunk);
  if (tr >= g.TR || col >= g.CV) return;
  float mu[V], rs[V], ga[V], bt[V], m1[V], m2[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const int c = col * V + e, st = b * s.G + c / s.Cg;
    mu[e] = mean[st];
    rs[e] = rstd[st];
    ga[e] = gamma ? gamma[c] : 1.f;
    bt[e] = beta ? beta[c] : 0.f;
    m1[e] = avg[st].x;
    m2[e] = avg[st].y;
  }
  const long long row0 = (long long)b * s.S;
#pragma unroll 2
  for (int r = r0 + tr; r < r1; r += g.TR) {
    float v[V], d[V];
    Vec<T, V>::unpack(Vec<T, V>::load(x + (row0 + r) * s.ldx + (long long)col * V), v);
    Vec<T, V>::unpack(Vec<T, V>::load(dy + (row0 + r) * s.lddy + (long long)col * V), d);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float h = (v[e] - mu[e]) * rs[e];
      const float du = act_grad(d[e], fmaf(ga[e], h, bt[e]), s.act);
      v[e] = rs[e] * (fmaf(ga[e], du, -m1[e]) - h * m2[e]);
    }
    Vec<T, V>::store(dx + (row0 + r) * s.ldy + (long long)col * V, v);
  }
}

// ------------------------------------------------------------------- host
constexpr long long kAlign = 16;
long long align_up(long long v) { return (v + kAlign - 1) / kAlign * kAlign; }

bool good_shape(int n, int spatial, int channels, int groups, ff_precision prec) {
  return n >= 0 && spatial >= 0 && channels >= 1 && groups >= 1 && channels % groups == 0 &&
         (prec == FF_FP32 || prec == FF_BF16);
}

// Widest vector of at most 16 bytes that every row of the (up to three)
// matrices and the row length allow.
int vec_of(int C, int esize, const void* a, long long lda, const void* b, long long ldb, const void* c,
           long long ldc) {
  int v = 16 / esize;
  while (v > 1 && !(C % v == 0 && rows_aligned(a, lda, esize, v * esize) && rows_aligned(b, ldb, esize, v * esize) &&
                    rows_aligned(c, ldc, esize, v * esize)))
    v /= 2;
  return v;
}

// The partials' chunks depend on the vector width, so the workspace covers
// the width that needs most.
long long partial_bytes(int n, int S, int C, ff_precision prec) {
  long long most = 0;
  for (int v = 16 / (prec == FF_BF16 ? 2 : 4); v >= 1; v /= 2) {
    if (C % v) continue;
    const long long b = (long long)n * col_geom(n, S, C, v).chunks * C * (long long)sizeof(float2);
    most = b > most ? b : most;
  }
  return align_up(most);
}
long long stats_bytes(int n, int G) { return align_up((long long)n * G * (long long)sizeof(float2)); }

template <typename T, int V>
ff_status norm_general(const T* x, const GnShape& s, const float* gamma, const float* beta, T* y, float* mean,
                       float* rstd, void* ws, cudaStream_t st) {
  const ColGeom g = col_geom(s.n, s.S, s.C, V);
  const long long blocks = (long long)s.n * g.chunks * g.ctiles;
  if (blocks > 0x7FFFFFFFll || (long long)s.n * s.G > 0x7FFFFFFFll) return FF_ERR_UNSUPPORTED;
  float2* part = static_cast<float2*>(ws);
  if (!mean) {
    mean = reinterpret_cast<float*>(static_cast<char*>(ws) + partial_bytes(s.n, s.S, s.C, sizeof(T) == 2 ? FF_BF16 : FF_FP32));
    rstd = mean + (long long)s.n * s.G;
  }
  const double bytes = (double)s.n * s.S * s.C * sizeof(T);
  PdlLaunch l1(dim3((unsigned)blocks), dim3(kColThreads), st);
  FF_LAUNCH(K_GNORM, bytes, st, cudaLaunchKernelEx(&l1.cfg, k_gn_colstats<T, V>, x, s, g, part), "group norm sums");
  PdlLaunch l2(dim3((unsigned)(s.n * s.G)), dim3(128), st);
  FF_LAUNCH(K_GNORM, 0, st,
            cudaLaunchKernelEx(&l2.cfg, k_gn_fold<T>, x, static_cast<const float2*>(part), s, g, mean, rstd),
            "group norm fold");
  PdlLaunch l3(dim3((unsigned)blocks), dim3(kColThreads), st);
  FF_LAUNCH(K_GNORM, 2 * bytes, st,
            cudaLaunchKernelEx(&l3.cfg, k_gn_apply<T, V>, x, s, g, gamma, beta, static_cast<const float*>(mean),
                               static_cast<const float*>(rstd), y),
            "group norm apply");
  return FF_OK;
}

template <typename T, int V>
ff_status grad_general(const T* dy, const T* x, const GnShape& s, const float* mean, const float* rstd,
                       const float* gamma, const float* beta, T* dx, float* dgamma, float* dbeta, void* ws,
                       cudaStream_t st) {
  const ColGeom g = col_geom(s.n, s.S, s.C, V);
  const long long blocks = (long long)s.n * g.chunks * g.ctiles;
  if (blocks > 0x7FFFFFFFll || (long long)s.n * s.G > 0x7FFFFFFFll) return FF_ERR_UNSUPPORTED;
  float2* part = static_cast<float2*>(ws);
  float2* avg = reinterpret_cast<float2*>(static_cast<char*>(ws) +
                                          partial_bytes(s.n, s.S, s.C, sizeof(T) == 2 ? FF_BF16 : FF_FP32));
  const double bytes = (double)s.n * s.S * s.C * sizeof(T);
  PdlLaunch l1(dim3((unsigned)blocks), dim3(kColThreads), st);
  FF_LAUNCH(K_GNORM_GRAD, 2 * bytes, st,
            cudaLaunchKernelEx(&l1.cfg, k_gn_grad_colsums<T, V>, dy, x, s, g, mean, rstd, gamma, beta, part),
            "group norm gradient sums");
  if (dx) {
    PdlLaunch l2(dim3((unsigned)(s.n * s.G)), dim3(128), st);
    FF_LAUNCH(K_GNORM_GRAD, 0, st,
              cudaLaunchKernelEx(&l2.cfg, k_gn_grad_fold, static_cast<const float2*>(part), s, g, gamma, avg),
              "group norm gradient fold");
    PdlLaunch l3(dim3((unsigned)blocks), dim3(kColThreads), st);
    FF_LAUNCH(K_GNORM_GRAD, 3 * bytes, st,
              cudaLaunchKernelEx(&l3.cfg, k_gn_grad_apply<T, V>, dy, x, s, g, mean, rstd, gamma, beta,
                                 static_cast<const float2*>(avg), dx),
              "group norm gradient apply");
  }
  if (dgamma) {
    PdlLaunch l4(dim3((unsigned)cdiv(s.C, kFoldCols)), dim3(kFoldCols * kFoldRows), st);
    FF_LAUNCH(K_GNORM_GRAD, 0, st,
              cudaLaunchKernelEx(&l4.cfg, k_gn_param_fold, static_cast<const float2*>(part),
                                 (long long)s.n * g.chunks, s.C, dgamma, dbeta),
              "group norm parameter gradients");
  }
  return FF_OK;
}

template <typename T>
ff_status norm_t(const T* x, const GnShape& s, const float* gamma, const float* beta, T* y, float* mean, float* rstd,
                 void* ws, cudaStream_t st) {
  const int v = vec_of(s.C, sizeof(T), x, s.ldx, y, s.ldy, y, s.ldy);
  if constexpr (sizeof(T) == 2)
    if (v == 8) return norm_general<T, 8>(x, s, gamma, beta, y, mean, rstd, ws, st);
  if (v >= 4) return norm_general<T, 4>(x, s, gamma, beta, y, mean, rstd, ws, st);
  if (v == 2) return norm_general<T, 2>(x, s, gamma, beta, y, mean, rstd, ws, st);
  return norm_general<T, 1>(x, s, gamma, beta, y, mean, rstd, ws, st);
}

template <typename T>
ff_status grad_t(const T* dy, const T* x, const GnShape& s, const float* mean, const float* rstd, const float* gamma,
                 const float* beta, T* dx, float* dgamma, float* dbeta, void* ws, cudaStream_t st) {
  const T* out = dx ? dx : x;
  const int v = vec_of(s.C, sizeof(T), x, s.ldx, dy, s.lddy, out, dx ? s.ldy : s.ldx);
  if constexpr (sizeof(T) == 2)
    if (v == 8) return grad_general<T, 8>(dy, x, s, mean, rstd, gamma, beta, dx, dgamma, dbeta, ws, st);
  if (v >= 4) return grad_general<T, 4>(dy, x, s, mean, rstd, gamma, beta, dx, dgamma, dbeta, ws, st);
  if (v == 2) return grad_general<T, 2>(dy, x, s, mean, rstd, gamma, beta, dx, dgamma, dbeta, ws, st);
  return grad_general<T, 1>(dy, x, s, mean, rstd, gamma, beta, dx, dgamma, dbeta, ws, st);
}

bool good_act(ff_activation a) { return a == FF_ACT_NONE || a == FF_ACT_RELU || a == FF_ACT_SILU; }
bool good_matrix(const void* p, long long ld, long long rows, int C, int esize) {
  return p && reinterpret_cast<uintptr_t>(p) % esize == 0 && (ld >= C || rows <= 1);
}

}  // namespace
}  // namespace ff

using namespace ff;

extern "C" FF_API long long ff_group_norm_workspace(int n, int spatial, int channels, int groups, ff_precision prec,
                                                    int backward) {
  (void)backward;
  if (!good_shape(n, spatial, channels, groups, prec)) return -1;
  if (n == 0 || spatial == 0) return 0;
  return partial_bytes(n, spatial, channels, prec) + stats_bytes(n, groups);
}

extern "C" FF_API ff_status ff_group_norm_act(const void* x, long long ldx, int n, int spatial, int channels,
                                              int groups, const float* gamma, const float* beta, float eps,
                                              ff_activation act, ff_precision prec, void* y, long long ldy,
                                              float* mean, float* rstd, void* workspace, long long workspace_bytes,
                                              void* stream) {
  if (!good_shape(n, spatial, channels, groups, prec) || !good_act(act)) return FF_ERR_INVALID_ARG;
  if (!(eps > 0.f) || !std::isfinite(eps) || (mean == nullptr) != (rstd == nullptr)) return FF_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (n == 0) return FF_OK;
  if (spatial == 0) {
    if (mean) {
      const size_t bytes = (size_t)n * groups * sizeof(float);
      if (cudaMemsetAsync(mean, 0, bytes, st) != cudaSuccess || cudaMemsetAsync(rstd, 0, bytes, st) != cudaSuccess)
        return FF_ERR_CUDA;
    }
    return FF_OK;
  }
  const long long rows = (long long)n * spatial;
  const int es = prec == FF_BF16 ? 2 : 4;
  if (!good_matrix(x, ldx, rows, channels, es) || !good_matrix(y, ldy, rows, channels, es)) return FF_ERR_INVALID_ARG;
  const long long need = ff_group_norm_workspace(n, spatial, channels, groups, prec, 0);
  if (need > 0 && (!workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(workspace) % kAlign))
    return FF_ERR_INVALID_ARG;
  const GnShape s{n, spatial, channels, groups, channels / groups, ldx, ldy, 0, eps, (int)act};
  if (prec == FF_BF16)
    return norm_t(static_cast<const bf16*>(x), s, gamma, beta, static_cast<bf16*>(y), mean, rstd, workspace, st);
  return norm_t(static_cast<const float*>(x), s, gamma, beta, static_cast<float*>(y), mean, rstd, workspace, st);
}

extern "C" FF_API ff_status ff_group_norm_act_backward(const void* dy, long long lddy, const void* x, long long ldx,
                                                       int n, int spatial, int channels, int groups,
                                                       const float* mean, const float* rstd, const float* gamma,
                                                       const float* beta, ff_activation act, ff_precision prec,
                                                       void* dx, long long lddx, float* dgamma, float* dbeta,
                                                       void* workspace, long long workspace_bytes, void* stream) {
  if (!good_shape(n, spatial, channels, groups, prec) || !good_act(act)) return FF_ERR_INVALID_ARG;
  if ((dgamma == nullptr) != (dbeta == nullptr)) return FF_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (n == 0 || spatial == 0) {
    if (dgamma) {
      const size_t bytes = (size_t)channels * sizeof(float);
      if (cudaMemsetAsync(dgamma, 0, bytes, st) != cudaSuccess || cudaMemsetAsync(dbeta, 0, bytes, st) != cudaSuccess)
        return FF_ERR_CUDA;
    }
    return FF_OK;
  }
  if (!dx && !dgamma) return FF_OK;
  const long long rows = (long long)n * spatial;
  const int es = prec == FF_BF16 ? 2 : 4;
  if (!good_matrix(x, ldx, rows, channels, es) || !good_matrix(dy, lddy, rows, channels, es) ||
      (dx && !good_matrix(dx, lddx, rows, channels, es)) || !mean || !rstd)
    return FF_ERR_INVALID_ARG;
  const long long need = ff_group_norm_workspace(n, spatial, channels, groups, prec, 1);
  if (need > 0 && (!workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(workspace) % kAlign))
    return FF_ERR_INVALID_ARG;
  const GnShape s{n, spatial, channels, groups, channels / groups, ldx, lddx, lddy, 0.f, (int)act};
  if (prec == FF_BF16)
    return grad_t(static_cast<const bf16*>(dy), static_cast<const bf16*>(x), s, mean, rstd, gamma, beta,
                  static_cast<bf16*>(dx), dgamma, dbeta, workspace, st);
  return grad_t(static_cast<const float*>(dy), static_cast<const float*>(x), s, mean, rstd, gamma, beta,
                static_cast<float*>(dx), dgamma, dbeta, workspace, st);
}
