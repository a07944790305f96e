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
//
// Bound by HBM and by what three dependent launches cost: 32 x 4096 x 512 in 32
// groups (bf16, silu) takes 74 us, 5.4 TB/s over two reads and a write, its
// gradient 127 us (four reads and a write); 32 x 3136 x 320 41 and 73 us.
// Reading once more from L2 instead of HBM was tried in two forms and lost.
// Passes over a few samples at a time pay about 10 us of ramps for every part
// (two parts: 87 us).  One persistent kernel that forms a piece's sums some
// pieces ahead of its outputs waits on its own barriers (113 us).
//
// Groups that fit registers or shared memory may take one of two paths that
// read x (and dy) once: rows (ff_norm_rows.cu) and blocks (ff_norm_block.cu).
#include <algorithm>
#include <cmath>

#include "ff_norm.cuh"

namespace ff {
namespace {

constexpr long long kAlign = 16;
long long align_up(long long v, long long to = kAlign) { return (v + to - 1) / to * to; }

// ------------------------------------------------------------ general path
constexpr int kColThreads = 256;
constexpr int kColVecs = 32;       // at most this many vectors of columns per block
// A thread's positions at most: they bound the rounding of its one-pass sums
// (see k_gn_colstats) and, in the gradient, of its plain ones.
constexpr int kRowsPerThread = 64, kGradRowsPerThread = 128;

struct ColGeom {
  int CV, TC, TR, ctiles, chunk, chunks;
  int wide;                              // gamma and beta are 16-byte aligned
  FastDiv by_tiles, by_chunks, by_TC, by_Cg, by_G;
};
// Blocks of TC vector columns x TR thread rows; `chunk` positions per block.
// The rounds of 4 (gradient: 3) blocks per SM cost what their slowest thread
// does: its positions and, for constants and the sums' way out, about 6 more.
// Whole rounds count more than their number (32 x 3136 x 320 bf16, gradient:
// 2.5 rounds of 29 positions 83 us, 4 whole ones of 19 80 us).
ColGeom col_geom(const GnShape& s, int V, int esize, bool grad, const float* gamma, const float* beta) {
  ColGeom g;
  g.CV = s.C / V;
  g.ctiles = cdiv(g.CV, kColVecs);
  // tiles of equal width, whole 32-byte sectors where a row has them
  g.TC = std::min(g.CV, (int)align_up(cdiv(g.CV, g.ctiles), std::max(1, 32 / (V * esize))));
  g.ctiles = cdiv(g.CV, g.TC);
  g.TR = kColThreads / g.TC;
  const long long room = 152 * (grad ? 3 : 4), tiles = (long long)s.n * g.ctiles;
  const int most = grad ? kGradRowsPerThread : kRowsPerThread;
  long long chunk = std::min<long long>(s.S, (long long)g.TR * most), least = 0;
  for (int k = 0; k <= 16; ++k) {
    // k = 0: the largest chunks, where even 16 rounds are too few
    const long long cut = cdiv(s.S, (int)std::min<long long>(s.S, std::max(1ll, k * room / tiles)));
    const long long c = k == 0 ? chunk : std::min<long long>(s.S, std::max(cut, g.TR * 8ll));  // (the fold reads every chunk)
    const int rows = cdiv((int)c, g.TR);
    if (rows > most) continue;
    const long long blocks = tiles * cdiv(s.S, (int)c), cost = (blocks + room - 1) / room * (rows + 6);
    if (least == 0 || cost < least) least = cost, chunk = c;
  }
  g.chunk = (int)chunk;
  g.chunks = cdiv(s.S, g.chunk);
  g.wide = ((reinterpret_cast<uintptr_t>(gamma) | reinterpret_cast<uintptr_t>(beta)) & 15) == 0;
  g.by_tiles = FastDiv(g.ctiles);
  g.by_chunks = FastDiv(g.chunks);
  g.by_TC = FastDiv(g.TC);
  g.by_Cg = FastDiv(s.Cg);
  g.by_G = FastDiv(s.G);
  return g;
}
// A thread's place: sample, chunk, its column of V channels, and its positions
// tr, tr + TR, .. below `rows`, counted from the chunk's first: a chunk's own
// count stays small, whereas positions counted from the sample's start would
// pass 2^31 in the last chunk of the longest samples.  The second passes take
// the blocks from the last to the first, since what the first pass read last
// is still in L2.
struct ColPlace {
  int b, ch, tc, tr, col, rows;
  long long r0;  // the thread's first position, from the sample's first
  bool on;
  __device__ __forceinline__ ColPlace(const GnShape& s, const ColGeom& g, bool backwards) {
    const uint32_t i = backwards ? gridDim.x - 1 - blockIdx.x : blockIdx.x;
    const uint32_t rest = g.by_tiles.div(i);
    b = (int)g.by_chunks.div(rest);
    ch = (int)rest - b * g.chunks;
    tr = (int)g.by_TC.div(threadIdx.x);
    tc = (int)threadIdx.x - tr * g.TC;
    col = (int)(i - rest * g.ctiles) * g.TC + tc;
    on = tr < g.TR && col < g.CV;
    const int first = ch * g.chunk;
    rows = min(g.chunk, s.S - first);
    r0 = (long long)first + tr;
  }
};

// f(which of kFlight positions are there) over a thread's positions: a run of
// them without conditions, so that their loads fly and their arithmetic
// overlaps, and what is left one at a time.
constexpr int kFlight = 4;
struct HasAll {
  __device__ constexpr bool operator()(int) const { return true; }
};
struct HasSome {
  int n;
  __device__ __forceinline__ bool operator()(int u) const { return u < n; }
};
template <typename F>
__device__ __forceinline__ void walk_rows(int r0, int r1, int step, F f) {
  int r = r0;
  for (; r + (kFlight - 1) * step < r1; r += kFlight * step) f(HasAll{});
  if (r < r1) f(HasSome{(r1 - r + step - 1) / step});
}

template <typename T>
__device__ __forceinline__ float group_pivot(const T* x, const GnShape& s, int b, int g) {
  const T* p = x + (long long)b * s.S * s.ldx + (long long)g * s.Cg;
  float v[1], w[1];
  Vec<T, 1>::unpack(Vec<T, 1>::load(p), v);
  Vec<T, 1>::unpack(Vec<T, 1>::load(p + second_of(s)), w);
  return pivot_of(v[0], w[0]);
}

// Column (mean - P, centred sum of squares) over a chunk of a sample's
// positions, P being the pivot of the column's group: what is combined later
// are differences of means, and those keep their bits when the means are
// large beside the spread only if they are held relative to a value nearby.  A
// thread sums x - p and (x - p)^2 with p its own first value: p belongs to the
// data, so it is off the mean by at most the root of the total it measures,
// and over at most 64 rows the difference loses at most 64 rounding units of
// that total.
template <typename T, int V>
__global__ void __launch_bounds__(kColThreads, 4) k_gn_colstats(const T* x, GnShape s, ColGeom g, float2* part) {
  using PV = Pairs<V>;
  __shared__ float2 red[kColThreads * V];
  ptx::griddep_wait();
  const ColPlace p(s, g, false);
  uint64_t np[PV::N], a1[PV::N], a2[PV::N];
#pragma unroll
  for (int e = 0; e < PV::N; ++e) np[e] = a1[e] = a2[e] = 0;
  if (p.on) {
    const T* q = x + ((long long)p.b * s.S + p.r0) * s.ldx + (long long)p.col * V;
    const long long step = (long long)g.TR * s.ldx;
    if (p.tr < p.rows) {
      float m[V];
      Vec<T, V>::unpack(Vec<T, V>::load(q), m);
#pragma unroll
      for (int e = 0; e < V; ++e) m[e] = -m[e];
      PV::of(m, np);
    }
    walk_rows(p.tr, p.rows, g.TR, [&](auto has) {
      typename Vec<T, V>::Raw raw[kFlight];
#pragma unroll
      for (int u = 0; u < kFlight; ++u)
        if (has(u)) raw[u] = Vec<T, V>::load(q + u * step);
#pragma unroll
      for (int u = 0; u < kFlight; ++u)
        if (has(u)) {
          float v[V];
          uint64_t d[PV::N];
          Vec<T, V>::unpack(raw[u], v);
          PV::of(v, d);
#pragma unroll
          for (int e = 0; e < PV::N; ++e) {
            d[e] = ptx::add2(d[e], np[e]);
            a1[e] = ptx::add2(a1[e], d[e]);
            a2[e] = ptx::fma2(d[e], d[e], a2[e]);
          }
        }
      q += kFlight * step;
    });
  }
  const int rows = p.rows;
  // thread row t has rows / TR positions, one more below the remainder
  const int lo = rows / g.TR, rem = rows - lo * g.TR, m = lo + (p.tr < rem ? 1 : 0);
  float s1[V], s2[V], minus[V];
  PV::to(a1, s1);
  PV::to(a2, s2);
  PV::to(np, minus);
  const float inv = m > 0 ? 1.f / (float)m : 0.f;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const float dm = s1[e] * inv;
    const float P = p.on ? group_pivot(x, s, p.b, (int)g.by_Cg.div((uint32_t)(p.col * V + e))) : 0.f;
    red[threadIdx.x * V + e] = make_float2((-minus[e] - P) + dm, s2[e] - s1[e] * dm);
  }
  __syncthreads();
  // one thread per channel: the thread rows together
  const int width = g.TC * V, c0 = (p.col - p.tc) * V;
  const int used = lo > 0 ? g.TR : rem;
  const float tot = 1.f / (float)rows;
  for (int c = threadIdx.x; c < width && c0 + c < s.C; c += kColThreads) {
    float mean = 0.f, M2 = 0.f;
    for (int t = 0; t < used; ++t) mean = fmaf(red[t * width + c].x, (float)(lo + (t < rem ? 1 : 0)), mean);
    mean *= tot;
    for (int t = 0; t < used; ++t) {
      const float2 q = red[t * width + c];
      const float d = q.x - mean;
      M2 += fmaf(d * d, (float)(lo + (t < rem ? 1 : 0)), q.y);
    }
    part[((long long)p.b * g.chunks + p.ch) * s.C + c0 + c] = make_float2(mean, M2);
  }
}

template <int THREADS>
__device__ __forceinline__ float block_sum(float v, float* sm) {
  v = warp_sum(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
  __syncthreads();
  float t = 0.f;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) t += sm[w];
  return t;
}
// f(partial sums, which of kKept, channel within the group, positions) over the
// chunks' columns of one group, kKept loads in flight.  The first `kept` of them stay
// with the thread for a second walk.
constexpr int kKept = 4;
template <int THREADS>
struct Cells {
  const float2* p;
  float2 kept[kKept];
  __device__ __forceinline__ explicit Cells(const float2* p) : p(p) {}
  template <bool AGAIN, typename F>
  __device__ __forceinline__ void walk(const GnShape& s, const ColGeom& g, F f) {
    const int cells = g.chunks * s.Cg;
    for (int i0 = threadIdx.x; i0 < cells; i0 += kKept * THREADS) {
      const bool first = i0 == (int)threadIdx.x;
      float2 q[kKept];
#pragma unroll
      for (int u = 0; u < kKept; ++u) {
        const int i = i0 + u * THREADS;
        const int ch = (int)g.by_Cg.div((uint32_t)i);
        if (i < cells) q[u] = AGAIN && first ? kept[u] : p[(long long)ch * s.C + (i - ch * s.Cg)];
        if (!AGAIN && first) kept[u] = q[u];
      }
#pragma unroll
      for (int u = 0; u < kKept; ++u) {
        const int i = i0 + u * THREADS;
        const int ch = (int)g.by_Cg.div((uint32_t)i);
        if (i < cells) f(q[u], u, i - ch * s.Cg, (float)min(g.chunk, s.S - ch * g.chunk));
      }
    }
  }
};

// Threads of the folds' blocks, one block per (sample, group): many where
// blocks are few (4 x 4096 x 130 in one group: 18 us with 128, all in all).
constexpr int kFoldMany = 512, kFoldFew = 128;
int fold_threads(const GnShape& s) { return (long long)s.n * s.G < 152 * 4 ? kFoldMany : kFoldFew; }

// One block per (sample, group): the chunks' column statistics to mean and rstd.
template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS) k_gn_fold(const T* x, const float2* part, GnShape s, ColGeom g,
                                                          float* mean_out, float* rstd_out) {
  __shared__ float sm[THREADS / 32];
  ptx::griddep_wait();
  const int b = (int)g.by_G.div(blockIdx.x), gr = (int)blockIdx.x - b * s.G;
  Cells<THREADS> cells(part + (long long)b * g.chunks * s.C + gr * s.Cg);
  const float total = (float)s.S * (float)s.Cg;
  float sum[kKept] = {}, M2[kKept] = {};  // short sums: less rounding
  cells.walk<false>(s, g, [&](float2 q, int u, int, float rows) { sum[u] = fmaf(q.x, rows, sum[u]); });
  const float mean = block_sum<THREADS>((sum[0] + sum[1]) + (sum[2] + sum[3]), sm) / total;
  cells.walk<true>(s, g, [&](float2 q, int u, int, float rows) {
    const float d = q.x - mean;
    M2[u] += fmaf(d * d, rows, q.y);
  });
  const float var = block_sum<THREADS>((M2[0] + M2[1]) + (M2[2] + M2[3]), sm) / total;
  if (threadIdx.x == 0) {
    mean_out[blockIdx.x] = group_pivot(x, s, b, gr) + mean;
    rstd_out[blockIdx.x] = 1.f / sqrtf(var + s.eps);
  }
}

template <typename T, int V>
__global__ void __launch_bounds__(kColThreads) k_gn_apply(const T* x, GnShape s, ColGeom g, const float* gamma,
                                                          const float* beta, const float* mean, const float* rstd,
                                                          T* y) {
  using PV = Pairs<V>;
  ptx::griddep_wait();
  const ColPlace p(s, g, true);
  if (!p.on) return;
  // y = (x - mean) (gamma rstd) + beta, the mean taken off first (see GradCols)
  float a[V], b[V], m[V];
  load_params<V>(a, gamma, p.col * V, 1.f, g.wide);
  load_params<V>(b, beta, p.col * V, 0.f, g.wide);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const int st = p.b * s.G + (int)g.by_Cg.div((uint32_t)(p.col * V + e));
    a[e] *= rstd[st];
    m[e] = -mean[st];
  }
  uint64_t A[PV::N], B[PV::N], M[PV::N];
  PV::of(a, A);
  PV::of(b, B);
  PV::of(m, M);
  const T* q = x + ((long long)p.b * s.S + p.r0) * s.ldx + (long long)p.col * V;
  T* o = y + ((long long)p.b * s.S + p.r0) * s.ldy + (long long)p.col * V;
  const long long sx = (long long)g.TR * s.ldx, so = (long long)g.TR * s.ldy;
  walk_rows(p.tr, p.rows, g.TR, [&](auto has) {
    typename Vec<T, V>::Raw raw[kFlight];
#pragma unroll
    for (int u = 0; u < kFlight; ++u)
      if (has(u)) raw[u] = Vec<T, V>::load(q + u * sx);
#pragma unroll
    for (int u = 0; u < kFlight; ++u)
      if (has(u)) {
        float v[V];
        uint64_t d[PV::N];
        Vec<T, V>::unpack(raw[u], v);
        PV::of(v, d);
#pragma unroll
        for (int e = 0; e < PV::N; ++e) d[e] = ptx::fma2(ptx::add2(d[e], M[e]), A[e], B[e]);
        act_pairs<T, V>(d, s.act);
        PV::to(d, v);
        Vec<T, V>::store(o + u * so, v);
      }
    q += kFlight * sx;
    o += kFlight * so;
  });
}

// What the gradient's passes share: a column's constants.  h = (x - mean) rs,
// u = gamma h + beta.  The mean is taken off first: x rs - mean rs in one
// multiply-add would bring the rounding of mean rs into h, mean / spread
// rounding units instead of one.
template <typename T, int V>
struct GradCols {
  uint64_t rs[Pairs<V>::N], minus[Pairs<V>::N], ga[Pairs<V>::N], be[Pairs<V>::N];
  __device__ __forceinline__ GradCols(const GnShape& s, const ColGeom& g, const ColPlace& p, const float* mean,
                                      const float* rstd, const float* gamma, const float* beta) {
    float r[V], m[V], a[V], b[V];
    load_params<V>(a, gamma, p.col * V, 1.f, g.wide);
    load_params<V>(b, beta, p.col * V, 0.f, g.wide);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int st = p.b * s.G + (int)g.by_Cg.div((uint32_t)(p.col * V + e));
      r[e] = rstd[st];
      m[e] = -mean[st];
    }
    Pairs<V>::of(r, rs);
    Pairs<V>::of(m, minus);
    Pairs<V>::of(a, ga);
    Pairs<V>::of(b, be);
  }
  // x and dy of a position to h and du
  __device__ __forceinline__ void forms(uint64_t (&x)[Pairs<V>::N], uint64_t (&d)[Pairs<V>::N], int act) const {
    uint64_t u[Pairs<V>::N];
#pragma unroll
    for (int e = 0; e < Pairs<V>::N; ++e) {
      x[e] = ptx::mul2(ptx::add2(x[e], minus[e]), rs[e]);
      u[e] = ptx::fma2(x[e], ga[e], be[e]);
    }
    act_grad_pairs<T, V>(d, u, act);
  }
};

// Column sums (du, du h) over a chunk of a sample's positions.
template <typename T, int V>
__global__ void __launch_bounds__(kColThreads, 3) k_gn_grad_colsums(const T* dy, const T* x, GnShape s, ColGeom g,
                                                                 const float* mean, const float* rstd,
                                                                 const float* gamma, const float* beta,
                                                                 float2* part) {
  using PV = Pairs<V>;
  __shared__ float2 red[kColThreads * V];
  ptx::griddep_wait();
  const ColPlace p(s, g, false);
  uint64_t p0[PV::N], p1[PV::N];
#pragma unroll
  for (int e = 0; e < PV::N; ++e) p0[e] = p1[e] = 0;
  if (p.on) {
    const GradCols<T, V> k(s, g, p, mean, rstd, gamma, beta);
    const T* qx = x + ((long long)p.b * s.S + p.r0) * s.ldx + (long long)p.col * V;
    const T* qd = dy + ((long long)p.b * s.S + p.r0) * s.lddy + (long long)p.col * V;
    const long long sx = (long long)g.TR * s.ldx, sd = (long long)g.TR * s.lddy;
    walk_rows(p.tr, p.rows, g.TR, [&](auto has) {
      typename Vec<T, V>::Raw rx[kFlight], rd[kFlight];
#pragma unroll
      for (int u = 0; u < kFlight; ++u)
        if (has(u)) {
          rx[u] = Vec<T, V>::load(qx + u * sx);
          rd[u] = Vec<T, V>::load(qd + u * sd);
        }
#pragma unroll
      for (int u = 0; u < kFlight; ++u)
        if (has(u)) {
          float v[V], w[V];
          uint64_t h[PV::N], d[PV::N];
          Vec<T, V>::unpack(rx[u], v);
          Vec<T, V>::unpack(rd[u], w);
          PV::of(v, h);
          PV::of(w, d);
          k.forms(h, d, s.act);
#pragma unroll
          for (int e = 0; e < PV::N; ++e) {
            p0[e] = ptx::add2(p0[e], d[e]);
            p1[e] = ptx::fma2(d[e], h[e], p1[e]);
          }
        }
      qx += kFlight * sx;
      qd += kFlight * sd;
    });
  }
  float s0[V], s1[V];
  PV::to(p0, s0);
  PV::to(p1, s1);
#pragma unroll
  for (int e = 0; e < V; ++e) red[threadIdx.x * V + e] = make_float2(s0[e], s1[e]);
  __syncthreads();
  const int width = g.TC * V, c0 = (p.col - p.tc) * V;
  for (int c = threadIdx.x; c < width && c0 + c < s.C; c += kColThreads) {
    float2 t = red[c];
    for (int r = 1; r < g.TR; ++r) {
      t.x += red[r * width + c].x;
      t.y += red[r * width + c].y;
    }
    part[((long long)p.b * g.chunks + p.ch) * s.C + c0 + c] = t;
  }
}

// A sum that keeps what its additions round off (Knuth's two-sum), so that it
// may be long.  An infinite or NaN sum has no such remainder.
struct LongSum {
  float sum = 0.f, lost = 0.f;
  __device__ __forceinline__ void add(float v) {
    const float s = sum + v, t = s - sum;
    lost += (sum - (s - t)) + (v - t);
    sum = s;
  }
  __device__ __forceinline__ float value() const { return lost == lost ? sum + lost : sum; }
};

// dbeta and dgamma of kFoldCols channels: the partial column sums [rows, C]
// added up, in an order that depends on the sizes only.  Few columns and many
// row threads per block: the sums are short and latency is what they cost.
// Long ones (the rows grow with the batch) go eight rows at a time.
constexpr int kFoldCols = 8, kFoldRows = 8;
template <int ROWS>
__device__ __forceinline__ void param_fold(int block, const float2* part, const GnFold& f, int C, float* dgamma,
                                           float* dbeta) {
  __shared__ float2 red[ROWS][kFoldCols];
  const int tc = threadIdx.x % kFoldCols, tr = threadIdx.x / kFoldCols;
  const int c = block * kFoldCols + tc;
  LongSum tx, ty;
  if (c < C) {
    long long rows = f.rows;
    if (f.units > 0) {
      const long long first = (long long)(c / f.W) * f.n;
      rows = (first + f.n - 1) / f.units - first / f.units + 1;
    }
    for (long long r = tr; r < rows; r += kFoldRows * ROWS) {
      float2 t = make_float2(0.f, 0.f);
#pragma unroll
      for (int u = 0; u < kFoldRows; ++u)
        if (r + u * ROWS < rows) {
          const float2 q = part[(r + u * ROWS) * C + c];
          t.x += q.x;
          t.y += q.y;
        }
      tx.add(t.x);
      ty.add(t.y);
    }
  }
  red[tr][tc] = make_float2(tx.value(), ty.value());
  for (int half = ROWS / 2; half > 0; half /= 2) {
    __syncthreads();
    if (tr < half) {
      red[tr][tc].x += red[tr + half][tc].x;
      red[tr][tc].y += red[tr + half][tc].y;
    }
  }
  if (tr == 0 && c < C) {
    dbeta[c] = red[0][tc].x;
    dgamma[c] = red[0][tc].y;
  }
}
constexpr int kParamRows = 64;
__global__ void __launch_bounds__(kFoldCols * kParamRows) k_gn_param_fold(const float2* part, GnFold f, int C,
                                                                         float* dgamma, float* dbeta) {
  ptx::griddep_wait();
  param_fold<kParamRows>((int)blockIdx.x, part, f, C, dgamma, dbeta);
}

// One block per (sample, group): the averages <gamma du> and <gamma du h>; the
// first blocks, where the parameters' gradients are wanted, take those.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) k_gn_grad_fold(const float2* part, GnShape s, ColGeom g,
                                                               const float* gamma, float2* avg, int param_blocks,
                                                               float* dgamma, float* dbeta) {
  __shared__ float sm[THREADS / 32];
  ptx::griddep_wait();
  if ((int)blockIdx.x < param_blocks) {
    param_fold<THREADS / kFoldCols>((int)blockIdx.x, part, GnFold{(long long)s.n * g.chunks, 0, 0, 0}, s.C, dgamma,
                                         dbeta);
    return;
  }
  const int i = (int)blockIdx.x - param_blocks;
  const int b = (int)g.by_G.div((uint32_t)i), gr = i - b * s.G;
  float s1[kKept] = {}, s2[kKept] = {};
  Cells<THREADS>(part + (long long)b * g.chunks * s.C + gr * s.Cg).walk<false>(s, g, [&](float2 q, int u, int c, float) {
    const float ga = gamma ? __ldg(gamma + gr * s.Cg + c) : 1.f;
    s1[u] = fmaf(ga, q.x, s1[u]);
    s2[u] = fmaf(ga, q.y, s2[u]);
  });
  const float total = (float)s.S * (float)s.Cg;
  const float m1 = block_sum<THREADS>((s1[0] + s1[1]) + (s1[2] + s1[3]), sm);
  const float m2 = block_sum<THREADS>((s2[0] + s2[1]) + (s2[2] + s2[3]), sm);
  if (threadIdx.x == 0) avg[i] = make_float2(m1 / total, m2 / total);
}

template <typename T, int V>
__global__ void __launch_bounds__(kColThreads, 3) k_gn_grad_apply(const T* dy, const T* x, GnShape s, ColGeom g,
                                                               const float* mean, const float* rstd,
                                                               const float* gamma, const float* beta,
                                                               const float2* avg, T* dx) {
  using PV = Pairs<V>;
  ptx::griddep_wait();
  const ColPlace p(s, g, true);
  if (!p.on) return;
  const GradCols<T, V> k(s, g, p, mean, rstd, gamma, beta);
  // dx = rs (gamma du - <.> - h <.>) = du (gamma rs) + (h c2 + c1)
  float f1[V], f2[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const int st = p.b * s.G + (int)g.by_Cg.div((uint32_t)(p.col * V + e));
    const float2 m = avg[st];
    f1[e] = -rstd[st] * m.x;
    f2[e] = -rstd[st] * m.y;
  }
  uint64_t c1[PV::N], c2[PV::N], gr[PV::N];
  PV::of(f1, c1);
  PV::of(f2, c2);
#pragma unroll
  for (int e = 0; e < PV::N; ++e) gr[e] = ptx::mul2(k.ga[e], k.rs[e]);
  const T* qx = x + ((long long)p.b * s.S + p.r0) * s.ldx + (long long)p.col * V;
  const T* qd = dy + ((long long)p.b * s.S + p.r0) * s.lddy + (long long)p.col * V;
  T* o = dx + ((long long)p.b * s.S + p.r0) * s.ldy + (long long)p.col * V;
  const long long sx = (long long)g.TR * s.ldx, sd = (long long)g.TR * s.lddy, so = (long long)g.TR * s.ldy;
  walk_rows(p.tr, p.rows, g.TR, [&](auto has) {
    typename Vec<T, V>::Raw rx[kFlight], rd[kFlight];
#pragma unroll
    for (int u = 0; u < kFlight; ++u)
      if (has(u)) {
        rx[u] = Vec<T, V>::load(qx + u * sx);
        rd[u] = Vec<T, V>::load(qd + u * sd);
      }
#pragma unroll
    for (int u = 0; u < kFlight; ++u)
      if (has(u)) {
        float v[V], w[V];
        uint64_t h[PV::N], d[PV::N];
        Vec<T, V>::unpack(rx[u], v);
        Vec<T, V>::unpack(rd[u], w);
        PV::of(v, h);
        PV::of(w, d);
        k.forms(h, d, s.act);
#pragma unroll
        for (int e = 0; e < PV::N; ++e) h[e] = ptx::fma2(d[e], gr[e], ptx::fma2(h[e], c2[e], c1[e]));
        PV::to(h, v);
        Vec<T, V>::store(o + u * so, v);
      }
    qx += kFlight * sx;
    qd += kFlight * sd;
    o += kFlight * so;
  });
}

// ------------------------------------------------------------------- host

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

// What a call runs: decided by its sizes, its type and the alignment of its
// rows.
enum Path { ROWS, BLOCK, GENERAL };
struct Plan {
  Path path;
  int V;              // values per access
  GnBlockPlan block;
  long long bytes;    // workspace
};

// v: the widest access that the rows' alignment allows.  Within the two
// register paths a vector must lie in one group; they have accesses of 16
// bytes, of 4 (bf16) and of one value.
// Estimated time of the column passes (us).  They read x (and dy) twice, at
// about 5.7 TB/s in all where a thread has many positions, and take 5 or 6 us
// beside; constants and the sums' way out cost as much as a few positions.
// (1000 x 64 x 128 bf16, 4 positions: 26 us, block path 13; 64 x 784 x 256, 11:
// 21 and 16; its gradient, 33: 31 and 38.)
double general_us(const GnShape& s, int V, int esize, bool grad) {
  const ColGeom g = col_geom(s, V, esize, grad, nullptr, nullptr);
  const double bytes = (double)s.n * s.S * s.C * esize, rows = cdiv(g.chunk, g.TR);
  const double more = esize == 2 ? (grad ? 3.5 : 4.5) : (grad ? 1.5 : 2.0);
  const double us = grad ? 6.0 + 5 * bytes / 5.6e6 : 5.0 + 3 * bytes / 5.8e6;
  return us * (1.0 + more / rows) * (V == 1 ? 1.3 : 1.0);
}

Plan make_plan(const GnShape& s, int esize, int v, bool grad, bool near) {
  Plan p{GENERAL, v, {}, 0};

  const int wide = 16 / esize;
  int in_group = v;
  while (s.Cg % in_group) in_group /= 2;
  const int V = in_group == wide ? wide : esize == 2 && in_group >= 2 ? 2 : 1;
  // A few positions of narrow groups would be fetched a fraction of a 32-byte
  // sector at a time: those go to slabs of several groups.
  const bool narrow = s.S > 1 && s.Cg * esize < 32 && s.G > 1;
  const bool rows_fit = gn_rows_fit(s) && near;
  if (rows_fit && !narrow) p.path = ROWS;
  if (p.path == GENERAL) {
    p.block = gn_block_plan(s, V, esize, grad);
    if (p.block.T > 0 && p.block.us <= general_us(s, grad && v > 4 ? 4 : v, esize, grad))
      p.path = BLOCK;
    else if (rows_fit)
      p.path = ROWS;
  }
  if (p.path == GENERAL) {
    // the gradient's constants of eight columns do not fit the registers of
    // three blocks per SM (32 x 4096 x 512 bf16: 210 us, with four 123 us)
    if (grad && p.V > 4) p.V = 4;
    p.bytes = align_up((long long)s.n * col_geom(s, p.V, esize, grad, nullptr, nullptr).chunks * s.C * (long long)sizeof(float2)) +
              align_up((long long)s.n * s.G * (long long)sizeof(float2));
    return p;
  }
  p.V = V;
  if (grad) {
    const long long rows =
        p.path == ROWS ? (long long)gn_rows_plan(s, V, true).P * s.S
                       : (long long)(s.n - 1) / p.block.units + 2;  // blocks that share a slab
    p.bytes = align_up(rows * s.C * (long long)sizeof(float2));
  }
  return p;
}

template <typename T, int V>
ff_status norm_general(const GnArgs<T>& a, cudaStream_t st) {
  const GnShape& s = a.s;
  const ColGeom g = col_geom(s, V, sizeof(T), false, a.gamma, a.beta);
  const long long blocks = (long long)s.n * g.chunks * g.ctiles;
  if (blocks > 0x7FFFFFFFll) return FF_ERR_UNSUPPORTED;
  float2* part = static_cast<float2*>(a.ws);
  float *mean = a.mean, *rstd = a.rstd;
  if (!mean) {
    mean = reinterpret_cast<float*>(static_cast<char*>(a.ws) +
                                    align_up((long long)s.n * g.chunks * s.C * (long long)sizeof(float2)));
    rstd = mean + (long long)s.n * s.G;
  }
  const double bytes = (double)s.n * s.S * s.C * sizeof(T);
  PdlLaunch l1(dim3((unsigned)blocks), dim3(kColThreads), st);
  FF_LAUNCH(K_GNORM, bytes, st, cudaLaunchKernelEx(&l1.cfg, k_gn_colstats<T, V>, a.x, s, g, part), "group norm sums");
  const int ft = fold_threads(s);
  PdlLaunch l2(dim3((unsigned)(s.n * s.G)), dim3((unsigned)ft), st);
  FF_LAUNCH(K_GNORM, 0, st,
            cudaLaunchKernelEx(&l2.cfg, ft == kFoldMany ? k_gn_fold<T, kFoldMany> : k_gn_fold<T, kFoldFew>, a.x, static_cast<const float2*>(part), s, g, mean, rstd),
            "group norm fold");
  PdlLaunch l3(dim3((unsigned)blocks), dim3(kColThreads), st);
  FF_LAUNCH(K_GNORM, 2 * bytes, st,
            cudaLaunchKernelEx(&l3.cfg, k_gn_apply<T, V>, a.x, s, g, a.gamma, a.beta, static_cast<const float*>(mean),
                               static_cast<const float*>(rstd), a.out),
            "group norm apply");
  return FF_OK;
}

template <typename T, int V>
ff_status grad_general(const GnArgs<T>& a, cudaStream_t st) {
  const GnShape& s = a.s;
  const ColGeom g = col_geom(s, V, sizeof(T), true, a.gamma, a.beta);
  const long long blocks = (long long)s.n * g.chunks * g.ctiles;
  if (blocks > 0x7FFFFFFFll) return FF_ERR_UNSUPPORTED;
  float2* part = static_cast<float2*>(a.ws);
  float2* avg = reinterpret_cast<float2*>(static_cast<char*>(a.ws) +
                                          align_up((long long)s.n * g.chunks * s.C * (long long)sizeof(float2)));
  const float *mean = a.mean, *rstd = a.rstd;
  const double bytes = (double)s.n * s.S * s.C * sizeof(T);
  PdlLaunch l1(dim3((unsigned)blocks), dim3(kColThreads), st);
  FF_LAUNCH(K_GNORM_GRAD, 2 * bytes, st,
            cudaLaunchKernelEx(&l1.cfg, k_gn_grad_colsums<T, V>, a.dy, a.x, s, g, mean, rstd, a.gamma, a.beta, part),
            "group norm gradient sums");
  if (!a.out) return gn_param_fold(part, GnFold{(long long)s.n * g.chunks, 0, 0, 0}, s.C, a.dgamma, a.dbeta, st);
  const int params = a.dgamma ? cdiv(s.C, kFoldCols) : 0;
  if ((long long)s.n * s.G + params > 0x7FFFFFFFll) return FF_ERR_UNSUPPORTED;
  const int ft = fold_threads(s);
  PdlLaunch l2(dim3((unsigned)(s.n * s.G + params)), dim3((unsigned)ft), st);
  FF_LAUNCH(K_GNORM_GRAD, 0, st,
            cudaLaunchKernelEx(&l2.cfg, ft == kFoldMany ? k_gn_grad_fold<kFoldMany> : k_gn_grad_fold<kFoldFew>, static_cast<const float2*>(part), s, g, a.gamma, avg, params,
                               a.dgamma, a.dbeta),
            "group norm gradient fold");
  PdlLaunch l3(dim3((unsigned)blocks), dim3(kColThreads), st);
  FF_LAUNCH(K_GNORM_GRAD, 3 * bytes, st,
            cudaLaunchKernelEx(&l3.cfg, k_gn_grad_apply<T, V>, a.dy, a.x, s, g, mean, rstd, a.gamma, a.beta,
                               static_cast<const float2*>(avg), a.out),
            "group norm gradient apply");
  return FF_OK;
}

template <typename T, int V>
ff_status general(const GnArgs<T>& a, bool grad, cudaStream_t st) {
  return grad ? grad_general<T, V>(a, st) : norm_general<T, V>(a, st);
}

// The plan of a call.  It follows from sizes, type, alignment and whether
// offsets within a sample fit 32 bits (a lone position has no stride); making
// one takes a microsecond or more, so each thread keeps the last ones.
Plan plan_of(const GnShape& s, int esize, int v, bool grad) {
  struct Entry {
    int n = -1, S, C, G, kind;
    Plan plan;
  };
  thread_local Entry kept[64];
  const long long ld = std::max(std::max(s.ldx, s.ldy), s.lddy);
  const bool near = s.S == 1 || (ld < 0x3FFFFFFF && s.S * ld < 0x3FFFFFFF);
  const int kind = ((esize * 16 + v) * 2 + grad) * 2 + near;
  uint32_t h = (uint32_t)s.n;
  for (const int part : {s.S, s.C, s.G, kind}) h = h * 0x9E3779B1u + (uint32_t)part;
  Entry& e = kept[(h * 0x9E3779B1u) >> 26];
  if (e.n != s.n || e.S != s.S || e.C != s.C || e.G != s.G || e.kind != kind)
    e = Entry{s.n, s.S, s.C, s.G, kind, make_plan(s, esize, v, grad, near)};
  return e.plan;
}

// The workspace of the path that needs most among those that some stride or
// alignment of the rows leads to.
long long workspace_of(int n, int spatial, int channels, int groups, int esize, bool grad) {
  // the strides only say whether a sample's offsets fit 32 bits: both ways count
  const GnShape tight{n, spatial, channels, groups, channels / groups, channels, channels, channels, 0.f, 0};
  GnShape wide = tight;
  wide.ldx = wide.ldy = wide.lddy = 0x7FFFFFFF;
  long long most = 0;
  for (int v = 16 / esize; v >= 1; v /= 2) {
    if (channels % v) continue;
    for (const GnShape* s : {&tight, static_cast<const GnShape*>(&wide)}) {
      const long long b = plan_of(*s, esize, v, grad).bytes;
      most = b > most ? b : most;
    }
  }
  return most;
}

template <typename T>
ff_status call(const GnArgs<T>& a, long long ws_bytes, bool grad, cudaStream_t st) {
  const GnShape& s = a.s;
  const int v = grad ? vec_of(s.C, sizeof(T), a.x, s.ldx, a.dy, s.lddy, a.out ? a.out : a.x, a.out ? s.ldy : s.ldx)
                     : vec_of(s.C, sizeof(T), a.x, s.ldx, a.out, s.ldy, a.out, s.ldy);
  if ((long long)s.n * s.G > 0x7FFFFFFFll) return FF_ERR_UNSUPPORTED;
  const Plan p = plan_of(s, sizeof(T), v, grad);
  // what the query promises for the shape, whether or not these rows' strides
  // and alignment need all of it: a buffer is too small for all calls or none
  const long long need = workspace_of(s.n, s.S, s.C, s.G, sizeof(T), grad);
  if (need > 0 && (!a.ws || ws_bytes < need || reinterpret_cast<uintptr_t>(a.ws) % kAlign)) return FF_ERR_INVALID_ARG;
  if (p.path == ROWS) return gn_rows(a, p.V, grad, st);
  if (p.path == BLOCK) return gn_block(a, p.V, p.block, grad, st);
  if constexpr (sizeof(T) == 2)
    if (p.V == 8) return norm_general<T, 8>(a, st);
  if (p.V >= 4) return general<T, 4>(a, grad, st);
  if (p.V == 2) return general<T, 2>(a, grad, st);
  return general<T, 1>(a, grad, st);
}

bool good_act(ff_activation a) { return a == FF_ACT_NONE || a == FF_ACT_RELU || a == FF_ACT_SILU; }
bool good_matrix(const void* p, long long ld, long long rows, int C, int esize) {
  return p && reinterpret_cast<uintptr_t>(p) % esize == 0 && (ld >= C || rows <= 1);
}

}  // namespace

ff_status gn_param_fold(const float2* part, const GnFold& f, int C, float* dgamma, float* dbeta, cudaStream_t st) {
  PdlLaunch l(dim3((unsigned)cdiv(C, kFoldCols)), dim3(kFoldCols * kParamRows), st);
  FF_LAUNCH(K_GNORM_GRAD, 0, st, cudaLaunchKernelEx(&l.cfg, k_gn_param_fold, part, f, C, dgamma, dbeta),
            "group norm parameter gradients");
  return FF_OK;
}

}  // namespace ff

using namespace ff;

extern "C" FF_API long long ff_group_norm_workspace(int n, int spatial, int channels, int groups, ff_precision prec,
                                                    int backward) {
  if (!good_shape(n, spatial, channels, groups, prec)) return -1;
  return n == 0 || spatial == 0 ? 0 : workspace_of(n, spatial, channels, groups, prec == FF_BF16 ? 2 : 4, backward != 0);
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
  if (rows == 1) ldx = ldy = channels;
  const GnShape s{n, spatial, channels, groups, channels / groups, ldx, ldy, channels, eps, (int)act};
  if (prec == FF_BF16)
    return call(GnArgs<bf16>{s, static_cast<const bf16*>(x), nullptr, static_cast<bf16*>(y), gamma, beta, mean, rstd,
                             nullptr, nullptr, workspace},
                workspace_bytes, false, st);
  return call(GnArgs<float>{s, static_cast<const float*>(x), nullptr, static_cast<float*>(y), gamma, beta, mean, rstd,
                            nullptr, nullptr, workspace},
              workspace_bytes, false, st);
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
  if (rows == 1) ldx = lddy = lddx = channels;
  const GnShape s{n, spatial, channels, groups, channels / groups, ldx, dx ? lddx : channels, lddy, 0.f, (int)act};
  float *mu = const_cast<float*>(mean), *rs = const_cast<float*>(rstd);  // read only by the gradient
  if (prec == FF_BF16)
    return call(GnArgs<bf16>{s, static_cast<const bf16*>(x), static_cast<const bf16*>(dy), static_cast<bf16*>(dx), gamma,
                             beta, mu, rs, dgamma, dbeta, workspace},
                workspace_bytes, true, st);
  return call(GnArgs<float>{s, static_cast<const float*>(x), static_cast<const float*>(dy), static_cast<float*>(dx),
                            gamma, beta, mu, rs, dgamma, dbeta, workspace},
              workspace_bytes, true, st);
}
