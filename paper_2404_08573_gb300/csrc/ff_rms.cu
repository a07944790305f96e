// RMS norm with the residual's addition, its output rounded to the input's
// type or to e4m3 blocks, and its gradient:
//
//   h = x + residual, rstd = 1 / sqrt(mean h^2 + eps), y = gamma h rstd
//   du = gamma dy, n = h rstd, dx = rstd (du - n <du n>) + dh, dgamma = sum dy n
//
// A row is cut into units of 128 values, four to a lane, so that a warp holds
// whole e4m3 blocks; `warps` warps share a row.
#include "ff_api_internal.h"
#include "ff_e4m3.cuh"
#include "ff_ptx.cuh"
#include "ff_vec.cuh"

namespace ff {
namespace {

constexpr int UNIT = 128;
constexpr int kMaxWarps = 32;

// A lane's four values of the unit at column c0, V of them consecutive: 16 or
// 8 bytes (V = 4), a pair of bf16 (V = 2), or one (V = 1, the lanes side by
// side), as the rows' alignment allows.
template <typename T, int V>
struct Unit {
  static constexpr int N = 4 / V;
  typename Vec<T, V>::Raw raw[N];
  static __device__ __forceinline__ int col(int e, int lane) { return (e / V) * 32 * V + lane * V + e % V; }
  __device__ __forceinline__ void load(const T* row, int c0, int lane, int cols) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = c0 + i * 32 * V + lane * V;
      if (c + V <= cols) {
        raw[i] = Vec<T, V>::load(row + c);
      } else {
        T t[V];
#pragma unroll
        for (int e = 0; e < V; ++e) t[e] = c + e < cols ? row[c + e] : T(0.f);
        memcpy(&raw[i], t, sizeof(raw[i]));
      }
    }
  }
  __device__ __forceinline__ void values(float (&v)[4]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float t[V];
      Vec<T, V>::unpack(raw[i], t);
#pragma unroll
      for (int e = 0; e < V; ++e) v[i * V + e] = t[e];
    }
  }
  __device__ __forceinline__ void set(const float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float t[V];
#pragma unroll
      for (int e = 0; e < V; ++e) t[e] = v[i * V + e];
      Vec<T, V>::store(reinterpret_cast<T*>(&raw[i]), t);
    }
  }
  __device__ __forceinline__ void store(T* row, int c0, int lane, int cols) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = c0 + i * 32 * V + lane * V;
      if (c + V <= cols) {
        *reinterpret_cast<typename Vec<T, V>::Raw*>(row + c) = raw[i];
      } else {
        T t[V];
        memcpy(t, &raw[i], sizeof(raw[i]));
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (c + e < cols) row[c + e] = t[e];
      }
    }
  }
};

// A lane's four gammas of the unit (null: ones); zero past the row.
template <int V>
__device__ __forceinline__ void gammas(float (&g)[4], const float* gamma, int c0, int lane, int cols, bool wide) {
  if (V == 4 && wide && gamma && c0 + lane * 4 + 4 <= cols) {
    const float4 f = __ldg(reinterpret_cast<const float4*>(gamma + c0 + lane * 4));
    g[0] = f.x;
    g[1] = f.y;
    g[2] = f.z;
    g[3] = f.w;
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int c = c0 + Unit<float, V>::col(e, lane);
    g[e] = c < cols ? (gamma ? __ldg(gamma + c) : 1.f) : 0.f;
  }
}

// The sum over a row's warps of v, in a fixed order; `part` holds two rows'
// worth of [kMaxWarps] in turn (one barrier a row).
__device__ __forceinline__ float row_sum(float v, int warps, int warp, int lane, float* part) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (warps == 1) return v;
  if (lane == 0) part[warp] = v;
  __syncthreads();
  v = lane < warps ? part[lane] : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

template <typename T>
struct RmsArgs {
  const T *x, *r;
  T *h, *y;
  uint8_t* q;
  const float* gamma;
  float *scale, *rstd;
  long long ldx, ldr, ldh, ldy;
  int rows, cols, ldq, warps;
  float eps;
  bool wide;  // gamma is 16-byte aligned
};

// One unit of a row's output from its h values.
template <typename T, int V>
__device__ __forceinline__ void put_unit(const RmsArgs<T>& a, long long row, int c0, int lane, const float (&v)[4],
                                         float rstd) {
  float y[4], g[4];
  gammas<V>(g, a.gamma, c0, lane, a.cols, a.wide);
#pragma unroll
  for (int e = 0; e < 4; ++e)
    y[e] = c0 + Unit<T, V>::col(e, lane) < a.cols ? __fmul_rn(__fmul_rn(v[e], rstd), g[e]) : 0.f;
  if (a.y) {
    Unit<T, V> u;
    u.set(y);
    u.store(a.y + row * a.ldy, c0, lane, a.cols);
  }
  if (a.q) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) m = max(m, __float_as_uint(y[e]) & 0x7FFFFFFFu);
    m = __reduce_max_sync(0xffffffffu, m);
    const float s = scale_of(m), inv = __frcp_rn(s);
    if (lane == 0) a.scale[(long long)(c0 / UNIT) * a.rows + row] = s;
    uint8_t* q = a.q + row * a.ldq + c0;
    const uint32_t lo = e4m3x2(__fmul_rn(y[0], inv), __fmul_rn(y[1], inv));
    const uint32_t hi = e4m3x2(__fmul_rn(y[2], inv), __fmul_rn(y[3], inv));
    // ldq is a multiple of 16: a vector lies inside or outside
    if constexpr (V == 4) {
      if (c0 + 4 * lane < a.ldq) *reinterpret_cast<uint32_t*>(q + 4 * lane) = lo | hi << 16;
    } else if constexpr (V == 2) {
      if (c0 + 2 * lane < a.ldq) *reinterpret_cast<uint16_t*>(q + 2 * lane) = (uint16_t)lo;
      if (c0 + 64 + 2 * lane < a.ldq) *reinterpret_cast<uint16_t*>(q + 64 + 2 * lane) = (uint16_t)hi;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c0 + 32 * e + lane < a.ldq) q[32 * e + lane] = (uint8_t)((e < 2 ? lo : hi) >> 8 * (e & 1));
    }
  }
}

// NU units a warp, the row in registers.  blockDim: a row's warps, or with one
// warp a row, several rows.
template <typename T, int V, int NU>
__global__ void __launch_bounds__(kMaxWarps * 32) k_rms(const RmsArgs<T> a) {
  __shared__ float part[kMaxWarps];
  ptx::griddep_wait();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int warp = a.warps == 1 ? 0 : w;
  const long long row = a.warps == 1 ? (long long)blockIdx.x * (blockDim.x >> 5) + w : blockIdx.x;
  if (row >= a.rows) return;
  Unit<T, V> u[NU];
  const int c0 = warp * NU * UNIT;
#pragma unroll
  for (int i = 0; i < NU; ++i) u[i].load(a.x + row * a.ldx, c0 + i * UNIT, lane, a.cols);
  if (a.r) {
    Unit<T, V> t[NU];
#pragma unroll
    for (int i = 0; i < NU; ++i) t[i].load(a.r + row * a.ldr, c0 + i * UNIT, lane, a.cols);
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      float v[4], s[4];
      u[i].values(v);
      t[i].values(s);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += s[e];
      u[i].set(v);
      u[i].store(a.h + row * a.ldh, c0 + i * UNIT, lane, a.cols);
    }
  }
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    float v[4];
    u[i].values(v);
    ss += (v[0] * v[0] + v[1] * v[1]) + (v[2] * v[2] + v[3] * v[3]);
  }
  ss = row_sum(ss, a.warps, warp, lane, part);
  const float rstd = __frsqrt_rn(__fdiv_rn(ss, (float)a.cols) + a.eps);
  if (a.rstd && warp == 0 && lane == 0) a.rstd[row] = rstd;
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    if (c0 + i * UNIT >= a.cols) break;
    float v[4];
    u[i].values(v);
    put_unit<T, V>(a, row, c0 + i * UNIT, lane, v, rstd);
  }
}

// Rows too long for registers: read twice (the second time h, which is in L2).
template <typename T, int V>
__global__ void __launch_bounds__(kMaxWarps * 32) k_rms_long(const RmsArgs<T> a) {
  __shared__ float part[kMaxWarps];
  ptx::griddep_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long row = blockIdx.x;
  float ss = 0.f;
  for (long long c = (long long)warp * UNIT; c < a.cols; c += kMaxWarps * UNIT) {
    Unit<T, V> u, t;
    float v[4], s[4];
    u.load(a.x + row * a.ldx, (int)c, lane, a.cols);
    u.values(v);
    if (a.r) {
      t.load(a.r + row * a.ldr, (int)c, lane, a.cols);
      t.values(s);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += s[e];
      u.set(v);
      u.store(a.h + row * a.ldh, (int)c, lane, a.cols);
      u.values(v);
    }
    ss += (v[0] * v[0] + v[1] * v[1]) + (v[2] * v[2] + v[3] * v[3]);
  }
  ss = row_sum(ss, kMaxWarps, warp, lane, part);
  const float rstd = __frsqrt_rn(__fdiv_rn(ss, (float)a.cols) + a.eps);
  if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
  const T* h = a.r ? a.h + row * a.ldh : a.x + row * a.ldx;  // each thread reads what it wrote itself
  for (long long c = (long long)warp * UNIT; c < a.cols; c += kMaxWarps * UNIT) {
    Unit<T, V> u;
    float v[4];
    u.load(h, (int)c, lane, a.cols);
    u.values(v);
    put_unit<T, V>(a, row, (int)c, lane, v, rstd);
  }
}

// -------------------------------------------------------------- gradient
template <typename T>
struct GradArgs {
  const T *dy, *h, *dh;
  T* dx;
  const float *rstd, *gamma;
  float* part;  // [gridDim.x, cols] sums of dgamma, or null
  long long lddy, ldh, lddh, lddx;
  int rows, cols, warps;
  bool wide;
};

// Rows blockIdx.x + i gridDim.x; each lane keeps its columns' sums of dgamma in
// registers over the block's rows, so that dy and h are read once.  With one
// warp a row the block's warps take rows of their own and join their sums in
// shared memory ([warps][cols]).
template <typename T, int V, int NU>
__global__ void __launch_bounds__(kMaxWarps * 32) k_rms_grad(const GradArgs<T> a) {
  extern __shared__ float joined[];
  __shared__ float part[2][kMaxWarps];
  ptx::griddep_wait();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const bool own = a.warps == 1;  // a warp a row
  const int warp = own ? 0 : w, team = own ? w : 0, teams = own ? blockDim.x >> 5 : 1;
  const int c0 = warp * NU * UNIT;
  float acc[NU][4];
#pragma unroll
  for (int i = 0; i < NU; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[i][e] = 0.f;
  int turn = 0;
  for (long long row = (long long)blockIdx.x * teams + team; row < a.rows; row += (long long)gridDim.x * teams, turn ^= 1) {
    Unit<T, V> h[NU], d[NU];
    const float rstd = __ldg(a.rstd + row);
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      h[i].load(a.h + row * a.ldh, c0 + i * UNIT, lane, a.cols);
      d[i].load(a.dy + row * a.lddy, c0 + i * UNIT, lane, a.cols);
    }
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      float x[4], y[4], g[4];
      h[i].values(x);
      d[i].values(y);
      gammas<V>(g, a.gamma, c0 + i * UNIT, lane, a.cols, a.wide);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float yn = y[e] * (x[e] * rstd);
        acc[i][e] += yn;
        dot += yn * g[e];
      }
    }
    dot = row_sum(dot, a.warps, warp, lane, part[turn]) / (float)a.cols;
    if (!a.dx) continue;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      if (c0 + i * UNIT >= a.cols) break;
      float x[4], y[4], g[4];
      h[i].values(x);
      d[i].values(y);
      gammas<V>(g, a.gamma, c0 + i * UNIT, lane, a.cols, a.wide);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = rstd * (g[e] * y[e] - (x[e] * rstd) * dot);
      if (a.dh) {
        Unit<T, V> t;
        t.load(a.dh + row * a.lddh, c0 + i * UNIT, lane, a.cols);
        t.values(y);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += y[e];
      }
      Unit<T, V> o;
      o.set(x);
      o.store(a.dx + row * a.lddx, c0 + i * UNIT, lane, a.cols);
    }
  }
  if (!a.part) return;
  float* out = a.part + (long long)blockIdx.x * a.cols;
  if (teams == 1) {
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = c0 + i * UNIT + Unit<T, V>::col(e, lane);
        if (c < a.cols) out[c] = acc[i][e];
      }
    return;
  }
#pragma unroll
  for (int i = 0; i < NU; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = i * UNIT + Unit<T, V>::col(e, lane);
      if (c < a.cols) joined[team * a.cols + c] = acc[i][e];
    }
  __syncthreads();
  for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
    float s = joined[c];
    for (int t = 1; t < teams; ++t) s += joined[t * a.cols + c];
    out[c] = s;
  }
}

// Rows too long for registers, in two passes: <du n> of each row, then its
// terms by strips of 32 x UNIT columns.
template <typename T, int V>
__global__ void __launch_bounds__(kMaxWarps * 32) k_rms_dot(const GradArgs<T> a, float* dots) {
  __shared__ float part[kMaxWarps];
  ptx::griddep_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long row = blockIdx.x;
  const float rstd = __ldg(a.rstd + row);
  float dot = 0.f;
  for (long long c = (long long)warp * UNIT; c < a.cols; c += kMaxWarps * UNIT) {
    Unit<T, V> h, d;
    float x[4], y[4], g[4];
    h.load(a.h + row * a.ldh, (int)c, lane, a.cols);
    d.load(a.dy + row * a.lddy, (int)c, lane, a.cols);
    h.values(x);
    d.values(y);
    gammas<V>(g, a.gamma, (int)c, lane, a.cols, a.wide);
#pragma unroll
    for (int e = 0; e < 4; ++e) dot += y[e] * (x[e] * rstd) * g[e];
  }
  dot = row_sum(dot, kMaxWarps, warp, lane, part);
  if (threadIdx.x == 0) dots[row] = dot / (float)a.cols;
}
// Block (strip, rows blockIdx.y + i gridDim.y): a warp a unit.
template <typename T, int V>
__global__ void __launch_bounds__(8 * 32) k_rms_strip(const GradArgs<T> a, const float* dots) {
  ptx::griddep_wait();
  const int lane = threadIdx.x & 31;
  const long long c = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * UNIT;
  if (c >= a.cols) return;
  float g[4], acc[4] = {0.f, 0.f, 0.f, 0.f};
  gammas<V>(g, a.gamma, (int)c, lane, a.cols, a.wide);
#pragma unroll 4
  for (long long row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const float rstd = __ldg(a.rstd + row), dot = dots ? dots[row] : 0.f;
    Unit<T, V> h, d;
    float x[4], y[4];
    h.load(a.h + row * a.ldh, (int)c, lane, a.cols);
    d.load(a.dy + row * a.lddy, (int)c, lane, a.cols);
    h.values(x);
    d.values(y);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float n = x[e] * rstd;
      acc[e] += y[e] * n;
      x[e] = rstd * (g[e] * y[e] - n * dot);
    }
    if (!a.dx) continue;
    if (a.dh) {
      d.load(a.dh + row * a.lddh, (int)c, lane, a.cols);
      d.values(y);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] += y[e];
    }
    h.set(x);
    h.store(a.dx + row * a.lddx, (int)c, lane, a.cols);
  }
  if (a.part) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int k = (int)c + Unit<T, V>::col(e, lane);
      if (k < a.cols) a.part[(long long)blockIdx.y * a.cols + k] = acc[e];
    }
  }
}

// dgamma[c] = sum of `rows` partial sums, 32 columns a block: 32 threads a
// column add up every 32nd, and then each other's, in a fixed order.
__global__ void __launch_bounds__(1024) k_rms_fold(const float* part, int rows, int cols, float* out) {
  __shared__ float s[32][33];
  ptx::griddep_wait();
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const long long c = (long long)blockIdx.x * 32 + tx;
  float v = 0.f;
  if (c < cols)
    for (int r = ty; r < rows; r += 32) v += part[(long long)r * cols + c];
  s[tx][ty] = v;
  __syncthreads();
  v = s[ty][tx];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  const long long k = (long long)blockIdx.x * 32 + ty;
  if (tx == 0 && k < cols) out[k] = v;
}

// ------------------------------------------------------------------ host
// Units per warp of the row kernels: the most (fewest barriers, most loads in
// flight a thread) that still give the GPU 16 warps an SM, else the fewest
// (2432 = 152 x 16; 0: the row does not fit `most` units a warp).
int units_per_warp(long long rows, int cols, int most) {
  const int units = cdiv(cols, UNIT);
  if (cdiv(units, most) > kMaxWarps) return 0;
  for (int nu = most; nu > 1; nu /= 2) {
    if (rows * cdiv(units, nu) >= 2432) return nu;
    if (cdiv(units, nu / 2) > kMaxWarps) return nu;
  }
  return 1;
}
constexpr int kOwnRows = 8;      // rows a block with one warp a row
constexpr int kGradRows = 128;   // rows whose terms of dgamma one thread adds up in a row
constexpr int kFwdUnits = 8, kGradUnits = 4;

// The vector that every array's rows are aligned for.
template <typename T, typename... P>
int vector_of(const P&... p) {
  auto all = [&](int bytes) { return ((!p.first || rows_aligned(p.first, p.second, sizeof(T), bytes)) && ...); };
  if (all(4 * (int)sizeof(T))) return 4;
  return sizeof(T) == 2 && all(4) ? 2 : 1;
}
template <typename T, typename F>
auto with_vector(int v, F f) {
  if (v == 4) return f(std::integral_constant<int, 4>{});
  if constexpr (sizeof(T) == 2)
    if (v == 2) return f(std::integral_constant<int, 2>{});
  return f(std::integral_constant<int, 1>{});
}
bool wide_of(const float* gamma) { return reinterpret_cast<uintptr_t>(gamma) % 16 == 0; }

template <typename T>
ff_status rms_t(RmsArgs<T> a, cudaStream_t st) {
  using P = std::pair<const void*, long long>;
  const int v = vector_of<T>(P{a.x, a.ldx}, P{a.r, a.ldr}, P{a.h, a.ldh}, P{a.y, a.ldy});
  const int nu = units_per_warp(a.rows, a.cols, kFwdUnits);
  const double bytes = (double)a.rows * a.cols * (sizeof(T) * (1 + (a.r ? 2 : 0) + (a.y ? 1 : 0)) + (a.q ? 1 : 0));
  a.wide = wide_of(a.gamma);
  auto go = [&]() -> cudaError_t {
    return with_vector<T>(v, [&](auto V) {
      if (nu == 0) {
        PdlLaunch l(dim3((unsigned)a.rows), dim3(kMaxWarps * 32), st);
        return cudaLaunchKernelEx(&l.cfg, k_rms_long<T, V.value>, a);
      }
      a.warps = cdiv(cdiv(a.cols, UNIT), nu);
      PdlLaunch l(dim3((unsigned)(a.warps == 1 ? cdiv(a.rows, kOwnRows) : a.rows)),
                  dim3((unsigned)(a.warps == 1 ? kOwnRows : a.warps) * 32), st);
      switch (nu) {
        case 1: return cudaLaunchKernelEx(&l.cfg, k_rms<T, V.value, 1>, a);
        case 2: return cudaLaunchKernelEx(&l.cfg, k_rms<T, V.value, 2>, a);
        case 4: return cudaLaunchKernelEx(&l.cfg, k_rms<T, V.value, 4>, a);
        default: return cudaLaunchKernelEx(&l.cfg, k_rms<T, V.value, 8>, a);
      }
    });
  };
  FF_LAUNCH(K_RMS, bytes, st, go(), "RMS norm");
  return FF_OK;
}

// Blocks of the gradient kernels along the rows: about two rounds' worth of
// warps for the GPU, and at most kGradRows rows a thread.
struct GradPlan {
  int nu, warps, teams, blocks;
};
GradPlan grad_plan(int rows, int cols) {
  GradPlan p{};
  p.nu = units_per_warp(rows, cols, kGradUnits);
  const int units = cdiv(cols, UNIT);
  p.warps = p.nu ? cdiv(units, p.nu) : kMaxWarps;
  p.teams = p.nu && p.warps == 1 ? kOwnRows : 1;
  const long long per = p.nu ? (long long)p.warps * p.teams : units;  // warps along the columns
  const long long fill = 152ll * 32 / per < 1 ? 1 : 152ll * 32 / per;
  const long long sets = cdiv(rows, p.teams), least = cdiv(sets, kGradRows);
  p.blocks = (int)(sets < fill ? sets : fill < least ? least : fill);
  if (!p.nu && p.blocks > 65535) p.blocks = 65535;
  return p;
}
long long grad_bytes(int rows, int cols) {
  const GradPlan p = grad_plan(rows, cols);
  const long long part = p.blocks > 1 ? 4ll * p.blocks * cols : 0;
  return ((part + 15) & ~15ll) + (p.nu ? 0 : 4ll * rows);
}

template <typename T>
ff_status rms_grad_t(GradArgs<T> a, float* dgamma, void* ws, cudaStream_t st) {
  using P = std::pair<const void*, long long>;
  const int v = vector_of<T>(P{a.dy, a.lddy}, P{a.h, a.ldh}, P{a.dh, a.lddh}, P{a.dx, a.lddx});
  const GradPlan p = grad_plan(a.rows, a.cols);
  a.warps = p.warps;
  a.wide = wide_of(a.gamma);
  a.part = !dgamma ? nullptr : p.blocks > 1 ? static_cast<float*>(ws) : dgamma;
  const double count = (double)a.rows * a.cols;
  const double bytes = count * sizeof(T) * (2 + (a.dx ? 1 : 0) + (a.dh ? 1 : 0));
  if (p.nu) {
    auto go = [&]() -> cudaError_t {
      return with_vector<T>(v, [&](auto V) {
        const size_t smem = p.teams > 1 && a.part ? (size_t)p.teams * a.cols * 4 : 0;
        PdlLaunch l(dim3((unsigned)p.blocks), dim3((unsigned)(p.teams > 1 ? p.teams : p.warps) * 32), st, smem);
        switch (p.nu) {
          case 1: return cudaLaunchKernelEx(&l.cfg, k_rms_grad<T, V.value, 1>, a);
          case 2: return cudaLaunchKernelEx(&l.cfg, k_rms_grad<T, V.value, 2>, a);
          default: return cudaLaunchKernelEx(&l.cfg, k_rms_grad<T, V.value, 4>, a);
        }
      });
    };
    FF_LAUNCH(K_RMS_GRAD, bytes, st, go(), "RMS norm gradient");
  } else {
    const long long part = p.blocks > 1 ? 4ll * p.blocks * a.cols : 0;
    float* dots = reinterpret_cast<float*>(static_cast<char*>(ws) + ((part + 15) & ~15ll));
    if (a.dx) {
      auto dot = [&]() -> cudaError_t {
        return with_vector<T>(v, [&](auto V) {
          PdlLaunch l(dim3((unsigned)a.rows), dim3(kMaxWarps * 32), st);
          return cudaLaunchKernelEx(&l.cfg, k_rms_dot<T, V.value>, a, dots);
        });
      };
      FF_LAUNCH(K_RMS_GRAD, 2 * count * sizeof(T), st, dot(), "RMS norm gradient");
    }
    auto strip = [&]() -> cudaError_t {
      return with_vector<T>(v, [&](auto V) {
        PdlLaunch l(dim3((unsigned)cdiv(cdiv(a.cols, UNIT), 8), (unsigned)p.blocks), dim3(8 * 32), st);
        return cudaLaunchKernelEx(&l.cfg, k_rms_strip<T, V.value>, a, (const float*)(a.dx ? dots : nullptr));
      });
    };
    FF_LAUNCH(K_RMS_GRAD, bytes, st, strip(), "RMS norm gradient");
  }
  if (dgamma && p.blocks > 1) {
    PdlLaunch l(dim3((unsigned)cdiv(a.cols, 32)), dim3(1024), st);
    FF_LAUNCH(K_RMS_GRAD, 4.0 * p.blocks * a.cols, st,
              cudaLaunchKernelEx(&l.cfg, k_rms_fold, (const float*)a.part, p.blocks, a.cols, dgamma), "RMS norm gradient");
  }
  return FF_OK;
}

bool aligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
// A matrix argument: there (or null and not needed), aligned for its type, rows apart.
bool matrix_ok(const void* p, long long ld, int rows, int cols, int es) {
  return !p || (aligned(p, es) && (ld >= cols || rows <= 1));
}

}  // namespace
}  // namespace ff

using namespace ff;

extern "C" FF_API ff_status ff_rms_norm(const void* x, long long ldx, const void* residual, long long ldr, int rows, int cols,
                                        const float* gamma, float eps, ff_precision prec, void* h, long long ldh, void* y,
                                        long long ldy, void* q, float* scale, float* rstd, void* stream) {
  if (rows < 0 || cols < 1 || cols > 0x7FFFFF00 || (prec != FF_FP32 && prec != FF_BF16) || !(eps > 0.f) || isinf(eps))
    return FF_ERR_INVALID_ARG;
  if (rows == 0) return FF_OK;
  const int es = prec == FF_BF16 ? 2 : 4;
  if (!x || (residual == nullptr) != (h == nullptr) || (q == nullptr) != (scale == nullptr) || (!y && !q) ||
      !matrix_ok(x, ldx, rows, cols, es) || !matrix_ok(residual, ldr, rows, cols, es) ||
      !matrix_ok(h, ldh, rows, cols, es) || !matrix_ok(y, ldy, rows, cols, es) || (y && y == h) || !aligned(q, 16) ||
      !aligned(scale, 4) || !aligned(gamma, 4) || !aligned(rstd, 4))
    return FF_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  auto run = [&](auto t) {
    using T = decltype(t);
    RmsArgs<T> a{};
    a.x = static_cast<const T*>(x);
    a.r = static_cast<const T*>(residual);
    a.h = static_cast<T*>(h);
    a.y = static_cast<T*>(y);
    a.q = static_cast<uint8_t*>(q);
    a.gamma = gamma;
    a.scale = scale;
    a.rstd = rstd;
    a.ldx = ldx;
    a.ldr = ldr;
    a.ldh = ldh;
    a.ldy = ldy;
    a.rows = rows;
    a.cols = cols;
    a.ldq = (cols + 15) & ~15;
    a.eps = eps;
    return rms_t(a, st);
  };
  return prec == FF_BF16 ? run(bf16{}) : run(float{});
}

extern "C" FF_API long long ff_rms_norm_workspace(int rows, int cols) {
  if (rows < 0 || cols < 1 || cols > 0x7FFFFF00) return -1;
  return rows == 0 ? 0 : grad_bytes(rows, cols);
}

extern "C" FF_API ff_status ff_rms_norm_backward(const void* dy, long long lddy, const void* h, long long ldh, int rows,
                                                 int cols, const float* rstd, const float* gamma, const void* dh,
                                                 long long lddh, ff_precision prec, void* dx, long long lddx,
                                                 float* dgamma, void* workspace, long long workspace_bytes, void* stream) {
  if (rows < 0 || cols < 1 || cols > 0x7FFFFF00 || (prec != FF_FP32 && prec != FF_BF16) || !aligned(dgamma, 4))
    return FF_ERR_INVALID_ARG;
  if (!dx && !dgamma) return FF_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (rows == 0) {
    if (dgamma) FF_TRY(cudaMemsetAsync(dgamma, 0, 4ull * cols, st), "RMS norm gradient");
    return FF_OK;
  }
  const int es = prec == FF_BF16 ? 2 : 4;
  const long long need = grad_bytes(rows, cols);
  if (!dy || !h || !rstd || !matrix_ok(dy, lddy, rows, cols, es) || !matrix_ok(h, ldh, rows, cols, es) ||
      !matrix_ok(dh, lddh, rows, cols, es) || !matrix_ok(dx, lddx, rows, cols, es) || !aligned(rstd, 4) ||
      !aligned(gamma, 4) || (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))))
    return FF_ERR_INVALID_ARG;
  auto run = [&](auto t) {
    using T = decltype(t);
    GradArgs<T> a{};
    a.dy = static_cast<const T*>(dy);
    a.h = static_cast<const T*>(h);
    a.dh = static_cast<const T*>(dh);
    a.dx = static_cast<T*>(dx);
    a.rstd = rstd;
    a.gamma = gamma;
    a.lddy = lddy;
    a.ldh = ldh;
    a.lddh = lddh;
    a.lddx = lddx;
    a.rows = rows;
    a.cols = cols;
    return rms_grad_t(a, dgamma, workspace, st);
  };
  return prec == FF_BF16 ? run(bf16{}) : run(float{});
}
