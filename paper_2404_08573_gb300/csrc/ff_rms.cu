// RMS norm with the residual's addition, its output rounded to the input's
// type or to e4m3 blocks, and its gradient:
//
//   h = x + residual, rstd = 1 / sqrt(mean h^2 + eps), y = gamma h rstd
//   du = gamma dy, n = h rstd, dx = rstd (du - n <du n>) + dh, dgamma = sum dy n
//
// A row is cut into units of 128 values, four to a lane, so that a warp holds
// whole e4m3 blocks; `warps` warps share a row.  The forward pass is bound by HBM:
// 16384 x 8192 bf16 with a residual to e4m3 138 us, at the copy rate; to bf16 155 us.
// Fewer instructions made it so (169 us before): sums and products on pairs of
// values, the residual added in bf16, one division a lane for all of a warp's
// scales.  A single row is a launch (1 x 2000: 2.1 us).  Rows that are aligned to
// single values only take 1.6 times as long (8000 x 4097 bf16 with a residual to
// e4m3: 55 us, floor 34).
#include <algorithm>
#include <type_traits>
#include <utility>

#include "ff_api_internal.h"
#include "ff_e4m3.cuh"
#include "ff_ptx.cuh"
#include "ff_vec.cuh"

namespace ff {
namespace {

constexpr int UNIT = 128;
constexpr int kMaxWarps = 32;
constexpr int kGradWarps = 16;  // of the gradient's row kernel

// A lane's four values of the unit at column c0, V of them consecutive: 16 or
// 8 bytes (V = 4), a pair of bf16 (V = 2), or one (V = 1, the lanes side by
// side), as the rows' alignment allows.  Held as loaded, bf16 in pairs.
template <typename T>
struct Held;
template <>
struct Held<float> {
  float w[4];
  __device__ __forceinline__ void pairs(uint64_t (&p)[2]) const {
    p[0] = ptx::pack2(w[0], w[1]);
    p[1] = ptx::pack2(w[2], w[3]);
  }
  __device__ __forceinline__ void set(const uint64_t (&p)[2]) {
    const float2 a = ptx::unpack2(p[0]), b = ptx::unpack2(p[1]);
    w[0] = a.x;
    w[1] = a.y;
    w[2] = b.x;
    w[3] = b.y;
  }
  __device__ __forceinline__ void add(const Held& o) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] += o.w[e];
  }
};
template <>
struct Held<bf16> {
  uint32_t w[2];
  __device__ __forceinline__ void pairs(uint64_t (&p)[2]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) p[i] = ptx::pack2(w[i] << 16, w[i] & 0xFFFF0000u);
  }
  __device__ __forceinline__ void set(const uint64_t (&p)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float2 f = ptx::unpack2(p[i]);
      const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
  }
  // One rounding, which is also that of an fp32 sum rounded once more: where
  // fp32 cannot hold the sum of two bf16 values exactly, one is below 2^-15 of the
  // other, and the sum far from halfway between two of them.
  __device__ __forceinline__ void add(const Held& o) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const __nv_bfloat162 h = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&w[i]), *reinterpret_cast<const __nv_bfloat162*>(&o.w[i]));
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
  }
};

template <typename T, int V>
struct Unit : Held<T> {
  static constexpr int N = 4 / V;  // accesses
  using Raw = typename Vec<T, V>::Raw;
  static __device__ __forceinline__ int first(int i, int lane) { return i * 32 * V + lane * V; }
  static __device__ __forceinline__ int col(int e, int lane) { return first(e / V, lane) + e % V; }
  __device__ __forceinline__ Raw* raw() { return reinterpret_cast<Raw*>(this->w); }
  __device__ __forceinline__ const Raw* raw() const { return reinterpret_cast<const Raw*>(this->w); }
  // (cols is a multiple of V: a vector lies inside the row or outside, where it
  // reads as zero; whole: the unit lies inside)
  __device__ __forceinline__ void load(const T* row, int c0, int lane, int cols, bool whole = false) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = c0 + first(i, lane);
      if (whole || c < cols)
        raw()[i] = Vec<T, V>::load(row + c);
      else
        memset(&raw()[i], 0, sizeof(Raw));
    }
  }
  __device__ __forceinline__ void store(T* row, int c0, int lane, int cols, bool whole = false) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = c0 + first(i, lane);
      if (whole || c < cols) *reinterpret_cast<Raw*>(row + c) = raw()[i];
    }
  }
};

// A lane's four gammas of the unit (null: ones); zero past the row.
template <int V>
__device__ __forceinline__ void gammas(uint64_t (&g)[2], const float* gamma, int c0, int lane, int cols, bool wide) {
  if (V == 4 && wide && gamma && c0 + lane * 4 < cols) {
    const float4 f = __ldg(reinterpret_cast<const float4*>(gamma + c0 + lane * 4));
    g[0] = ptx::pack2(f.x, f.y);
    g[1] = ptx::pack2(f.z, f.w);
    return;
  }
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int c = c0 + Unit<float, V>::col(e, lane);
    v[e] = c < cols ? (gamma ? __ldg(gamma + c) : 1.f) : 0.f;
  }
  g[0] = ptx::pack2(v[0], v[1]);
  g[1] = ptx::pack2(v[2], v[3]);
}
__device__ __forceinline__ uint64_t both(float v) { return ptx::pack2(v, v); }
__device__ __forceinline__ float sum_of(uint64_t v) {
  const float2 f = ptx::unpack2(v);
  return f.x + f.y;
}

// The warps of one row meet.  A named barrier, since warps come to it from either
// twin of the code below (a block-wide one has to be one place for all threads).
__device__ __forceinline__ void row_barrier(int warps) { ptx::named_bar(1, warps * 32); }

// The sum over a row's warps of v, in a fixed order, through part[kMaxWarps]
// (not used again before the row's warps have met once more), the same bits in
// every lane.
__device__ __forceinline__ float row_sum(float v, int warps, int warp, int lane, float* part) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (warps == 1) return v;
  if (lane == 0) part[warp] = v;
  row_barrier(warps);
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

// y of one unit from its h values.  (Past the row h and gamma are zero and so is
// y, but for a row with a NaN, which is NaN there too.)
template <typename T, int V>
__device__ __forceinline__ void outputs(const RmsArgs<T>& a, uint64_t (&y)[2], int c0, int lane, float rstd) {
  uint64_t g[2];
  gammas<V>(g, a.gamma, c0, lane, a.cols, a.wide);
#pragma unroll
  for (int i = 0; i < 2; ++i) y[i] = ptx::mul2(ptx::mul2(y[i], both(rstd)), g[i]);
}
// The bits of the largest magnitude over the warp (a NaN's above all others).
__device__ __forceinline__ uint32_t amax_of(const uint64_t (&y)[2]) {
  const float2 a = ptx::unpack2(y[0]), b = ptx::unpack2(y[1]);
  float m, n;
  asm("{\n\t.reg .f32 p, q;\n\tabs.f32 p, %1;\n\tabs.f32 q, %2;\n\tmax.NaN.f32 %0, p, q;\n\t}" : "=f"(m) : "f"(a.x), "f"(a.y));
  asm("{\n\t.reg .f32 p, q;\n\tabs.f32 p, %1;\n\tabs.f32 q, %2;\n\tmax.NaN.f32 %0, p, q;\n\t}" : "=f"(n) : "f"(b.x), "f"(b.y));
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(n));
  return __reduce_max_sync(0xffffffffu, __float_as_uint(m));
}
template <typename T, int V>
__device__ __forceinline__ void put_fp8(const RmsArgs<T>& a, long long row, const uint64_t (&y)[2], int c0, int lane, float inv,
                                        bool whole = false) {
  const float2 f = ptx::unpack2(ptx::mul2(y[0], both(inv))), g = ptx::unpack2(ptx::mul2(y[1], both(inv)));
  const uint32_t lo = e4m3x2(f.x, f.y), hi = e4m3x2(g.x, g.y);
  uint8_t* q = a.q + row * a.ldq + c0;
  // ldq is a multiple of 16: a vector lies inside or outside
  if constexpr (V == 4) {
    if (whole || c0 + 4 * lane < a.ldq) *reinterpret_cast<uint32_t*>(q + 4 * lane) = lo | hi << 16;
  } else if constexpr (V == 2) {
    if (whole || c0 + 2 * lane < a.ldq) *reinterpret_cast<uint16_t*>(q + 2 * lane) = (uint16_t)lo;
    if (whole || c0 + 64 + 2 * lane < a.ldq) *reinterpret_cast<uint16_t*>(q + 64 + 2 * lane) = (uint16_t)hi;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (whole || c0 + 32 * e + lane < a.ldq) q[32 * e + lane] = (uint8_t)((e < 2 ? lo : hi) >> 8 * (e & 1));
  }
}
__device__ __forceinline__ float rstd_of(float sum, int cols, float eps) { return __frsqrt_rn(__fdiv_rn(sum, (float)cols) + eps); }
// A row that is not held in registers: a warp reads its units at columns c0,
// c0 + step, .. before `end` (and before the row's) again.
struct Units {
  long long c0, end;
  int step;
};
template <typename T>
__device__ __forceinline__ const T* h_of(const RmsArgs<T>& a, long long row) {  // each thread reads what it wrote itself
  return a.r ? a.h + row * a.ldh : a.x + row * a.ldx;
}
// rstd from the squares of h 2^-80, for a row whose own squares' sum is past
// fp32's range: of no finite row theirs is, and all that vanishes in it does so
// beside a value of 2^64 / sqrt(cols) at least.
template <typename T, int V>
__device__ __forceinline__ float far_rstd(const RmsArgs<T>& a, long long row, Units at, int warps, int warp, int lane, float* part) {
  constexpr float by = 0x1p-80f;
  const T* h = h_of(a, row);
  uint64_t ss = 0;
#pragma unroll 1
  for (long long c = at.c0; c < at.end; c += at.step) {
    Unit<T, V> u;
    uint64_t v[2];
    u.load(h, (int)c, lane, a.cols);
    u.pairs(v);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint64_t w = ptx::mul2(v[e], both(by));
      ptx::fma2_to(ss, w, w);
    }
  }
  return rstd_of(row_sum(sum_of(ss), warps, warp, lane, part), a.cols, a.eps * by * by) * by;
}
template <typename T, int V>
__device__ __forceinline__ void outputs_from_memory(const RmsArgs<T>& a, long long row, Units at, int lane, float rstd) {
  const T* h = h_of(a, row);
  for (long long c = at.c0; c < at.end; c += at.step) {
    Unit<T, V> u;
    uint64_t y[2];
    u.load(h, (int)c, lane, a.cols);
    u.pairs(y);
    outputs<T, V>(a, y, (int)c, lane, rstd);
    if (a.q) {
      const float s = scale_of(amax_of(y));
      if (lane == 0) a.scale[c / UNIT * a.rows + row] = s;
      put_fp8<T, V>(a, row, y, (int)c, lane, __frcp_rn(s));
    }
    if (a.y) {
      u.set(y);
      u.store(a.y + row * a.ldy, (int)c, lane, a.cols);
    }
  }
}

// NU units a warp, the row in registers.  blockDim: a row's warps, or with one
// warp a row, several rows.  whole: all of the warp's units lie inside the row
// (without this twin the rows of single values, with four comparisons a unit,
// took half as long again).  Returns false, for all of the row's warps, where the
// squares are past fp32's range; rstd and outputs are then still to be written.
template <typename T, int V, int NU>
__device__ __forceinline__ bool rms_row(const RmsArgs<T>& a, long long row, int warp, int lane, float* part, bool whole) {
  Unit<T, V> u[NU];
  const int c0 = warp * NU * UNIT;
#pragma unroll
  for (int i = 0; i < NU; ++i) u[i].load(a.x + row * a.ldx, c0 + i * UNIT, lane, a.cols, whole);
  if (a.r) {
    Unit<T, V> t[NU];
#pragma unroll
    for (int i = 0; i < NU; ++i) t[i].load(a.r + row * a.ldr, c0 + i * UNIT, lane, a.cols, whole);
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      u[i].add(t[i]);
      u[i].store(a.h + row * a.ldh, c0 + i * UNIT, lane, a.cols, whole);
    }
  }
  uint64_t ss[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    uint64_t v[2];
    u[i].pairs(v);
    ptx::fma2_to(ss[0], v[0], v[0]);
    ptx::fma2_to(ss[1], v[1], v[1]);
  }
  const float sum = row_sum(sum_of(ptx::add2(ss[0], ss[1])), a.warps, warp, lane, part);
  if (sum == INFINITY) return false;
  const float rstd = rstd_of(sum, a.cols, a.eps);
  if (a.rstd && warp == 0 && lane == 0) a.rstd[row] = rstd;
  if (a.y) {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      uint64_t y[2];
      u[i].pairs(y);
      outputs<T, V>(a, y, c0 + i * UNIT, lane, rstd);
      Unit<T, V> o;
      o.set(y);
      o.store(a.y + row * a.ldy, c0 + i * UNIT, lane, a.cols, whole);
    }
  }
  if (a.q) {
    // The units' maxima first, so that lane i divides for unit i once.  (The
    // outputs are kept meanwhile; formed again, 4000 x 8192 took 29 us for 26.)
    uint64_t y[NU][2];
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      u[i].pairs(y[i]);
      outputs<T, V>(a, y[i], c0 + i * UNIT, lane, rstd);
      const uint32_t m = amax_of(y[i]);
      mine = lane == i ? m : mine;
    }
    const float s = scale_of(mine), inv = __frcp_rn(s);
    if (lane < NU && c0 + lane * UNIT < a.cols) a.scale[(long long)(c0 / UNIT + lane) * a.rows + row] = s;
#pragma unroll
    for (int i = 0; i < NU; ++i)
      put_fp8<T, V>(a, row, y[i], c0 + i * UNIT, lane, __shfl_sync(0xffffffffu, inv, i), whole);
  }
  return true;
}
// The rest of such a row, apart from the kernel's own code, whose registers it
// would take.  The arguments by reference to the kernel's own (a __grid_constant__)
// where units are whole vectors, else by value: the other way round, or with all of it
// in line, one or another of the kernels spills and takes 5 to 12 % longer
// (4096 x 8192 fp32 43.2 and 45.2 us; 8000 x 4097 fp32 with a residual 83.0 and 92.6).
template <typename T, int V>
using FarArgs = std::conditional_t<V == 4, const RmsArgs<T>&, const RmsArgs<T>>;
template <typename T, int V, int NU>
__device__ __noinline__ void far_row(FarArgs<T, V> a) {
  __shared__ float part[kMaxWarps];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int warp = a.warps == 1 ? 0 : w;
  const long long row = a.warps == 1 ? (long long)blockIdx.x * (blockDim.x >> 5) + w : blockIdx.x;
  const long long c0 = (long long)warp * NU * UNIT;
  const Units at{c0, min((long long)a.cols, c0 + NU * UNIT), UNIT};
  const float rstd = far_rstd<T, V>(a, row, at, a.warps, warp, lane, part);
  if (a.rstd && warp == 0 && lane == 0) a.rstd[row] = rstd;
  outputs_from_memory<T, V>(a, row, at, lane, rstd);
}
template <typename T, int V, int NU>
__device__ __forceinline__ void rms_rows(const RmsArgs<T>& a) {
  __shared__ float part[kMaxWarps];
  ptx::griddep_wait();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int warp = a.warps == 1 ? 0 : w;
  const long long row = a.warps == 1 ? (long long)blockIdx.x * (blockDim.x >> 5) + w : blockIdx.x;
  if (row >= a.rows) return;
  const bool done = (warp + 1) * NU * UNIT <= a.cols ? rms_row<T, V, NU>(a, row, warp, lane, part, true)
                                                    : rms_row<T, V, NU>(a, row, warp, lane, part, false);
  if (!done) far_row<T, V, NU>(a);
}
template <typename T, int NU>
__global__ void __launch_bounds__(kMaxWarps * 32) k_rms(const __grid_constant__ RmsArgs<T> a) {
  rms_rows<T, 4, NU>(a);
}
template <typename T, int V, int NU>
__global__ void __launch_bounds__(kMaxWarps * 32) k_rms_narrow(const RmsArgs<T> a) {
  rms_rows<T, V, NU>(a);
}

// Rows too long for registers: read twice (the second time h, which is in L2).
template <typename T, int V>
__global__ void __launch_bounds__(kMaxWarps * 32) k_rms_long(const RmsArgs<T> a) {
  __shared__ float part[2 * kMaxWarps];
  ptx::griddep_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long row = blockIdx.x;
  uint64_t ss[2] = {0, 0};
  for (long long c = (long long)warp * UNIT; c < a.cols; c += kMaxWarps * UNIT) {
    Unit<T, V> u, t;
    uint64_t v[2];
    u.load(a.x + row * a.ldx, (int)c, lane, a.cols);
    if (a.r) {
      t.load(a.r + row * a.ldr, (int)c, lane, a.cols);
      u.add(t);
      u.store(a.h + row * a.ldh, (int)c, lane, a.cols);
    }
    u.pairs(v);
    ptx::fma2_to(ss[0], v[0], v[0]);
    ptx::fma2_to(ss[1], v[1], v[1]);
  }
  const float sum = row_sum(sum_of(ptx::add2(ss[0], ss[1])), kMaxWarps, warp, lane, part);
  float rstd = rstd_of(sum, a.cols, a.eps);
  const Units at{(long long)warp * UNIT, a.cols, kMaxWarps * UNIT};
  if (sum == INFINITY) rstd = far_rstd<T, V>(a, row, at, kMaxWarps, warp, lane, part + kMaxWarps);
  if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
  outputs_from_memory<T, V>(a, row, at, lane, rstd);
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
  int depth;    // rows on their way
  float inv_cols;
  bool wide;
};

// How NU units of a row lie in the row and in shared memory.  V = 8 (bf16, NU
// even): units in twos of 2 x UNIT columns, a lane's eight values of which are one
// 16-byte copy, which goes past L1 (8-byte copies go through it, and L1 is what
// the slots leave: 16384 x 2000 60 us, so 49).  A lane reads back its own copies,
// but for single bf16 values (WORDS), which come as the 4-byte words that cover
// them, in the row's order, with half a word more at either end.
template <typename T, int V>
struct Lay {
  static constexpr bool WORDS = sizeof(T) * V < 4;
  static constexpr int P = V == 8 ? 2 : 1;  // units together
  static constexpr uint32_t PITCH = 32 * sizeof(Held<T>);               // bytes of a warp's unit
  static constexpr uint32_t LANE = WORDS ? 0 : P * sizeof(Held<T>);     // from a lane's slot to the next one's
  static __host__ __device__ constexpr uint32_t part(int nu) { return nu * PITCH + (WORDS ? 16 : 0); }  // of a warp's units
  static __device__ __forceinline__ int col(int i, int e, int lane) {   // of value e of unit i
    if constexpr (V == 8) return (i & ~1) * UNIT + lane * 8 + (i & 1) * 4 + e;
    else return i * UNIT + Unit<T, V>::col(e, lane);
  }
};
// Whether a row of bf16 values starts in the middle of a word.
__device__ __forceinline__ uint32_t odd_at(const void* p) { return (uint32_t)(reinterpret_cast<uintptr_t>(p) >> 1) & 1u; }

// Copies these by the bytes that the alignment allows.  A word before an odd row's
// first value belongs to the row before; matrix_start: there is none.
template <typename T, int V, int NU>
__device__ __forceinline__ void fetch(uint32_t slot, const T* row, int c0, int lane, int cols, bool whole, bool matrix_start) {
  using L = Lay<T, V>;
  if constexpr (!L::WORDS) {
    constexpr int BYTES = (int)sizeof(T) * V;
#pragma unroll
    for (int u = 0; u < NU; u += L::P)
#pragma unroll
      for (int i = 0; i < 4 * L::P / V; ++i) {
        const int c = c0 + L::col(u, i * V, lane);
        const bool in = whole || c < cols;
        ptx::cp_async_zfill<BYTES>(slot + u * L::PITCH + i * BYTES, row + (in ? c : 0), in ? BYTES : 0);
      }
  } else {
    const int odd = (int)odd_at(row);
    const char* from = reinterpret_cast<const char*>(row + c0 - odd);
    auto word = [&](int w, int most) {
      const int n = whole ? most : max(0, min(most, (cols - c0 + odd - 2 * w) * 2));
      ptx::cp_async_zfill<4>(slot + 4 * w, n > 0 ? from + 4 * w : reinterpret_cast<const char*>(row - odd), n);  // (of none: not read)
    };
#pragma unroll
    for (int i = 0; i < NU * 2; ++i) {
      if (i == 0 && odd && matrix_start && c0 == 0 && lane == 0) {
        const uint16_t v = Vec<T, 1>::load(row);
        asm volatile("st.shared.u16 [%0], %1;" ::"r"(slot + 2), "h"(v) : "memory");
        continue;
      }
      word(i * 32 + lane, 4);
    }
    if (odd && lane == 0) word(NU * 64, 2);
  }
}

// The units in a slot.
__device__ __forceinline__ void read_slot(Held<bf16> (&h)[1], uint32_t slot) {
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(h[0].w[0]), "=r"(h[0].w[1]) : "r"(slot));
}
__device__ __forceinline__ void read_slot(Held<bf16> (&h)[2], uint32_t slot) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(h[0].w[0]), "=r"(h[0].w[1]), "=r"(h[1].w[0]), "=r"(h[1].w[1])
               : "r"(slot));
}
__device__ __forceinline__ void read_slot(Held<float> (&h)[1], uint32_t slot) {
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(h[0].w[0]), "=f"(h[0].w[1]), "=f"(h[0].w[2]), "=f"(h[0].w[3])
               : "r"(slot));
}
// Unit i (and the next, if they lie together) of a warp's part.
template <typename T, int V, int P>
__device__ __forceinline__ void part_pairs(uint64_t (&p)[P][2], uint32_t slot, int i, uint32_t odd, int lane) {
  if constexpr (Lay<T, V>::WORDS) {
    uint32_t v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      asm volatile("{\n\t.reg .u16 h;\n\tld.shared.u16 h, [%1];\n\tcvt.u32.u16 %0, h;\n\t}"
                   : "=r"(v[e])
                   : "r"(slot + 2 * (odd + Lay<T, V>::col(i, e, lane))));
    p[0][0] = ptx::pack2(v[0] << 16, v[1] << 16);
    p[0][1] = ptx::pack2(v[2] << 16, v[3] << 16);
  } else {
    Held<T> h[P];
    read_slot(h, slot + i * Lay<T, V>::PITCH);
#pragma unroll
    for (int j = 0; j < P; ++j) h[j].pairs(p[j]);
  }
}

// The sums over a row's warps of R values (rows), in a fixed order, in every
// lane; of two, half a warp each.  `part` is [2][kMaxWarps], one of two that
// callers use in turn (one barrier a call).
template <int R>
__device__ __forceinline__ void row_sums(float (&v)[R], int warps, int warp, int lane, float (*part)[kMaxWarps]) {
  if constexpr (R == 1) {
    v[0] = row_sum(v[0], warps, warp, lane, part[0]);
  } else {
    const int r = lane >> 4, i = lane & 15;
    float s = (r ? v[1] : v[0]) + __shfl_xor_sync(0xffffffffu, r ? v[0] : v[1], 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (warps > 1) {
      if (i == 0) part[r][warp] = s;
      row_barrier(warps);
      s = i < warps ? part[r][i] : 0.f;
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    }
    v[0] = __shfl_sync(0xffffffffu, s, 0);
    v[1] = __shfl_sync(0xffffffffu, s, 16);
  }
}

// A block takes R rows at a time, sets of them gridDim.x apart; each lane keeps
// gamma and its columns' sums of dgamma in registers over all of them, so that
// dy and h are read once.  The rows to come are on their way into shared memory
// (`depth` sets, each thread its own values, so that no barrier is needed; of
// single bf16 values a warp's words, and a __syncwarp) while these are worked on.  With one warp a row the block's warps take rows of
// their own and join their sums in shared memory ([warps][cols]).
// h comes into products as n = h rstd (0.2 us of 47, bf16): dy h or rstd^2 may
// leave fp32's range where n, dy and dx do not.
// Bound by HBM in fp32 (4096 x 8192 with dh: 85 us, floor 80) and in bf16 by the
// latency of a set's two halves and the barrier between them (42 us and the fold's
// 5, floor 40).  (gamma read anew each time came from L2, since the copies take
// L1's place, and one row at a time pays the barrier for each: 60 us in all.)
template <typename T, int V, int NU, int R>
__device__ __forceinline__ void grad_rows(const GradArgs<T>& a, uint64_t (&acc)[NU][2], uint32_t slots, int teams, int team, int warp,
                                          int lane, float (*part)[2][kMaxWarps], bool whole) {
  const int c0 = warp * NU * UNIT;
  const long long first = ((long long)blockIdx.x * teams + team) * R, step = (long long)gridDim.x * teams * R;
  const T *hp = a.h + first * a.ldh, *dp = a.dy + first * a.lddy, *tp = a.dh ? a.dh + first * a.lddh : nullptr;
  using L = Lay<T, V>;
  constexpr uint32_t part1 = L::part(NU);
  constexpr int P = L::P;
  const uint32_t rb = (a.dh ? 3 : 2) * part1;  // of a row
  const uint32_t stage = R * rb * (blockDim.x >> 5);
  long long ahead = first;
  auto issue = [&](uint32_t to) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (ahead + r < a.rows) {
        fetch<T, V, NU>(to + r * rb, hp + r * a.ldh, c0, lane, a.cols, whole, ahead + r == 0);
        fetch<T, V, NU>(to + r * rb + part1, dp + r * a.lddy, c0, lane, a.cols, whole, ahead + r == 0);
        if (a.dh) fetch<T, V, NU>(to + r * rb + 2 * part1, tp + r * a.lddh, c0, lane, a.cols, whole, ahead + r == 0);
      }
    }
    hp += step * a.ldh;
    dp += step * a.lddy;
    if (a.dh) tp += step * a.lddh;
    ahead += step;
    ptx::cp_async_commit();
  };
  for (int d = 0; d < a.depth; ++d) issue(slots + d * stage);
  auto odd = [](const T* m, long long ld, long long row) { return L::WORDS ? odd_at(m + row * ld) : 0u; };
  uint64_t g[NU][2];
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    if constexpr (V == 8) gammas<4>(g[i], a.gamma, c0 + L::col(i, 0, lane) - lane * 4, lane, a.cols, a.wide);
    else gammas<V>(g[i], a.gamma, c0 + i * UNIT, lane, a.cols, a.wide);
  }
  T* out = a.dx ? a.dx + first * a.lddx : nullptr;
  int turn = 0, at = 0;
  float coming[R];  // the next set's rstd, so that its load is not waited for either (4096 x 8192: 2 us)
  auto rstds = [&](float (&to)[R], long long row) {
#pragma unroll
    for (int r = 0; r < R; ++r) to[r] = row + r < a.rows ? __ldg(a.rstd + row + r) : 0.f;
  };
  constexpr bool AHEAD = !L::WORDS;  // (those have no registers for it)
  if constexpr (AHEAD) rstds(coming, first);
  for (long long row = first; row < a.rows; row += step, turn ^= 1) {
    float rstd[R], dot[R];
    if constexpr (AHEAD) {
#pragma unroll
      for (int r = 0; r < R; ++r) rstd[r] = coming[r];
      rstds(coming, row + step);
    } else {
      rstds(rstd, row);
    }
    if (a.depth >= 4) ptx::cp_async_wait<3>();
    else if (a.depth == 3) ptx::cp_async_wait<2>();
    else if (a.depth == 2) ptx::cp_async_wait<1>();
    else ptx::cp_async_wait<0>();
    if constexpr (L::WORDS) __syncwarp();  // the other lanes' copies too
    const uint32_t now = slots + at * stage;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      uint64_t dot2 = 0;
      if (row + r < a.rows) {
#pragma unroll
        for (int i = 0; i < NU; i += P) {
          uint64_t x[P][2], y[P][2];
          part_pairs<T, V>(x, now + r * rb, i, odd(a.h, a.ldh, row + r), lane);
          part_pairs<T, V>(y, now + r * rb + part1, i, odd(a.dy, a.lddy, row + r), lane);
#pragma unroll
          for (int j = 0; j < P; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint64_t yn = ptx::mul2(y[j][e], ptx::mul2(x[j][e], both(rstd[r])));
              acc[i + j][e] = ptx::add2(acc[i + j][e], yn);
              ptx::fma2_to(dot2, yn, g[i + j][e]);
            }
        }
      }
      dot[r] = sum_of(dot2);
    }
    row_sums<R>(dot, a.warps, warp, lane, part[turn]);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (row + r >= a.rows || !out) break;
      const uint64_t off = both(-dot[r] * a.inv_cols * rstd[r]), by = both(rstd[r]);  // -<du n> rstd
#pragma unroll
      for (int i = 0; i < NU; i += P) {
        if (!whole && c0 + i * UNIT >= a.cols) break;
        uint64_t x[P][2], y[P][2];
        part_pairs<T, V>(x, now + r * rb, i, odd(a.h, a.ldh, row + r), lane);
        part_pairs<T, V>(y, now + r * rb + part1, i, odd(a.dy, a.lddy, row + r), lane);
#pragma unroll
        for (int j = 0; j < P; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            x[j][e] = ptx::mul2(by, ptx::fma2(x[j][e], off, ptx::mul2(g[i + j][e], y[j][e])));
        if (a.dh) {
          part_pairs<T, V>(y, now + r * rb + 2 * part1, i, odd(a.dh, a.lddh, row + r), lane);
#pragma unroll
          for (int j = 0; j < P; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) x[j][e] = ptx::add2(x[j][e], y[j][e]);
        }
        if constexpr (V == 8) {
          Held<T> o[2];
          o[0].set(x[0]);
          o[1].set(x[1]);
          const int c = c0 + L::col(i, 0, lane);
          if (whole || c < a.cols)
            *reinterpret_cast<uint4*>(out + r * a.lddx + c) = make_uint4(o[0].w[0], o[0].w[1], o[1].w[0], o[1].w[1]);
        } else {
          Unit<T, V> o;
          o.set(x[0]);
          o.store(out + r * a.lddx, c0 + i * UNIT, lane, a.cols, whole);
        }
      }
    }
    if (out) out += step * a.lddx;
    if constexpr (L::WORDS) __syncwarp();
    issue(now);  // into the slots just read
    if (++at == a.depth) at = 0;
  }
}
template <typename T, int V, int NU, int R>
__global__ void __launch_bounds__(kGradWarps * 32) k_rms_grad(const GradArgs<T> a) {
  extern __shared__ __align__(16) uint8_t dyn[];
  __shared__ float part[2][2][kMaxWarps];
  ptx::griddep_wait();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const bool own = a.warps == 1;  // a warp a row
  const int warp = own ? 0 : w, team = own ? w : 0, teams = own ? blockDim.x >> 5 : 1;
  const int c0 = warp * NU * UNIT;
  uint64_t acc[NU][2];
#pragma unroll
  for (int i = 0; i < NU; ++i) acc[i][0] = acc[i][1] = 0;
  const uint32_t slots = ptx::smem_u32(dyn) + (uint32_t)(w * R * (a.dh ? 3 : 2)) * Lay<T, V>::part(NU) + lane * Lay<T, V>::LANE;
  if (c0 + NU * UNIT <= a.cols)
    grad_rows<T, V, NU, R>(a, acc, slots, teams, team, warp, lane, part, true);
  else
    grad_rows<T, V, NU, R>(a, acc, slots, teams, team, warp, lane, part, false);
  ptx::griddep_launch_dependents();  // the fold's blocks may take their places
  if (!a.part) return;
  float* out = a.part + (long long)blockIdx.x * a.cols;
  float* joined = reinterpret_cast<float*>(dyn);
  if (teams > 1) __syncthreads();  // every warp is done with its slots
  float* const to = teams > 1 ? joined + team * a.cols : out;
  const bool wide = reinterpret_cast<uintptr_t>(to) % 16 == 0;  // (dgamma itself may not be)
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const float2 f[2] = {ptx::unpack2(acc[i][0]), ptx::unpack2(acc[i][1])};
    if constexpr (V >= 4) {
      // (single values here, 16 or 32 bytes apart, cost 3 us of 50 at 4096 x 8192)
      const int c = c0 + Lay<T, V>::col(i, 0, lane);
      if (wide && c < a.cols) {
        *reinterpret_cast<float4*>(to + c) = make_float4(f[0].x, f[0].y, f[1].x, f[1].y);
        continue;
      }
    }
    const float v[4] = {f[0].x, f[0].y, f[1].x, f[1].y};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = c0 + Lay<T, V>::col(i, e, lane);
      if (c < a.cols) to[c] = v[e];
    }
  }
  if (teams == 1) return;
  __syncthreads();
  for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
    float s = joined[c];
    for (int t = 1; t < teams; ++t) s += joined[t * a.cols + c];
    out[c] = s;
  }
}

// Rows too long for registers, in two passes: <du n> of each row, then its
// terms by strips of 8 x UNIT columns.
template <typename T, int V>
__global__ void __launch_bounds__(kMaxWarps * 32) k_rms_dot(const GradArgs<T> a, float* dots) {
  __shared__ float part[kMaxWarps];
  ptx::griddep_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long row = blockIdx.x;
  const float rstd = __ldg(a.rstd + row);
  uint64_t dot = 0;
  for (long long at = (long long)warp * UNIT; at < a.cols; at += 4 * kMaxWarps * UNIT) {
    Unit<T, V> h[4], d[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const long long c = at + j * (kMaxWarps * UNIT);
      if (c < a.cols) {
        h[j].load(a.h + row * a.ldh, (int)c, lane, a.cols);
        d[j].load(a.dy + row * a.lddy, (int)c, lane, a.cols);
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const long long c = at + j * (kMaxWarps * UNIT);
      if (c >= a.cols) break;
      uint64_t x[2], y[2], g[2];
      h[j].pairs(x);
      d[j].pairs(y);
      gammas<V>(g, a.gamma, (int)c, lane, a.cols, a.wide);
#pragma unroll
      for (int e = 0; e < 2; ++e) ptx::fma2_to(dot, ptx::mul2(y[e], ptx::mul2(x[e], both(rstd))), g[e]);
    }
  }
  const float sum = row_sum(sum_of(dot), kMaxWarps, warp, lane, part);
  if (threadIdx.x == 0) dots[row] = sum / (float)a.cols;
}
// Block (strip, rows blockIdx.y + i gridDim.y): a warp a unit.  Four such blocks an SM
// in bf16 (2000 x 32768: 148 us in all, three 175, two 158), three in fp32.
constexpr int strip_blocks(int esize) { return esize == 2 ? 4 : 3; }
template <typename T, int V>
__global__ void __launch_bounds__(8 * 32, strip_blocks(sizeof(T))) k_rms_strip(const GradArgs<T> a, const float* dots) {
  ptx::griddep_wait();
  const int lane = threadIdx.x & 31;
  const long long c = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * UNIT;
  if (c >= a.cols) return;
  uint64_t g[2], acc[2] = {0, 0};
  gammas<V>(g, a.gamma, (int)c, lane, a.cols, a.wide);
  for (long long row0 = blockIdx.y; row0 < a.rows; row0 += 4ll * gridDim.y) {
    Unit<T, V> h[4], d[4], t[4];  // four rows' loads together
    float rstd[4], dot[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const long long row = row0 + (long long)j * gridDim.y;
      if (row < a.rows) {
        h[j].load(a.h + row * a.ldh, (int)c, lane, a.cols);
        d[j].load(a.dy + row * a.lddy, (int)c, lane, a.cols);
        if (a.dh) t[j].load(a.dh + row * a.lddh, (int)c, lane, a.cols);
        rstd[j] = __ldg(a.rstd + row);
        dot[j] = dots ? dots[row] : 0.f;
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const long long row = row0 + (long long)j * gridDim.y;
      if (row >= a.rows) break;
      uint64_t x[2], y[2];
      h[j].pairs(x);
      d[j].pairs(y);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint64_t n = ptx::mul2(x[e], both(rstd[j]));
        ptx::fma2_to(acc[e], y[e], n);
        x[e] = ptx::mul2(both(rstd[j]), ptx::fma2(n, both(-dot[j]), ptx::mul2(g[e], y[e])));
      }
      if (!a.dx) continue;
      if (a.dh) {
        t[j].pairs(y);
#pragma unroll
        for (int e = 0; e < 2; ++e) x[e] = ptx::add2(x[e], y[e]);
      }
      Unit<T, V> o;
      o.set(x);
      o.store(a.dx + row * a.lddx, (int)c, lane, a.cols);
    }
  }
  if (a.part) {
    const float2 f[2] = {ptx::unpack2(acc[0]), ptx::unpack2(acc[1])};
    const float v[4] = {f[0].x, f[0].y, f[1].x, f[1].y};
    float* const to = a.part + (long long)blockIdx.y * a.cols;
    if (V == 4 && reinterpret_cast<uintptr_t>(to) % 16 == 0) {
      const int k = (int)c + Unit<T, V>::col(0, lane);
      if (k < a.cols) *reinterpret_cast<float4*>(to + k) = make_float4(v[0], v[1], v[2], v[3]);
      return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int k = (int)c + Unit<T, V>::col(e, lane);
      if (k < a.cols) to[k] = v[e];
    }
  }
}

// dgamma[c] = sum of `rows` partial sums, W columns a block: 1024 / W threads a
// column add up every (1024 / W)th, and then each other's, in a fixed order.
template <int W>
__global__ void __launch_bounds__(1024) k_rms_fold(const float* part, int rows, int cols, float* out) {
  constexpr int G = 1024 / W, AHEAD = 4;
  __shared__ float s[32][W + 1];
  ptx::griddep_wait();
  const int tx = threadIdx.x % W, ty = threadIdx.x / W, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long c = (long long)blockIdx.x * W + tx;
  float v = 0.f;
  if (c < cols)
    for (int r = ty; r < rows; r += AHEAD * G) {
      float t[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) t[i] = r + i * G < rows ? part[(long long)(r + i * G) * cols + c] : 0.f;
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) v += t[i];
    }
#pragma unroll
  for (int o = 16; o >= W; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (lane < W) s[warp][lane] = v;
  __syncthreads();
  if (warp >= W) return;
  v = s[lane][warp];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  const long long k = (long long)blockIdx.x * W + warp;
  if (lane == 0 && k < cols) out[k] = v;
}

// ------------------------------------------------------------------ host
// Units per warp of the row kernels: the most (fewest barriers, most loads in
// flight a thread) that still give the GPU 16 warps an SM, else the fewest
// (2432 = 152 x 16; 0: the row does not fit `most` units a warp).
int units_per_warp(long long rows, int cols, int most, int warps) {
  const int units = cdiv(cols, UNIT);
  if (cdiv(units, most) > warps) return 0;
  while (most > 1 && most / 2 >= units) most /= 2;
  for (int nu = most; nu > 1; nu /= 2) {
    if (rows * cdiv(units, nu) >= 2432) return nu;
    if (cdiv(units, nu / 2) > warps) return nu;
  }
  return 1;
}
constexpr int kOwnRows = 8;      // rows a block with one warp a row
constexpr int kGradRows = 128;   // rows whose terms of dgamma one thread adds up in a row

// The vector that every array's rows are aligned for and the columns fill.
template <typename T, typename... P>
int vector_of(int cols, const P&... p) {
  auto all = [&](int bytes) { return ((!p.first || rows_aligned(p.first, p.second, sizeof(T), bytes)) && ...); };
  if (cols % 4 == 0 && all(4 * (int)sizeof(T))) return 4;
  return sizeof(T) == 2 && cols % 2 == 0 && all(4) ? 2 : 1;
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
  const int v = vector_of<T>(a.cols, P{a.x, a.ldx}, P{a.r, a.ldr}, P{a.h, a.ldh}, P{a.y, a.ldy});
  // (4096 x 2000: 8.1 us with up to four units a warp, 8.8 with eight; 4000 x 8192 to e4m3 35 and 26)
  const int nu = units_per_warp(a.rows, a.cols, cdiv(a.cols, UNIT) <= 16 ? 4 : 8, kMaxWarps);
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
      auto go_on = [&](auto N) {
        if constexpr (V.value == 4) return cudaLaunchKernelEx(&l.cfg, k_rms<T, N.value>, a);
        else return cudaLaunchKernelEx(&l.cfg, k_rms_narrow<T, V.value, N.value>, a);
      };
      switch (nu) {
        case 1: return go_on(std::integral_constant<int, 1>{});
        case 2: return go_on(std::integral_constant<int, 2>{});
        case 4: return go_on(std::integral_constant<int, 4>{});
        default: return go_on(std::integral_constant<int, 8>{});
      }
    });
  };
  FF_LAUNCH(K_RMS, bytes, st, go(), "RMS norm");
  return FF_OK;
}

// The gradient's blocks: as many an SM as 512 threads (128 registers each) and
// two sets of rows in shared memory allow, and at most kGradRows rows a thread.
// Two rows a set where that leaves two blocks an SM or costs none (16384 x 3000 bf16: 72
// us, one a set 79).  The rest of the shared memory deepens the queue.  (Sized for three arrays whether dh is there or not, so that the
// workspace does not depend on it.)
constexpr int kGradSmem = 200 * 1024;
static_assert(kGradWarps * 8 * 32 * (int)sizeof(Held<float>) * 3 <= kGradSmem, "the longest row of the row kernel");
constexpr int kGradEnds = 4 * 2 * 3 * kGradWarps * 16;  // and at most what single bf16 values add to their copies
struct GradPlan {
  int nu, warps, teams, set, blocks, depth;
};
GradPlan grad_plan(int rows, int cols, int esize) {
  GradPlan p{};
  // four units a warp, or eight where four do not reach or their warps leave a
  // quarter of an SM's empty
  const int units = cdiv(cols, UNIT);
  p.nu = units_per_warp(rows, cols, 4, kGradWarps);
  if (!p.nu || (p.nu == 4 && kGradWarps % cdiv(units, 4) > kGradWarps / 4)) p.nu = units_per_warp(rows, cols, 8, kGradWarps);
  int row = 0, threads = 0;
  if (p.nu) {
    p.warps = cdiv(units, p.nu);
    p.teams = p.warps == 1 ? kOwnRows : 1;
    threads = p.warps * p.teams * 32;
    row = threads * p.nu * 4 * esize * 3;  // bytes
  }
  long long fill;
  if (p.nu) {
    const int most = kGradWarps * 32 / threads;
    auto room_of = [&](int set) { return std::max(1, std::min(most, kGradSmem / (2 * set * row))); };
    p.set = 4 * row <= kGradSmem && (room_of(2) >= 2 || room_of(2) == room_of(1)) ? 2 : 1;
    const int room = room_of(p.set);
    p.depth = std::max(1, std::min(4, kGradSmem / (room * p.set * row)));
    fill = 152ll * room;
  } else {
    p.warps = kMaxWarps;
    p.teams = p.set = 1;
    fill = std::max(1, 152 * strip_blocks(esize) / cdiv(units, 8));
  }
  const long long sets = cdiv(rows, p.teams * p.set), least = cdiv(rows, (long long)p.teams * kGradRows);
  p.blocks = (int)(sets < fill ? sets : fill < least ? least : fill);
  if (!p.nu && p.blocks > 65535) p.blocks = 65535;
  return p;
}
long long grad_bytes(int rows, int cols, int esize) {
  const GradPlan p = grad_plan(rows, cols, esize);
  const long long part = p.blocks > 1 ? 4ll * p.blocks * cols : 0;
  return ((part + 15) & ~15ll) + (p.nu ? 0 : 4ll * rows);
}

template <typename T>
ff_status rms_grad_t(GradArgs<T> a, float* dgamma, void* ws, cudaStream_t st) {
  using P = std::pair<const void*, long long>;
  const int v = vector_of<T>(a.cols, P{a.dy, a.lddy}, P{a.h, a.ldh}, P{a.dh, a.lddh}, P{a.dx, a.lddx});
  const GradPlan p = grad_plan(a.rows, a.cols, (int)sizeof(T));
  a.warps = p.warps;
  a.depth = p.depth;
  a.inv_cols = 1.f / (float)a.cols;
  a.wide = wide_of(a.gamma);
  a.part = !dgamma ? nullptr : p.blocks > 1 ? static_cast<float*>(ws) : dgamma;
  const double count = (double)a.rows * a.cols;
  const double bytes = count * sizeof(T) * (2 + (a.dx ? 1 : 0) + (a.dh ? 1 : 0));
  if (p.nu) {
    auto go = [&]() -> cudaError_t {
      // (eight bf16 values a vector where two units go together)
      const bool eight = sizeof(T) == 2 && v == 4 && p.nu > 1 && a.cols % 8 == 0 && rows_aligned(a.dy, a.lddy, 2, 16) &&
                         rows_aligned(a.h, a.ldh, 2, 16) && (!a.dh || rows_aligned(a.dh, a.lddh, 2, 16)) &&
                         (!a.dx || rows_aligned(a.dx, a.lddx, 2, 16));
      auto with = [&](auto f) -> cudaError_t {
        if constexpr (sizeof(T) == 2)
          if (eight) return f(std::integral_constant<int, 8>{});
        return with_vector<T>(v, f);
      };
      return with([&](auto V) {
        const int threads = p.teams * p.warps * 32;
        // (single bf16 values: 16384 x 2001 70 us with one row a set, with two 83)
        const int set = Lay<T, V.value>::WORDS && p.blocks >= 152 ? 1 : p.set;
        const size_t ring = (size_t)p.depth * set * (a.dh ? 3 : 2) * (threads / 32) * Lay<T, V.value>::part(p.nu);
        const size_t smem = std::max(ring, p.teams > 1 && a.part ? (size_t)p.teams * a.cols * 4 : 0);
        PdlLaunch l(dim3((unsigned)p.blocks), dim3((unsigned)threads), st, smem);
        auto go = [&](auto N, auto R) -> cudaError_t {
          // what grad_plan gives: one row a set with eight units, with four of fp32 and
          // with single bf16 values; two with less than eight (and see `eight`)
          constexpr bool planned =
              R.value == 2 ? N.value < 8 : N.value == 8 || (N.value == 4 && sizeof(T) == 4) || Lay<T, V.value>::WORDS;
          if constexpr (!planned || (V.value == 8 && N.value == 1)) {
            return cudaErrorInvalidValue;
          } else {
            const cudaError_t e = allow_smem<k_rms_grad<T, V.value, N.value, R.value>>(kGradSmem + kGradEnds);
            return e != cudaSuccess ? e : cudaLaunchKernelEx(&l.cfg, k_rms_grad<T, V.value, N.value, R.value>, a);
          }
        };
        using One = std::integral_constant<int, 1>;
        using Two = std::integral_constant<int, 2>;
        using Four = std::integral_constant<int, 4>;
        using Eight = std::integral_constant<int, 8>;
        switch (p.nu) {
          case 1: return set == 2 ? go(One{}, Two{}) : go(One{}, One{});
          case 2: return set == 2 ? go(Two{}, Two{}) : go(Two{}, One{});
          case 4: return set == 2 ? go(Four{}, Two{}) : go(Four{}, One{});
          default: return set == 2 ? go(Eight{}, Two{}) : go(Eight{}, One{});
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
    // (16384 x 1000: 33.7 us in all with 8, 35.1 with 32; x 3000 71.0 and 70.1)
    const int w = a.cols < 32 * 76 ? 8 : 32;
    PdlLaunch l(dim3((unsigned)cdiv(a.cols, w)), dim3(1024), st);
    auto* const fold = w == 32 ? k_rms_fold<32> : k_rms_fold<8>;
    FF_LAUNCH(K_RMS_GRAD, 4.0 * p.blocks * a.cols, st,
              cudaLaunchKernelEx(&l.cfg, fold, (const float*)a.part, p.blocks, a.cols, dgamma), "RMS norm gradient");
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
      !matrix_ok(h, ldh, rows, cols, es) || !matrix_ok(y, ldy, rows, cols, es) || !aligned(q, 16) || !aligned(scale, 4) ||
      !aligned(gamma, 4) || !aligned(rstd, 4) || !apart(y, ldy, h, ldh, rows, cols, es) ||
      !apart_or_one(y, ldy, x, ldx, rows, cols, es) || !apart_or_one(y, ldy, residual, ldr, rows, cols, es) ||
      !apart_or_one(h, ldh, x, ldx, rows, cols, es) || !apart_or_one(h, ldh, residual, ldr, rows, cols, es))
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
  return rows == 0 ? 0 : std::max(grad_bytes(rows, cols, 2), grad_bytes(rows, cols, 4));
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
  const long long need = ff_rms_norm_workspace(rows, cols);
  if (!dy || !h || !rstd || !matrix_ok(dy, lddy, rows, cols, es) || !matrix_ok(h, ldh, rows, cols, es) ||
      !matrix_ok(dh, lddh, rows, cols, es) || !matrix_ok(dx, lddx, rows, cols, es) || !aligned(rstd, 4) ||
      !aligned(gamma, 4) || (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) ||
      !apart_or_one(dx, lddx, dy, lddy, rows, cols, es) || !apart_or_one(dx, lddx, h, ldh, rows, cols, es) ||
      !apart_or_one(dx, lddx, dh, lddh, rows, cols, es))
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
