// Group norm with an activation: what its kernel files share.  Sizes, the
// activation and its slope, and the three paths' entry points (ff_norm.cu
// picks one by sizes and alignment).
#pragma once

#include "ff_api_internal.h"
#include "ff_ptx.cuh"
#include "ff_vec.cuh"

namespace ff {

struct GnShape {
  int n, S, C, G, Cg;
  long long ldx, ldy, lddy;  // forward: x -> y; gradient: (dy, x) -> dx with ldy the stride of dx
  float eps;
  int act;
};

// Everything a call passes; mean and rstd are outputs of the forward pass
// (or null) and inputs of the gradient.
template <typename T>
struct GnArgs {
  GnShape s;
  const T *x, *dy;
  T* out;                    // y or dx (null: no dx)
  const float *gamma, *beta; // or null: ones, zeros
  float *mean, *rstd;
  float *dgamma, *dbeta;     // or null
  void* ws;
};

// Samples whose terms of dgamma and dbeta one thread adds up in a row: the
// rounding of a plain sum grows with its length, and a batch has no bound.
constexpr int kGradSamples = 128;

// The rows path: groups in the registers of up to a warp, or of a block.
// `lanes` lanes per group (a power of 2), sets of groups side by side.
struct GnRowsPlan {
  int lanes, sets, P;  // P: blocks along the samples
};
bool gn_rows_fit(const GnShape& s);
// The block path: a slab of whole groups of one sample stays in the shared
// memory of a thread block.
struct GnBlockPlan {
  int T, GS, nv;      // threads, groups per slab, vectors per thread; T = 0: does not fit
  int blocks, units;  // blocks launched, and (slab, sample) units each takes
  double us;          // estimated time
};

GnRowsPlan gn_rows_plan(const GnShape& s, int V, bool grad);
GnBlockPlan gn_block_plan(const GnShape& s, int V, int esize, bool grad);

template <typename T>
ff_status gn_rows(const GnArgs<T>& a, int V, bool grad, cudaStream_t st);
template <typename T>
ff_status gn_block(const GnArgs<T>& a, int V, const GnBlockPlan& p, bool grad, cudaStream_t st);
// dbeta and dgamma from partial column sums (du, du h) [., C]: `rows` of them,
// or, with units > 0, as many as the blocks that took the column's slab (slabs
// of W columns, n units each; `units` consecutive ones per block).
struct GnFold {
  long long rows;
  int units, n, W;
};
ff_status gn_param_fold(const float2* part, const GnFold& f, int C, float* dgamma, float* dbeta, cudaStream_t st);

// Division of non-negative 31-bit numbers by a number fixed per launch
// (Granlund and Montgomery's multiply-and-shift): q = (hi(n mul) + n) >> s.
struct FastDiv {
  uint32_t d, mul;
  int s;
  FastDiv() = default;
  explicit FastDiv(uint32_t by) : d(by), s(0) {
    while ((1ull << s) < by) ++s;
    mul = (uint32_t)(((1ull << 32) * ((1ull << s) - by)) / by + 1);
  }
  __device__ __forceinline__ uint32_t div(uint32_t n) const { return (__umulhi(n, mul) + n) >> s; }
};

// What a group's sums are held relative to, from its first two values: the
// first where it is large beside their distance, so that a large mean costs
// the small spread no bits; else zero, since a mean near zero would come out
// as the difference of two numbers of the spread's size.
__device__ __forceinline__ float pivot_of(float first, float second) {
  return fabsf(first) >= 16.f * fabsf(second - first) ? first : 0.f;
}
// How far a group's second value lies from its first.
__device__ __forceinline__ long long second_of(const GnShape& s) { return s.Cg > 1 ? 1 : s.S > 1 ? s.ldx : 0; }

__device__ __forceinline__ uint64_t both(float v) { return ptx::pack2(v, v); }
// 1 / (1 + e^-u) from e = e^-|u|, which is at most one: 1 / (1 + e) for u >= 0
// and e / (1 + e) below, so that nothing overflows and the result goes to zero
// as it should however far out u is.  T = float: e by expf, and a reciprocal
// each (within 2^-21 of itself in all).  T = bf16, where the output's rounding
// is 2^-9: the approximate exponential, whose rounded argument costs up to
// 2^-17, and of a pair one approximate reciprocal for both: with a = 1 + e and
// r = 1 / (a b), 1 / a is r b and 1 / b is r a.  (These units take 16 values a
// clock and SM, and with two calls a value they, not HBM, would bound the bf16
// forms.)
__device__ __forceinline__ float rcp_approx(float v) {  // of 1 to 4: within one unit of the last place
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
template <typename T>
__device__ __forceinline__ float exp_minus_abs(float u) {
  if constexpr (sizeof(T) == 4) return expf(-fabsf(u));
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(fabsf(u) * -1.44269504f));
  return r;
}
template <typename T>
__device__ __forceinline__ float sigmoid1(float u) {
  const float e = exp_minus_abs<T>(u), r = rcp_approx(1.f + e);
  return u < 0.f ? e * r : r;
}
template <typename T>
__device__ __forceinline__ uint64_t sigmoid2(uint64_t u) {
  const float2 v = ptx::unpack2(u);
  if constexpr (sizeof(T) == 4) return ptx::pack2(sigmoid1<T>(v.x), sigmoid1<T>(v.y));
  const float x = exp_minus_abs<T>(v.x), y = exp_minus_abs<T>(v.y);
  const float a = 1.f + x, b = 1.f + y, r = rcp_approx(a * b);
  const float p = b * r, q = a * r;
  return ptx::pack2(v.x < 0.f ? x * p : p, v.y < 0.f ? y * q : q);
}
__device__ __forceinline__ float max0(float u) {  // max(u, 0), NaN kept
  float r;
  asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(u));
  return r;
}

// A vector of V values as pairs (V = 1: one pair whose second value is zero).
template <int V>
struct Pairs {
  static constexpr int N = V < 2 ? 1 : V / 2;
  static __device__ __forceinline__ void of(const float (&v)[V], uint64_t (&p)[N]) {
    if constexpr (V == 1) {
      p[0] = ptx::pack2(v[0], 0.f);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) p[i] = ptx::pack2(v[2 * i], v[2 * i + 1]);
    }
  }
  static __device__ __forceinline__ void to(const uint64_t (&p)[N], float (&v)[V]) {
    if constexpr (V == 1) {
      v[0] = ptx::unpack2(p[0]).x;
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float2 f = ptx::unpack2(p[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
      }
    }
  }
};

// u = act(u) and d = d act'(u) over pairs (V = 1: the first value only).
template <typename T, int V>
__device__ __forceinline__ void act_pairs(uint64_t (&u)[Pairs<V>::N], int act) {
  constexpr int N = Pairs<V>::N;
  if (act == FF_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      u[i] = V == 1 ? ptx::pack2(ptx::unpack2(u[i]).x * sigmoid1<T>(ptx::unpack2(u[i]).x), 0.f)
                    : ptx::mul2(u[i], sigmoid2<T>(u[i]));
  } else if (act == FF_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float2 v = ptx::unpack2(u[i]);
      u[i] = ptx::pack2(max0(v.x), max0(v.y));
    }
  }
}
template <typename T, int V>
__device__ __forceinline__ void act_grad_pairs(uint64_t (&d)[Pairs<V>::N], const uint64_t (&u)[Pairs<V>::N], int act) {
  constexpr int N = Pairs<V>::N;
  if (act == FF_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint64_t p = V == 1 ? ptx::pack2(sigmoid1<T>(ptx::unpack2(u[i]).x), 0.f) : sigmoid2<T>(u[i]);
      const uint64_t q = ptx::fma2(p, both(-1.f), both(1.f));  // 1 - p
      d[i] = ptx::mul2(d[i], ptx::mul2(p, ptx::fma2(u[i], q, both(1.f))));
    }
  } else if (act == FF_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float2 v = ptx::unpack2(u[i]), w = ptx::unpack2(d[i]);
      d[i] = ptx::pack2(v.x > 0.f ? w.x : 0.f, v.y > 0.f ? w.y : 0.f);
    }
  }
}

// V parameters from index c (a multiple of V), or `none` everywhere; wide: p
// is 16-byte aligned.
template <int V>
__device__ __forceinline__ void load_params(float (&v)[V], const float* p, long long c, float none, bool wide) {
  if (!p) {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = none;
  } else if (V % 4 == 0 && wide) {
#pragma unroll
    for (int e = 0; e + 3 < V; e += 4) {
      const float4 f = __ldg(reinterpret_cast<const float4*>(p + c + e));
      v[e] = f.x;
      v[e + 1] = f.y;
      v[e + 2] = f.z;
      v[e + 3] = f.w;
    }
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = __ldg(p + c + e);
  }
}

}  // namespace ff
