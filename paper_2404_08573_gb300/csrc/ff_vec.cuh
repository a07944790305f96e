// Vectors of V consecutive bf16 or fp32 values of a row, held as loaded (a
// bf16 pair stays packed in one register) until their values are wanted.
#pragma once

#include "ff_internal.cuh"

namespace ff {

template <int BYTES>
struct RawOf;
template <>
struct RawOf<16> { using type = uint4; };
template <>
struct RawOf<8> { using type = uint2; };
template <>
struct RawOf<4> { using type = uint32_t; };
template <>
struct RawOf<2> { using type = uint16_t; };

template <typename T, int V>
struct Vec {
  using Raw = typename RawOf<(int)sizeof(T) * V>::type;
  static __device__ __forceinline__ Raw load(const T* p) { return *reinterpret_cast<const Raw*>(p); }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&v)[V]) {
    if constexpr (sizeof(T) == 4) {
      const float* f = reinterpret_cast<const float*>(&r);
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = f[e];
    } else if constexpr (V == 1) {
      v[0] = __uint_as_float((uint32_t)r << 16);
    } else {
      const uint32_t* w = reinterpret_cast<const uint32_t*>(&r);
#pragma unroll
      for (int e = 0; e < V / 2; ++e) {
        v[2 * e] = __uint_as_float(w[e] << 16);
        v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
      }
    }
  }
  static __device__ __forceinline__ void store(T* p, const float (&v)[V]) {
    Raw r;
    if constexpr (sizeof(T) == 4) {
      float* f = reinterpret_cast<float*>(&r);
#pragma unroll
      for (int e = 0; e < V; ++e) f[e] = v[e];
    } else if constexpr (V == 1) {
      const bf16 h = __float2bfloat16_rn(v[0]);
      r = *reinterpret_cast<const uint16_t*>(&h);
    } else {
      uint32_t* w = reinterpret_cast<uint32_t*>(&r);
#pragma unroll
      for (int e = 0; e < V / 2; ++e) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
        w[e] = *reinterpret_cast<const uint32_t*>(&h);
      }
    }
    *reinterpret_cast<Raw*>(p) = r;
  }
};

// Whether rows of a matrix (base p, row stride ld elements of esize bytes)
// all start on a multiple of `bytes`.
inline bool rows_aligned(const void* p, long long ld, int esize, int bytes) {
  return reinterpret_cast<uintptr_t>(p) % bytes == 0 && (ld * esize) % bytes == 0;
}

}  // namespace ff
