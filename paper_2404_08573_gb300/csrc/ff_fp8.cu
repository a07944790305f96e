// 8-bit matrices (e4m3 values, an fp32 scale per block of 128 along the
// contraction): the quantizer, and the C entries of both operations.
#include <cuda_fp8.h>

#include "ff_api_internal.h"
#include "ff_fp8.h"
#include "ff_vec.cuh"

namespace ff {
namespace {

constexpr float kE4m3Max = 448.f;
constexpr float kScaleMin = 1.17549435e-38f;  // 2^-126

// The scale of a block whose largest magnitude has these bits (the bits of
// non-negative floats order like the floats, with infinity and then NaN above
// all of them, so an integer maximum keeps both).
__device__ __forceinline__ float scale_of(uint32_t amax_bits) {
  const float s = __fdiv_rn(__uint_as_float(amax_bits), kE4m3Max);
  return s < kScaleMin ? kScaleMin : s;  // keeps NaN
}
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Two values as e4m3 (to nearest even, saturating; NaN stays NaN), a in the low byte.
__device__ __forceinline__ uint32_t e4m3x2(float a, float b) {
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}

constexpr int QB = 128;          // a block of the matrix: 128 x 128
constexpr int kQThreads = 256;
constexpr int kTPitch = QB + 8;  // bytes per column of the transposed tile in shared memory

// One thread block per 128 x 128 tile.  Thread (rg, cg) holds rows
// 8 rg .. 8 rg + 7 of columns 8 cg .. 8 cg + 7 in registers: a row block's
// maximum is 8 values and a shuffle over the 16 threads of a row group, a
// column block's 8 values and one pass over the 16 row groups, and both
// orientations are formed from one read.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kQThreads) k_fp8_quantize(const T* x, long long ldx, int rows, int k, int tile,
                                                            uint8_t* q, float* scale, uint8_t* qt, float* scale_t,
                                                            int ldq, int ldqt, int kblocks, int rblocks) {
  __shared__ uint32_t cmax[16][QB];
  __shared__ float cinv[QB];
  __shared__ uint32_t wmax[kQThreads / 32];
  __shared__ __align__(16) uint8_t tq[QB * kTPitch];
  const int kb = blockIdx.x % kblocks, rb = blockIdx.x / kblocks;
  const int rg = threadIdx.x >> 4, cg = threadIdx.x & 15;
  const int row0 = rb * QB + rg * 8, c0 = kb * QB + cg * 8;
  float v[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = row0 + i;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
    if (r < rows) {
      const T* p = x + (long long)r * ldx + c0;
      if (VEC && c0 + 8 <= k) {
        Vec8<T>::load(p, v[i]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c0 + e < k) {
            float one[1];
            Vec<T, 1>::unpack(Vec<T, 1>::load(p + e), one);
            v[i][e] = one[0];
          }
      }
    }
  }
  float inv_tile = 0.f;
  if (tile) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) m = max(m, abs_bits(v[i][e]));
    m = __reduce_max_sync(0xffffffffu, m);
    if ((threadIdx.x & 31) == 0) wmax[threadIdx.x >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kQThreads / 32; ++w) m = max(m, wmax[w]);
    const float s = scale_of(m);
    inv_tile = __frcp_rn(s);
    if (threadIdx.x == 0) {
      if (q) scale[(long long)kb * rblocks + rb] = s;
      if (qt) scale_t[(long long)rb * kblocks + kb] = s;
    }
  }
  if (q) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = row0 + i;
      float inv = inv_tile;
      if (!tile) {
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, abs_bits(v[i][e]));
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
        const float s = scale_of(m);
        inv = __frcp_rn(s);
        if (cg == 0 && r < rows) scale[(long long)kb * rows + r] = s;
      }
      if (r < rows && c0 < ldq) {  // ldq is a multiple of 16: a group of 8 columns lies inside or outside
        uint2 w;
        w.x = e4m3x2(__fmul_rn(v[i][0], inv), __fmul_rn(v[i][1], inv)) |
              e4m3x2(__fmul_rn(v[i][2], inv), __fmul_rn(v[i][3], inv)) << 16;
        w.y = e4m3x2(__fmul_rn(v[i][4], inv), __fmul_rn(v[i][5], inv)) |
              e4m3x2(__fmul_rn(v[i][6], inv), __fmul_rn(v[i][7], inv)) << 16;
        *reinterpret_cast<uint2*>(q + (long long)r * ldq + c0) = w;
      }
    }
  }
  if (qt) {
    if (!tile) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, abs_bits(v[i][e]));
        cmax[rg][cg * 8 + e] = m;
      }
      __syncthreads();
      if (threadIdx.x < QB) {
        uint32_t m = 0;
#pragma unroll
        for (int t = 0; t < 16; ++t) m = max(m, cmax[t][threadIdx.x]);
        const float s = scale_of(m);
        cinv[threadIdx.x] = __frcp_rn(s);
        const int c = kb * QB + threadIdx.x;
        if (c < k) scale_t[(long long)rb * k + c] = s;
      }
      __syncthreads();
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float inv = tile ? inv_tile : cinv[cg * 8 + e];
      uint2 w;
      w.x = e4m3x2(__fmul_rn(v[0][e], inv), __fmul_rn(v[1][e], inv)) |
            e4m3x2(__fmul_rn(v[2][e], inv), __fmul_rn(v[3][e], inv)) << 16;
      w.y = e4m3x2(__fmul_rn(v[4][e], inv), __fmul_rn(v[5][e], inv)) |
            e4m3x2(__fmul_rn(v[6][e], inv), __fmul_rn(v[7][e], inv)) << 16;
      *reinterpret_cast<uint2*>(tq + (cg * 8 + e) * kTPitch + rg * 8) = w;
    }
    __syncthreads();
    // 16 threads per column of the tile, 8 bytes each
    for (int c = threadIdx.x >> 4; c < QB; c += kQThreads / 16) {
      const int col = kb * QB + c, r = rb * QB + (threadIdx.x & 15) * 8;
      if (col < k && r < ldqt)
        *reinterpret_cast<uint2*>(qt + (long long)col * ldqt + r) =
            *reinterpret_cast<const uint2*>(tq + c * kTPitch + (threadIdx.x & 15) * 8);
    }
  }
}

template <typename T>
ff_status quantize_t(const T* x, long long ldx, int rows, int k, int tile, uint8_t* q, float* scale, uint8_t* qt,
                     float* scale_t, cudaStream_t st) {
  const int kblocks = cdiv(k, QB), rblocks = cdiv(rows, QB);
  const long long blocks = (long long)kblocks * rblocks;
  if (blocks > 0x7FFFFFFFll) return FF_ERR_UNSUPPORTED;
  const double bytes = (double)rows * k * (sizeof(T) + (q ? 1 : 0) + (qt ? 1 : 0));
  const int ldq = fp8_stride(k), ldqt = fp8_stride(rows);
  const bool vec = rows_aligned(x, ldx, sizeof(T), 16);
  FF_LAUNCH(K_FP8_QUANT, bytes, st,
            ((vec ? k_fp8_quantize<T, true><<<(unsigned)blocks, kQThreads, 0, st>>>(
                        x, ldx, rows, k, tile, q, scale, qt, scale_t, ldq, ldqt, kblocks, rblocks)
                  : k_fp8_quantize<T, false><<<(unsigned)blocks, kQThreads, 0, st>>>(
                        x, ldx, rows, k, tile, q, scale, qt, scale_t, ldq, ldqt, kblocks, rblocks)),
             cudaGetLastError()),
            "8-bit quantize");
  return FF_OK;
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
bool aligned4(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

}  // namespace
}  // namespace ff

using namespace ff;

extern "C" FF_API int ff_fp8_stride(int k) { return k > 0 && k <= 0x7FFFFFF0 ? fp8_stride(k) : 0; }

extern "C" FF_API ff_status ff_fp8_quantize(const void* x, long long ldx, int rows, int k, ff_precision prec,
                                            ff_fp8_blocks blocks, void* q, float* scale, void* qt, float* scale_t,
                                            void* stream) {
  if (rows < 0 || k < 1 || rows > 0x7FFFFF00 || k > 0x7FFFFF00 || (prec != FF_FP32 && prec != FF_BF16) ||
      (blocks != FF_FP8_ROWS && blocks != FF_FP8_TILES))
    return FF_ERR_INVALID_ARG;
  if (rows == 0) return FF_OK;
  const int es = prec == FF_BF16 ? 2 : 4;
  if (!x || reinterpret_cast<uintptr_t>(x) % es != 0 || (ldx < k && rows > 1)) return FF_ERR_INVALID_ARG;
  if ((q == nullptr) != (scale == nullptr) || (qt == nullptr) != (scale_t == nullptr) || (!q && !qt))
    return FF_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(qt) || !aligned4(scale) || !aligned4(scale_t)) return FF_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int tile = blocks == FF_FP8_TILES;
  if (prec == FF_BF16)
    return quantize_t(static_cast<const bf16*>(x), ldx, rows, k, tile, static_cast<uint8_t*>(q), scale,
                      static_cast<uint8_t*>(qt), scale_t, st);
  return quantize_t(static_cast<const float*>(x), ldx, rows, k, tile, static_cast<uint8_t*>(q), scale,
                    static_cast<uint8_t*>(qt), scale_t, st);
}

extern "C" FF_API ff_status ff_fp8_matmul(const void* a, const float* a_scale, const void* b, const float* b_scale,
                                          ff_fp8_blocks b_blocks, int m, int n, int k, const float* bias, int relu,
                                          ff_precision out_prec, void* c, long long ldc, int* device_status,
                                          void* stream) {
  if (m < 0 || n < 0 || k < 1 || m > 0x7FFFFF00 || n > 0x7FFFFF00 || k > 0x7FFFFF00 ||
      (out_prec != FF_FP32 && out_prec != FF_BF16) || (b_blocks != FF_FP8_ROWS && b_blocks != FF_FP8_TILES))
    return FF_ERR_INVALID_ARG;
  if (m == 0 || n == 0) return FF_OK;
  const int es = out_prec == FF_BF16 ? 2 : 4;
  if (!a || !a_scale || !b || !b_scale || !c || !aligned16(a) || !aligned16(b) || !aligned4(a_scale) ||
      !aligned4(b_scale) || !aligned4(bias) || !aligned4(device_status) || reinterpret_cast<uintptr_t>(c) % es != 0 ||
      (ldc < n && m > 1))
    return FF_ERR_INVALID_ARG;
  if (!tc_supported()) return FF_ERR_UNSUPPORTED;
  Fp8Gemm g{};
  g.a = static_cast<const uint8_t*>(a);
  g.b = static_cast<const uint8_t*>(b);
  g.sa = a_scale;
  g.sb = b_scale;
  g.b_tiles = b_blocks == FF_FP8_TILES;
  g.M = m;
  g.N = n;
  g.K = k;
  g.bias = bias;
  g.relu = relu != 0;
  g.out_bf16 = out_prec == FF_BF16;
  g.c = c;
  g.ldc = ldc;
  g.status = device_status;
  return fp8_gemm(g, static_cast<cudaStream_t>(stream));
}
