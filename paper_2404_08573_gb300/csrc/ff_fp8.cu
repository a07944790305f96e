// 8-bit matrices (e4m3 values, an fp32 scale per block of 128 along the
// contraction): the quantizer, and the C entries of both operations.
#include <cuda_fp8.h>

#include "ff_api_internal.h"
#include "ff_fp8.h"
#include "ff_ptx.cuh"
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

// Two values as e4m3 (to nearest even, saturating; NaN stays NaN), a in the low byte.
__device__ __forceinline__ uint32_t e4m3x2(float a, float b) {
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ uint2 e4m3x8(const float (&v)[8]) {
  return make_uint2(e4m3x2(v[0], v[1]) | e4m3x2(v[2], v[3]) << 16, e4m3x2(v[4], v[5]) | e4m3x2(v[6], v[7]) << 16);
}

// Eight values of a row as loaded: bf16 in pairs (the low half first), or fp32.
// Magnitudes are compared as integers, bf16 two at a time.
template <typename T>
struct Eight;
template <>
struct Eight<bf16> {
  static constexpr int WORDS = 4, PER = 2;  // PER: values per word
  static constexpr uint32_t ABS = 0x7FFF7FFFu;
  static __device__ __forceinline__ uint32_t max_of(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ float value(const uint32_t (&w)[WORDS], int e) {
    return __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
  }
  // the magnitude in half `h` of a word, as the bits of a float
  static __device__ __forceinline__ uint32_t bits(uint32_t w, int h) { return h ? w & 0xFFFF0000u : w << 16; }
};
template <>
struct Eight<float> {
  static constexpr int WORDS = 8, PER = 1;
  static constexpr uint32_t ABS = 0x7FFFFFFFu;
  static __device__ __forceinline__ uint32_t max_of(uint32_t a, uint32_t b) { return max(a, b); }
  static __device__ __forceinline__ float value(const uint32_t (&w)[WORDS], int e) { return __uint_as_float(w[e]); }
  static __device__ __forceinline__ uint32_t bits(uint32_t w, int) { return w; }
};

constexpr int QB = 128;          // a block of the matrix: 128 x 128
constexpr int kQThreads = 256;

// One thread block per 128 x 128 tile.  Thread (rg, cg) holds rows
// 8 rg .. 8 rg + 7 of columns 8 cg .. 8 cg + 7 as loaded (all loads in flight
// together).  A row block's maximum is formed by the 16 threads of a row
// group, each step handing half of the rows to the partner, so that a thread
// ends with one row, divides once, and passes the reciprocal round; a column
// block's by one pass over the 16 row groups in shared memory.  Both
// orientations come from one read.  Bound by HBM: x once, each orientation
// once (4096 x 8192 bf16, both: 25 us, 5.4 TB/s; 2000 x 784 fp32 in tiles, both:
// 4.0 us, a launch and one round of 112 blocks).  Rows that start on 4 bytes
// only are read in pairs (7455 x 7374 bf16, both: 43 us, value by value 64, and
// 7376 columns 38); odd widths of bf16 stay value by value, since five words
// shifted into place took as long.
// LOAD: bytes of x per access that its rows' alignment allows.
template <typename T, int LOAD>
__global__ void __launch_bounds__(kQThreads, sizeof(T) == 2 ? 4 : 2)
    k_fp8_quantize(const T* x, long long ldx, int rows, int k, int tile, uint8_t* q, float* scale, uint8_t* qt,
                   float* scale_t, int ldq, int ldqt, int kblocks, int rblocks) {
  using E = Eight<T>;
  constexpr int W = E::WORDS, PER = E::PER;
  __shared__ uint32_t cmax[16][QB / PER];
  __shared__ float cinv[QB];
  __shared__ uint32_t wmax[kQThreads / 32];
  // the transposed tile: 128 bytes per column, its 8-byte units permuted so
  // that the 16 column groups of a warp's writes fall into different banks
  __shared__ __align__(16) uint8_t tq[QB * QB];
  ptx::griddep_wait();
  const int kb = blockIdx.x % kblocks, rb = blockIdx.x / kblocks;
  const int rg = threadIdx.x >> 4, cg = threadIdx.x & 15;
  const int row0 = rb * QB + rg * 8, c0 = kb * QB + cg * 8;
  uint32_t v[8][W];
  if (LOAD == 16 && c0 + 8 <= k) {
    const T* p = x + (long long)row0 * ldx + c0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < W / 4; ++j)
        *reinterpret_cast<uint4*>(&v[i][4 * j]) =
            row0 + i < rows ? reinterpret_cast<const uint4*>(p + i * ldx)[j] : make_uint4(0, 0, 0, 0);
  } else if (LOAD == 4 && c0 + 8 <= k) {
    const T* p = x + (long long)row0 * ldx + c0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < W; ++j)
        v[i][j] = row0 + i < rows ? reinterpret_cast<const uint32_t*>(p + i * ldx)[j] : 0u;
  } else {
    const T* p = x + (long long)row0 * ldx + c0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < W; ++j) {
        uint32_t w = 0;
#pragma unroll
        for (int h = 0; h < PER; ++h)
          if (row0 + i < rows && c0 + j * PER + h < k)
            w |= (uint32_t)Vec<T, 1>::load(p + i * ldx + j * PER + h) << (16 * h);
        v[i][j] = w;
      }
  }
  float inv_tile = 0.f;
  if (tile) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < W; ++j) m = E::max_of(m, v[i][j] & E::ABS);
    m = max(E::bits(m, 0), E::bits(m, 1));
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
    float inv_row = inv_tile;
    if (!tile) {
      // word j of m: rows j PER .. (one per half of the word)
      uint32_t m[8 / PER];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint32_t t = v[i][0] & E::ABS;
#pragma unroll
        for (int j = 1; j < W; ++j) t = E::max_of(t, v[i][j] & E::ABS);
        if constexpr (PER == 2) {
          t = max(t & 0xFFFFu, t >> 16);
          m[i / 2] = i & 1 ? m[i / 2] | t << 16 : t;
        } else {
          m[i] = t;
        }
      }
      int bit = 8;
#pragma unroll
      for (int n = 8 / PER; n > 1; n /= 2) {
#pragma unroll
        for (int j = 0; j < n / 2; ++j) {
          const bool up = (cg & bit) != 0;
          const uint32_t give = up ? m[j] : m[j + n / 2], keep = up ? m[j + n / 2] : m[j];
          m[j] = E::max_of(keep, __shfl_xor_sync(0xffffffffu, give, bit));
        }
        bit >>= 1;
      }
      for (; bit > 0; bit >>= 1) m[0] = E::max_of(m[0], __shfl_xor_sync(0xffffffffu, m[0], bit));
      // this thread's row: the bits of cg that chose, from the top (bf16: 8, 4,
      // and bit 0 picks the half; fp32: 8, 4, 2)
      const int mine = PER == 2 ? (cg >> 3 & 1) * 4 + (cg >> 2 & 1) * 2 + (cg & 1) : cg >> 1;
      const float s = scale_of(E::bits(m[0], cg & 1));
      inv_row = __frcp_rn(s);
      const bool writer = PER == 2 ? (cg & 2) == 0 : (cg & 1) == 0;
      if (writer && row0 + mine < rows) scale[(long long)kb * rows + row0 + mine] = s;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int src = PER == 2 ? (i >> 2) * 8 + (i >> 1 & 1) * 4 + (i & 1) : i * 2;
      const float inv = tile ? inv_tile : __shfl_sync(0xffffffffu, inv_row, (threadIdx.x & 16) | src);
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = __fmul_rn(E::value(v[i], e), inv);
      const int r = row0 + i;
      // ldq is a multiple of 16: a group of 8 columns lies inside or outside
      if (r < rows && c0 < ldq) *reinterpret_cast<uint2*>(q + (long long)r * ldq + c0) = e4m3x8(f);
    }
  }
  if (qt) {
    if (!tile) {
#pragma unroll
      for (int j = 0; j < W; ++j) {
        uint32_t m = v[0][j] & E::ABS;
#pragma unroll
        for (int i = 1; i < 8; ++i) m = E::max_of(m, v[i][j] & E::ABS);
        cmax[rg][cg * W + j] = m;
      }
      __syncthreads();
      if (threadIdx.x < QB) {
        uint32_t m = 0;
#pragma unroll
        for (int t = 0; t < 16; ++t) m = E::max_of(m, cmax[t][threadIdx.x / PER]);
        const float s = scale_of(E::bits(m, threadIdx.x & 1));
        cinv[threadIdx.x] = __frcp_rn(s);
        const int c = kb * QB + threadIdx.x;
        if (c < k) scale_t[(long long)rb * k + c] = s;
      }
      __syncthreads();
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float inv = tile ? inv_tile : cinv[cg * 8 + e];
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = __fmul_rn(E::value(v[i], e), inv);
      *reinterpret_cast<uint2*>(tq + (cg * 8 + e) * QB + ((rg ^ cg) << 3)) = e4m3x8(f);
    }
    __syncthreads();
    // 8 threads per column of the tile, 16 bytes each (ldqt is a multiple of 16)
    const int u = threadIdx.x & 7, r = rb * QB + u * 16;
    if (r < ldqt) {
#pragma unroll
      for (int c = threadIdx.x >> 3; c < QB; c += kQThreads / 8) {
        const int col = kb * QB + c;
        if (col >= k) break;
        const uint8_t* t = tq + c * QB;
        const uint2 a = *reinterpret_cast<const uint2*>(t + (((2 * u) ^ (c >> 3)) << 3));
        const uint2 b = *reinterpret_cast<const uint2*>(t + (((2 * u + 1) ^ (c >> 3)) << 3));
        *reinterpret_cast<uint4*>(qt + (long long)col * ldqt + r) = make_uint4(a.x, a.y, b.x, b.y);
      }
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
  PdlLaunch l(dim3((unsigned)blocks), dim3(kQThreads), st);
  auto go = [&](auto* kernel) {
    return cudaLaunchKernelEx(&l.cfg, kernel, x, ldx, rows, k, tile, q, scale, qt, scale_t, ldq, ldqt, kblocks, rblocks);
  };
  FF_LAUNCH(K_FP8_QUANT, bytes, st,
            rows_aligned(x, ldx, sizeof(T), 16)  ? go(k_fp8_quantize<T, 16>)
            : rows_aligned(x, ldx, sizeof(T), 4) ? go(k_fp8_quantize<T, 4>)
                                                 : go(k_fp8_quantize<T, sizeof(T)>),
            "8-bit quantize");
  return FF_OK;
}

// Where products without a status word of the caller's latch a timeout: a word
// on each device, so that no invalid result goes unreported.
__device__ int g_fp8_status;
cudaError_t own_status(int** word) {
  static PerDevice<void*> kept;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  void* p = nullptr;
  e = kept.get(dev, &p, [](void** p) { return cudaGetSymbolAddress(p, g_fp8_status); });
  *word = static_cast<int*>(p);
  return e;
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
  if (!device_status) FF_TRY(own_status(&g.status), "8-bit matrix product");
  return fp8_gemm(g, static_cast<cudaStream_t>(stream));
}

extern "C" FF_API ff_status ff_fp8_check(void* stream) {
  int *word = nullptr, err = 0;
  FF_TRY(own_status(&word), "8-bit check");
  FF_TRY(cudaStreamSynchronize(static_cast<cudaStream_t>(stream)), "8-bit check");
  FF_TRY(cudaMemcpy(&err, word, sizeof(int), cudaMemcpyDeviceToHost), "8-bit check");
  if (!err) return FF_OK;
  const int zero = 0;
  FF_TRY(cudaMemcpy(word, &zero, sizeof(int), cudaMemcpyHostToDevice), "8-bit check");
  return FF_ERR_TIMEOUT;
}

extern "C" FF_API ff_status ff_fp8_selftest_wait(unsigned int timeout_us, void* stream) {
  if (timeout_us < 1 || timeout_us > 10000000u) return FF_ERR_INVALID_ARG;
  int* word = nullptr;
  FF_TRY(own_status(&word), "8-bit self-test");
  FF_TRY(launch_wait_selftest(word, 1000ull * timeout_us, static_cast<cudaStream_t>(stream)), "8-bit self-test");
  return FF_OK;
}
