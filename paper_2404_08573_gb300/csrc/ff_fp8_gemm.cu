// The 8-bit matrix product C = act(A B^T + bias) with a scale per block of 128
// along the contraction, on CUDA cores: a 64 x 64 tile of C per thread block,
// each k-block's products summed in fp32 and then scaled by the block's scales.
#include <cuda_fp8.h>

#include "ff_api_internal.h"
#include "ff_fp8.h"

namespace ff {
namespace {

constexpr int ST = 64, SK = 32, SBLOCK = 128;

__device__ __forceinline__ float from_e4m3(uint8_t v) {
  return __half2float(__half(__nv_cvt_fp8_to_halfraw(v, __NV_E4M3)));
}

__global__ void __launch_bounds__(256) k_fp8_simple(Fp8Gemm g, int ntn) {
  __shared__ float sA[SK][ST + 4], sB[SK][ST + 4];
  const int m0 = (int)(blockIdx.x / ntn) * ST, n0 = (int)(blockIdx.x % ntn) * ST;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int ld = (g.K + 15) & ~15;
  float acc[4][4] = {};
  for (int kb = 0; kb * SBLOCK < g.K; ++kb) {
    float p[4][4] = {};
    for (int k0 = kb * SBLOCK; k0 < min(g.K, (kb + 1) * SBLOCK); k0 += SK) {
      __syncthreads();
      for (int i = threadIdx.x; i < ST * SK; i += 256) {
        const int r = i / SK, k = i % SK;
        const bool in = k0 + k < g.K;
        sA[k][r] = in && m0 + r < g.M ? from_e4m3(g.a[(long long)(m0 + r) * ld + k0 + k]) : 0.f;
        sB[k][r] = in && n0 + r < g.N ? from_e4m3(g.b[(long long)(n0 + r) * ld + k0 + k]) : 0.f;
      }
      __syncthreads();
      for (int k = 0; k < SK; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) p[i][j] = fmaf(sA[k][ty * 4 + i], sB[k][tx * 4 + j], p[i][j]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int m = m0 + ty * 4 + i, n = n0 + tx * 4 + j;
        if (m < g.M && n < g.N) {
          const float sb = g.b_tiles ? g.sb[(long long)kb * ((g.N + 127) / 128) + n / 128] : g.sb[(long long)kb * g.N + n];
          acc[i][j] = fmaf(g.sa[(long long)kb * g.M + m] * sb, p[i][j], acc[i][j]);
        }
      }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int m = m0 + ty * 4 + i, n = n0 + tx * 4 + j;
      if (m >= g.M || n >= g.N) continue;
      float v = acc[i][j] + (g.bias ? g.bias[n] : 0.f);
      if (g.relu) v = v < 0.f ? 0.f : v;
      if (g.out_bf16)
        static_cast<bf16*>(g.c)[(long long)m * g.ldc + n] = __float2bfloat16_rn(v);
      else
        static_cast<float*>(g.c)[(long long)m * g.ldc + n] = v;
    }
}

}  // namespace

ff_status fp8_gemm(const Fp8Gemm& g, cudaStream_t st) {
  const int ntm = cdiv(g.M, ST), ntn = cdiv(g.N, ST);
  if ((long long)ntm * ntn > 0x7FFFFFFFll) return FF_ERR_UNSUPPORTED;
  FF_LAUNCH(K_FP8_GEMM, 2.0 * g.M * g.N * g.K, st,
            (k_fp8_simple<<<(unsigned)(ntm * ntn), 256, 0, st>>>(g, ntn), cudaGetLastError()), "8-bit matrix product");
  return FF_OK;
}

}  // namespace ff
