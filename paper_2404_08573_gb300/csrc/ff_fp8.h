// The 8-bit matrix product behind ff_fp8_matmul (see include/ff.h).
#pragma once

#include "ff_internal.cuh"

namespace ff {

inline int fp8_stride(int k) { return (k + 15) & ~15; }

struct Fp8Gemm {
  const uint8_t *a, *b;   // e4m3 [M, fp8_stride(K)], [N, fp8_stride(K)]
  const float *sa, *sb;   // [k blocks, M]; [k blocks, N] or, b_tiles, [k blocks, ceil(N / 128)]
  bool b_tiles;
  int M, N, K;
  const float* bias;      // [N] or null
  bool relu, out_bf16;
  void* c;
  long long ldc;
  int* status;            // latches timeouts
};

ff_status fp8_gemm(const Fp8Gemm& g, cudaStream_t st);

}  // namespace ff
