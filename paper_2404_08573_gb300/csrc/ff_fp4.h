// 4-bit matrices (see ff_fp4_quantize in include/ff.h): their layout, and the
// product behind ff_fp4_matmul.
#pragma once

#include "ff_internal.cuh"

namespace ff {

constexpr int kFp4Block = 32;       // contraction indices that share a scale
constexpr int kFp4ScaleTile = 512;  // bytes of a scale tile: 128 rows x 4 blocks

inline int fp4_blocks(int k) { return cdiv(k, kFp4Block); }
inline int fp4_stride(int k) { return fp4_blocks(k) * 16; }
inline long long fp4_scale_bytes(int rows, int k) { return (long long)cdiv(rows, 128) * cdiv(k, 128) * kFp4ScaleTile; }

struct Fp4Gemm {
  const uint8_t *a, *b;    // e2m1 pairs [M, fp4_stride(K)], [N, fp4_stride(K)]
  const uint8_t *sa, *sb;  // scale tiles
  int M, N, K;
  const float* bias;       // [N] or null
  bool relu, out_bf16;
  void* c;
  long long ldc;
  int* status;             // latches timeouts
};

ff_status fp4_gemm(const Fp4Gemm& g, cudaStream_t st);

}  // namespace ff
