// Dropout from the library's counter-based generator: the mask is a function
// of (seed, offset, element) and is formed wherever it is needed, forward and
// backward, so nothing of it is stored or read.
//
// One 64-bit word of the generator covers four neighbouring elements of a row,
// 16 bits each.
#include <cmath>

#include "ff_api_internal.h"
#include "ff_vec.cuh"

namespace ff {
namespace {

constexpr unsigned long long kStreamDropout = 7;

struct DropShape {
  long long rows, cols, words, ldx, ldr, ldy;  // words: per row
  unsigned long long state, offset;
  const unsigned long long* offset_dev;
  uint32_t thresh;  // elements whose 16 bits are below it are dropped
  float scale;
};

// One thread per word: four elements of a row, element by element.
template <typename T>
__global__ void __launch_bounds__(256) k_dropout(const T* x, const T* res, T* y, DropShape s) {
  const unsigned long long off = s.offset + (s.offset_dev ? *s.offset_dev : 0ull);
  const long long total = s.rows * s.words;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < total;
       i += (long long)gridDim.x * blockDim.x) {
    const long long r = i / s.words, j0 = (i - r * s.words) * 4;
    const unsigned long long w = sm64_mix(s.state + (off + (unsigned long long)i + 1) * kGamma);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const long long j = j0 + e;
      if (j >= s.cols) break;
      float v[1], q[1] = {0.f};
      Vec<T, 1>::unpack(Vec<T, 1>::load(x + r * s.ldx + j), v);
      if (res) Vec<T, 1>::unpack(Vec<T, 1>::load(res + r * s.ldr + j), q);
      const bool keep = ((uint32_t)(w >> (16 * e)) & 0xFFFFu) >= s.thresh;
      q[0] = keep ? fmaf(v[0], s.scale, q[0]) : q[0];
      Vec<T, 1>::store(y + r * s.ldy + j, q);
    }
  }
}

template <typename T>
ff_status dropout_t(const T* x, const T* res, T* y, const DropShape& s, cudaStream_t st) {
  const long long total = s.rows * s.words;
  const long long blocks = (total + 255) / 256;
  const unsigned grid = (unsigned)(blocks < 152 * 64 ? blocks : 152 * 64);
  const double bytes = (double)s.rows * s.cols * sizeof(T) * (res ? 3 : 2);
  FF_LAUNCH(K_DROPOUT, bytes, st, (k_dropout<T><<<grid, 256, 0, st>>>(x, res, y, s), cudaGetLastError()), "dropout");
  return FF_OK;
}

}  // namespace
}  // namespace ff

using namespace ff;

extern "C" FF_API long long ff_dropout_words(long long rows, long long cols) {
  return rows > 0 && cols > 0 ? rows * ((cols + 3) / 4) : 0;
}

extern "C" FF_API ff_status ff_dropout(const void* x, long long ldx, long long rows, long long cols, double p,
                                       unsigned long long seed, unsigned long long offset,
                                       const unsigned long long* offset_dev, const void* residual, long long ldr,
                                       ff_precision prec, void* y, long long ldy, void* stream) {
  if (rows < 0 || cols < 0 || !(p >= 0.0 && p <= 1.0) || (prec != FF_FP32 && prec != FF_BF16))
    return FF_ERR_INVALID_ARG;
  if (rows == 0 || cols == 0) return FF_OK;
  const int es = prec == FF_BF16 ? 2 : 4;
  auto bad = [&](const void* q, long long ld) {
    return !q || reinterpret_cast<uintptr_t>(q) % es != 0 || (ld < cols && rows > 1);
  };
  if (bad(x, ldx) || bad(y, ldy) || (residual && bad(residual, ldr)) ||
      (offset_dev && reinterpret_cast<uintptr_t>(offset_dev) % 8 != 0))
    return FF_ERR_INVALID_ARG;
  if (rows > (1ll << 62) / ((cols + 3) / 4 * 4)) return FF_ERR_INVALID_ARG;
  DropShape s{};
  s.rows = rows;
  s.cols = cols;
  s.words = (cols + 3) / 4;
  s.ldx = ldx;
  s.ldr = ldr;
  s.ldy = ldy;
  s.state = sm64_mix((seed << 8) | kStreamDropout);
  s.offset = offset;
  s.offset_dev = offset_dev;
  s.thresh = (uint32_t)std::nearbyint(p * 65536.0);
  s.scale = s.thresh < 65536u ? 65536.f / (float)(65536u - s.thresh) : 0.f;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (prec == FF_BF16)
    return dropout_t(static_cast<const bf16*>(x), static_cast<const bf16*>(residual), static_cast<bf16*>(y), s, st);
  return dropout_t(static_cast<const float*>(x), static_cast<const float*>(residual), static_cast<float*>(y), s, st);
}
