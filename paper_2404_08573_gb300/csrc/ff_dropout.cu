// Dropout from the library's counter-based generator: the mask is a function
// of (seed, offset, element) and is formed wherever it is needed, forward and
// backward, so nothing of it is stored or read.
//
// One 64-bit word of the generator covers four neighbouring elements of a row,
// 16 bits each.
#include <cmath>

#include "ff_api_internal.h"
#include "ff_ptx.cuh"
#include "ff_vec.cuh"

namespace ff {
namespace {

constexpr unsigned long long kStreamDropout = 7;

struct DropShape {
  long long rows, cols, ldx, ldr, ldy;
  long long words;        // of the generator per row
  long long count, total; // elements; units
  long long span, step;   // elements of a row as the units count them, and of a unit
  long long dr, dc;       // a block's width (256 units) further on: rows, and elements within a row
  int small;              // positions fit 32 bits
  unsigned long long state, offset;
  const unsigned long long* offset_dev;
  uint32_t thresh;        // elements whose 16 bits are below it are dropped
  float scale;
};

constexpr int kDropThreads = 256;
constexpr int kDropUnits = 4;  // units per thread, loaded together

// How a unit lies in memory:
//   FLAT   a 16-byte vector of one long row (dense, whole vectors)
//   ROWS   a 16-byte vector of a row: every row starts on 16 bytes and holds
//          whole vectors, at any stride
//   DENSE  a 16-byte vector of a dense matrix of any width: it may start
//          anywhere in a row, so its bits come from up to one word more, and
//          it may cross into the next row
//   WORDS  the four elements of one word, one by one (anything else)
enum DropMode { FLAT, ROWS, DENSE, WORDS };

// A block takes kDropUnits * 256 consecutive units.  Bound by HBM: the
// generator's 25 or so integer instructions per word of four elements stay
// under the time that reading and writing them takes (16384 x 8192 bf16 with
// residual: 115 us, 7.0 TB/s).
template <typename T, DropMode MODE, bool RES>
__global__ void __launch_bounds__(kDropThreads) k_dropout(const T* x, const T* res, T* y, DropShape s) {
  constexpr int E = MODE == WORDS ? 4 : 16 / (int)sizeof(T);  // elements of a unit
  constexpr int A = MODE == WORDS ? 1 : E;                    // elements of an access
  using V = Vec<T, A>;
  ptx::griddep_wait();
  const unsigned long long off = s.offset + (s.offset_dev ? *s.offset_dev : 0ull);
  const long long i0 = (long long)blockIdx.x * (kDropThreads * kDropUnits) + threadIdx.x;
  // row and column (in elements) of this thread's units, one block's width apart
  const long long first = i0 * s.step;
  long long r = 0, c = first;
  if (MODE != FLAT && s.rows > 1) {
    r = s.small ? (long long)((uint32_t)first / (uint32_t)s.span) : first / s.span;
    c = first - r * s.span;
  }
  typename V::Raw a[kDropUnits][E / A], b[kDropUnits][E / A];
  long long rr[kDropUnits], cc[kDropUnits];
#pragma unroll
  for (int u = 0; u < kDropUnits; ++u) {
    rr[u] = r;
    cc[u] = c;
    if (MODE != FLAT) {
      r += s.dr;
      c += s.dc;
      if (c >= s.span) {
        c -= s.span;
        ++r;
      }
    }
    const long long i = i0 + (long long)u * kDropThreads;
    if (i >= s.total) continue;
    if (MODE == DENSE && (i + 1) * E > s.count) continue;  // the last, partial vector: below
#pragma unroll
    for (int e = 0; e < E; e += A)
      if (MODE != WORDS || cc[u] + e < s.cols) {
        a[u][e / A] = V::load(x + (MODE == FLAT || MODE == DENSE ? i * E : rr[u] * s.ldx + cc[u] + e));
        if constexpr (RES) b[u][e / A] = V::load(res + (MODE == FLAT || MODE == DENSE ? i * E : rr[u] * s.ldr + cc[u] + e));
      }
  }
  auto key = [&](unsigned long long w) { return s.state + (off + w + 1) * kGamma; };  // of word w; the next is kGamma on
  auto one = [&](float v, float q, uint32_t bits) { return bits >= s.thresh ? fmaf(v, s.scale, q) : q; };
#pragma unroll
  for (int u = 0; u < kDropUnits; ++u) {
    const long long i = i0 + (long long)u * kDropThreads;
    if (i >= s.total) break;
    unsigned long long w[E / 4];
    // units of whole words follow one another as the words do
    const unsigned long long w0 = MODE == DENSE ? (unsigned long long)(rr[u] * s.words + (cc[u] >> 2))
                                                : (unsigned long long)i * (E / 4);
    const unsigned long long k0 = key(w0);
    if constexpr (MODE == DENSE) if (cc[u] + E > s.cols || (i + 1) * E > s.count) {
      // across rows, or past the end: a word whenever the next element is in another
      const int there = (int)min((long long)E, s.count - i * E);
      float v[E], q[E];
      if (there == E) {
        V::unpack(a[u][0], v);
        if constexpr (RES) V::unpack(b[u][0], q);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (e < there) {
            Vec<T, 1>::unpack(Vec<T, 1>::load(x + i * E + e), reinterpret_cast<float(&)[1]>(v[e]));
            if constexpr (RES)
              Vec<T, 1>::unpack(Vec<T, 1>::load(res + i * E + e), reinterpret_cast<float(&)[1]>(q[e]));
          }
      }
      unsigned long long word = (unsigned long long)(rr[u] * s.words + (cc[u] >> 2)), m = 0;
      long long ec = cc[u];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (e == 0 || (ec & 3) == 0) m = sm64_mix(key(word));
        q[e] = one(v[e], RES ? q[e] : 0.f, (uint32_t)(m >> (16 * (ec & 3))) & 0xFFFFu);
        ++ec;
        if (ec == s.cols) ec = 0;
        if ((ec & 3) == 0) ++word;  // the next word of the row, or the first of the next
      }
      if (there == E) {
        V::store(y + i * E, q);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (e < there) Vec<T, 1>::store(y + i * E + e, reinterpret_cast<const float(&)[1]>(q[e]));
      }
      continue;
    }
#pragma unroll
    for (int j = 0; j < E / 4; ++j) w[j] = sm64_mix(k0 + j * kGamma);
    if (MODE == DENSE) {
      const int sh = 16 * (int)(cc[u] & 3);
      if (sh) {
        const unsigned long long last = sm64_mix(k0 + E / 4 * kGamma);
#pragma unroll
        for (int j = 0; j < E / 4; ++j) w[j] = w[j] >> sh | (j + 1 < E / 4 ? w[j + 1] : last) << (64 - sh);
      }
    }
#pragma unroll
    for (int e = 0; e < E; e += A) {
      if (MODE == WORDS && cc[u] + e >= s.cols) break;
      float v[A], q[A];
      V::unpack(a[u][e / A], v);
      if constexpr (RES) {
        V::unpack(b[u][e / A], q);
      } else {
#pragma unroll
        for (int t = 0; t < A; ++t) q[t] = 0.f;
      }
#pragma unroll
      for (int t = 0; t < A; ++t)
        q[t] = one(v[t], q[t], (uint32_t)(w[(e + t) / 4] >> (16 * ((e + t) & 3))) & 0xFFFFu);
      V::store(y + (MODE == FLAT || MODE == DENSE ? i * E : rr[u] * s.ldy + cc[u] + e), q);
    }
  }
}

template <typename T>
ff_status dropout_t(const T* x, const T* res, T* y, DropShape s, cudaStream_t st) {
  constexpr int E = 16 / (int)sizeof(T);
  const double bytes = (double)s.rows * s.cols * sizeof(T) * (res ? 3 : 2);
  const bool one_row = s.rows == 1;
  const bool dense = one_row || (s.ldx == s.cols && s.ldy == s.cols && (!res || s.ldr == s.cols));
  s.words = (s.cols + 3) / 4;
  // rows that follow one another whole, words included, are one long row
  if (dense && s.cols % 4 == 0) {
    s.cols *= s.rows;
    s.words *= s.rows;
    s.rows = 1;
    s.ldx = s.ldy = s.ldr = s.cols;
  }
  auto on16 = [&](bool rows) {
    auto ok = [&](const T* p, long long ld) { return rows_aligned(p, rows && s.rows > 1 ? ld : 0, sizeof(T), 16); };
    return ok(x, s.ldx) && ok(y, s.ldy) && (!res || ok(res, s.ldr));
  };
  const DropMode mode = s.cols % E == 0 && on16(true) ? (s.rows == 1 ? FLAT : ROWS)
                        : dense && on16(false)        ? DENSE
                                                      : WORDS;
  const long long e = mode == WORDS ? 4 : E;  // elements of a unit
  s.count = s.rows * s.cols;
  // positions run over rows of `span` elements: whole words where units are words
  s.span = mode == WORDS ? s.words * 4 : s.cols;
  s.total = mode == DENSE ? (s.count + e - 1) / e : s.rows * (s.span / e);
  s.step = e;
  s.dr = kDropThreads * e / s.span;
  s.dc = kDropThreads * e % s.span;
  s.small = s.rows * s.span <= 0x7FFFFFFFll;
  const long long blocks = (s.total + kDropThreads * kDropUnits - 1) / (kDropThreads * kDropUnits);
  if (blocks > 0x7FFFFFFFll) return FF_ERR_UNSUPPORTED;
  PdlLaunch l(dim3((unsigned)blocks), dim3(kDropThreads), st);
  auto go = [&](auto* plain, auto* with) { return cudaLaunchKernelEx(&l.cfg, res ? with : plain, x, res, y, s); };
  FF_LAUNCH(K_DROPOUT, bytes, st,
            mode == FLAT    ? go(k_dropout<T, FLAT, false>, k_dropout<T, FLAT, true>)
            : mode == ROWS  ? go(k_dropout<T, ROWS, false>, k_dropout<T, ROWS, true>)
            : mode == DENSE ? go(k_dropout<T, DENSE, false>, k_dropout<T, DENSE, true>)
                            : go(k_dropout<T, WORDS, false>, k_dropout<T, WORDS, true>),
            "dropout");
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
