// 4-bit matrices (e2m1 values, a power-of-two scale per block of 32 along the
// contraction): the quantizer, its inverse, and the C entries of all three
// operations.
#include <algorithm>

#include <cuda_fp16.h>

#include "ff_api_internal.h"
#include "ff_fp4.h"
#include "ff_fp8.h"
#include "ff_ptx.cuh"
#include "ff_vec.cuh"

namespace ff {
namespace {

// The scale of a block by its largest magnitude, given as the exponent field
// of that float: 2^(floor(log2 amax) - 2), which maps amax to [4, 8), held as
// its own exponent field and at least 2^-127 (field 0, also for a block of
// zeros).  255 marks a block that holds an infinity or a NaN.
__device__ __forceinline__ uint32_t scale_field(uint32_t field) { return field == 255u ? 255u : field < 2u ? 0u : field - 2u; }
// 1 / scale: 2^(127 - field), exact in fp32 (for the mark -infinity: whatever the
// block's codes are then, it stands for NaN).
__device__ __forceinline__ float scale_inverse(uint32_t field) { return __uint_as_float((254u - field) << 23); }

// Four pairs times f as e2m1 codes (to nearest even, saturating), the first lowest.
__device__ __forceinline__ uint32_t e2m1x8(const uint64_t (&p)[4], float f) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 t = ptx::unpack2(ptx::mul2(p[i], ptx::pack2(f, f)));
    v[2 * i] = t.x;
    v[2 * i + 1] = t.y;
  }
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}
// The two values of a byte, the low four bits' first.
__device__ __forceinline__ float2 e2m1x2_values(uint32_t byte) {
  uint32_t h;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t}"
      : "=r"(h)
      : "r"(byte));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// Eight values of a row as loaded, as in the 8-bit quantizer: bf16 in pairs
// (the low half first), or fp32; magnitudes are compared as integers.
template <typename T>
struct Eight;
template <>
struct Eight<bf16> {
  static constexpr int WORDS = 4, PER = 2;
  // the larger magnitudes of two words (of a NaN and another: NaN)
  static __device__ __forceinline__ uint32_t abs_max(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("{\n\t.reg .b32 p, q;\n\tabs.bf16x2 p, %1;\n\tabs.bf16x2 q, %2;\n\tmax.NaN.bf16x2 %0, p, q;\n\t}" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ uint32_t max_of(uint32_t a, uint32_t b) {  // of magnitudes
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ float value(const uint32_t (&w)[WORDS], int e) {
    return __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
  }
  static __device__ __forceinline__ uint32_t field(uint32_t w, int h) { return h ? w >> 23 : (w >> 7) & 0xFFu; }  // of a magnitude
  static __device__ __forceinline__ uint64_t pair(const uint32_t (&w)[WORDS], int i) {  // values 2i, 2i + 1
    return ptx::pack2(w[i] << 16, w[i] & 0xFFFF0000u);
  }
};
template <>
struct Eight<float> {
  static constexpr int WORDS = 8, PER = 1;
  static __device__ __forceinline__ uint32_t abs_max(uint32_t a, uint32_t b) {
    float r;
    asm("{\n\t.reg .f32 p, q;\n\tabs.f32 p, %1;\n\tabs.f32 q, %2;\n\tmax.NaN.f32 %0, p, q;\n\t}"
        : "=f"(r)
        : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)));
    return __float_as_uint(r);
  }
  static __device__ __forceinline__ uint32_t max_of(uint32_t a, uint32_t b) { return max(a, b); }
  static __device__ __forceinline__ float value(const uint32_t (&w)[WORDS], int e) { return __uint_as_float(w[e]); }
  static __device__ __forceinline__ uint32_t field(uint32_t w, int) { return w >> 23; }
  static __device__ __forceinline__ uint64_t pair(const uint32_t (&w)[WORDS], int i) { return ptx::pack2(w[2 * i], w[2 * i + 1]); }
};

constexpr int QT = 128;  // a tile: 128 x 128 values, one scale tile each way
constexpr int kQThreads = 256;
constexpr int kPitch = 17;  // words a staged column: 16, and one against bank conflicts

// One thread block per 128 x 128 tile; a warp takes 32 rows x 64 columns of
// it, a thread 8 x 8 (all its loads in flight together), so that both a row's
// block of 32 columns and a column's block of 32 rows lie within a warp and
// their maxima take two shuffles.  Bound by HBM and, at two thirds of the
// issue slots, by the maxima and conversions of both directions: 4096 x 8192 bf16
// both ways 20.6 us, 5.0 TB/s (floor 15.5); 2000 x 784 fp32 4.6 us, a launch and one round of
// 112 blocks.
// LOAD: bytes of x per access that its rows' alignment allows.
template <typename T, int LOAD>
__global__ void __launch_bounds__(kQThreads, sizeof(T) == 2 ? 4 : 2)
    k_fp4_quantize(const T* x, long long ldx, int rows, int k, uint8_t* q, uint8_t* scale, uint8_t* qt, uint8_t* scale_t,
                   int ldq, int ldqt, int ktiles, int rtiles) {
  using E = Eight<T>;
  constexpr int W = E::WORDS, PER = E::PER;
  __shared__ uint32_t tq[QT * kPitch];
  __shared__ __align__(16) uint8_t sc[kFp4ScaleTile], sct[kFp4ScaleTile];
  ptx::griddep_wait();
  const int kt = blockIdx.x % ktiles, rt = blockIdx.x / ktiles;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int wr = warp >> 1, wc = warp & 1, rg = lane >> 3, cg = lane & 7;
  const int r_in = wr * 32 + rg * 8, c_in = wc * 64 + cg * 8;
  const int row0 = rt * QT + r_in, c0 = kt * QT + c_in;
  uint32_t v[8][W];
  const T* p = x + (long long)row0 * ldx + c0;
  if (LOAD == 16 && c0 + 8 <= k) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < W / 4; ++j)
        *reinterpret_cast<uint4*>(&v[i][4 * j]) =
            row0 + i < rows ? reinterpret_cast<const uint4*>(p + i * ldx)[j] : make_uint4(0, 0, 0, 0);
  } else if (LOAD == 4 && c0 + 8 <= k) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < W; ++j) v[i][j] = row0 + i < rows ? reinterpret_cast<const uint32_t*>(p + i * ldx)[j] : 0u;
  } else {
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
  if (q) {
    uint8_t* const to = q + (long long)row0 * ldq + c0 / 2;
    uint32_t m[8 / PER];  // word j: rows j PER .. (one per half of the word)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t t = E::abs_max(v[i][0], v[i][1]);
#pragma unroll
      for (int j = 2; j < W; ++j) t = E::abs_max(t, v[i][j]);
      if constexpr (PER == 2) {
        t = max(t & 0xFFFFu, t >> 16);
        m[i / 2] = i & 1 ? m[i / 2] | t << 16 : t;
      } else {
        m[i] = t;
      }
    }
#pragma unroll
    for (int o = 1; o <= 2; o *= 2)
#pragma unroll
      for (int j = 0; j < 8 / PER; ++j) m[j] = E::max_of(m[j], __shfl_xor_sync(0xffffffffu, m[j], o));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t f = scale_field(E::field(m[i / PER], i % PER));
      uint64_t y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = E::pair(v[i], e);
      // ldq covers whole blocks of 32: eight columns lie inside or outside
      if (row0 + i < rows && c0 / 2 < ldq) *reinterpret_cast<uint32_t*>(to + (long long)i * ldq) = e2m1x8(y, scale_inverse(f));
      if ((cg & 3) == 0) sc[(rg * 8 + i) * 16 + wr * 4 + wc * 2 + (cg >> 2)] = (uint8_t)f;
    }
  }
  if (qt) {
    uint32_t m[W];  // word j: columns j PER ..
#pragma unroll
    for (int j = 0; j < W; ++j) {
      m[j] = E::abs_max(v[0][j], v[1][j]);
#pragma unroll
      for (int i = 2; i < 8; ++i) m[j] = E::abs_max(m[j], v[i][j]);
    }
#pragma unroll
    for (int o = 8; o <= 16; o *= 2)
#pragma unroll
      for (int j = 0; j < W; ++j) m[j] = E::max_of(m[j], __shfl_xor_sync(0xffffffffu, m[j], o));
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t f = scale_field(E::field(m[e / PER], e % PER));
      uint64_t y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = ptx::pack2(E::value(v[2 * i], e), E::value(v[2 * i + 1], e));
      const int c = c_in + e;
      tq[c * kPitch + wr * 4 + rg] = e2m1x8(y, scale_inverse(f));
      if (rg == 0) sct[(c & 31) * 16 + (c >> 5) * 4 + wr] = (uint8_t)f;
    }
  }
  __syncthreads();
  if (q && threadIdx.x < 32)
    reinterpret_cast<uint4*>(scale + ((long long)rt * ktiles + kt) * kFp4ScaleTile)[threadIdx.x] = reinterpret_cast<uint4*>(sc)[threadIdx.x];
  if (qt) {
    if (threadIdx.x >= 32 && threadIdx.x < 64)
      reinterpret_cast<uint4*>(scale_t + ((long long)kt * rtiles + rt) * kFp4ScaleTile)[threadIdx.x - 32] =
          reinterpret_cast<uint4*>(sct)[threadIdx.x - 32];
    // 4 threads per column of the tile, 16 bytes (a block of 32 rows) each
    const int u = threadIdx.x & 3, at = rt * (QT / 2) + u * 16;
    if (at < ldqt) {
#pragma unroll
      for (int c = threadIdx.x >> 2; c < QT; c += kQThreads / 4) {
        const long long col = (long long)kt * QT + c;
        if (col >= k) break;
        const uint32_t* t = tq + c * kPitch + u * 4;
        *reinterpret_cast<uint4*>(qt + col * ldqt + at) = make_uint4(t[0], t[1], t[2], t[3]);
      }
    }
  }
}

// The rows alone: a lane takes eight values of a row at a time (four lanes a
// block of 32), so a warp 256 columns: of rows j, j + 32, j + 64 and j + 96 of a
// scale tile, with their loads in flight together, since these rows' scale bytes
// lie side by side (rows one after the other: 3 us of 18 for 4-byte stores all
// over the tiles, 4096 x 8192 bf16).  Rows past the matrix write zero scales.
// Bound by HBM: x once, its half-bytes once: 4096 x 8192 bf16 13.7 us, 6.2 TB/s.
template <typename T, int LOAD>
__global__ void __launch_bounds__(kQThreads)
    k_fp4_rows(const T* x, long long ldx, int rows, int k, uint8_t* q, uint8_t* scale, int ldq, int ktiles, int strips, int units) {
  using E = Eight<T>;
  constexpr int W = E::WORDS, PER = E::PER;
  ptx::griddep_wait();
  const int lane = threadIdx.x & 31;
  const int unit = blockIdx.x * (kQThreads / 32) + (threadIdx.x >> 5);  // (row tile, j, strip of 256 columns)
  if (unit >= units) return;
  const int strip = unit % strips, rj = unit / strips, j0 = rj & 31, rt = rj >> 5;
  const int row0 = rt * QT + j0, c0 = strip * 256 + lane * 8;
  uint32_t v[4][W];
  if constexpr (sizeof(T) == 4 && LOAD == 4) {
    // A lane's own values from rows that only four bytes align would be eight
    // times the wavefronts (4096 x 8191: 36 us, so 25): the warp loads them side by side.
    // (bf16, with half the bytes, was not faster so, nor were the tiles above.)
    __shared__ __align__(16) uint32_t staged[kQThreads / 32][4 * 256];
    uint32_t* const own = staged[threadIdx.x >> 5];
#pragma unroll
    for (int h = 0; h < 4; h += 2) {
      uint32_t t[16];
#pragma unroll
      for (int n = 0; n < 16; ++n) {
        const int r = row0 + (h + n / 8) * 32, c = strip * 256 + n % 8 * 32 + lane;
        t[n] = r < rows && c < k ? Vec<T, 1>::load(x + (long long)r * ldx + c) : 0u;
      }
#pragma unroll
      for (int n = 0; n < 16; ++n) own[(h * 8 + n) * 32 + lane] = t[n];
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < W / 4; ++j)
        *reinterpret_cast<uint4*>(&v[i][4 * j]) = reinterpret_cast<const uint4*>(own + i * 256 + lane * 8)[j];
  } else {
    const T* p = x + (long long)row0 * ldx + c0;
#pragma unroll
    for (int i = 0; i < 4; ++i, p += 32 * ldx) {
      const bool in = row0 + 32 * i < rows;
      if (LOAD == 16 && c0 + 8 <= k) {
#pragma unroll
        for (int j = 0; j < W / 4; ++j)
          *reinterpret_cast<uint4*>(&v[i][4 * j]) = in ? reinterpret_cast<const uint4*>(p)[j] : make_uint4(0, 0, 0, 0);
      } else if (LOAD == 4 && c0 + 8 <= k) {
#pragma unroll
        for (int j = 0; j < W; ++j) v[i][j] = in ? reinterpret_cast<const uint32_t*>(p)[j] : 0u;
      } else {
#pragma unroll
        for (int j = 0; j < W; ++j) {
          uint32_t w = 0;
#pragma unroll
          for (int h = 0; h < PER; ++h)
            if (in && c0 + j * PER + h < k) w |= (uint32_t)Vec<T, 1>::load(p + j * PER + h) << (16 * h);
          v[i][j] = w;
        }
      }
    }
  }
  uint32_t s[4];
  uint8_t* to = q + (long long)row0 * ldq + c0 / 2;
#pragma unroll
  for (int i = 0; i < 4; ++i, to += 32ll * ldq) {
    uint32_t m = E::abs_max(v[i][0], v[i][1]);
#pragma unroll
    for (int j = 2; j < W; ++j) m = E::abs_max(m, v[i][j]);
    if constexpr (PER == 2) m = max(m & 0xFFFFu, m >> 16);
#pragma unroll
    for (int o = 1; o <= 2; o *= 2) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    const uint32_t f = scale_field(E::field(m, 0));
    uint64_t y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = E::pair(v[i], e);
    if (row0 + 32 * i < rows && c0 / 2 < ldq) *reinterpret_cast<uint32_t*>(to) = e2m1x8(y, scale_inverse(f));
    // the tile's four blocks' bytes of this row, to its first lane
    s[i] = f | __shfl_down_sync(0xffffffffu, f, 4) << 8;
    s[i] |= __shfl_down_sync(0xffffffffu, s[i], 8) << 16;
  }
  const int tile = strip * 2 + (lane >> 4);  // of 128 columns, along k
  if ((lane & 15) == 0 && tile < ktiles)
    *reinterpret_cast<uint4*>(scale + ((long long)rt * ktiles + tile) * kFp4ScaleTile + j0 * 16) = make_uint4(s[0], s[1], s[2], s[3]);
}

__device__ __forceinline__ float scale_value(uint32_t field) {  // 2^(field - 127)
  return __uint_as_float(field == 0u ? 0x00400000u : field == 255u ? 0x7FC00000u : field << 23);
}

// The values of a unit of N columns from its N / 2 bytes.
template <int N>
__device__ __forceinline__ void unit_values(float (&v)[N], uint32_t w, float s) {
#pragma unroll
  for (int h = 0; h < N / 2; ++h) {
    const float2 t = e2m1x2_values(w >> (8 * h));
    v[2 * h] = t.x * s;
    v[2 * h + 1] = t.y * s;
  }
}
struct DequantArgs {
  const uint8_t *q, *scale;
  int rows, k, ldq, ktiles;
  long long ldy;
  int lanes_log, strips, groups;
};

// y = value * scale, exact in either type.  A thread takes the same unit of
// columns of rows j, j + 32, j + 64 and j + 96 of a scale tile, with their loads in
// flight together: their scales come with one load.  A block of 256 covers
// 2^lanes_log units side by side and the rest of its threads' j.  WIDE: y's rows
// are 16-byte aligned and a unit is that many; else one column.  (Rows one after
// the other, each with its own scale load, left it bound by the instructions of
// their addresses: 4096 x 8192 to bf16 13.5 us, now 11.7, at 7.2 TB/s HBM's.  To fp32
// 24; with units of 8 there, stores of half sectors, 34.)
template <typename T, bool WIDE>
__global__ void __launch_bounds__(256) k_fp4_dequantize(const DequantArgs a, T* y) {
  constexpr int UNIT = WIDE ? 16 / (int)sizeof(T) : 1;
  ptx::griddep_wait();
  const int lanes = 1 << a.lanes_log, per = 256 >> a.lanes_log;
  const int strip = blockIdx.x % a.strips, g = blockIdx.x / a.strips;
  const int j = g % a.groups * per + (threadIdx.x >> a.lanes_log), rt = g / a.groups;
  const long long row0 = (long long)rt * QT + j;
  const long long c = ((long long)strip * lanes + (threadIdx.x & (lanes - 1))) * UNIT;
  if (c >= a.k || row0 >= a.rows) return;
  const uint8_t* p = a.q + row0 * a.ldq + c / 2;
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i, p += 32ll * a.ldq) {
    w[i] = 0u;
    if (row0 + 32 * i < a.rows)
      w[i] = UNIT == 8   ? __ldg(reinterpret_cast<const uint32_t*>(p))
             : UNIT == 4 ? (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(p))
                         : (uint32_t)__ldg(p);
  }
  const uint4 s4 = __ldg(reinterpret_cast<const uint4*>(a.scale + ((long long)rt * a.ktiles + c / QT) * kFp4ScaleTile + j * 16));
  const uint32_t fields[4] = {s4.x, s4.y, s4.z, s4.w};
  const int shift = (int)(c / kFp4Block & 3) * 8;
  T* to = y + row0 * a.ldy + c;
#pragma unroll
  for (int i = 0; i < 4; ++i, to += 32 * a.ldy) {
    if (row0 + 32 * i >= a.rows) break;
    const float s = scale_value(fields[i] >> shift & 0xFFu);
    if constexpr (WIDE) {
      float v[UNIT];
      unit_values<UNIT>(v, w[i], s);
      if (c + UNIT <= a.k) {
        Vec<T, UNIT>::store(to, v);
      } else {
#pragma unroll
        for (int e = 0; e < UNIT; ++e) {
          const float one[1] = {v[e]};
          if (c + e < a.k) Vec<T, 1>::store(to + e, one);
        }
      }
    } else {
      const float2 t = e2m1x2_values(w[i]);
      const float one[1] = {(c & 1 ? t.y : t.x) * s};
      Vec<T, 1>::store(to, one);
    }
  }
}

// The same where y's rows are not 16-byte aligned and there are many: units of 8
// columns (2^lanes_log <= 32 of them), which a warp passes through shared memory,
// so that its stores of STORE bytes lie side by side: 4096 x 8191 to bf16 32 us, 4095 x
// 8190 22, to fp32 32; a value a thread 55 each.  (But 154 x 1789 3.0 for 1.7: a
// million values divide them.)
template <typename T, int STORE>
__global__ void __launch_bounds__(256) k_fp4_dequantize_staged(const DequantArgs a, T* y) {
  constexpr int A = STORE / (int)sizeof(T), N = 16 / (int)sizeof(T);  // values a store; and a staging store
  __shared__ __align__(16) T staged[256 / 32][4][256];
  ptx::griddep_wait();
  const int lane = threadIdx.x & 31, lanes = 1 << a.lanes_log, per = 256 >> a.lanes_log, wide_log = a.lanes_log + 3;
  const int strip = blockIdx.x % a.strips, g = blockIdx.x / a.strips;
  const int j = g % a.groups * per + (threadIdx.x >> a.lanes_log), rt = g / a.groups;
  const long long row0 = (long long)rt * QT + j, c0 = (long long)strip << wide_log;
  const long long c = c0 + (threadIdx.x & (lanes - 1)) * 8;
  uint32_t w[4] = {0u, 0u, 0u, 0u};
  uint4 s4 = make_uint4(0, 0, 0, 0);
  if (c < a.k && row0 < a.rows) {
    const uint8_t* p = a.q + row0 * a.ldq + c / 2;
#pragma unroll
    for (int i = 0; i < 4; ++i, p += 32ll * a.ldq)
      if (row0 + 32 * i < a.rows) w[i] = __ldg(reinterpret_cast<const uint32_t*>(p));
    s4 = __ldg(reinterpret_cast<const uint4*>(a.scale + ((long long)rt * a.ktiles + c / QT) * kFp4ScaleTile + j * 16));
  }
  const uint32_t fields[4] = {s4.x, s4.y, s4.z, s4.w};
  const int shift = (int)(c / kFp4Block & 3) * 8;
  auto& own = staged[threadIdx.x >> 5];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float v[8];
    unit_values<8>(v, w[i], scale_value(fields[i] >> shift & 0xFFu));
#pragma unroll
    for (int h = 0; h < 8; h += N) {
      float t[N];
#pragma unroll
      for (int e = 0; e < N; ++e) t[e] = v[h + e];
      Vec<T, N>::store(&own[i][lane * 8 + h], t);
    }
  }
  __syncwarp();
  // the warp's 256 values of each i: 2^wide_log columns of one row or of several
  const int j0 = g % a.groups * per + ((threadIdx.x & ~31) >> a.lanes_log);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int n = 0; n < 256 / 32 / A; ++n) {
      const int at = (n * 32 + lane) * A;
      const long long row = (long long)rt * QT + 32 * i + j0 + (at >> wide_log), col = c0 + (at & ((1 << wide_log) - 1));
      if (row >= a.rows || col >= a.k) continue;
      T* const to = y + row * a.ldy + col;
      if (col + A <= a.k) *reinterpret_cast<typename Vec<T, A>::Raw*>(to) = *reinterpret_cast<const typename Vec<T, A>::Raw*>(&own[i][at]);
      else *to = own[i][at];
    }
}

template <typename T>
ff_status quantize_t(const T* x, long long ldx, int rows, int k, uint8_t* q, uint8_t* scale, uint8_t* qt, uint8_t* scale_t,
                     cudaStream_t st) {
  const int ktiles = cdiv(k, QT), rtiles = cdiv(rows, QT);
  const long long blocks = (long long)ktiles * rtiles;
  if (blocks > 0x7FFFFFFFll) return FF_ERR_UNSUPPORTED;
  const double bytes = (double)rows * k * (sizeof(T) + (q ? 0.5 : 0) + (qt ? 0.5 : 0));
  const int ldq = fp4_stride(k), ldqt = fp4_stride(rows);
  const int load = rows_aligned(x, ldx, sizeof(T), 16) ? 16 : rows_aligned(x, ldx, sizeof(T), 4) ? 4 : (int)sizeof(T);
  if (!qt) {
    const int strips = cdiv(k, 256);
    const long long units = (long long)strips * rtiles * 32;
    if (units > 0x7FFFFFFFll) return FF_ERR_UNSUPPORTED;
    auto* const rows_kernel = load == 16 ? k_fp4_rows<T, 16> : load == 4 ? k_fp4_rows<T, 4> : k_fp4_rows<T, sizeof(T)>;
    PdlLaunch l(dim3((unsigned)cdiv(units, kQThreads / 32)), dim3(kQThreads), st);
    FF_LAUNCH(K_FP4_QUANT, bytes, st,
              cudaLaunchKernelEx(&l.cfg, rows_kernel, x, ldx, rows, k, q, scale, ldq, ktiles, strips, (int)units), "4-bit quantize");
    return FF_OK;
  }
  PdlLaunch l(dim3((unsigned)blocks), dim3(kQThreads), st);
  auto go = [&](auto* kernel) {
    return cudaLaunchKernelEx(&l.cfg, kernel, x, ldx, rows, k, q, scale, qt, scale_t, ldq, ldqt, ktiles, rtiles);
  };
  auto* const kernel = load == 16 ? k_fp4_quantize<T, 16> : load == 4 ? k_fp4_quantize<T, 4> : k_fp4_quantize<T, sizeof(T)>;
  FF_LAUNCH(K_FP4_QUANT, bytes, st, go(kernel), "4-bit quantize");
  return FF_OK;
}

template <typename T>
ff_status dequantize_t(const uint8_t* q, const uint8_t* scale, int rows, int k, T* y, long long ldy, cudaStream_t st) {
  if (rows == 1) ldy = 0;
  const bool wide = rows_aligned(y, ldy, sizeof(T), 16), staged = !wide && (long long)rows * k >= 1 << 20;
  const int units = wide ? cdiv(k, 16 / (int)sizeof(T)) : staged ? cdiv(k, 8) : k, most = staged ? 5 : 8;
  DequantArgs a{q, scale, rows, k, fp4_stride(k), cdiv(k, QT), ldy, 3, 0, 0};
  while (a.lanes_log < most && (1 << a.lanes_log) < units) ++a.lanes_log;
  a.strips = cdiv(units, 1 << a.lanes_log);
  // (a matrix of less than 32 rows leaves the other j out)
  const int per = 256 >> a.lanes_log;
  a.groups = rows < QT ? cdiv(std::min(rows, 32), per) : 32 / per;
  const long long blocks = (long long)a.strips * cdiv(rows, QT) * a.groups;
  if (blocks > 0x7FFFFFFFll) return FF_ERR_UNSUPPORTED;
  const double bytes = (double)rows * k * (sizeof(T) + 0.5);
  PdlLaunch l(dim3((unsigned)blocks), dim3(256), st);
  auto* const kernel = wide      ? k_fp4_dequantize<T, true>
                       : !staged ? k_fp4_dequantize<T, false>
                       : rows_aligned(y, ldy, sizeof(T), 4) ? k_fp4_dequantize_staged<T, 4>
                                                            : k_fp4_dequantize_staged<T, sizeof(T)>;
  FF_LAUNCH(K_FP4_DEQUANT, bytes, st, cudaLaunchKernelEx(&l.cfg, kernel, a, y), "4-bit dequantize");
  return FF_OK;
}

bool aligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

}  // namespace
}  // namespace ff

using namespace ff;

constexpr int kMostSize = 0x7FFFFF00;

extern "C" FF_API int ff_fp4_stride(int k) { return k > 0 && k <= kMostSize ? fp4_stride(k) : 0; }
extern "C" FF_API long long ff_fp4_scale_bytes(int rows, int k) {
  return rows < 0 || rows > kMostSize || k < 1 || k > kMostSize ? -1 : fp4_scale_bytes(rows, k);
}

extern "C" FF_API ff_status ff_fp4_quantize(const void* x, long long ldx, int rows, int k, ff_precision prec, void* q, void* scale,
                                            void* qt, void* scale_t, void* stream) {
  if (rows < 0 || k < 1 || rows > kMostSize || k > kMostSize || (prec != FF_FP32 && prec != FF_BF16)) return FF_ERR_INVALID_ARG;
  if (rows == 0) return FF_OK;
  const int es = prec == FF_BF16 ? 2 : 4;
  if (!x || !aligned(x, es) || (ldx < k && rows > 1) || (q == nullptr) != (scale == nullptr) ||
      (qt == nullptr) != (scale_t == nullptr) || (!q && !qt) || !aligned(q, 16) || !aligned(qt, 16) || !aligned(scale, 16) ||
      !aligned(scale_t, 16))
    return FF_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  auto run = [&](auto t) {
    using T = decltype(t);
    return quantize_t(static_cast<const T*>(x), ldx, rows, k, static_cast<uint8_t*>(q), static_cast<uint8_t*>(scale),
                      static_cast<uint8_t*>(qt), static_cast<uint8_t*>(scale_t), st);
  };
  return prec == FF_BF16 ? run(bf16{}) : run(float{});
}

extern "C" FF_API ff_status ff_fp4_dequantize(const void* q, const void* scale, int rows, int k, ff_precision prec, void* y,
                                              long long ldy, void* stream) {
  if (rows < 0 || k < 1 || rows > kMostSize || k > kMostSize || (prec != FF_FP32 && prec != FF_BF16)) return FF_ERR_INVALID_ARG;
  if (rows == 0) return FF_OK;
  const int es = prec == FF_BF16 ? 2 : 4;
  if (!q || !scale || !y || !aligned(q, 16) || !aligned(scale, 16) || !aligned(y, es) || (ldy < k && rows > 1))
    return FF_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const uint8_t *qb = static_cast<const uint8_t*>(q), *sb = static_cast<const uint8_t*>(scale);
  return prec == FF_BF16 ? dequantize_t(qb, sb, rows, k, static_cast<bf16*>(y), ldy, st)
                         : dequantize_t(qb, sb, rows, k, static_cast<float*>(y), ldy, st);
}

extern "C" FF_API ff_status ff_fp4_matmul(const void* a, const void* a_scale, const void* b, const void* b_scale, int m, int n,
                                          int k, const float* bias, int relu, ff_precision out_prec, void* c, long long ldc,
                                          int* device_status, void* stream) {
  if (m < 0 || n < 0 || k < 1 || m > kMostSize || n > kMostSize || k > kMostSize ||
      (out_prec != FF_FP32 && out_prec != FF_BF16))
    return FF_ERR_INVALID_ARG;
  if (m == 0 || n == 0) return FF_OK;
  const int es = out_prec == FF_BF16 ? 2 : 4;
  if (!a || !a_scale || !b || !b_scale || !c || !aligned(a, 16) || !aligned(b, 16) || !aligned(a_scale, 16) ||
      !aligned(b_scale, 16) || !aligned(bias, 4) || !aligned(device_status, 4) || !aligned(c, es) || (ldc < n && m > 1))
    return FF_ERR_INVALID_ARG;
  if (!tc_supported()) return FF_ERR_UNSUPPORTED;
  Fp4Gemm g{};
  g.a = static_cast<const uint8_t*>(a);
  g.b = static_cast<const uint8_t*>(b);
  g.sa = static_cast<const uint8_t*>(a_scale);
  g.sb = static_cast<const uint8_t*>(b_scale);
  g.M = m;
  g.N = n;
  g.K = k;
  g.bias = bias;
  g.relu = relu != 0;
  g.out_bf16 = out_prec == FF_BF16;
  g.c = c;
  g.ldc = ldc;
  g.status = device_status;
  if (!device_status) FF_TRY(own_status(&g.status), "4-bit matrix product");
  return fp4_gemm(g, static_cast<cudaStream_t>(stream));
}
