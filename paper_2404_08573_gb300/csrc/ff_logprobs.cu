// Log-probabilities of given labels under a row's logits, with the entropy and
// the likeliest classes, and their gradient.  With m = max x, d = x - m:
//
//   s = sum e^d, t = sum d e^d
//   log p = d - ln s,  entropy = ln s - t / s
//   dx = g (1[label] - p) - g' p (log p + entropy)   (g, g' from above)
//
// One pass: every thread carries (m, s, t) over its part of the row, rescaled
// when m grows, and they are joined at the end.  The likeliest classes come
// from the same pass: a warp keeps its best 32 in its lanes, and takes up a
// value only if it beats the least of those it needs.
#include <algorithm>

#include "ff_api_internal.h"
#include "ff_ptx.cuh"
#include "ff_vec.cuh"

namespace ff {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kFar = -1e4f;  // e^d is zero in fp32 from here on: d is held above, so that e^d d is never 0 * inf
constexpr float kLowest = -3.402823466e38f;
constexpr int kMostTop = 32;
constexpr int kMostWarps = 32;

__device__ __forceinline__ float max_nan(float a, float b) {  // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float exp2_approx(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

// m starts at the lowest finite value, not at -infinity, so that x - m is
// -infinity (and its term zero) for a masked class and never NaN.  s == 0 at
// the end: every class was masked.
struct Sums {
  float m, s, t;
};
__device__ __forceinline__ void raise(Sums& a, float m) {  // to a maximum m >= a.m
  const float d = max_nan(a.m - m, kFar), f = exp2_approx(d * kLog2e);
  a.t = (a.t + a.s * d) * f;
  a.s *= f;
  a.m = m;
}
__device__ __forceinline__ void join(Sums& a, Sums b) {
  const float m = fmaxf(a.m, b.m);
  raise(a, m);
  raise(b, m);
  a.s += b.s;
  a.t += b.t;
}

// Floats in the order of whole numbers (-0 as 0; a NaN above infinity).
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t o) {
  return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}
// A class as one number: larger is likelier, the lower index first.
__device__ __forceinline__ unsigned long long key_of(uint32_t o, uint32_t index) {
  return (unsigned long long)o << 32 | (0xFFFFFFFFu - index);
}

// A warp's best 32 classes, lane i the i-th, and the value that a later class
// has to beat to be among the first k: the k-th of the warp's own, or the k-th of
// another warp of the block (which one with the same value may still precede).
struct Best {
  unsigned long long key;
  uint32_t least;
  int k;
  __device__ __forceinline__ void insert(unsigned long long n, int lane) {
    const int pos = __popc(__ballot_sync(0xffffffffu, key > n));
    const unsigned long long up = __shfl_up_sync(0xffffffffu, key, 1);
    key = lane < pos ? key : lane == pos ? n : up;
  }
  __device__ __forceinline__ uint32_t kth() const { return (uint32_t)(__shfl_sync(0xffffffffu, key, k - 1) >> 32); }
};

// N values of a vector into the warp's list: `top` is the largest of each
// lane's, index0 the class of the lane's first.  A lane's classes, and the
// lanes', follow each other in index order.
template <int N>
__device__ __forceinline__ void take(Best& b, const float (&v)[N], int count, uint32_t index0, int lane, uint32_t* shared) {
  uint32_t left = count < N ? (1u << (count < 0 ? 0 : count)) - 1u : (1u << N) - 1u;
  const uint32_t others = *reinterpret_cast<volatile uint32_t*>(shared);
  uint32_t least = max(b.kth(), others ? others - 1u : 0u);
  while (true) {
    uint32_t o = 0, at = 0;
#pragma unroll
    for (int e = N - 1; e >= 0; --e) {
      const uint32_t c = left >> e & 1u ? ordered(v[e]) : 0u;
      if (c >= o && c > 0u) {
        o = c;
        at = (uint32_t)e;
      }
    }
    const uint32_t most = __reduce_max_sync(0xffffffffu, o);
    if (most <= least) break;
    const int src = __ffs(__ballot_sync(0xffffffffu, o == most)) - 1;
    const uint32_t index = __shfl_sync(0xffffffffu, index0 + at, src);
    if (lane == src) left &= ~(1u << at);
    b.insert(key_of(most, index), lane);
    least = max(least, b.kth());
  }
  const uint32_t own = b.kth();
  if (lane == 0 && own > others) atomicMax(shared, own);
  b.least = max(own, others ? others - 1u : 0u);
}

// Two warp lists into one: the larger of one and of the other reversed are the
// 32 largest, and a bitonic merge orders them.
__device__ __forceinline__ unsigned long long merge(unsigned long long a, unsigned long long b, int lane) {
  const unsigned long long r = __shfl_sync(0xffffffffu, b, 31 - lane);
  a = a > r ? a : r;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const unsigned long long p = __shfl_xor_sync(0xffffffffu, a, o);
    const bool low = (lane & o) == 0;
    a = (a > p) == low ? a : p;
  }
  return a;
}

template <typename T>
struct Args {
  const T* x;
  long long ldx;
  int rows, classes, top, warps, cluster;
  const int* labels;
  float *logp, *entropy, *top_logp;
  int* top_index;
  float2* stats;
};

template <typename T>
struct Load {
  static constexpr int N = 16 / (int)sizeof(T);
};

// A row on `cluster` blocks of `warps` warps (or, warps == 1, several rows a
// block).  The row's 16-byte aligned middle is read as vectors, its ends value
// by value by the first block's first and the last block's last warp.
template <typename T, bool TOP>
__global__ void __launch_bounds__(kMostWarps * 32, 1) k_logprobs(const Args<T> a) {
  constexpr int N = Load<T>::N;
  constexpr int AHEAD = 4;
  __shared__ Sums sums[kMostWarps];
  __shared__ Sums blocks[8];
  __shared__ unsigned long long keys[TOP ? kMostWarps : 1][32];
  __shared__ unsigned long long block_keys[TOP ? 8 : 1][32];
  __shared__ uint32_t least[8];
  if (a.cluster > 1) ptx::cluster_arrive();  // so that the first block is known to run before it is written to
  ptx::griddep_wait();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const bool own = a.warps == 1;
  const int warp = own ? 0 : w;
  const int rank = a.cluster > 1 ? (int)ptx::cluster_ctarank() : 0;
  const long long row = own ? (long long)blockIdx.x * (blockDim.x >> 5) + w : blockIdx.x / (unsigned)a.cluster;
  uint32_t* shared_least = &least[own ? w : 0];
  if (TOP) {
    if (own ? lane == 0 : threadIdx.x == 0) *shared_least = 0;
    if (own) __syncwarp();
    else __syncthreads();
  }
  if (row >= a.rows) return;
  const T* p = a.x + row * a.ldx;
  const int label = a.labels ? __ldg(a.labels + row) : -1;
  const bool has = label >= 0 && label < a.classes;
  float at_label = 0.f;
  if (has) {
    float one[1];
    Vec<T, 1>::unpack(Vec<T, 1>::load(p + label), one);
    at_label = one[0];
  }

  Sums f{kLowest, 0.f, 0.f};
  Best best{0ull, 0u, a.top};
  auto one_by_one = [&](int from, int to) {  // values from .. to of the row (fewer than a vector) on a warp's lanes
    const int i = from + lane;
    float v[1] = {kLowest};
    const bool in = i < to;
    if (in) {
      Vec<T, 1>::unpack(Vec<T, 1>::load(p + i), v);
      if (v[0] > f.m) raise(f, v[0]);
      const float d = max_nan(v[0] - f.m, kFar), e = exp2_approx(d * kLog2e);
      f.s += e;
      f.t += e * d;
    }
    if (TOP) take<1>(best, v, in ? 1 : 0, (uint32_t)i, lane, shared_least);
  };
  const int off = (int)(reinterpret_cast<uintptr_t>(p) / sizeof(T) % N);
  const int head = min(off ? N - off : 0, a.classes), vecs = (a.classes - head) / N;
  const int v0 = (int)((long long)vecs * rank / a.cluster), v1 = (int)((long long)vecs * (rank + 1) / a.cluster);
  if (rank == 0 && warp == 0 && head) one_by_one(0, head);
  const uint4* src = reinterpret_cast<const uint4*>(p + head);
  const int step = a.warps * 32;
  for (long long i0 = v0; i0 < v1; i0 += (long long)AHEAD * step) {  // the same for a warp's lanes
    uint4 raw[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const long long i = i0 + j * step + warp * 32 + lane;
      if (i < v1) raw[j] = src[i];
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const long long first = i0 + j * step + warp * 32, i = first + lane;
      if (first >= v1) break;
      float v[N];
      Vec<T, N>::unpack(raw[j], v);
      float most = kLowest;
      if (i < v1) {
        most = v[0];
#pragma unroll
        for (int e = 1; e < N; ++e) most = fmaxf(most, v[e]);
        if (most > f.m) raise(f, most);
        const uint64_t m2 = ptx::pack2(-f.m, -f.m), l2 = ptx::pack2(kLog2e, kLog2e);
        uint64_t s2 = 0, t2 = 0;
#pragma unroll
        for (int e = 0; e < N; e += 2) {
          float2 d = ptx::unpack2(ptx::add2(ptx::pack2(v[e], v[e + 1]), m2));
          d.x = max_nan(d.x, kFar);
          d.y = max_nan(d.y, kFar);
          const uint64_t d2 = ptx::pack2(d.x, d.y);
          const float2 g = ptx::unpack2(ptx::mul2(d2, l2));
          const uint64_t e2 = ptx::pack2(exp2_approx(g.x), exp2_approx(g.y));
          s2 = ptx::add2(s2, e2);
          ptx::fma2_to(t2, e2, d2);
        }
        const float2 s = ptx::unpack2(s2), t = ptx::unpack2(t2);
        f.s += s.x + s.y;
        f.t += t.x + t.y;
      }
      if (TOP && __any_sync(0xffffffffu, i < v1 && (ordered(most) > best.least || best.least == 0u)))
        take<N>(best, v, i < v1 ? N : 0, (uint32_t)(head + i * N), lane, shared_least);
    }
  }
  if (rank == a.cluster - 1 && warp == a.warps - 1 && head + vecs * N < a.classes) one_by_one(head + vecs * N, a.classes);

#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Sums b{__shfl_xor_sync(0xffffffffu, f.m, o), __shfl_xor_sync(0xffffffffu, f.s, o), __shfl_xor_sync(0xffffffffu, f.t, o)};
    join(f, b);
  }
  if (!own) {
    if (lane == 0) sums[warp] = f;
    if (TOP) keys[warp][lane] = best.key;
    __syncthreads();
    if (warp == 0) {
      f = lane < a.warps ? sums[lane] : Sums{kLowest, 0.f, 0.f};
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        Sums b{__shfl_xor_sync(0xffffffffu, f.m, o), __shfl_xor_sync(0xffffffffu, f.s, o),
               __shfl_xor_sync(0xffffffffu, f.t, o)};
        join(f, b);
      }
      if (TOP)
        for (int i = 1; i < a.warps; ++i) best.key = merge(best.key, keys[i][lane], lane);
    }
    if (a.cluster > 1) {
      ptx::cluster_wait();
      if (warp == 0) {  // to the first block
        if (lane == 0) {
          ptx::st_remote_f32(&blocks[rank].m, 0, f.m);
          ptx::st_remote_f32(&blocks[rank].s, 0, f.s);
          ptx::st_remote_f32(&blocks[rank].t, 0, f.t);
        }
        if (TOP)
          ptx::st_remote_u2(reinterpret_cast<uint2*>(&block_keys[rank][lane]), 0,
                            make_uint2((uint32_t)best.key, (uint32_t)(best.key >> 32)));
      }
      __syncwarp();
      ptx::cluster_sync();
      if (rank == 0 && warp == 0) {
        f = blocks[0];
        for (int i = 1; i < a.cluster; ++i) join(f, blocks[i]);
        if (TOP)
          for (int i = 1; i < a.cluster; ++i) best.key = merge(best.key, block_keys[i][lane], lane);
      }
    }
    if (rank != 0 || warp != 0) return;
  }
  // an empty row, and one with a NaN or +infinity, has no distribution
  const bool none = !(f.s > 0.f);
  const float nan = __int_as_float(0x7FC00000), m = f.s == 0.f ? -INFINITY : f.m;
  const float ln = none ? nan : logf(f.s);
  if (lane == 0) {
    if (a.logp) a.logp[row] = has ? (at_label - m) - ln : 0.f;
    if (a.entropy) a.entropy[row] = ln - f.t / f.s;
    if (a.stats) a.stats[row] = make_float2(f.s != f.s ? nan : m, ln);
  }
  if (TOP && lane < a.top) {
    const bool got = best.key != 0ull;
    a.top_index[row * a.top + lane] = got ? (int)(0xFFFFFFFFu - (uint32_t)best.key) : lane;
    a.top_logp[row * a.top + lane] = got ? (unordered((uint32_t)(best.key >> 32)) - m) - ln : nan;
  }
}

// -------------------------------------------------------------- gradient
template <typename T>
struct GradArgs {
  const T* x;
  T* dx;
  long long ldx, lddx;
  int rows, classes;
  const int* labels;
  const float2* stats;
  const float *dlogp, *entropy, *dentropy;
  int team;      // threads a row's segment has
  int segments;  // segments a row is cut into
};

// What a row's gradient needs, and one value of it.
struct Row {
  float m, ln, scale, g, ge, h;
  int label;
};
template <typename T>
__device__ __forceinline__ float grad_of(const Row& r, float x, int c) {
  const float d = max_nan(x - r.m, kFar);
  const float p = (sizeof(T) == 4 ? expf(d) : exp2_approx(d * kLog2e)) * r.scale;
  float v = -p * (r.g + r.ge * (d - r.ln + r.h));
  if (c == r.label) v += r.g;
  return v;
}

// WIDE: both rows lie alike to 16 bytes, and all but their ends go as vectors.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(256) k_logprobs_grad(const GradArgs<T> a) {
  constexpr int N = Load<T>::N;
  ptx::griddep_wait();
  const int tid = threadIdx.x & (a.team - 1);
  const long long unit = (long long)blockIdx.x * (256 / a.team) + threadIdx.x / a.team;
  const long long row = unit / a.segments;
  const int seg = (int)(unit - row * a.segments);
  if (row >= a.rows) return;
  const T* p = a.x + row * a.ldx;
  T* out = a.dx + row * a.lddx;
  Row r;
  const float2 st = __ldg(a.stats + row);
  r.m = st.x;
  r.ln = st.y;
  r.scale = expf(-st.y);
  r.label = a.labels ? __ldg(a.labels + row) : -1;
  if (r.label >= a.classes) r.label = -1;
  r.g = a.dlogp && r.label >= 0 ? __ldg(a.dlogp + row) : 0.f;
  r.ge = a.dentropy ? __ldg(a.dentropy + row) : 0.f;
  r.h = a.dentropy ? __ldg(a.entropy + row) : 0.f;
  const bool zero = r.g == 0.f && r.ge == 0.f;  // nothing asked of the row: zeros, whatever it holds
  auto one = [&](int c) {
    float v[1];
    Vec<T, 1>::unpack(Vec<T, 1>::load(p + c), v);
    v[0] = zero ? 0.f : grad_of<T>(r, v[0], c);
    Vec<T, 1>::store(out + c, v);
  };
  if constexpr (WIDE) {
    const int off = (int)(reinterpret_cast<uintptr_t>(p) / sizeof(T) % N);
    const int head = min(off ? N - off : 0, a.classes), vecs = (a.classes - head) / N;
    const int v0 = (int)((long long)vecs * seg / a.segments), v1 = (int)((long long)vecs * (seg + 1) / a.segments);
    if (seg == 0 && tid < head) one(tid);
    if (seg == a.segments - 1 && head + vecs * N + tid < a.classes) one(head + vecs * N + tid);
#pragma unroll 4
    for (int i = v0 + tid; i < v1; i += a.team) {
      float v[N];
      Vec<T, N>::unpack(Vec<T, N>::load(p + head + (long long)i * N), v);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = zero ? 0.f : grad_of<T>(r, v[e], head + i * N + e);
      Vec<T, N>::store(out + head + (long long)i * N, v);
    }
  } else {
    const int c0 = (int)((long long)a.classes * seg / a.segments), c1 = (int)((long long)a.classes * (seg + 1) / a.segments);
#pragma unroll 8
    for (int c = c0 + tid; c < c1; c += a.team) one(c);
  }
}

// ------------------------------------------------------------------ host
template <typename T, bool TOP>
cudaError_t launch(const Args<T>& a, unsigned grid, unsigned threads, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)a.cluster;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = a.cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, k_logprobs<T, TOP>, a);
}

template <typename T>
ff_status logprobs_t(Args<T> a, cudaStream_t st) {
  constexpr int N = Load<T>::N;
  const int vecs = cdiv(a.classes, N);
  // Short rows take a warp each.  Others a block of 8 warps; with fewer rows
  // than the GPU has room for, more warps and then more blocks, as long as
  // each thread has a vector or two to read.
  a.warps = vecs <= 256 && a.rows >= 152 ? 1 : 8;
  a.cluster = 1;
  if (a.warps == 8 && a.rows < 152 * 4) {
    while (a.warps < kMostWarps && (long long)a.warps * 2 * 32 <= vecs && (long long)a.rows * a.warps < 152 * 32) a.warps *= 2;
    while (a.cluster < 8 && (long long)a.cluster * 2 * a.warps * 32 <= vecs && (long long)a.rows * a.cluster * 2 <= 152) a.cluster *= 2;
  }
  const unsigned threads = a.warps == 1 ? 256 : (unsigned)a.warps * 32;
  const long long grid = a.warps == 1 ? cdiv(a.rows, 8) : (long long)a.rows * a.cluster;
  if (grid > 0x7FFFFFFFll) return FF_ERR_UNSUPPORTED;
  const double bytes = (double)a.rows * a.classes * sizeof(T);
  auto* const go = a.top ? launch<T, true> : launch<T, false>;
  FF_LAUNCH(K_LOGPROBS, bytes, st, go(a, (unsigned)grid, threads, st), "label log-probabilities");
  return FF_OK;
}

template <typename T>
ff_status grad_t(GradArgs<T> a, cudaStream_t st) {
  constexpr int N = Load<T>::N;
  const bool wide = (reinterpret_cast<uintptr_t>(a.x) - reinterpret_cast<uintptr_t>(a.dx)) % 16 == 0 &&
                    (a.rows == 1 || (a.ldx - a.lddx) * (long long)sizeof(T) % 16 == 0);
  const int units = wide ? cdiv(a.classes, N) : a.classes;
  a.team = 32;
  while (a.team < 256 && a.team * 4 <= units) a.team *= 2;
  a.segments = std::max(1, cdiv(units, (long long)a.team * (wide ? 8 : 16)));
  const long long blocks = ((long long)a.rows * a.segments + 256 / a.team - 1) / (256 / a.team);
  if (blocks > 0x7FFFFFFFll) return FF_ERR_UNSUPPORTED;
  const double bytes = 2.0 * a.rows * a.classes * sizeof(T);
  PdlLaunch l(dim3((unsigned)blocks), dim3(256), st);
  auto* const kernel = wide ? k_logprobs_grad<T, true> : k_logprobs_grad<T, false>;
  FF_LAUNCH(K_LOGPROBS_GRAD, bytes, st, cudaLaunchKernelEx(&l.cfg, kernel, a), "label log-probabilities' gradient");
  return FF_OK;
}

bool aligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

}  // namespace
}  // namespace ff

using namespace ff;

extern "C" FF_API ff_status ff_label_logprobs(const void* logits, long long ld, int rows, int classes, ff_precision prec,
                                              const int* labels, float* logp, float* entropy, int top, float* top_logp,
                                              int* top_index, float* stats, void* stream) {
  if (rows < 0 || classes < 1 || classes > 0x7FFFFF00 || (prec != FF_FP32 && prec != FF_BF16) || top < 0 || top > kMostTop ||
      top > classes)
    return FF_ERR_INVALID_ARG;
  if (rows == 0) return FF_OK;
  const int es = prec == FF_BF16 ? 2 : 4;
  if (!logits || !aligned(logits, es) || (ld < classes && rows > 1) || (logp && !labels) || !aligned(labels, 4) ||
      !aligned(logp, 4) || !aligned(entropy, 4) || (top > 0 && (!top_logp || !top_index)) || !aligned(top_logp, 4) ||
      !aligned(top_index, 4) || !aligned(stats, 8))
    return FF_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  auto run = [&](auto t) {
    using T = decltype(t);
    Args<T> a{};
    a.x = static_cast<const T*>(logits);
    a.ldx = ld;
    a.rows = rows;
    a.classes = classes;
    a.top = top;
    a.labels = labels;
    a.logp = logp;
    a.entropy = entropy;
    a.top_logp = top_logp;
    a.top_index = top_index;
    a.stats = reinterpret_cast<float2*>(stats);
    return logprobs_t(a, st);
  };
  return prec == FF_BF16 ? run(bf16{}) : run(float{});
}

extern "C" FF_API ff_status ff_label_logprobs_backward(const void* logits, long long ld, int rows, int classes,
                                                       ff_precision prec, const int* labels, const float* stats,
                                                       const float* dlogp, const float* entropy, const float* dentropy,
                                                       void* dlogits, long long lddx, void* stream) {
  if (rows < 0 || classes < 1 || classes > 0x7FFFFF00 || (prec != FF_FP32 && prec != FF_BF16)) return FF_ERR_INVALID_ARG;
  if (rows == 0) return FF_OK;
  const int es = prec == FF_BF16 ? 2 : 4;
  if (!logits || !dlogits || !stats || !aligned(logits, es) || !aligned(dlogits, es) || !aligned(stats, 8) ||
      ((ld < classes || lddx < classes) && rows > 1) || (dlogp && !labels) || (dentropy && !entropy) || !aligned(labels, 4) ||
      !aligned(dlogp, 4) || !aligned(entropy, 4) || !aligned(dentropy, 4))
    return FF_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  auto run = [&](auto t) {
    using T = decltype(t);
    GradArgs<T> a{};
    a.x = static_cast<const T*>(logits);
    a.dx = static_cast<T*>(dlogits);
    a.ldx = ld;
    a.lddx = lddx;
    a.rows = rows;
    a.classes = classes;
    a.labels = labels;
    a.stats = reinterpret_cast<const float2*>(stats);
    a.dlogp = dlogp;
    a.entropy = entropy;
    a.dentropy = dentropy;
    return grad_t(a, st);
  };
  return prec == FF_BF16 ? run(bf16{}) : run(float{});
}
