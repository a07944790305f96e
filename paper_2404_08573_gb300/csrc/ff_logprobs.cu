// Log-probabilities of given labels under a row's logits, with the entropy and
// the likeliest classes, and their gradient.  With m = max x, d = x - m:
//
//   s = sum e^d, t = sum d e^d
//   log p = d - ln s,  entropy = ln s - t / s
//   dx = g (1[label] - p) - g' p (log p + entropy)   (g, g' from above)
//
// One pass: every thread carries (m, s, t) over its part of the row, rescaled
// when m grows, and they are joined at the end.
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
constexpr int kOwnRows = 8;  // rows a block with a warp a row

__device__ __forceinline__ float max_nan(float a, float b) {  // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// 2^v to 2^-22 of itself, below 2^-126 zero: enough for the sums of either type,
// since a class's error counts by its probability, as does that of rounding the
// exponent (|d| e^d 2^-24, at most 2^-25), and ln s and t / s are then within some
// 2^-21.  The fp32 gradient, whose elements stand for themselves, has expf.
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

// A warp's 32 numbers, largest first: by a bitonic sort; and two such lists
// into one (the larger of one and of the other reversed are the 32 largest, and
// a bitonic merge orders them).
template <typename K>
__device__ __forceinline__ K step(K a, int o, bool keep_larger) {
  const K p = __shfl_xor_sync(0xffffffffu, a, o);
  return (a > p) == keep_larger ? a : p;
}
template <typename K>
__device__ __forceinline__ K sorted(K a, int lane) {
#pragma unroll
  for (int size = 2; size <= 32; size *= 2)
#pragma unroll
    for (int o = size / 2; o > 0; o /= 2) a = step(a, o, ((lane & o) == 0) == ((lane & size) == 0 || size == 32));
  return a;
}
template <typename K>
__device__ __forceinline__ K merged(K a, K b, int lane) {
  const K r = __shfl_sync(0xffffffffu, b, 31 - lane);
  a = a > r ? a : r;
#pragma unroll
  for (int o = 16; o > 0; o /= 2) a = step(a, o, (lane & o) == 0);
  return a;
}
// The 32 largest of n keys in shared memory, largest first; `place` (32 of them)
// is scratch.  A few by counting how many are larger (keys differ), which is one
// broadcast read each; many by sorting and merging.
__device__ __forceinline__ unsigned long long first_of(const unsigned long long* keys, int n, int lane, unsigned long long* place) {
  if (n > 96) {
    unsigned long long best = 0;
    for (int i = 0; i < n; i += 32) {
      const unsigned long long a = sorted(i + lane < n ? keys[i + lane] : 0ull, lane);
      best = i == 0 ? a : merged(best, a, lane);
    }
    return best;
  }
  place[lane] = 0ull;
  __syncwarp();
  for (int i = lane; i < n; i += 32) {
    const unsigned long long mine = keys[i];
    int larger = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) larger += keys[j] > mine;
    if (larger < 32 && mine != 0ull) place[larger] = mine;
  }
  __syncwarp();
  return place[lane];
}
// The k-th largest of n <= 128 numbers in shared memory.
__device__ __forceinline__ uint32_t kth_of(const uint32_t* numbers, int n, int k, int lane) {
  uint32_t best = 0;
  for (int i = 0; i < n; i += 32) {
    const uint32_t a = sorted(i + lane < n ? numbers[i + lane] : 0u, lane);
    best = i == 0 ? a : merged(best, a, lane);
  }
  return __shfl_sync(0xffffffffu, best, k - 1);
}

template <typename T>
struct Args {
  const T* x;
  long long ldx;
  int rows, classes, top, warps, cluster, groups;
  const int* labels;
  float *logp, *entropy, *top_logp;
  int* top_index;
  float2* stats;
};

__device__ __forceinline__ float nan_value() { return __int_as_float(0x7FC00000); }

// What a row's sums come to.  An empty row, and one with a NaN or +infinity, has
// no distribution.
struct Result {
  float m, s, t, ln;
  __device__ __forceinline__ Result(float most, float sum, float dsum) : m(sum == 0.f ? -INFINITY : most), s(sum), t(dsum) {
    ln = sum > 0.f ? logf(sum) : nan_value();
  }
  __device__ __forceinline__ float logp(float x) const { return (x - m) - ln; }
  template <typename T>
  __device__ __forceinline__ void put(const Args<T>& a, long long row, bool has, float at_label) const {
    if (a.logp) a.logp[row] = has ? logp(at_label) : 0.f;
    if (a.entropy) a.entropy[row] = ln - t / s;
    if (a.stats) a.stats[row] = make_float2(s != s ? nan_value() : m, ln);
  }
};

template <typename T>
struct Load {
  static constexpr int N = 16 / (int)sizeof(T);
};

// How a thread block reads its part of a row: the row's 16-byte aligned middle
// as vectors, v0 .. v1 of them the block's, vector v0 + j step + 32 warp + lane
// being the j-th of a thread; the row's ends value by value on a warp's lanes,
// by the first block's first and the last block's last warp.
template <typename T>
struct Part {
  const T* p;
  int classes, head, vecs, v0, v1, step;
  bool has_head, has_tail;  // this warp's
  __device__ __forceinline__ Part(const T* row, int n, int rank, int blocks, int warp, int warps) : p(row), classes(n) {
    constexpr int N = Load<T>::N;
    const int off = (int)(reinterpret_cast<uintptr_t>(p) / sizeof(T) % N);
    head = min(off ? N - off : 0, classes);
    vecs = (classes - head) / N;
    v0 = (int)((long long)vecs * rank / blocks);
    v1 = (int)((long long)vecs * (rank + 1) / blocks);
    step = warps * 32;
    has_head = rank == 0 && warp == 0 && head > 0;
    has_tail = rank == blocks - 1 && warp == warps - 1 && tail_at() < classes;
  }
  __device__ __forceinline__ int tail_at() const { return head + vecs * Load<T>::N; }
  __device__ __forceinline__ const uint4* vectors() const { return reinterpret_cast<const uint4*>(p + head); }
  // the lane's value of the row's head or tail, if it has one
  __device__ __forceinline__ float end_value(int from, int to, int lane, bool* in) const {
    float v[1] = {kLowest};
    *in = from + lane < to;
    if (*in) Vec<T, 1>::unpack(Vec<T, 1>::load(p + from + lane), v);
    return v[0];
  }
};

// The likeliest classes of a part of a row by one insertion after the other: a
// warp keeps its best 32 in its lanes, and takes up a value only if it beats
// the top-th of them.  For rows that the quick way below does not serve: many
// equal values, or fewer than `top` above -infinity.  (A lane's classes, and the
// lanes', follow each other in index order, so of equal values the first
// found stays.)
struct Best {
  unsigned long long key;
  uint32_t least;
  int top;
  template <int N>
  __device__ __forceinline__ void take(const float (&v)[N], bool in, uint32_t index0, int lane) {
    uint32_t left = in ? (1u << N) - 1u : 0u;
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
      const unsigned long long n = key_of(most, index);
      const int pos = __popc(__ballot_sync(0xffffffffu, key > n));
      const unsigned long long up = __shfl_up_sync(0xffffffffu, key, 1);
      key = lane < pos ? key : lane == pos ? n : up;
      least = (uint32_t)(__shfl_sync(0xffffffffu, key, top - 1) >> 32);
    }
  }
};
template <typename T>
__device__ __noinline__ unsigned long long best_by_insertion(const Part<T> part, int top, int warp, int lane) {
  constexpr int N = Load<T>::N;
  Best best{0ull, 0u, top};
  if (part.has_head) {
    bool in;
    const float v[1] = {part.end_value(0, part.head, lane, &in)};
    best.template take<1>(v, in, (uint32_t)lane, lane);
  }
  for (long long first = part.v0 + warp * 32; first < part.v1; first += part.step) {
    const long long i = first + lane;
    float v[N];
    Vec<T, N>::unpack(i < part.v1 ? part.vectors()[i] : make_uint4(0, 0, 0, 0), v);
    best.template take<N>(v, i < part.v1, (uint32_t)(part.head + i * N), lane);
  }
  if (part.has_tail) {
    bool in;
    const float v[1] = {part.end_value(part.tail_at(), part.classes, lane, &in)};
    best.template take<1>(v, in, (uint32_t)(part.tail_at() + lane), lane);
  }
  return best.key;
}

constexpr int kPool = 2048;               // candidates a block holds; a warp with a row of its own an eighth
constexpr int kOwnPool = kPool / kOwnRows;

// A row on `cluster` blocks of `warps` warps (or, warps == 1, kOwnRows rows a
// block).
//
// The likeliest classes: each thread has its largest value from the sums' pass.
// Of any groups of threads, the top-th largest of the groups' largest values is
// at most the row's top-th largest value, so every class wanted is at least
// that, and lies with one of the threads whose largest is.  Their values are
// read again (from L2) and those large enough are sorted.  Groups: whole warps,
// or the lanes of a warp in `a.groups` classes, so that there are at least 1.5
// top of them (then some 1.1 top values are found, 2 at worst).
//
// Bound by HBM, the selection beside it (2048 x 49999 fp32, top 4: 77 us, floor 61), or
// with few rows by the latency of its steps (1 x 131072 bf16, top 8, on 8 blocks of 32
// warps: 7.3 us, of which the sums alone are 4.3).
//
// WARPS: the most a block has.  Rows are many with 8: five blocks an SM keep
// 80 KB of loads in flight while others select (2048 x 49999 fp32: top 0 66 us, with
// four 71, with six 73; top 4 77, 82, 88).  bf16 with the likeliest spills a few words
// at five, all of them at six.
template <typename T, bool TOP, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, WARPS == 8 ? 5 : 1) k_logprobs(const Args<T> a) {
  constexpr int N = Load<T>::N;
  constexpr int AHEAD = 4;
  __shared__ Sums sums[kMostWarps];
  __shared__ Sums blocks[8];
  __shared__ uint32_t largest[TOP ? 128 : 1];
  __shared__ unsigned long long pool[TOP ? kPool : 1];
  __shared__ unsigned long long place[TOP ? kOwnRows : 1][32];
  __shared__ unsigned long long block_keys[TOP ? 8 * 32 : 1];
  __shared__ uint32_t counts[kOwnRows];
  if (a.cluster > 1) ptx::cluster_arrive();  // so that the first block is known to run before it is written to
  ptx::griddep_wait();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const bool own = a.warps == 1;
  const int warp = own ? 0 : w;
  const int rank = a.cluster > 1 ? (int)ptx::cluster_ctarank() : 0;
  const long long row = own ? (long long)blockIdx.x * kOwnRows + w : blockIdx.x / (unsigned)a.cluster;
  uint32_t* count = &counts[own ? w : 0];
  if (TOP && (own ? lane == 0 : threadIdx.x == 0)) *count = 0;
  if (row >= a.rows) return;
  const T* p = a.x + row * a.ldx;
  const int label = a.labels ? __ldg(a.labels + row) : -1;
  const Part<T> part(p, a.classes, rank, a.cluster, warp, a.warps);
  Sums f{kLowest, 0.f, 0.f};
  auto one_value = [&](float v) {
    if (v > f.m) raise(f, v);
    const float d = max_nan(v - f.m, kFar), e = exp2_approx(d * kLog2e);
    f.s += e;
    f.t += e * d;
  };
  bool in_head = false, in_tail = false;
  float head = kLowest, tail = kLowest;
  if (part.has_head) head = part.end_value(0, part.head, lane, &in_head);
  if (part.has_tail) tail = part.end_value(part.tail_at(), a.classes, lane, &in_tail);
  const uint4* src = part.vectors();
  for (long long i0 = part.v0 + warp * 32 + lane; i0 < part.v1; i0 += (long long)AHEAD * part.step) {
    uint4 raw[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
      if (i0 + j * part.step < part.v1) raw[j] = src[i0 + j * part.step];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (i0 + j * part.step >= part.v1) break;
      float v[N];
      Vec<T, N>::unpack(raw[j], v);
      float most = v[0];
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
  }
  if (in_head) one_value(head);
  if (in_tail) one_value(tail);
  __syncwarp();
  const bool has = label >= 0 && label < a.classes;
  float at_label = 0.f;
  if (has && rank == 0 && warp == 0) {
    float one[1];
    Vec<T, 1>::unpack(Vec<T, 1>::load(p + label), one);
    at_label = one[0];
  }

  const uint32_t mine = ordered(f.m);  // the thread's largest (the lowest finite value if it has none)
  uint32_t group = mine;
  if (TOP && !own) {
    for (int o = 16; o >= a.groups; o >>= 1) group = max(group, __shfl_xor_sync(0xffffffffu, group, o));
    if (lane < a.groups) largest[warp * a.groups + lane] = group;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Sums b{__shfl_xor_sync(0xffffffffu, f.m, o), __shfl_xor_sync(0xffffffffu, f.s, o), __shfl_xor_sync(0xffffffffu, f.t, o)};
    join(f, b);
  }
  if (!own) {
    if (lane == 0) sums[warp] = f;
    __syncthreads();
    if (warp == 0) {
      f = lane < a.warps ? sums[lane] : Sums{kLowest, 0.f, 0.f};
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        Sums b{__shfl_xor_sync(0xffffffffu, f.m, o), __shfl_xor_sync(0xffffffffu, f.s, o),
               __shfl_xor_sync(0xffffffffu, f.t, o)};
        join(f, b);
      }
    }
  }

  unsigned long long key = 0;  // of the part's classes, likeliest first, in the lanes of its first warp
  if (TOP) {
    unsigned long long* const to = pool + (own ? w * kOwnPool : 0);
    const uint32_t room = own ? kOwnPool : kPool;
    const uint32_t least =
        own ? __shfl_sync(0xffffffffu, sorted(mine, lane), a.top - 1) : kth_of(largest, a.warps * a.groups, a.top, lane);
    const float floor = unordered(least);
    auto add = [&](float v, bool in, uint32_t index) {  // NaN is not at least anything
      const bool hit = in && v >= floor;
      const uint32_t hits = __ballot_sync(0xffffffffu, hit);
      if (!hits) return;
      uint32_t at = 0;
      if (lane == 0) at = atomicAdd(count, (uint32_t)__popc(hits));
      at = __shfl_sync(0xffffffffu, at, 0) + (uint32_t)__popc(hits & ((1u << lane) - 1u));
      if (hit && at < room) to[at] = key_of(ordered(v), index);
    };
    if (part.has_head) add(head, in_head, (uint32_t)lane);
    if (part.has_tail) add(tail, in_tail, (uint32_t)(part.tail_at() + lane));
    auto add_all = [&](long long i) {  // vector i on each lane
      const bool in = i < part.v1;
      float v[N];
      Vec<T, N>::unpack(in ? src[i] : make_uint4(0, 0, 0, 0), v);
      bool any = false;
#pragma unroll
      for (int e = 0; e < N; ++e) any |= in && v[e] >= floor;
      if (__any_sync(0xffffffffu, any)) {
#pragma unroll
        for (int e = 0; e < N; ++e) add(v[e], in, (uint32_t)(part.head + i * N + e));
      }
    };
    uint32_t who = __ballot_sync(0xffffffffu, mine >= least);
    if (part.v1 - part.v0 <= 4 * part.step) {  // a few vectors a thread: each lane its own
      if (who)
        for (long long i = part.v0 + warp * 32; i < part.v1; i += part.step) add_all(i + lane);
    } else {  // else 32 lanes to one's
      for (; who; who &= who - 1u)
        for (long long i = part.v0 + warp * 32 + (__ffs(who) - 1); i < part.v1; i += 32ll * part.step)
          add_all(i + (long long)lane * part.step);
    }
    if (own) __syncwarp();
    else __syncthreads();
    const uint32_t found = *reinterpret_cast<volatile uint32_t*>(count);
    if (found < (uint32_t)a.top || found > room) {
      key = best_by_insertion(part, a.top, warp, lane);
      if (!own) {
        __syncthreads();  // the pool is no longer read
        pool[warp * 32 + lane] = key;
        __syncthreads();
        if (warp == 0) key = first_of(pool, a.warps * 32, lane, place[0]);
      }
    } else if (warp == 0) {
      key = first_of(to, (int)found, lane, place[own ? w : 0]);
    }
  }
  if (a.cluster > 1) {
    ptx::cluster_wait();
    if (warp == 0) {  // to the first block
      if (lane == 0) {
        ptx::st_remote_f32(&blocks[rank].m, 0, f.m);
        ptx::st_remote_f32(&blocks[rank].s, 0, f.s);
        ptx::st_remote_f32(&blocks[rank].t, 0, f.t);
      }
      if (TOP && lane < a.top)
        ptx::st_remote_u2(reinterpret_cast<uint2*>(&block_keys[rank * a.top + lane]), 0,
                          make_uint2((uint32_t)key, (uint32_t)(key >> 32)));
    }
    __syncwarp();
    ptx::cluster_sync();
    if (rank == 0 && warp == 0) {
      f = blocks[0];
      for (int i = 1; i < a.cluster; ++i) join(f, blocks[i]);
      if (TOP) key = first_of(block_keys, a.cluster * a.top, lane, place[0]);
    }
  }
  if (rank != 0 || warp != 0) return;
  const Result r(f.m, f.s, f.t);
  if (lane == 0) r.put(a, row, has, at_label);
  if (TOP && lane < a.top) {
    const bool got = key != 0ull;
    a.top_index[row * a.top + lane] = got ? (int)(0xFFFFFFFFu - (uint32_t)key) : lane;
    a.top_logp[row * a.top + lane] = got ? r.logp(unordered((uint32_t)(key >> 32))) : nan_value();
  }
}

// Rows of up to 32 E classes: 2^lanes_log lanes a row (32 if E > 1), lane l with
// the classes l, l + 32, ..  The likeliest: a class's place is the number of larger
// ones, counted over the row's keys in shared memory, four a load.  Bound by latency
// and, with many rows, by this counting: bf16, 11562 x 8, top 1: 2.4 us (by a warp a row
// below 11.5); 60000 x 10: 6.2 (26), with top 8 9.5 (58); 16384 x 64, top 8: 13 (20);
// 16384 x 100: 4.7 (8.9), but with top 8 29 (19), so that rows with the likeliest
// classes wanted come here up to 64.
template <typename T, bool TOP, int E>
__global__ void __launch_bounds__(256) k_logprobs_short(const Args<T> a, int lanes_log) {
  ptx::griddep_wait();
  const int lanes = 1 << lanes_log, l = threadIdx.x & (lanes - 1);
  const long long row = (long long)blockIdx.x * (256 >> lanes_log) + (threadIdx.x >> lanes_log);
  const bool in = row < a.rows;  // (lanes without a row take part in the shuffles)
  const T* p = a.x + (in ? row : 0) * a.ldx;
  int label = -1;
  if (a.labels && in) label = __ldg(a.labels + row);
  float x[E], m = kLowest;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    x[e] = -INFINITY;
    if (in && l + 32 * e < a.classes) {
      float one[1];
      Vec<T, 1>::unpack(Vec<T, 1>::load(p + l + 32 * e), one);
      x[e] = one[0];
    }
    m = fmaxf(m, x[e]);
  }
  for (int o = lanes >> 1; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float s = 0.f, t = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float d = max_nan(x[e] - m, kFar), y = exp2_approx(d * kLog2e);
    s += y;
    t += y * d;
  }
  for (int o = lanes >> 1; o > 0; o >>= 1) {
    s += __shfl_xor_sync(0xffffffffu, s, o);
    t += __shfl_xor_sync(0xffffffffu, t, o);
  }
  const Result r(m, s, t);
  const bool has = label >= 0 && label < a.classes;
  float at_label = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float v = __shfl_sync(0xffffffffu, x[e], label & (lanes - 1), lanes);
    if (e == label >> 5) at_label = v;
  }
  if (l == 0 && in) r.put(a, row, has, at_label);
  if constexpr (TOP) {
    // Of classes in other sets a comparison knows which comes first; in a class's own
    // set the equal ones are all counted, and those from itself on taken off again.
    __shared__ __align__(16) uint32_t keys[256 * E];
    uint32_t* const to = keys + (threadIdx.x & ~31u) * E;
    const int lane = threadIdx.x & 31, row0 = lane - l;
    // the row's lanes from this one on
    const uint32_t rest = (lanes == 32 ? 0xFFFFFFFFu : ((1u << lanes) - 1u) << row0) >> lane << lane;
    uint32_t mine[E];
    int place[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      mine[e] = l + 32 * e < a.classes ? ordered(x[e]) : 0u;
      to[32 * e + lane] = mine[e];
      place[e] = -__popc(__match_any_sync(0xffffffffu, mine[e]) & rest);
    }
    __syncwarp();
#pragma unroll
    for (int f = 0; f < E; ++f) {
      const uint4* from = reinterpret_cast<const uint4*>(to + 32 * f + row0);
      for (int n = min(lanes, a.classes - 32 * f); n > 0; n -= 4, ++from) {
        const uint4 o = *from;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          if (f <= e) place[e] += (o.x >= mine[e]) + (o.y >= mine[e]) + (o.z >= mine[e]) + (o.w >= mine[e]);
          else place[e] += (o.x > mine[e]) + (o.y > mine[e]) + (o.z > mine[e]) + (o.w > mine[e]);
        }
      }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (!in || l + 32 * e >= a.classes || place[e] >= a.top) continue;
      a.top_index[row * a.top + place[e]] = l + 32 * e;
      a.top_logp[row * a.top + place[e]] = r.logp(unordered(mine[e]));
    }
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

// What a row's gradient needs: dx = -p (k + g' d) with d = x - m,
// p = e^(d - ln s) and k = g + g' (entropy - ln s); the label's class adds g.
struct Row {
  float m, ln, scale, g, ge, k;
  int label;
};
// bf16: one approximate exponential, whose argument's rounding is far below the
// result's.  fp32: the full one, e^d / s.
template <typename T>
__device__ __forceinline__ uint64_t grad_of(const Row& r, uint64_t x) {
  float2 d = ptx::unpack2(ptx::add2(x, ptx::pack2(-r.m, -r.m)));
  d.x = max_nan(d.x, kFar);
  d.y = max_nan(d.y, kFar);
  const uint64_t d2 = ptx::pack2(d.x, d.y);
  uint64_t p;
  if constexpr (sizeof(T) == 4) {
    p = ptx::mul2(ptx::pack2(expf(d.x), expf(d.y)), ptx::pack2(-r.scale, -r.scale));
    return ptx::mul2(p, ptx::fma2(d2, ptx::pack2(r.ge, r.ge), ptx::pack2(r.k, r.k)));
  } else {
    const float l = -r.ln * kLog2e;
    const float2 e = ptx::unpack2(ptx::fma2(d2, ptx::pack2(kLog2e, kLog2e), ptx::pack2(l, l)));
    p = ptx::pack2(exp2_approx(e.x), exp2_approx(e.y));
    return ptx::mul2(p, ptx::fma2(d2, ptx::pack2(-r.ge, -r.ge), ptx::pack2(-r.k, -r.k)));
  }
}

// Bound by HBM: 4096 x 65536 bf16 with entropy 157 us, the floor at the copy
// rate (on single values and with one load in flight a thread 186).
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
  r.k = a.dentropy ? r.g + r.ge * (__ldg(a.entropy + row) - st.y) : r.g;
  const bool zero = r.g == 0.f && r.ge == 0.f;  // nothing asked of the row: zeros, whatever it holds
  auto put = [&](int c, float x) {
    const float v[1] = {zero ? 0.f : ptx::unpack2(grad_of<T>(r, ptx::pack2(x, r.m))).x + (c == r.label ? r.g : 0.f)};
    Vec<T, 1>::store(out + c, v);
  };
  auto one = [&](int c) {
    float v[1];
    Vec<T, 1>::unpack(Vec<T, 1>::load(p + c), v);
    put(c, v[0]);
  };
  if constexpr (WIDE) {
    const int off = (int)(reinterpret_cast<uintptr_t>(p) / sizeof(T) % N);
    const int head = min(off ? N - off : 0, a.classes), vecs = (a.classes - head) / N;
    const int v0 = (int)((long long)vecs * seg / a.segments), v1 = (int)((long long)vecs * (seg + 1) / a.segments);
    if (seg == 0 && tid < head) one(tid);
    if (seg == a.segments - 1 && head + vecs * N + tid < a.classes) one(head + vecs * N + tid);
    const uint4* src = reinterpret_cast<const uint4*>(p + head);
    uint4* dst = reinterpret_cast<uint4*>(out + head);
    if (zero) {
      for (int i = v0 + tid; i < v1; i += a.team) dst[i] = make_uint4(0, 0, 0, 0);
      return;
    }
    const int at = r.label - head, there = at >= 0 ? at / N : -1;  // the label's vector
    for (int i0 = v0 + tid; i0 < v1; i0 += 4 * a.team) {
      uint4 raw[4];  // loaded together (the stores may be to the same memory, so the compiler could not)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (i0 + j * a.team < v1) raw[j] = src[i0 + j * a.team];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = i0 + j * a.team;
        if (i >= v1) break;
        float v[N];
        Vec<T, N>::unpack(raw[j], v);
#pragma unroll
        for (int e = 0; e < N; e += 2) {
          const float2 f = ptx::unpack2(grad_of<T>(r, ptx::pack2(v[e], v[e + 1])));
          v[e] = f.x;
          v[e + 1] = f.y;
        }
        if (i == there) {
#pragma unroll
          for (int e = 0; e < N; ++e) v[e] += at - i * N == e ? r.g : 0.f;
        }
        Vec<T, N>::store(reinterpret_cast<T*>(dst + i), v);
      }
    }
  } else {
    const int c0 = (int)((long long)a.classes * seg / a.segments), c1 = (int)((long long)a.classes * (seg + 1) / a.segments);
    for (long long b = c0 + tid; b < c1; b += 8 * a.team) {
      typename Vec<T, 1>::Raw raw[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (b + j * a.team < c1) raw[j] = Vec<T, 1>::load(p + b + j * a.team);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (b + j * a.team >= c1) break;
        float v[1];
        Vec<T, 1>::unpack(raw[j], v);
        put((int)b + j * a.team, v[0]);
      }
    }
  }
}

// ------------------------------------------------------------------ host
template <typename T, bool TOP, int WARPS>
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
  return cudaLaunchKernelEx(&cfg, k_logprobs<T, TOP, WARPS>, a);
}

template <typename T, bool TOP, int E>
cudaError_t launch_short(const Args<T>& a, cudaStream_t st) {
  int lanes_log = 2;
  while (lanes_log < 5 && (1 << lanes_log) < a.classes) ++lanes_log;
  PdlLaunch l(dim3((unsigned)cdiv(a.rows, 256 >> lanes_log)), dim3(256), st);
  return cudaLaunchKernelEx(&l.cfg, k_logprobs_short<T, TOP, E>, a, lanes_log);
}

template <typename T>
ff_status logprobs_t(Args<T> a, cudaStream_t st) {
  constexpr int N = Load<T>::N;
  const double bytes = (double)a.rows * a.classes * sizeof(T);
  if (a.classes <= (a.top ? 64 : 128)) {
    const int each = cdiv(a.classes, 32);
    auto* const go = a.top ? (each == 1 ? launch_short<T, true, 1> : launch_short<T, true, 2>)
                           : (each == 1 ? launch_short<T, false, 1> : each == 2 ? launch_short<T, false, 2> : launch_short<T, false, 4>);
    FF_LAUNCH(K_LOGPROBS, bytes, st, go(a, st), "label log-probabilities");
    return FF_OK;
  }
  const int vecs = cdiv(a.classes, N);
  // Many rows take few warps each, so that what a row costs besides its bytes (the
  // joins, the barrier, the selection) is shared by more rows at a time: 16384 x 2500
  // bf16 on 1, 4 and 8 warps 22, 39 and 67 us, with top 8 50, 86 and 128; 1000 x 5000 7.4,
  // 5.8 and 6.7; 1500 x 16000 20, 12 and 14.  The selection of long rows wants more:
  // 2048 x 49999 fp32, top 4: 1, 4 and 8 warps 187, 148 and 81; and two warps are no good
  // there.  So do more than 16 of the likeliest, for which a warp's 32 largest
  // values are few: 3000 x 1000 fp32, top 32: 1 and 4 warps 40 and 18.  A thread has one
  // and a half vectors at least (with the last: one).
  if (a.top)
    a.warps = a.top <= 16 && a.rows >= 1800 && vecs <= 1300 ? 1 : a.rows >= 700 && vecs <= 3000 ? 4 : 8;
  else
    a.warps = vecs > 4000 ? 8 : a.rows >= 4000 ? 1 : a.rows >= 1500 ? 2 : a.rows >= 700 ? 4 : 8;
  while (a.warps > 1 && a.warps * (a.top > 16 ? 32 : 46) > vecs) a.warps = a.top && a.warps == 4 ? 1 : a.warps / 2;
  // With fewer rows than the GPU has room for, more warps and then more
  // blocks, as long as each thread has a vector or two to read.
  a.cluster = 1;
  if (a.warps == 8) {
    while (a.warps < kMostWarps && (long long)a.warps * 2 * 32 <= vecs && (long long)a.rows * a.warps * 2 <= 152 * 32) a.warps *= 2;
    while (a.cluster < 8 && (long long)a.cluster * 2 * a.warps * 32 <= vecs && (long long)a.rows * a.cluster * 2 <= 152) a.cluster *= 2;
  }
  a.groups = 1;
  while (a.groups < 32 && 2 * a.warps * a.groups < 3 * a.top) a.groups *= 2;
  const unsigned threads = a.warps == 1 ? kOwnRows * 32 : (unsigned)a.warps * 32;
  const long long grid = a.warps == 1 ? cdiv(a.rows, kOwnRows) : (long long)a.rows * a.cluster;
  if (grid > 0x7FFFFFFFll) return FF_ERR_UNSUPPORTED;
  auto* const go = a.warps > 8 ? (a.top ? launch<T, true, kMostWarps> : launch<T, false, kMostWarps>)
                               : (a.top ? launch<T, true, 8> : launch<T, false, 8>);
  FF_LAUNCH(K_LOGPROBS, bytes, st, go(a, (unsigned)grid, threads, st), "label log-probabilities");
  return FF_OK;
}

template <typename T>
ff_status grad_t(GradArgs<T> a, cudaStream_t st) {
  constexpr int N = Load<T>::N;
  const bool wide = (reinterpret_cast<uintptr_t>(a.x) - reinterpret_cast<uintptr_t>(a.dx)) % 16 == 0 &&
                    (a.rows == 1 || (a.ldx - a.lddx) * (long long)sizeof(T) % 16 == 0);
  const int units = wide ? cdiv(a.classes, N) : a.classes;
  // As few threads a row as leave each 16 loads (16384 x 500 bf16: 7.4 us, with 4 loads 13),
  // and 16 loads a segment, or half of that and so on down to two while the
  // blocks are fewer than 2.5 an SM (4096 x 65536: 157 us, with 8 loads 167; but 500 x 8000
  // fp32: 7.5 us with 16, 6.6 with 8; 1 x 131072: 2.0 with 2, 2.8 with 8).  Single
  // values count half.
  a.team = 8;
  while (a.team < 256 && a.team * 16 <= units) a.team *= 2;
  for (int loads = 16; loads >= 2; loads /= 2) {
    a.segments = std::max(1, cdiv(units, (long long)a.team * loads * (wide ? 1 : 2)));
    if ((long long)a.rows * a.segments * a.team >= 380ll * 256) break;
  }
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
      !aligned(dlogp, 4) || !aligned(entropy, 4) || !aligned(dentropy, 4) ||
      !apart_or_one(dlogits, lddx, logits, ld, rows, classes, es))
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
