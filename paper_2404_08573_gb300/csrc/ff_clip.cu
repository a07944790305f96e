// The 2-norm over many gradients, and the gradients scaled so that it is at
// most max_norm:  norm = sqrt(sum g^2), out = g min(1, max_norm / norm).
//
// The tensors are cut into pieces of 16 KB that thread groups of 256 take in
// turn.  Few pieces: one cluster of blocks keeps them in registers between the
// sum and the product (one read; 24010 fp32 values: 4.6 us).  Many: a pass for the
// sums, one partial a block, and a pass in the opposite order for the products,
// which finds the last pieces in L2 (all others are read and written as first to
// be evicted; where it clips nothing in place it gives them their ordinary
// priority back).  Bound by HBM, two reads and a write: 268 M fp32 values in 486 us, 6.6 TB/s
// (without the policies 503).
#include <algorithm>
#include <vector>

#include "ff_api_internal.h"
#include "ff_ptx.cuh"
#include "ff_vec.cuh"

namespace ff {
namespace {

constexpr int GROUP = 256;             // threads that take a piece
constexpr int VECS = 4;                // 16-byte vectors of it per thread
constexpr int PIECE = GROUP * VECS * 16;  // bytes
constexpr int kTable = 120;            // tensors a launch
constexpr int kResident = 5;           // blocks of the two passes an SM holds (one group each): 80 KB of loads in flight
constexpr int kBlocks = 152 * kResident;
constexpr int kKeep = (64 << 20) / PIECE;  // pieces that the first pass leaves in L2 for the second
constexpr int kClusterBlocks = 8, kClusterGroups = 4, kKept = 2;  // pieces kept: 8 * 4 * 2

struct Table {
  const void* in[kTable];
  void* out[kTable];
  long long count[kTable];
  int first[kTable + 1];  // a tensor's first piece; [n]: all pieces
  uint8_t bf16s[kTable];
  int n;
};

__device__ __forceinline__ int tensor_of(const Table& t, int piece) {
  int lo = 0, hi = t.n - 1;  // the last tensor whose first piece is not behind this one
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= piece) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// min(1, max_norm / norm) as two factors, the first a power of two: 1, but where the
// ratio lies near or below the end of fp32's normal range and would be rounded to
// few bits.  Gradients are brought to the norm's order of magnitude there.
struct Factor {
  float first, then;
  __device__ __forceinline__ bool one() const { return then == 1.f && first == 1.f; }
};
// 1 where nothing is to be clipped, as with an infinite max_norm whatever the
// norm is; else NaN for a NaN norm.
__device__ __forceinline__ Factor factor(float norm, float max_norm) {
  const float by = __fdiv_rn(max_norm, norm);
  if (by >= 0x1p-100f && by < INFINITY) return Factor{1.f, fminf(by, 1.f)};
  if (isinf(max_norm) || norm == 0.f || by > 1.f) return Factor{1.f, 1.f};
  if (!(by < 0x1p-100f) || isinf(norm) || max_norm == 0.f) return Factor{1.f, by};
  // 2^-floor(log2 norm), at least 2^-126 (norm > 2^-49, since no max_norm is below 2^-149)
  const float first = __uint_as_float(max(254u - (__float_as_uint(norm) >> 23), 1u) << 23);
  return Factor{first, __fdiv_rn(max_norm, norm * first)};
}

// One thread's part of a piece, as loaded.  Past the end: zeros.
template <typename T>
struct Piece {
  static constexpr int N = 16 / (int)sizeof(T);
  static __device__ __forceinline__ void load(uint4 (&r)[VECS], const T* p, long long left, int tid, bool wide, uint64_t policy) {
#pragma unroll
    for (int j = 0; j < VECS; ++j) {
      const int i = (j * GROUP + tid) * N;
      if (wide && i + N <= left) {
        r[j] = ptx::ld_hint(p + i, policy);
      } else {
        T v[N];
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = i + e < left ? p[i + e] : T(0.f);
        memcpy(&r[j], v, 16);
      }
    }
  }
  // The sum of the squares; SCALED: of the values times `by`.
  template <bool SCALED>
  static __device__ __forceinline__ float squares(const uint4 (&r)[VECS], float by) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < VECS; ++j) {
      float v[N];
      Vec<T, N>::unpack(r[j], v);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        if (SCALED) v[e] *= by;
        s = fmaf(v[e], v[e], s);
      }
    }
    return s;
  }
  static __device__ __forceinline__ void store(const uint4 (&r)[VECS], T* p, long long left, int tid, bool wide, Factor by,
                                               uint64_t policy) {
#pragma unroll
    for (int j = 0; j < VECS; ++j) {
      const int i = (j * GROUP + tid) * N;
      float v[N];
      Vec<T, N>::unpack(r[j], v);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = v[e] * by.first * by.then;
      if (wide && i + N <= left) {
        uint4 o;
        Vec<T, N>::store(reinterpret_cast<T*>(&o), v);
        ptx::st_hint(p + i, o, policy);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float one[1] = {v[e]};
          if (i + e < left) Vec<T, 1>::store(p + i + e, one);
        }
      }
    }
  }
};
__device__ __forceinline__ bool wide_at(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// What a piece is: its tensor, where it starts and what is left of the tensor from there.
struct At {
  int t;
  long long from, left;
};
__device__ __forceinline__ At at_piece(const Table& t, int piece) {
  At a;
  a.t = tensor_of(t, piece);
  a.from = (long long)(piece - t.first[a.t]) * (PIECE / (t.bf16s[a.t] ? 2 : 4));
  a.left = t.count[a.t] - a.from;
  return a;
}
__device__ __forceinline__ void load_piece(const Table& t, const At& a, uint4 (&r)[VECS], int tid, uint64_t policy) {
  const bool wide = wide_at(t.in[a.t]);
  if (t.bf16s[a.t]) Piece<bf16>::load(r, static_cast<const bf16*>(t.in[a.t]) + a.from, a.left, tid, wide, policy);
  else Piece<float>::load(r, static_cast<const float*>(t.in[a.t]) + a.from, a.left, tid, wide, policy);
}
template <bool SCALED>
__device__ __forceinline__ float piece_squares(const Table& t, const At& a, const uint4 (&r)[VECS], float by) {
  return t.bf16s[a.t] ? Piece<bf16>::template squares<SCALED>(r, by) : Piece<float>::template squares<SCALED>(r, by);
}
__device__ __forceinline__ void store_piece(const Table& t, const At& a, const uint4 (&r)[VECS], int tid, Factor by, uint64_t policy) {
  const bool wide = wide_at(t.out[a.t]);
  if (t.bf16s[a.t]) Piece<bf16>::store(r, static_cast<bf16*>(t.out[a.t]) + a.from, a.left, tid, wide, by, policy);
  else Piece<float>::store(r, static_cast<float*>(t.out[a.t]) + a.from, a.left, tid, wide, by, policy);
}

// Takes back the priority with which a piece was left in L2.
__device__ __forceinline__ void release_piece(const Table& t, const At& a, int tid) {
  const int es = t.bf16s[a.t] ? 2 : 4;
  const char* const p = static_cast<const char*>(t.in[a.t]) + a.from * es;
  const char* const line = reinterpret_cast<const char*>(reinterpret_cast<uintptr_t>(p) & ~uintptr_t(127)) + 128 * tid;
  if (line < p + min((long long)PIECE, a.left * es)) ptx::l2_evict_normal_line(line);
}

// The fp64 units take two lanes a clock and SM, so a thread's sums are fp32 (two
// of them: the sum and what its roundings lost), a warp's too, and only one lane
// a warp goes on in fp64, one thread to the square root (with both on every
// thread 24010 values took 8.2 us, 2 M 24).
//
// fp32 holds these sums where a piece's lies in [2^-115, 2^96]: what its 32 squares lost
// by underflow, at most 2^-150 each, is then below 2^-30 of it, and neither 2^22 pieces nor
// a warp's overflow.  A thread whose piece lies elsewhere (vanished or exploding
// gradients) squares it again, times a power of two that brings every fp32
// magnitude of that side into range, and adds that to `far` in fp64 (24000 such values
// 7.3 us for 4.9; 67 M, at HBM's rate, as others).
__device__ __forceinline__ bool any_bit(const uint4 (&r)[VECS]) {
  uint32_t o = 0;
#pragma unroll
  for (int j = 0; j < VECS; ++j) o |= r[j].x | r[j].y | r[j].z | r[j].w;
  return o != 0;
}
struct Sum {
  float hi = 0.f, lo = 0.f;
  double far = 0.0;
  bool has_far = false;  // (the comparison far != 0 takes the fp64 units a quarter us in a block of 1024)
  __device__ __forceinline__ void add(float v) {  // Knuth's two-sum
    const float s = __fadd_rn(hi, v), t = __fsub_rn(s, hi);
    lo = __fadd_rn(lo, __fadd_rn(__fsub_rn(hi, __fsub_rn(s, t)), __fsub_rn(v, t)));
    hi = s;
  }
  __device__ __forceinline__ void add(const Table& t, const At& a, const uint4 (&r)[VECS]) {
    const float s = piece_squares<false>(t, a, r, 1.f);
    if (s >= 0x1p-115f && s <= 0x1p96f) {
      add(s);
    } else if (s != 0.f || any_bit(r)) {  // (a NaN comes here too)
      const bool small = s < 1.f;
      const float q = piece_squares<true>(t, a, r, small ? 0x1p96f : 0x1p-70f);
      if (q != 0.f) {
        far = fma((double)q, small ? 0x1p-192 : 0x1p140, far);
        has_far = true;
      }
    }
  }
  __device__ __forceinline__ float value() const { return hi + lo; }
};
template <typename F>
__device__ __forceinline__ F warp_sum(F v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// The block's warps' sums, to be read after the call.
__device__ __forceinline__ void warp_totals(const Sum& s, double* warps, int warp, int lane) {
  const float f = warp_sum(s.value());
  if (lane == 0) warps[warp] = f;
  if (__syncthreads_or(s.has_far)) {
    const double d = warp_sum(s.far);
    if (lane == 0) warps[warp] += d;
    __syncthreads();
  }
}
// sqrt of a sum of squares, in fp32: past its range either way, by powers of two.
__device__ __forceinline__ float norm_of(double s) {
  const bool big = s > 1e38, small = s < 1e-30;
  const float r = __fsqrt_rn((float)(s * (big ? 0x1p-128 : small ? 0x1p192 : 1.0)));
  return big ? r * 0x1p64f : small ? r * 0x1p-96f : r;  // an infinity and NaN stay
}

// All pieces in one cluster's registers.
__global__ void __launch_bounds__(GROUP * kClusterGroups, 1)
    k_clip_small(const __grid_constant__ Table t, float max_norm, float* norm_out, int pieces, int nblocks) {
  __shared__ double part[kClusterBlocks];
  __shared__ double warps[GROUP * kClusterGroups / 32];
  __shared__ float shared_norm;
  if (nblocks > 1) ptx::cluster_arrive();
  ptx::griddep_wait();
  const int rank = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int groups = blockDim.x / GROUP, tid = threadIdx.x & (GROUP - 1);
  const int first = rank * groups + threadIdx.x / GROUP, step = groups * nblocks;
  uint4 r[kKept][VECS];
  At at[kKept];
  Sum s;
#pragma unroll
  for (int k = 0; k < kKept; ++k)
    if (first + k * step < pieces) {
      at[k] = at_piece(t, first + k * step);
      load_piece(t, at[k], r[k], tid, ptx::l2_evict_normal());
    }
#pragma unroll
  for (int k = 0; k < kKept; ++k)
    if (first + k * step < pieces) s.add(t, at[k], r[k]);
  warp_totals(s, warps, warp, lane);
  if (nblocks > 1) ptx::cluster_wait();
  if (warp == 0) {
    const double d = warp_sum(lane < (int)(blockDim.x >> 5) ? warps[lane] : 0.0);
    if (nblocks == 1) {
      if (lane == 0) part[0] = d;
    } else if (lane < nblocks) {
      const uint2 w = make_uint2((uint32_t)__double2loint(d), (uint32_t)__double2hiint(d));
      ptx::st_remote_u2(reinterpret_cast<uint2*>(&part[rank]), (uint32_t)lane, w);
    }
    __syncwarp();
  }
  if (nblocks > 1) ptx::cluster_sync();
  if (threadIdx.x == 0) {
    double d = part[0];
    for (int b = 1; b < nblocks; ++b) d += part[b];
    shared_norm = norm_of(d);
    if (rank == 0) *norm_out = shared_norm;
  }
  __syncthreads();
  const Factor by = factor(shared_norm, max_norm);
#pragma unroll
  for (int k = 0; k < kKept; ++k)
    if (first + k * step < pieces && (!by.one() || t.in[at[k].t] != t.out[at[k].t])) store_piece(t, at[k], r[k], tid, by, ptx::l2_evict_normal());
}

// part[blockIdx.x] = the sum of squares of the block's pieces.
__global__ void __launch_bounds__(GROUP, kResident) k_clip_sums(const __grid_constant__ Table t, int pieces, int keep_from, double* part) {
  __shared__ double warps[GROUP / 32];
  ptx::griddep_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint64_t first = ptx::l2_evict_first(), last = ptx::l2_evict_last();
  Sum s;
  for (int p = blockIdx.x; p < pieces; p += gridDim.x) {
    uint4 r[VECS];
    const At a = at_piece(t, p);
    load_piece(t, a, r, threadIdx.x, p >= keep_from ? last : first);
    s.add(t, a, r);
  }
  warp_totals(s, warps, warp, lane);
  if (threadIdx.x == 0) {
    double d = warps[0];
    for (int w = 1; w < GROUP / 32; ++w) d += warps[w];
    part[blockIdx.x] = d;
  }
}
__global__ void __launch_bounds__(GROUP, kResident)
    k_clip_scale(const __grid_constant__ Table t, int pieces, int keep_from, const double* part, int parts, float max_norm,
                 float* norm_out) {
  __shared__ float shared_norm;
  ptx::griddep_wait();
  if (threadIdx.x < 32) {
    double d = 0.0;
    for (int i = threadIdx.x; i < parts; i += 32) d += part[i];
    d = warp_sum(d);
    if (threadIdx.x == 0) {
      shared_norm = norm_of(d);
      if (blockIdx.x == 0) *norm_out = shared_norm;
    }
  }
  __syncthreads();
  const Factor by = factor(shared_norm, max_norm);
  const uint64_t first = ptx::l2_evict_first();
  for (int p = pieces - 1 - (int)blockIdx.x; p >= 0; p -= gridDim.x) {
    const At a = at_piece(t, p);
    if (by.one() && t.in[a.t] == t.out[a.t]) {
      if (p >= keep_from) release_piece(t, a, threadIdx.x);
      continue;
    }
    uint4 r[VECS];
    load_piece(t, a, r, threadIdx.x, first);
    store_piece(t, a, r, threadIdx.x, by, first);
  }
}

struct Tensor {
  const void* in;
  void* out;
  long long count;
  bool half;
  long long bytes() const { return count * (half ? 2 : 4); }
};

int tables_of(int n) { return n <= kTable ? 1 : cdiv(n, kTable); }

ff_status clip(const std::vector<Tensor>& all, float max_norm, float* norm, double* part, cudaStream_t st) {
  const int n = (int)all.size(), tables = tables_of(n);
  std::vector<Table> ts((size_t)tables);
  std::vector<long long> bytes((size_t)tables, 0);
  long long total = 0;
  for (int k = 0; k < tables; ++k) {
    Table& t = ts[k];
    t.n = 0;
    long long pieces = 0;
    for (int i = k * kTable; i < n && i < (k + 1) * kTable; ++i) {
      const Tensor& e = all[i];
      t.in[t.n] = e.in;
      t.out[t.n] = e.out;
      t.count[t.n] = e.count;
      t.bf16s[t.n] = e.half;
      t.first[t.n++] = (int)pieces;
      pieces += (e.bytes() + PIECE - 1) / PIECE;
      if (pieces > 0x7FFF0000ll) return FF_ERR_UNSUPPORTED;
      bytes[k] += e.bytes();
    }
    t.first[t.n] = (int)pieces;
    total += pieces;
  }
  if (tables == 1 && total <= kClusterBlocks * kClusterGroups * kKept) {
    const int blocks = total <= kClusterGroups ? 1 : total <= 2 * kClusterGroups ? 2 : total <= 4 * kClusterGroups ? 4 : kClusterBlocks;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3((unsigned)(GROUP * std::max(1, (int)std::min<long long>(total, kClusterGroups))));
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)blocks;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    FF_LAUNCH(K_CLIP, 2.0 * bytes[0], st, cudaLaunchKernelEx(&cfg, k_clip_small, ts[0], max_norm, norm, (int)total, blocks),
              "gradient clipping");
    return FF_OK;
  }
  for (int k = 0; k < tables; ++k) {
    PdlLaunch l(dim3(kBlocks), dim3(GROUP), st);
    FF_LAUNCH(K_CLIP, (double)bytes[k], st,
              cudaLaunchKernelEx(&l.cfg, k_clip_sums, ts[k], ts[k].first[ts[k].n], std::max(0, ts[k].first[ts[k].n] - kKeep), part + (long long)k * kBlocks),
              "gradient clipping");
  }
  for (int k = tables - 1; k >= 0; --k) {
    PdlLaunch l(dim3(kBlocks), dim3(GROUP), st);
    FF_LAUNCH(K_CLIP, 2.0 * bytes[k], st,
              cudaLaunchKernelEx(&l.cfg, k_clip_scale, ts[k], ts[k].first[ts[k].n], std::max(0, ts[k].first[ts[k].n] - kKeep),
                                 (const double*)part, tables * kBlocks, max_norm, norm),
              "gradient clipping");
  }
  return FF_OK;
}

}  // namespace
}  // namespace ff

using namespace ff;

extern "C" FF_API long long ff_clip_grad_norm_workspace(int n) {
  return n < 0 ? -1 : 8ll * kBlocks * tables_of(n);
}

extern "C" FF_API ff_status ff_clip_grad_norm(const void* const* grads, void* const* out, const long long* counts,
                                              const int* precs, int n, float max_norm, float* norm, void* workspace,
                                              long long workspace_bytes, void* stream) {
  if (n < 0 || !(max_norm >= 0.f) || !norm || reinterpret_cast<uintptr_t>(norm) % 4 != 0 ||
      (n > 0 && (!grads || !out || !counts || !precs)))
    return FF_ERR_INVALID_ARG;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 16 != 0 || workspace_bytes < ff_clip_grad_norm_workspace(n))
    return FF_ERR_INVALID_ARG;
  try {
    std::vector<Tensor> all;
    all.reserve((size_t)n);
    for (int i = 0; i < n; ++i) {
      if (precs[i] != FF_FP32 && precs[i] != FF_BF16) return FF_ERR_INVALID_ARG;
      const int es = precs[i] == FF_BF16 ? 2 : 4;
      if (counts[i] < 0 || counts[i] > (1ll << 60)) return FF_ERR_INVALID_ARG;
      if (counts[i] == 0) continue;
      if (!grads[i] || !out[i] || reinterpret_cast<uintptr_t>(grads[i]) % es != 0 ||
          reinterpret_cast<uintptr_t>(out[i]) % es != 0)
        return FF_ERR_INVALID_ARG;
      all.push_back(Tensor{grads[i], out[i], counts[i], precs[i] == FF_BF16});
    }
    // An output may be its own gradient; otherwise no output overlaps another
    // output or any gradient (a piece is read long after others are written).
    struct Span {
      uintptr_t from, to;
      int owner;
      bool write;
    };
    std::vector<Span> spans;
    spans.reserve(2 * all.size());
    for (size_t i = 0; i < all.size(); ++i) {
      const Tensor& e = all[i];
      const uintptr_t o = reinterpret_cast<uintptr_t>(e.out), g = reinterpret_cast<uintptr_t>(e.in);
      spans.push_back(Span{o, o + (uintptr_t)e.bytes(), (int)i, true});
      if (g != o) spans.push_back(Span{g, g + (uintptr_t)e.bytes(), (int)i, false});
    }
    std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.from < b.from; });
    uintptr_t written = 0, read = 0;  // ends of what outputs and gradients have covered so far
    for (const Span& s : spans) {
      if (s.from < written || (s.write && s.from < read)) return FF_ERR_INVALID_ARG;
      if (s.write) written = std::max(written, s.to);
      else read = std::max(read, s.to);
    }
    return clip(all, max_norm, norm, static_cast<double*>(workspace), static_cast<cudaStream_t>(stream));
  } catch (...) {
    return FF_ERR_OOM;
  }
}
