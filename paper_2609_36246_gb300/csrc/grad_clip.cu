// grad_clip.cu -- the 2-norm over all elements of a list of gradients, and the
// gradients scaled so that it is at most a limit (olive_grad_clip).
//
// The tensors are cut into units of 16 KB, numbered through; block b takes units
// b, b + blocks, ...  A thread squares 64 bytes of a unit at a time (32 bf16 or 16
// fp32 values) into one fp32 sum and adds that to an fp64 sum.  Where that fp32
// sum is not finite, large or nearly zero the same values, still in registers,
// are squared again scaled by a power of two: squares leave fp32's range long
// before the values do.  Every block's total goes to the workspace.  Values that are
// not in whole 16-byte pieces (a tensor's last few, all of one that starts off 16 bytes)
// are read one by one and squared in fp64.
//
// The second launch adds the blocks' totals (each block by itself: a few KB from
// L2), and scales, from the last unit to the first: what the first launch read
// last is still in the L2.
//
// What bounds it: HBM, each gradient read twice and written once (read once where
// all of them fit the L2): 2 GB in 915 us, of which the norm 282 (7.15 TB/s).  Of a
// tensor that starts off 16 bytes, the single loads and the fp64 squares: 1 GB of bf16
// takes 1819 us for the norm and 2946 with the scaling (176 and 477 where it is aligned;
// from empty caches).
#include <algorithm>
#include <cmath>

#include "internal.h"
#include "sm103.cuh"

namespace olive {
namespace {

constexpr int kThreads = 256;
constexpr int kVecs = 4;                               // 16-byte vectors of a thread's part of a unit
constexpr int kUnitBytes = kThreads * kVecs * 16;
constexpr int kBlocksPerSm = 6;
constexpr int kMaxBlocks = 192 * kBlocksPerSm;
constexpr int kMaxList = 512;                          // tensors of a launch

struct Entry {
  const void* src;
  void* dst;
  long long n;
  uint32_t unit0;  // its first unit
  uint32_t f32;
};
template <int N>
struct List {
  int count;
  uint32_t units;
  Entry e[N];
};

__device__ __forceinline__ bool aligned16_dev(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Values of a 16-byte vector.
template <bool kF32>
__device__ __forceinline__ void widen(const uint4& v, float (&x)[kF32 ? 4 : 8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (kF32) {
      x[i] = __uint_as_float(w[i]);
    } else {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}

// Sum of squares of a thread's vectors.
template <bool kF32>
__device__ __forceinline__ double squares(const uint4 (&v)[kVecs]) {
  constexpr int kPer = kF32 ? 4 : 8;
  float q = 0.f;
  uint32_t any = 0;
#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
    float x[kPer];
    widen<kF32>(v[k], x);
    any |= v[k].x | v[k].y | v[k].z | v[k].w;
#pragma unroll
    for (int i = 0; i < kPer; ++i) q = fmaf(x[i], x[i], q);
  }
  if (q < 1e36f && q > 1e-28f) return q;
  if (q != q) return q;  // a NaN among them: so it is in any width
  if ((any & (kF32 ? 0x7fffffffu : 0x7fff7fffu)) == 0) return 0.0;
  // The squares again, of values scaled by a power of two.  Small: none is above 1e-14,
  // so that 2^100 of it is at most 1.3e16, and the least fp32 value becomes 1.8e-15.
  // Large: 2^-70 of the largest fp32 value is 2.9e17; what it flushes is nothing beside
  // a value of 1.7e17 or more.  (The norm of 1 GB of values like 1e-30 or 1e30 takes
  // 168 us, 1902 with squares in fp64; in range 143.)
  const bool small = q <= 1e-28f;
  const float by = small ? 0x1p100f : 0x1p-70f;
  q = 0.f;
#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
    float x[kPer];
    widen<kF32>(v[k], x);
#pragma unroll
    for (int i = 0; i < kPer; ++i) q = fmaf(x[i] * by, x[i] * by, q);
  }
  return static_cast<double>(q) * (small ? 0x1p-200 : 0x1p140);
}

// A vector scaled by f.
template <bool kF32>
__device__ __forceinline__ uint4 scaled(const uint4& v, float f) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (kF32) {
      w[i] = __float_as_uint(__uint_as_float(w[i]) * f);
    } else {
      const __nv_bfloat162 h =
          __floats2bfloat162_rn(__uint_as_float(w[i] << 16) * f, __uint_as_float(w[i] & 0xffff0000u) * f);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ float value_at(const void* p, bool f32, int i) {
  return f32 ? static_cast<const float*>(p)[i] : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}
__device__ __forceinline__ void store_at(void* p, bool f32, int i, float v) {
  if (f32)
    static_cast<float*>(p)[i] = v;
  else
    static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
}

// Sum over the block, in a fixed order, in every thread.
__device__ double block_sum(double v, double* sums) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (threadIdx.x % 32 == 0) sums[threadIdx.x / 32] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) v += sums[i];
  return v;
}

// Unit u's place in the list, whose entry is at e or behind it (before it, in
// descending order).
struct Span {
  const char* src;
  char* dst;
  int n;      // values
  bool f32, whole;
};
template <int N>
__device__ __forceinline__ Span span(const List<N>& list, int e, uint32_t u) {
  const Entry& t = list.e[e];
  Span s;
  s.f32 = t.f32 != 0;
  const int per = kUnitBytes / (s.f32 ? 4 : 2);
  const long long at = static_cast<long long>(u - t.unit0);
  const long long left = t.n - at * per;
  s.n = static_cast<int>(min(left, static_cast<long long>(per)));
  s.whole = left >= per;
  s.src = static_cast<const char*>(t.src) + at * kUnitBytes;
  s.dst = static_cast<char*>(t.dst) + at * kUnitBytes;
  return s;
}

template <int N>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
    grad_norm_kernel(const __grid_constant__ List<N> list, double* part) {
  __shared__ double sums[kThreads / 32];
  double acc = 0.0;
  int e = 0;
  for (uint32_t u = blockIdx.x; u < list.units; u += gridDim.x) {
    while (e + 1 < list.count && u >= list.e[e + 1].unit0) ++e;
    const Span s = span(list, e, u);
    if (aligned16_dev(s.src)) {
      const uint4* v = reinterpret_cast<const uint4*>(s.src) + threadIdx.x;
      uint4 x[kVecs];
      if (s.whole) {
#pragma unroll
        for (int k = 0; k < kVecs; ++k) x[k] = __ldg(v + k * kThreads);
      } else {
        const int per = s.f32 ? 4 : 8, vecs = s.n / per, tail = s.n % per;
#pragma unroll
        for (int k = 0; k < kVecs; ++k)
          x[k] = k * kThreads + static_cast<int>(threadIdx.x) < vecs ? __ldg(v + k * kThreads) : make_uint4(0, 0, 0, 0);
        if (static_cast<int>(threadIdx.x) < tail) {  // values behind the last whole vector
          const double y = value_at(s.src, s.f32, s.n - tail + threadIdx.x);
          acc = fma(y, y, acc);
        }
      }
      acc += s.f32 ? squares<true>(x) : squares<false>(x);
    } else {
      for (int i = threadIdx.x; i < s.n; i += kThreads) {
        const double y = value_at(s.src, s.f32, i);
        acc = fma(y, y, acc);
      }
    }
  }
  grid_launch_dependents();
  const double s = block_sum(acc, sums);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

template <int N>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
    grad_scale_kernel(const __grid_constant__ List<N> list, const double* part, int parts, float max_norm,
                      float* norm) {
  __shared__ double sums[kThreads / 32];
  grid_wait();
  double total = 0.0;
  for (int i = threadIdx.x; i < parts; i += kThreads) total += part[i];
  total = sqrt(block_sum(total, sums));
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = static_cast<float>(total);
  const double ratio = static_cast<double>(max_norm) / (total + 1e-6);
  const float f = ratio >= 1.0 ? 1.f : static_cast<float>(ratio);  // (NaN stays NaN)

  int e = list.count - 1;
  for (long long w = static_cast<long long>(list.units) - 1 - blockIdx.x; w >= 0; w -= gridDim.x) {
    const uint32_t u = static_cast<uint32_t>(w);
    while (u < list.e[e].unit0) --e;
    const Span s = span(list, e, u);
    if (f == 1.f && s.src == s.dst) continue;
    if (aligned16_dev(s.src) && aligned16_dev(s.dst)) {
      const uint4* v = reinterpret_cast<const uint4*>(s.src) + threadIdx.x;
      uint4* o = reinterpret_cast<uint4*>(s.dst) + threadIdx.x;
      const int per = s.f32 ? 4 : 8, vecs = s.n / per, tail = s.n % per;
      uint4 x[kVecs];
      if (s.whole) {
#pragma unroll
        for (int k = 0; k < kVecs; ++k) x[k] = v[k * kThreads];
#pragma unroll
        for (int k = 0; k < kVecs; ++k) o[k * kThreads] = s.f32 ? scaled<true>(x[k], f) : scaled<false>(x[k], f);
      } else {
#pragma unroll
        for (int k = 0; k < kVecs; ++k)
          if (k * kThreads + static_cast<int>(threadIdx.x) < vecs) x[k] = v[k * kThreads];
#pragma unroll
        for (int k = 0; k < kVecs; ++k)
          if (k * kThreads + static_cast<int>(threadIdx.x) < vecs)
            o[k * kThreads] = s.f32 ? scaled<true>(x[k], f) : scaled<false>(x[k], f);
        if (static_cast<int>(threadIdx.x) < tail) {
          const int i = s.n - tail + threadIdx.x;
          store_at(s.dst, s.f32, i, value_at(s.src, s.f32, i) * f);
        }
      }
    } else {
      for (int i = threadIdx.x; i < s.n; i += kThreads) store_at(s.dst, s.f32, i, value_at(s.src, s.f32, i) * f);
    }
  }
}

// Tensors [i0, i1) of the caller's list.
template <int N>
List<N> make_list(const void* const* src, void* const* dst, const int64_t* numel, const int32_t* dtype, int i0,
                  int i1) {
  List<N> l;
  l.count = 0;
  l.units = 0;
  for (int i = i0; i < i1; ++i) {
    if (numel[i] == 0) continue;
    Entry& e = l.e[l.count++];
    e.src = src[i];
    e.dst = dst ? dst[i] : nullptr;
    e.n = numel[i];
    e.unit0 = l.units;
    e.f32 = dtype[i] == OLIVE_DTYPE_F32;
    l.units += static_cast<uint32_t>(ceil_div(numel[i] * (e.f32 ? 4 : 2), kUnitBytes));
  }
  return l;
}

template <int N>
olive_status run(const Ctx& c, const void* const* src, void* const* dst, const int64_t* numel, const int32_t* dtype,
                 int32_t n, float max_norm, float* norm, double* part) {
  const int most = std::min(c.num_sms * kBlocksPerSm, kMaxBlocks);
  int parts = 0;
  for (int i = 0; i < n; i += N) {
    const List<N> l = make_list<N>(src, dst, numel, dtype, i, std::min(n, i + N));
    const int blocks = static_cast<int>(std::min<int64_t>(l.units, most));
    if (blocks > 0) grad_norm_kernel<N><<<blocks, kThreads, 0, c.stream>>>(l, part + parts);
    parts += blocks;
  }
  for (int i = 0; i < std::max(n, 1); i += N) {
    List<N> l = make_list<N>(src, dst, numel, dtype, i, dst ? std::min(n, i + N) : i);
    const int blocks = static_cast<int>(std::min<int64_t>(l.units, most));
    // starts while the launch ahead ends, and waits for it by itself
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(std::max(blocks, 1)));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = c.stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaLaunchKernelEx(&cfg, grad_scale_kernel<N>, l, static_cast<const double*>(part), parts, max_norm, norm);
    if (!dst) break;
  }
  return cudaGetLastError() == cudaSuccess ? OLIVE_OK : OLIVE_ERR_CUDA;
}

}  // namespace

size_t grad_clip_ws_bytes(int64_t n) { return align_up(8ull * kMaxBlocks * ceil_div(n, kMaxList), kWsAlign); }

olive_status launch_grad_clip(const Ctx& c, const void* const* src, void* const* dst, const int64_t* numel,
                              const int32_t* dtype, int32_t n, float max_norm, float* norm, void* ws) {
  double* part = static_cast<double*>(ws);
  // (the list travels in the launch's parameters: the short one costs less to launch)
  return n <= 48 ? run<48>(c, src, dst, numel, dtype, n, max_norm, norm, part)
                 : run<kMaxList>(c, src, dst, numel, dtype, n, max_norm, norm, part);
}

}  // namespace olive
