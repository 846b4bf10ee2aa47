// row_norm.cu -- layer norm and RMS norm of the hidden rows, forward and backward,
// with the residual's sum on the way and the weights' gradients.
//
// A row is held in registers by a group of threads, eight values a vector and up to
// four vectors a thread, so it is read once: the mean, the mean square of what is
// left and the result all come from the same registers.  The forward keeps each row's
// mean and reciprocal deviation for the backward, whose two sums (of a = dy w and of
// a n) then come from one exchange.
//
// Backward: a block takes every so-manieth row, so that a thread keeps the weights'
// gradients of its columns in registers from beginning to end; the blocks' sums are
// stored and added in a second launch, in fp64 and a fixed order.
#include <algorithm>

#include "internal.h"
#include "sm103.cuh"

namespace olive {
namespace {

constexpr int kMaxBlocks = 1024;  // blocks whose partial weight gradients the workspace holds

// Eight values of a row.
template <typename T>
struct Eight;
template <>
struct Eight<__nv_bfloat16> {
  using Raw = uint4;
  static __device__ __forceinline__ void get(const Raw& r, float (&v)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ Raw put(const float (&v)[8]) {
    return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                      pack_bf16x2(v[6], v[7]));
  }
};
template <>
struct Eight<float> {
  struct alignas(16) Raw {
    float4 a, b;
  };
  static __device__ __forceinline__ void get(const Raw& r, float (&v)[8]) {
    v[0] = r.a.x, v[1] = r.a.y, v[2] = r.a.z, v[3] = r.a.w;
    v[4] = r.b.x, v[5] = r.b.y, v[6] = r.b.z, v[7] = r.b.w;
  }
  static __device__ __forceinline__ Raw put(const float (&v)[8]) {
    return {make_float4(v[0], v[1], v[2], v[3]), make_float4(v[4], v[5], v[6], v[7])};
  }
};

template <int G>
constexpr int threads_of() {
  return G < 128 ? 128 : G;
}

// Sums of kN values over a group of G threads, the same bits in every thread.  `slot`
// alternates between calls, so that one barrier a call is enough.
template <int G, int kN>
__device__ __forceinline__ void group_sum(float (&v)[kN], float (*red)[threads_of<G>() / 32][kN], int slot) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  if constexpr (G > 32) {
    const int warp = threadIdx.x / 32;
    if (threadIdx.x % 32 == 0)
#pragma unroll
      for (int i = 0; i < kN; ++i) red[slot][warp][i] = v[i];
    __syncthreads();
    const int first = warp / (G / 32) * (G / 32);
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = 0.f;
#pragma unroll
    for (int w = 0; w < G / 32; ++w)
#pragma unroll
      for (int i = 0; i < kN; ++i) v[i] += red[slot][first + w][i];
  }
}

template <typename T, int G, int NV, bool kCentre>
__global__ void __launch_bounds__(threads_of<G>()) norm_fwd_kernel(const NormArgs p) {
  using V = Eight<T>;
  using Raw = typename V::Raw;
  constexpr int kGroups = threads_of<G>() / G;
  __shared__ float red[2][threads_of<G>() / 32][1];
  const int lane = threadIdx.x % G;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kGroups + threadIdx.x / G;
  const bool live = row < p.T;
  const int nv = p.d / 8;
  const Raw* x = static_cast<const Raw*>(p.x) + row * nv;
  const float inv_d = 1.f / p.d;

  Raw raw[NV];
  if (live) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (lane + G * k < nv) raw[k] = x[lane + G * k];
  }
  if (live && p.residual) {
    const Raw* res = static_cast<const Raw*>(p.residual) + row * nv;
    Raw* sum = static_cast<Raw*>(p.sum) + row * nv;
    Raw add[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (lane + G * k < nv) add[k] = res[lane + G * k];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      if (lane + G * k >= nv) continue;
      float a[8], b[8];
      V::get(raw[k], a);
      V::get(add[k], b);
#pragma unroll
      for (int e = 0; e < 8; ++e) a[e] += b[e];
      // (the norm is that of the sum as it is kept, which the backward reads)
      raw[k] = V::put(a);
      sum[lane + G * k] = raw[k];
    }
  }

  float s[1] = {0.f}, mean = 0.f;
  if constexpr (kCentre) {
    if (live) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        if (lane + G * k >= nv) continue;
        float a[8];
        V::get(raw[k], a);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] += a[e];
      }
    }
    group_sum<G>(s, red, 0);
    mean = s[0] * inv_d;
    s[0] = 0.f;
  }
  if (live) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      if (lane + G * k >= nv) continue;
      float a[8];
      V::get(raw[k], a);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[0] = fmaf(a[e] - mean, a[e] - mean, s[0]);
    }
  }
  group_sum<G>(s, red, 1);
  const float r = rsqrtf(fmaf(s[0], inv_d, p.eps));
  if (!live) return;
  if (p.stats && lane == 0) {
    p.stats[row] = mean;
    p.stats[p.T + row] = r;
  }
  Raw* y = static_cast<Raw*>(p.y) + row * nv;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int at = lane + G * k;
    if (at >= nv) continue;
    float a[8], w[8], b[8] = {};
    V::get(raw[k], a);
    V::get(static_cast<const Raw*>(p.w)[at], w);
    if (p.b) V::get(static_cast<const Raw*>(p.b)[at], b);
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = fmaf((a[e] - mean) * r, w[e], b[e]);
    y[at] = V::put(a);
  }
}

template <typename T, int G, int NV, bool kCentre>
__global__ void __launch_bounds__(threads_of<G>()) norm_bwd_kernel(const NormArgs p) {
  using V = Eight<T>;
  using Raw = typename V::Raw;
  constexpr int kGroups = threads_of<G>() / G;
  __shared__ float red[2][threads_of<G>() / 32][2];
  const int lane = threadIdx.x % G;
  const int nv = p.d / 8;
  const float inv_d = 1.f / p.d;
  float dw[NV][8] = {}, db[NV][8] = {};
  int slot = 0;
  // (all groups of a block go round as often: they share its barriers)
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * kGroups; first < p.T;
       first += static_cast<int64_t>(gridDim.x) * kGroups, slot ^= 1) {
    const int64_t row = first + threadIdx.x / G;
    const bool live = row < p.T;
    Raw xr[NV], gr[NV];
    float mean = 0.f, r = 0.f;
    if (live) {
      const Raw* x = static_cast<const Raw*>(p.x) + row * nv;
      const Raw* g = static_cast<const Raw*>(p.dy) + row * nv;
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (lane + G * k < nv) {
          xr[k] = x[lane + G * k];
          gr[k] = g[lane + G * k];
        }
      mean = kCentre ? p.stats[row] : 0.f;
      r = p.stats[p.T + row];
    }
    float s[2] = {0.f, 0.f};
    if (live) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int at = lane + G * k;
        if (at >= nv) continue;
        float n[8], g[8], w[8];
        V::get(xr[k], n);
        V::get(gr[k], g);
        V::get(static_cast<const Raw*>(p.w)[at], w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          n[e] = (n[e] - mean) * r;
          dw[k][e] = fmaf(g[e], n[e], dw[k][e]);
          db[k][e] += g[e];
          const float a = g[e] * w[e];
          s[0] += a;
          s[1] = fmaf(a, n[e], s[1]);
        }
      }
    }
    group_sum<G>(s, red, slot);
    const float ma = kCentre ? s[0] * inv_d : 0.f, man = s[1] * inv_d;
    if (!live) continue;
    const Raw* gs = static_cast<const Raw*>(p.g_sum) + row * nv;
    Raw* dx = static_cast<Raw*>(p.dx) + row * nv;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int at = lane + G * k;
      if (at >= nv) continue;
      float n[8], g[8], w[8], more[8] = {};
      V::get(xr[k], n);
      V::get(gr[k], g);
      V::get(static_cast<const Raw*>(p.w)[at], w);
      if (p.g_sum) V::get(gs[at], more);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        n[e] = (n[e] - mean) * r;
        g[e] = fmaf(r, fmaf(-n[e], man, g[e] * w[e] - ma), more[e]);
      }
      dx[at] = V::put(g);
    }
  }
  grid_launch_dependents();
  // [block's group][dw, db][d]
  float* part = static_cast<float*>(p.ws) + (static_cast<size_t>(blockIdx.x) * kGroups + threadIdx.x / G) * 2 * p.d;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int at = lane + G * k;
    if (at >= nv) continue;
    float4* a = reinterpret_cast<float4*>(part + 8 * at);
    float4* b = reinterpret_cast<float4*>(part + p.d + 8 * at);
    a[0] = make_float4(dw[k][0], dw[k][1], dw[k][2], dw[k][3]);
    a[1] = make_float4(dw[k][4], dw[k][5], dw[k][6], dw[k][7]);
    b[0] = make_float4(db[k][0], db[k][1], db[k][2], db[k][3]);
    b[1] = make_float4(db[k][4], db[k][5], db[k][6], db[k][7]);
  }
}

// dw (blockIdx.y = 0) and db (1): the groups' sums added, 32 columns a block.
__global__ void __launch_bounds__(1024) norm_dw_kernel(const float* part, int groups, int d, float* dw, float* db) {
  __shared__ double sums[32][32];
  grid_wait();
  const int lane = threadIdx.x % 32, g = threadIdx.x / 32, col = blockIdx.x * 32 + lane;
  double v = 0.0;
  if (col < d) {
    const float* at = part + static_cast<size_t>(blockIdx.y) * d + col;
#pragma unroll 8
    for (int b = g; b < groups; b += 32) v += static_cast<double>(at[static_cast<size_t>(b) * 2 * d]);
  }
  sums[g][lane] = v;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    __syncthreads();
    if (g < o) sums[g][lane] += sums[g + o][lane];
  }
  if (g == 0 && col < d) (blockIdx.y ? db : dw)[col] = static_cast<float>(sums[0][lane]);
}

template <typename T, int G, int NV>
void run_fwd(const Ctx& c, const NormArgs& a) {
  constexpr int kGroups = threads_of<G>() / G;
  const unsigned blocks = static_cast<unsigned>(ceil_div(a.T, kGroups));
  if (a.kind == OLIVE_NORM_LAYER)
    norm_fwd_kernel<T, G, NV, true><<<blocks, threads_of<G>(), 0, c.stream>>>(a);
  else
    norm_fwd_kernel<T, G, NV, false><<<blocks, threads_of<G>(), 0, c.stream>>>(a);
}

template <typename T, int G, int NV>
void run_bwd(const Ctx& c, const NormArgs& a) {
  constexpr int kThreads = threads_of<G>(), kGroups = kThreads / G;
  const int per_sm = std::max(1, 512 / kThreads);
  const int64_t most = std::min<int64_t>(static_cast<int64_t>(c.num_sms) * per_sm, kMaxBlocks / kGroups);
  const int blocks = static_cast<int>(std::min<int64_t>(most, ceil_div(a.T, kGroups)));
  if (blocks > 0) {
    if (a.kind == OLIVE_NORM_LAYER)
      norm_bwd_kernel<T, G, NV, true><<<blocks, kThreads, 0, c.stream>>>(a);
    else
      norm_bwd_kernel<T, G, NV, false><<<blocks, kThreads, 0, c.stream>>>(a);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(ceil_div(a.d, 32)), a.db ? 2 : 1);
  cfg.blockDim = dim3(1024);
  cfg.stream = c.stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cudaLaunchKernelEx(&cfg, norm_dw_kernel, static_cast<const float*>(a.ws), blocks * kGroups, static_cast<int>(a.d),
                     a.dw, a.db);
}

// Threads of a row and vectors of a thread for rows of d / 8 vectors.
template <bool kBwd, typename T>
olive_status by_width(const Ctx& c, const NormArgs& a) {
  auto go = [&](auto group, auto vecs) {
    constexpr int G = decltype(group)::value, NV = decltype(vecs)::value;
    if constexpr (kBwd)
      run_bwd<T, G, NV>(c, a);
    else
      run_fwd<T, G, NV>(c, a);
  };
  const int nv = a.d / 8;
  using std::integral_constant;
  if (nv <= 32)
    go(integral_constant<int, 32>{}, integral_constant<int, 1>{});
  else if (nv <= 64)
    go(integral_constant<int, 32>{}, integral_constant<int, 2>{});
  else if (nv <= 128)
    go(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  else if (nv <= 256)
    go(integral_constant<int, 128>{}, integral_constant<int, 2>{});
  else if (nv <= 512)
    go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  else if (nv <= 1024)
    go(integral_constant<int, 512>{}, integral_constant<int, 2>{});
  else
    go(integral_constant<int, 512>{}, integral_constant<int, 4>{});
  return cudaGetLastError() == cudaSuccess ? OLIVE_OK : OLIVE_ERR_CUDA;
}

}  // namespace

size_t norm_bwd_ws_bytes(int64_t d) { return align_up(8ull * kMaxBlocks * d, kWsAlign); }

olive_status launch_norm_fwd(const Ctx& c, const NormArgs& a) {
  return a.dtype == OLIVE_DTYPE_BF16 ? by_width<false, __nv_bfloat16>(c, a) : by_width<false, float>(c, a);
}

olive_status launch_norm_bwd(const Ctx& c, const NormArgs& a) {
  return a.dtype == OLIVE_DTYPE_BF16 ? by_width<true, __nv_bfloat16>(c, a) : by_width<true, float>(c, a);
}

}  // namespace olive
