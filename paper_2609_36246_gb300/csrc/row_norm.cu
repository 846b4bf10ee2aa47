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
// gradients of its columns in registers from beginning to end, in fp32: T / groups rows in
// turn (at most 1024 groups, 152 above a width of 4096); the blocks' sums are stored and
// added in a second launch, in a fixed order.
//
// Bound by memory.  32768 rows of 4096, bf16, with a residual and its gradient: forward 152
// us (7.1 TB/s), backward 179 (6.0) and 6 for the weights'.  3001 rows of 2040 in fp32: 10,
// 17 and 4 us.
#include <algorithm>
#include <atomic>

#include "internal.h"
#include "sm103.cuh"

namespace olive {
namespace {

constexpr int kMaxBlocks = 1024;  // blocks whose partial weight gradients the workspace holds
// blocks an SM of rows that a whole block works on, and a block's stages
template <typename T, int G>
constexpr int staged_blocks() { return G > 256 ? 1 : (sizeof(T) == 2 ? 768 : 512) / G; }
template <typename T, int G>
constexpr int staged_smem() { return 216 * 1024 / staged_blocks<T, G>(); }

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

// The same as pairs, for two operations an instruction.
template <typename T>
__device__ __forceinline__ void get_pairs(const typename Eight<T>::Raw& r, uint64_t (&v)[4]) {
  float f[8];
  Eight<T>::get(r, f);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = pair(f[2 * i], f[2 * i + 1]);
}
template <typename T>
__device__ __forceinline__ typename Eight<T>::Raw put_pairs(const uint64_t (&v)[4]) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) unpair(v[i], f[2 * i], f[2 * i + 1]);
  return Eight<T>::put(f);
}

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

// The two passes of the backward over a vector.  First the weights' sums and the row's,
// of a = dy w and of a n; then dx = r (a - mean(a) - n mean(a n)) + more.
struct RowStats {
  uint64_t minus_mean, r;  // both in each half
};
template <typename T>
__device__ __forceinline__ void first_pass(const typename Eight<T>::Raw& xr, const typename Eight<T>::Raw& gr, const typename Eight<T>::Raw& wr,
                                           const RowStats& st, uint64_t (&dw)[4], uint64_t (&db)[4], uint64_t (&s)[2]) {
  uint64_t x[4], g[4], w[4];
  get_pairs<T>(xr, x);
  get_pairs<T>(gr, g);
  get_pairs<T>(wr, w);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint64_t n = mul_pair(add_pair(x[e], st.minus_mean), st.r), a = mul_pair(g[e], w[e]);
    dw[e] = fma_pair(g[e], n, dw[e]);
    db[e] = add_pair(db[e], g[e]);
    s[0] = add_pair(s[0], a);
    s[1] = fma_pair(a, n, s[1]);
  }
}
template <typename T>
__device__ __forceinline__ typename Eight<T>::Raw second_pass(const typename Eight<T>::Raw& xr, const typename Eight<T>::Raw& gr,
                                                              const typename Eight<T>::Raw& wr, bool add, const typename Eight<T>::Raw& more,
                                                              const RowStats& st, uint64_t minus_ma, uint64_t minus_man) {
  uint64_t x[4], g[4], w[4], m[4] = {};
  get_pairs<T>(xr, x);
  get_pairs<T>(gr, g);
  get_pairs<T>(wr, w);
  if (add) get_pairs<T>(more, m);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint64_t n = mul_pair(add_pair(x[e], st.minus_mean), st.r);
    const uint64_t t = fma_pair(n, minus_man, fma_pair(g[e], w[e], minus_ma));
    x[e] = fma_pair(st.r, t, m[e]);
  }
  return put_pairs<T>(x);
}

// A group's sums to the workspace: [group][dw, db][d].
template <int NV, int G>
__device__ __forceinline__ void store_parts(const NormArgs& p, const uint64_t (&dw)[NV][4], const uint64_t (&db)[NV][4], int lane, int64_t group) {
  float* part = static_cast<float*>(p.ws) + group * 2 * p.d;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int at = lane + G * k;
    if (at >= p.d / 8) continue;
    ulonglong2* a = reinterpret_cast<ulonglong2*>(part + 8 * at);
    ulonglong2* b = reinterpret_cast<ulonglong2*>(part + p.d + 8 * at);
    a[0] = make_ulonglong2(dw[k][0], dw[k][1]);
    a[1] = make_ulonglong2(dw[k][2], dw[k][3]);
    b[0] = make_ulonglong2(db[k][0], db[k][1]);
    b[1] = make_ulonglong2(db[k][2], db[k][3]);
  }
}

template <typename T, int G, int NV, bool kCentre>
__global__ void __launch_bounds__(threads_of<G>()) norm_bwd_kernel(const NormArgs p) {
  using V = Eight<T>;
  using Raw = typename V::Raw;
  constexpr int kGroups = threads_of<G>() / G;
  // (registers for two rows: not with four vectors, nor with two of fp32)
  constexpr bool kAhead = NV * sizeof(T) <= 4;
  __shared__ float red[2][threads_of<G>() / 32][2];
  const int lane = threadIdx.x % G;
  const int nv = p.d / 8;
  const float inv_d = 1.f / p.d;
  uint64_t dw[NV][4] = {}, db[NV][4] = {};
  // a row's values and statistics, the next row's on their way while this one's are used
  struct Row {
    Raw x[NV], g[NV], more[NV];
    float mean, r;
  };
  const int64_t step = static_cast<int64_t>(gridDim.x) * kGroups;
  const auto load = [&](Row& t, int64_t row) {
    if (row >= p.T) return;
    const Raw* x = static_cast<const Raw*>(p.x) + row * nv;
    const Raw* g = static_cast<const Raw*>(p.dy) + row * nv;
    const Raw* more = static_cast<const Raw*>(p.g_sum) + row * nv;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int at = lane + G * k;
      if (at >= nv) continue;
      t.x[k] = x[at];
      t.g[k] = g[at];
      if (p.g_sum) t.more[k] = more[at];
    }
    t.mean = kCentre ? p.stats[row] : 0.f;
    t.r = p.stats[p.T + row];
  };
  int64_t row = static_cast<int64_t>(blockIdx.x) * kGroups + threadIdx.x / G;
  Row now, next;
  load(now, row);
  int slot = 0;
  // (all groups of a block go round as often: they share its barriers)
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * kGroups; first < p.T; first += step, row += step, slot ^= 1) {
    const bool live = row < p.T;
    if (kAhead) load(next, row + step);
    const RowStats st = {pair(-now.mean, -now.mean), pair(now.r, now.r)};
    uint64_t sp[2] = {0, 0};
    if (live) {
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (lane + G * k < nv)
          first_pass<T>(now.x[k], now.g[k], static_cast<const Raw*>(p.w)[lane + G * k], st, dw[k], db[k], sp);
    }
    float s[2], odd[2];
    unpair(sp[0], s[0], odd[0]);
    unpair(sp[1], s[1], odd[1]);
    s[0] += odd[0];
    s[1] += odd[1];
    group_sum<G>(s, red, slot);
    const float ma = kCentre ? -s[0] * inv_d : 0.f, man = -s[1] * inv_d;
    if (live) {
      Raw* dx = static_cast<Raw*>(p.dx) + row * nv;
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (lane + G * k < nv)
          dx[lane + G * k] = second_pass<T>(now.x[k], now.g[k], static_cast<const Raw*>(p.w)[lane + G * k],
                                            p.g_sum != nullptr, now.more[k], st, pair(ma, ma), pair(man, man));
    }
    if (kAhead)
      now = next;
    else
      load(now, row + step);
  }
  grid_launch_dependents();
  store_parts<NV, G>(p, dw, db, lane, static_cast<int64_t>(blockIdx.x) * kGroups + threadIdx.x / G);
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// The same for rows of a whole block: they come through shared memory, kStages rows ahead,
// every thread copying what it reads itself, so that nothing but the row's sums is waited
// for together.  (32768 rows of 4096 with g_sum, bf16: 179 us; 224 with the next row in
// registers, where a row takes as long as its loads.)
template <typename T, int G, int NV, bool kCentre, int kStages>
__global__ void __launch_bounds__(G, staged_blocks<T, G>()) norm_bwd_staged_kernel(const NormArgs p) {
  using V = Eight<T>;
  using Raw = typename V::Raw;
  extern __shared__ __align__(16) uint8_t stage_smem[];
  __shared__ float red[2][G / 32][2];
  const int lane = threadIdx.x, nv = p.d / 8, arrays = p.g_sum ? 3 : 2;
  const float inv_d = 1.f / p.d;
  Raw* const stages = reinterpret_cast<Raw*>(stage_smem);
  const auto fetch = [&](int stage, int64_t row) {
    if (row < p.T) {
      const auto copy = [&](Raw* to, const void* from) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const int at = lane + G * k;
          if (at >= nv) continue;
          const char* src = reinterpret_cast<const char*>(static_cast<const Raw*>(from) + row * nv + at);
#pragma unroll
          for (int b = 0; b < static_cast<int>(sizeof(Raw)); b += 16) copy16(smem_u32(to + at) + b, src + b);
        }
      };
      Raw* to = stages + stage * arrays * nv;
      copy(to, p.x);
      copy(to + nv, p.dy);
      if (p.g_sum) copy(to + 2 * nv, p.g_sum);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < kStages; ++i) fetch(i, blockIdx.x + static_cast<int64_t>(i) * gridDim.x);
  uint64_t dw[NV][4] = {}, db[NV][4] = {};
  int stage = 0, slot = 0;
  float mean = kCentre ? p.stats[blockIdx.x] : 0.f, r = p.stats[p.T + blockIdx.x];
  for (int64_t row = blockIdx.x; row < p.T; row += gridDim.x, slot ^= 1) {
    const RowStats st = {pair(-mean, -mean), pair(r, r)};
    if (row + gridDim.x < p.T) {  // (the next row's, while this one is worked on)
      if (kCentre) mean = p.stats[row + gridDim.x];
      r = p.stats[p.T + row + gridDim.x];
    }
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
    const Raw* x = stages + stage * arrays * nv;
    Raw xr[NV], gr[NV], more[NV];
    uint64_t sp[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int at = lane + G * k;
      if (at >= nv) continue;
      xr[k] = x[at];
      gr[k] = x[nv + at];
      if (p.g_sum) more[k] = x[2 * nv + at];
      first_pass<T>(xr[k], gr[k], static_cast<const Raw*>(p.w)[at], st, dw[k], db[k], sp);
    }
    fetch(stage, row + static_cast<int64_t>(kStages) * gridDim.x);
    if (++stage == kStages) stage = 0;
    float s[2], odd[2];
    unpair(sp[0], s[0], odd[0]);
    unpair(sp[1], s[1], odd[1]);
    s[0] += odd[0];
    s[1] += odd[1];
    group_sum<G>(s, red, slot);
    const float ma = kCentre ? -s[0] * inv_d : 0.f, man = -s[1] * inv_d;
    Raw* dx = static_cast<Raw*>(p.dx) + row * nv;
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (lane + G * k < nv)
        dx[lane + G * k] = second_pass<T>(xr[k], gr[k], static_cast<const Raw*>(p.w)[lane + G * k], p.g_sum != nullptr, more[k], st,
                                          pair(ma, ma), pair(man, man));
  }
  grid_launch_dependents();
  store_parts<NV, G>(p, dw, db, lane, blockIdx.x);
}

// dw (blockIdx.y = 0) and db (1): the groups' sums added, 32 columns a block, in a fixed
// order: each thread every 32nd group's, then the threads' as a tree.  (In fp64, of which
// there are two operations a cycle and SM, it took 15 us of 43 for 3001 rows of 2040.)
__global__ void __launch_bounds__(1024) norm_dw_kernel(const float* part, int groups, int d, float* dw, float* db) {
  __shared__ float sums[32][33];
  grid_wait();
  const int lane = threadIdx.x % 32, g = threadIdx.x / 32, col = blockIdx.x * 32 + lane;
  float v = 0.f;
  if (col < d) {
    const float* at = part + static_cast<size_t>(blockIdx.y) * d + col;
#pragma unroll 8
    for (int b = g; b < groups; b += 32) v += at[static_cast<size_t>(b) * 2 * d];
  }
  sums[g][lane] = v;
  __syncthreads();
  v = sums[lane][g];  // a warp a column
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  const int mine = blockIdx.x * 32 + g;
  if (lane == 0 && mine < d) (blockIdx.y ? db : dw)[mine] = v;
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

template <typename T, int G, int NV, bool kCentre, int kStages>
bool run_staged(const Ctx& c, const NormArgs& a, int blocks) {
  const int row = static_cast<int>(sizeof(T)) * a.d * (a.g_sum ? 3 : 2);
  static std::atomic<int> done[kMaxDevices];
  const auto kernel = norm_bwd_staged_kernel<T, G, NV, kCentre, kStages>;
  if (!set_smem_once(reinterpret_cast<const void*>(kernel), staged_smem<T, G>(), c.device, done)) return false;
  kernel<<<blocks, G, kStages * row, c.stream>>>(a);
  return true;
}

template <typename T, int G, int NV>
bool run_bwd(const Ctx& c, const NormArgs& a) {
  constexpr int kThreads = threads_of<G>(), kGroups = kThreads / G;
  const int per_sm = std::max(1, 512 / kThreads);
  const int64_t most = std::min<int64_t>(static_cast<int64_t>(c.num_sms) * per_sm, kMaxBlocks / kGroups);
  int blocks = static_cast<int>(std::min<int64_t>(most, ceil_div(a.T, kGroups)));
  if (blocks > 0) {
    // a block a row, in 2 or 3 arrays: staged where two rows of a block fit
    const bool centre = a.kind == OLIVE_NORM_LAYER;
    bool staged = false;
    if constexpr (G >= 128) {
      const int64_t fit = staged_smem<T, G>() / (static_cast<int64_t>(sizeof(T)) * a.d * (a.g_sum ? 3 : 2));
      if (fit >= 2) {
        staged = true;
        blocks = static_cast<int>(std::min<int64_t>(a.T, std::min(staged_blocks<T, G>() * c.num_sms, kMaxBlocks)));
        const auto run = [&](auto is_centred, auto n) { return run_staged<T, G, NV, decltype(is_centred)::value, decltype(n)::value>(c, a, blocks); };
        const auto by_stages = [&](auto is_centred) {
          if (fit >= 4) return run(is_centred, std::integral_constant<int, 4>{});
          if (fit == 3) return run(is_centred, std::integral_constant<int, 3>{});
          return run(is_centred, std::integral_constant<int, 2>{});
        };
        if (!(centre ? by_stages(std::true_type{}) : by_stages(std::false_type{}))) return false;
      }
    }
    if (staged) {
    } else if (centre) {
      norm_bwd_kernel<T, G, NV, true><<<blocks, kThreads, 0, c.stream>>>(a);
    } else {
      norm_bwd_kernel<T, G, NV, false><<<blocks, kThreads, 0, c.stream>>>(a);
    }
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
  return true;
}

// Threads of a row and vectors of a thread for rows of d / 8 vectors.
template <bool kBwd, typename T>
olive_status by_width(const Ctx& c, const NormArgs& a) {
  bool ok = true;
  auto go = [&](auto group, auto vecs) {
    constexpr int G = decltype(group)::value, NV = decltype(vecs)::value;
    if constexpr (kBwd)
      ok = run_bwd<T, G, NV>(c, a);
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
  return cudaGetLastError() == cudaSuccess && ok ? OLIVE_OK : OLIVE_ERR_CUDA;
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
