// qk_norm_rope.cu -- RMS norm of each query and key head and the rotation by the
// token's position in one pass, forward and backward, and the packed tokens'
// positions.
//
// A head's D values are held by the lanes of a group (8, 16 or 32 lanes for D up
// to 64, 128 or 256), eight values each as two runs of four: in the half layout
// j .. and j + R/2 .., so that both members of a pair are in one thread and a
// rotation needs no exchange; the mean square is a butterfly over the group.  A
// group takes several heads of one token and reads its cosines and sines once.
//
// What bounds it: HBM, 2 reads or writes of every value forward and 3 backward (6.3
// and 5.6 TB/s at 32768 tokens of 32 + 8 heads of 128, 107 and 180 us; at_once
// below), and the launch for a token or a few (2.8 us).  The backward with one or two
// key heads is bound by the keys' blocks: they are given by the number of heads, and
// each of their rounds holds one or two heads in place of four (32768 tokens of 32 query
// heads, us: 8 key heads 186, 4 176, 2 260, 1 420, caches empty).
#include <algorithm>

#include "internal.h"
#include "sm103.cuh"

namespace olive {
namespace {

constexpr int kThreads = 256;
constexpr int kFwdBlocks = 4, kBwdBlocks = 2;  // blocks an SM
// blocks whose partial weight gradients the workspace holds (a side of many heads
// may need more than run at once, for one token's chunks)
constexpr int kMaxBwdBlocks = 1024;
constexpr int kStatusToken = 1 << OLIVE_ERR_TOKEN_RANGE;

template <typename T>
struct Four;
template <>
struct Four<float> {
  using Raw = float4;
  static __device__ __forceinline__ void get(const Raw& r, float (&v)[4]) {
    v[0] = r.x;
    v[1] = r.y;
    v[2] = r.z;
    v[3] = r.w;
  }
  static __device__ __forceinline__ Raw put(const float (&v)[4]) { return make_float4(v[0], v[1], v[2], v[3]); }
};
template <>
struct Four<__nv_bfloat16> {
  using Raw = uint2;
  static __device__ __forceinline__ void get(const Raw& r, float (&v)[4]) {
    v[0] = __uint_as_float(r.x << 16);
    v[1] = __uint_as_float(r.x & 0xffff0000u);
    v[2] = __uint_as_float(r.y << 16);
    v[3] = __uint_as_float(r.y & 0xffff0000u);
  }
  static __device__ __forceinline__ Raw put(const float (&v)[4]) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
    return make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
  }
};

// What a lane holds of a head: two runs of four values.
struct Place {
  int a, b;       // their first elements
  bool in, turn;  // the lane has a part of the head; a rotated one
  int j;          // its first pair
};
template <bool kInter>
__device__ __forceinline__ Place place(int lane, int D, int R) {
  Place q;
  q.in = lane < D / 8;
  q.turn = lane < R / 8;
  q.j = 4 * lane;
  if (kInter || !q.turn) {
    q.a = 8 * lane;
    q.b = q.a + 4;
  } else {
    q.a = 4 * lane;
    q.b = R / 2 + 4 * lane;
  }
  return q;
}

// The pairs of (a, b) turned by the angles (c, s).
template <bool kInter>
__device__ __forceinline__ void rotate(float (&a)[4], float (&b)[4], const float (&c)[4], const float (&s)[4]) {
  if (kInter) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float x = a[2 * i], y = a[2 * i + 1], z = b[2 * i], w = b[2 * i + 1];
      a[2 * i] = x * c[i] - y * s[i];
      a[2 * i + 1] = y * c[i] + x * s[i];
      b[2 * i] = z * c[2 + i] - w * s[2 + i];
      b[2 * i + 1] = w * c[2 + i] + z * s[2 + i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = a[i], y = b[i];
      a[i] = x * c[i] - y * s[i];
      b[i] = y * c[i] + x * s[i];
    }
  }
}

template <int L>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Cosines and sines of a lane's pairs; `fine`: the position is inside the tables.
__device__ __forceinline__ bool angles(const QkArgs& p, int t, const Place& q, bool report, float (&c)[4], float (&s)[4]) {
  const int pos = p.positions[t];
  const bool fine = pos >= 0 && pos < p.P;
  if (!fine && report && p.dev_status) atomicOr(p.dev_status, kStatusToken);
  if (q.turn) {
    const size_t at = static_cast<size_t>(fine ? pos : 0) * (p.R / 2) + q.j;
    Four<float>::get(*reinterpret_cast<const float4*>(p.cos + at), c);
    Four<float>::get(*reinterpret_cast<const float4*>(p.sin + at), s);
  }
  return fine;
}

// Heads whose loads a thread has in flight together: 64 bytes of each operand.
// Measured, us on 32768 tokens of 32 + 8 heads of 128, bf16: forward, 4 blocks an
// SM, 106 with four heads (6.3 TB/s), 121 with two; 118 with four and 3 blocks;
// backward 180 with four heads and 2 blocks (5.6 TB/s), 184 with two and 3.
template <typename T>
constexpr int at_once() {
  return sizeof(T) == 2 ? 4 : 2;
}

// A group's heads: `per` of one token, all queries or all keys; chunk c of a
// token's nch, the first nq of them queries.
template <typename T, bool kInter, int L>
__global__ void __launch_bounds__(kThreads, kFwdBlocks) qk_fwd_kernel(const QkArgs p, int per, int nq, int nch) {
  using V = Four<T>;
  constexpr int kAtOnce = at_once<T>();
  const int lane = threadIdx.x % L;
  const long long i = static_cast<long long>(blockIdx.x) * (kThreads / L) + threadIdx.x / L;
  const bool live = i < static_cast<long long>(p.T) * nch;
  // (32-bit division where it is enough: the 64-bit one is a hundred instructions)
  const int t = !live ? 0 : i >> 32 ? static_cast<int>(i / nch) : static_cast<int>(static_cast<uint32_t>(i) / static_cast<uint32_t>(nch));
  int c0 = live ? static_cast<int>(i - static_cast<long long>(t) * nch) : 0;
  const int side = c0 >= nq;
  if (side) c0 -= nq;
  const int h0 = c0 * per, h1 = live ? min(h0 + per, p.heads[side]) : h0;
  const Place q = place<kInter>(lane, p.D, p.R);
  const HeadsView src = p.in[side], dst = p.out[side];
  const T* w = static_cast<const T*>(p.w[side]);
  const float inv_d = 1.f / p.D;
  // the lane's first run of a head; the second is `other` values on
  const int other = q.b - q.a;
  const T* x = static_cast<const T*>(src.x) + t * src.token_stride + h0 * src.head_stride + q.a;
  T* y = static_cast<T*>(const_cast<void*>(dst.x)) + t * dst.token_stride + h0 * dst.head_stride + q.a;

  // The rotation with the weights in it: out = r (a ca - b sb, b cb + a sa) with
  // ca = w_a cos, sa = w_a sin, cb = w_b cos, sb = w_b sin, formed once a token
  float ca[4], sa[4], cb[4], sb[4];
  bool fine = true;
  for (int h = h0; __any_sync(0xffffffffu, h < h1); h += kAtOnce) {
    typename V::Raw ra[kAtOnce], rb[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k, x += src.head_stride) {
      if (q.in && h + k < h1) {
        ra[k] = *reinterpret_cast<const typename V::Raw*>(x);
        rb[k] = *reinterpret_cast<const typename V::Raw*>(x + other);
      } else {
        ra[k] = rb[k] = typename V::Raw{};
      }
    }
    if (h == h0) {
      float wa[4] = {}, wb[4] = {}, c[4] = {}, s[4] = {};
      if (live) fine = angles(p, t, q, lane == 0, c, s);
      if (live && q.in) {
        V::get(*reinterpret_cast<const typename V::Raw*>(w + q.a), wa);
        V::get(*reinterpret_cast<const typename V::Raw*>(w + q.b), wb);
      }
      const auto fold = [&](float& cc, float& ss, float ww, int pair) {
        cc = q.turn ? ww * c[pair] : ww;
        ss = ww * s[pair];
      };
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        fold(ca[e], sa[e], wa[e], kInter ? e / 2 : e);
        fold(cb[e], sb[e], wb[e], kInter ? 2 + e / 2 : e);
      }
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k, y += dst.head_stride) {
      float a[4], b[4];
      V::get(ra[k], a);
      V::get(rb[k], b);
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) ss = fmaf(a[e], a[e], fmaf(b[e], b[e], ss));
      ss = group_sum<L>(ss);
      if (!(q.in && h + k < h1)) continue;
      float r = rsqrtf(fmaf(ss, inv_d, p.eps));
      if (!fine) r = __uint_as_float(0x7fffffffu);
      float oa[4], ob[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (!q.turn) {  // (not a turn by 0: an infinite partner would make it NaN)
          oa[e] = r * (a[e] * ca[e]);
          ob[e] = r * (b[e] * cb[e]);
        } else if (kInter) {  // pairs inside a run: even members -, odd ones +
          const int m = e ^ 1;
          oa[e] = r * fmaf(a[e], ca[e], e & 1 ? a[m] * sa[m] : -(a[m] * sa[m]));
          ob[e] = r * fmaf(b[e], cb[e], e & 1 ? b[m] * sb[m] : -(b[m] * sb[m]));
        } else {
          oa[e] = r * fmaf(a[e], ca[e], -(b[e] * sb[e]));
          ob[e] = r * fmaf(b[e], cb[e], a[e] * sa[e]);
        }
      }
      *reinterpret_cast<typename V::Raw*>(y) = V::put(oa);
      *reinterpret_cast<typename V::Raw*>(y + other) = V::put(ob);
    }
  }
}

// Backward.  With n = x r (r the reciprocal root mean square) and dn the
// gradient turned back, dx = r (dn w - n mean(dn w n)) and dw = sum of dn n over
// all tokens and heads: sum(x^2) and sum(dn w x) come from one butterfly.
// A block works on queries (the first `bq` blocks) or keys alone, a group on one
// chunk of the heads of every so-manieth token, so that a thread keeps the weight
// gradients of its eight columns in registers from beginning to end; the block
// adds its threads' up and stores them, and a second launch adds the blocks'.
template <typename T, bool kInter, int L>
__global__ void __launch_bounds__(kThreads, kBwdBlocks) qk_bwd_kernel(const QkArgs p, int per, int bq) {
  using V = Four<T>;
  constexpr int kAtOnce = at_once<T>();
  __shared__ float sums[kThreads / 32][8 * L];
  const int lane = threadIdx.x % L;
  const Place q = place<kInter>(lane, p.D, p.R);
  const float inv_d = 1.f / p.D;
  const int side = static_cast<int>(blockIdx.x) >= bq;
  const int block = static_cast<int>(blockIdx.x) - (side ? bq : 0);
  const int blocks = side ? static_cast<int>(gridDim.x) - bq : bq;
  const int nch = (p.heads[side] + per - 1) / per;
  const int group = block * (kThreads / L) + static_cast<int>(threadIdx.x) / L;
  const int step = blocks * (kThreads / L) / nch;  // tokens worked on at once
  const int chunk = group % nch;
  const int h0 = chunk * per, h1 = min(h0 + per, p.heads[side]);
  const int other = q.b - q.a;  // from the lane's first run of a head to its second
  const HeadsView src = p.in[side], grd = p.grad[side], dst = p.out[side];

  float w[8] = {}, dw[8] = {};
  if (q.in) {
    const T* v = static_cast<const T*>(p.w[side]);
    float a[4], b[4];
    V::get(*reinterpret_cast<const typename V::Raw*>(v + q.a), a);
    V::get(*reinterpret_cast<const typename V::Raw*>(v + q.b), b);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[e] = a[e];
      w[4 + e] = b[e];
    }
  }

  // (groups beyond the last whole set of chunks have no token)
  for (int t = group / nch < step ? group / nch : p.T; __any_sync(0xffffffffu, t < p.T); t = t < p.T - step ? t + step : p.T) {
    const bool live = t < p.T;
    const int tt = live ? t : 0, he = live ? h1 : h0;
    const T* x = static_cast<const T*>(src.x) + tt * src.token_stride + h0 * src.head_stride + q.a;
    const T* g = static_cast<const T*>(grd.x) + tt * grd.token_stride + h0 * grd.head_stride + q.a;
    T* y = static_cast<T*>(const_cast<void*>(dst.x)) + tt * dst.token_stride + h0 * dst.head_stride + q.a;
    float c[4] = {}, s[4] = {};
    bool fine = true;
    for (int h = h0; __any_sync(0xffffffffu, h < he); h += kAtOnce) {
      typename V::Raw xa[kAtOnce], xb[kAtOnce], ga[kAtOnce], gb[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k, x += src.head_stride, g += grd.head_stride) {
        if (q.in && h + k < he) {
          xa[k] = *reinterpret_cast<const typename V::Raw*>(x);
          xb[k] = *reinterpret_cast<const typename V::Raw*>(x + other);
          ga[k] = *reinterpret_cast<const typename V::Raw*>(g);
          gb[k] = *reinterpret_cast<const typename V::Raw*>(g + other);
        } else {
          xa[k] = xb[k] = ga[k] = gb[k] = typename V::Raw{};
        }
      }
      if (h == h0 && live) {
        fine = angles(p, t, q, lane == 0, c, s);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = -s[e];
      }
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k, y += dst.head_stride) {
        float v[8], d[8];
        {
          float a[4], b[4];
          V::get(xa[k], a);
          V::get(xb[k], b);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v[e] = a[e];
            v[4 + e] = b[e];
          }
          V::get(ga[k], a);
          V::get(gb[k], b);
          if (q.turn) rotate<kInter>(a, b, c, s);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            d[e] = a[e];
            d[4 + e] = b[e];
          }
        }
        float ss = 0.f, dot = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          ss = fmaf(v[e], v[e], ss);
          dot = fmaf(d[e] * w[e], v[e], dot);
        }
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) {
          ss += __shfl_xor_sync(0xffffffffu, ss, o);
          dot += __shfl_xor_sync(0xffffffffu, dot, o);
        }
        if (!(q.in && h + k < he)) continue;
        float r = rsqrtf(fmaf(ss, inv_d, p.eps));
        if (!fine) r = __uint_as_float(0x7fffffffu);
        const float mean = dot * r * inv_d;  // mean(dn w n)
        float a[4], b[4];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float n = v[e] * r;
          dw[e] = fmaf(d[e], n, dw[e]);
          const float o = r * fmaf(-n, mean, d[e] * w[e]);
          if (e < 4)
            a[e] = o;
          else
            b[e - 4] = o;
        }
        *reinterpret_cast<typename V::Raw*>(y) = V::put(a);
        *reinterpret_cast<typename V::Raw*>(y + other) = V::put(b);
      }
    }
  }
  grid_launch_dependents();

  // the warp's groups, then the block's warps
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float v = dw[e];
#pragma unroll
    for (int o = 16; o >= L; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (threadIdx.x % 32 < L && q.in) sums[threadIdx.x / 32][(e < 4 ? q.a : q.b - 4) + e] = v;
  }
  __syncthreads();
  float* part = static_cast<float*>(p.ws) + static_cast<size_t>(blockIdx.x) * p.D;
  for (int col = threadIdx.x; col < p.D; col += kThreads) {
    float v = 0.f;
#pragma unroll
    for (int wp = 0; wp < kThreads / 32; ++wp) v += sums[wp][col];
    part[col] = v;
  }
}

// dw of a side (blockIdx.y) = sum over its blocks, 32 columns a block, in a fixed
// order.
__global__ void __launch_bounds__(1024) qk_dw_kernel(const float* part, int bq, int blocks, int D, float* dw_q, float* dw_k) {
  __shared__ double sums[32][32];
  grid_wait();
  const int lane = threadIdx.x % 32, g = threadIdx.x / 32, col = blockIdx.x * 32 + lane;
  const int b0 = blockIdx.y ? bq : 0, b1 = blockIdx.y ? blocks : bq;
  double v = 0.0;
  if (col < D) {
#pragma unroll 4
    for (int b = b0 + g; b < b1; b += 32) v += static_cast<double>(part[static_cast<size_t>(b) * D + col]);
  }
  sums[g][lane] = v;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    __syncthreads();
    if (g < o) sums[g][lane] += sums[g + o][lane];
  }
  if (g == 0 && col < D) (blockIdx.y ? dw_k : dw_q)[col] = static_cast<float>(sums[0][lane]);
}

__global__ void positions_kernel(const int32_t* cu, int S, int T_cap, int32_t* positions) {
  const int64_t at = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  if (at >= T_cap) return;
  const int t = static_cast<int>(at);
  int lo = 0, hi = S;  // the last s with cu[s] <= t
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (cu[mid] <= t)
      lo = mid;
    else
      hi = mid - 1;
  }
  positions[t] = lo < S ? t - cu[lo] : 0;
}

template <typename T, bool kInter, int L>
void run_fwd(const Ctx& c, const QkArgs& a) {
  // as many heads a group as bring all of them into one wave, at most 8: their
  // loads are in flight together and the angles are read once
  const int64_t heads = static_cast<int64_t>(a.T) * (a.heads[0] + a.heads[1]);
  const int64_t room = static_cast<int64_t>(c.num_sms) * kFwdBlocks * (kThreads / L);
  int per = 1;
  while (per < 8 && heads > per * room) per *= 2;
  const int nq = static_cast<int>(ceil_div(a.heads[0], per));
  const int nch = nq + static_cast<int>(ceil_div(a.heads[1], per));
  const int64_t blocks = ceil_div(static_cast<int64_t>(a.T) * nch, kThreads / L);
  qk_fwd_kernel<T, kInter, L><<<static_cast<unsigned>(blocks), kThreads, 0, c.stream>>>(a, per, nq, nch);
}

template <typename T, bool kInter, int L>
void run_bwd(const Ctx& c, const QkArgs& a) {
  const int groups = kThreads / L;
  const int64_t heads = static_cast<int64_t>(a.T) * (a.heads[0] + a.heads[1]);
  // several heads a group where there are enough of them to fill the GPU anyway
  const int64_t room = static_cast<int64_t>(c.num_sms) * kBwdBlocks * groups;
  const int per = heads >= 16 * room ? 8 : heads >= 4 * room ? 4 : heads >= 2 * room ? 2 : 1;
  const int most = std::min(kBwdBlocks * c.num_sms, kMaxBwdBlocks);  // as many as run at once
  // blocks of a side: its share, at least one token's chunks
  int blocks[2] = {0, 0};
  for (int s = 0; s < 2 && a.T > 0; ++s) {
    if (a.heads[s] == 0) continue;
    const int64_t nch = ceil_div(a.heads[s], per);
    const int64_t share = std::max<int64_t>(1, static_cast<int64_t>(most) * a.heads[s] / (a.heads[0] + a.heads[1]));
    const int64_t least = ceil_div(nch, groups);
    blocks[s] = static_cast<int>(std::max(least, std::min(share, ceil_div(a.T * nch, groups))));
  }
  const int all = blocks[0] + blocks[1];
  if (all > 0) qk_bwd_kernel<T, kInter, L><<<all, kThreads, 0, c.stream>>>(a, per, blocks[0]);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(ceil_div(a.D, 32)), 2);
  cfg.blockDim = dim3(1024);
  cfg.stream = c.stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cudaLaunchKernelEx(&cfg, qk_dw_kernel, static_cast<const float*>(a.ws), blocks[0], all, static_cast<int>(a.D),
                     a.dw[0], a.dw[1]);
}

template <bool kBwd, typename T, bool kInter>
void by_width(const Ctx& c, const QkArgs& a) {
  auto go = [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    if constexpr (kBwd)
      run_bwd<T, kInter, L>(c, a);
    else
      run_fwd<T, kInter, L>(c, a);
  };
  if (a.D <= 64)
    go(std::integral_constant<int, 8>{});
  else if (a.D <= 128)
    go(std::integral_constant<int, 16>{});
  else
    go(std::integral_constant<int, 32>{});
}

template <bool kBwd>
olive_status by_type(const Ctx& c, const QkArgs& a) {
  if (a.dtype == OLIVE_DTYPE_BF16)
    a.interleaved ? by_width<kBwd, __nv_bfloat16, true>(c, a) : by_width<kBwd, __nv_bfloat16, false>(c, a);
  else
    a.interleaved ? by_width<kBwd, float, true>(c, a) : by_width<kBwd, float, false>(c, a);
  return cudaGetLastError() == cudaSuccess ? OLIVE_OK : OLIVE_ERR_CUDA;
}

}  // namespace

size_t qk_bwd_ws_bytes(int64_t D) { return align_up(4ull * kMaxBwdBlocks * D, kWsAlign); }

olive_status launch_qk_fwd(const Ctx& c, const QkArgs& a) { return by_type<false>(c, a); }

olive_status launch_qk_bwd(const Ctx& c, const QkArgs& a) { return by_type<true>(c, a); }

olive_status launch_packed_positions(const Ctx& c, const int32_t* cu_seqlens, int32_t S,
                                     int32_t T_cap, int32_t* positions) {
  positions_kernel<<<static_cast<unsigned>(ceil_div(T_cap, 256)), 256, 0, c.stream>>>(cu_seqlens, S, T_cap, positions);
  return cudaGetLastError() == cudaSuccess ? OLIVE_OK : OLIVE_ERR_CUDA;
}

}  // namespace olive
