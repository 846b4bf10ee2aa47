// packed_attention_bwd.cu -- attention inside packed sequences, backward.
//
// With p_ij = exp(s_ij - lse_i), dp_ij = <do_i, v_j>, delta_i = <do_i, o_i> and
// ds_ij = p_ij (dp_ij - delta_i) (1 - (t_ij)^2 where scores are capped, t the tanh):
//   dv_j = sum_i p_ij do_i,  dk_j = scale sum_i ds_ij q_i,  dq_i = scale sum_j ds_ij k_j
// over the rows i that see j, and the query heads of j's key head.
//
// Three launches: each row's lse (base 2) and delta; dk and dv, a CTA on a key tile that
// walks the query tiles of its heads; dq, a CTA on a query tile that walks the key tiles.
// Scores and dp are formed in both (seven products in place of five): so no gradient is
// added up in memory, results are the same bits from call to call, and no fp32 copy of
// dq exists.
#include <algorithm>

#include "packed_attention.cuh"

namespace olive {
namespace {

constexpr int kThreads = 384;
constexpr int kRegsLaunch = 168, kRegsRows = 224, kRegsRest = 56;
static_assert(2 * kRegsRows + kRegsRest <= 3 * kRegsLaunch, "the block's registers");
constexpr int kStages = 2;
constexpr int kTmaWarp = 8, kMmaWarp = 9, kVecWarp = 10;
constexpr int kRowWarps = 8;

// ------------------------------------------------------------------ delta ---
// Rows that see up to this many keys have their delta from the keys themselves: <do, o>
// carries o's rounding, which is large beside dp - delta where one key has all the weight.
constexpr int kFewKeys = 16;
constexpr int kDeltaThreads = 128;

__device__ __forceinline__ void eight(const __nv_bfloat16* at, bool in, float (&v)[8]) {
  const uint4 r = in ? *reinterpret_cast<const uint4*>(at) : make_uint4(0, 0, 0, 0);
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
// Sum over the 16 lanes of a row.
__device__ __forceinline__ float dot16(const float (&a)[8], const float (&b)[8]) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s = fmaf(a[e], b[e], s);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}
__device__ __forceinline__ const __nv_bfloat16* row_of(const HeadsView& x, int64_t t, int h) {
  return static_cast<const __nv_bfloat16*>(x.x) + t * x.token_stride + h * x.head_stride;
}
// A score in base 2 and the derivative of its cap.
__device__ __forceinline__ float score2(const AttArgs& p, float s, float slope2, float dist, float& bend) {
  bend = 1.f;
  float x = s * (p.scale * kAttLog2e);
  if (p.cap > 0.f) {
    const float t = tanh_of(x * (2.f / p.cap));
    bend = fmaf(-t, t, 1.f);
    x = p.cap * kAttLog2e * t;
  }
  return fmaf(-slope2, dist, x);
}

// stats: [Hq, T] of (lse in base 2, delta); a block works on a tile's rows of one head,
// 16 lanes a row.
__global__ void __launch_bounds__(kDeltaThreads) att_delta_kernel(const AttArgs p, float2* stats) {
  const int head = static_cast<int>(blockIdx.x % p.Hq);
  const Seq q = seq_of_slot<128>(p, static_cast<int>(blockIdx.x / p.Hq));
  if (q.tile < 0) return;
  const int lane = threadIdx.x % 16, group = threadIdx.x / 16, kv = head / (p.Hq / p.Hk);
  const bool in = 8 * lane < p.D;
  const float slope2 = p.slopes ? p.slopes[head] * kAttLog2e : 0.f;
#pragma unroll 1
  for (int r = group; r < 128; r += kDeltaThreads / 16) {
    const int i = q.tile * 128 + r;
    if (!__any_sync(0xffffffffu, i < q.n)) break;
    const bool live = i < q.n;
    const int64_t t = q.start + min(i, q.n - 1);
    float a[8], b[8];
    eight(row_of(p.d_o, t, head) + 8 * lane, in, a);
    eight(row_of(p.o, t, head) + 8 * lane, in, b);
    float delta = dot16(a, b);
    const float lse2 = p.lse[static_cast<int64_t>(head) * p.T + t] * kAttLog2e;
    const int keys = keys_seen(p, q, static_cast<int>(t) - q.start);
    if (__any_sync(0xffffffffu, keys <= kFewKeys)) {
      float qr[8], sum = 0.f;
      eight(row_of(p.q, t, head) + 8 * lane, in, qr);
      for (int j = 0; __any_sync(0xffffffffu, j < keys && keys <= kFewKeys); ++j) {
        const int64_t tj = q.start + min(j, keys - 1);
        eight(row_of(p.k, tj, kv) + 8 * lane, in, b);
        float bend;
        const float s = score2(p, dot16(qr, b), slope2, fabsf(static_cast<float>(t - tj)), bend);
        eight(row_of(p.v, tj, kv) + 8 * lane, in, b);
        const float dp = dot16(a, b);
        if (j < keys) sum = fmaf(fast_exp2(s - lse2), dp, sum);
      }
      if (keys <= kFewKeys) delta = sum;
    }
    if (live && lane == 0) stats[static_cast<int64_t>(head) * p.T + t] = make_float2(lse2, delta);
  }
}

// ---------------------------------------------------------- what both share ---
// A row's one key (a softmax of one: no gradient flows to the score): only a
// sequence's first row can have just one.
__device__ __forceinline__ bool first_row_alone(const AttArgs& p, const Seq& q) { return keys_seen(p, q, 0) == 1; }

// A warp's rows of an accumulator, scaled, to 32 columns of a head from `col` on.
__device__ __forceinline__ void store_cols(uint32_t taddr, __nv_bfloat16* row, bool store, int col, int D, float by) {
  uint32_t o[32];
  tmem_ld_32x32b_x32(taddr + col, o);
  tmem_ld_wait();
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    if (!store || col + 8 * v >= D) continue;
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(o[8 * v + e]) * by;
    reinterpret_cast<uint4*>(row + col)[v] = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]),
                                                        pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
  }
}

// The end of the MMA warp: what it issued is complete before the CTA retires.
__device__ __forceinline__ void drain_mmas(uint32_t bar, bool leader, uint64_t limit_ns) {
  if (leader) umma_commit(bar);
  volatile int keep_waiting = 0;
  const uint64_t floor_ns = 200ull * 1000 * 1000;
  const WaitCtl own{&keep_waiting, limit_ns > floor_ns ? limit_ns : floor_ns};
  mbar_wait_warp(bar, 0, own);
  __syncwarp();
}

// ----------------------------------------------------------------- dk, dv ---
// tensor memory: S^T (then P^T), dP^T (then dS^T), dV, dK.  The MMAs of step t run in
// the order dP_t, dV_t, S_{t+1}, dK_t: P_t is formed while dP_t runs and dS_t while
// dV_t and S_{t+1} do.
enum { A_KVFULL = 0, A_KVEMPTY, A_QFULL, A_QEMPTY = A_QFULL + kStages, A_FIX = A_QEMPTY + kStages,
       A_VECFULL = A_FIX + kStages, A_VECEMPTY = A_VECFULL + kStages, A_SFULL = A_VECEMPTY + kStages, A_PREADY,
       A_DPFULL, A_DSREADY, A_OFULL, A_OEMPTY, A_DRAIN, A_COUNT };

constexpr int kv_smem(int boxes) { return 1024 + (2 + 2 * kStages) * boxes * kBoxBytes + kStages * 1024 + 8 * A_COUNT + 16; }

struct KvItem {
  Seq q;
  int kv_head, k0, first, tiles, steps;  // first query tile, query tiles of a head, of all heads
};
__device__ __forceinline__ bool kv_item(const AttArgs& p, int64_t i, KvItem& it) {
  it.q = seq_of_slot<128>(p, static_cast<int>(i / p.Hk));
  if (it.q.tile < 0) return false;
  it.kv_head = static_cast<int>(i % p.Hk);
  it.k0 = 128 * it.q.tile;
  it.first = p.causal && it.k0 >= it.q.prefix ? it.q.tile : 0;
  it.tiles = (it.q.n + 127) / 128 - it.first;
  it.steps = it.tiles * (p.Hq / p.Hk);
  return true;
}
// Step t of an item: a query head and the first row of a query tile.
__device__ __forceinline__ void kv_step(const AttArgs& p, const KvItem& it, int t, int& head, int& q0) {
  head = it.kv_head * (p.Hq / p.Hk) + t / it.tiles;
  q0 = 128 * (it.first + t % it.tiles);
}

template <int kBoxes, bool kExtra>
__global__ void __launch_bounds__(kThreads, 1)
    att_dkdv_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                    const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do, const AttArgs p,
                    const float2* stats, int64_t items) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  constexpr uint32_t kTileBytes = kBoxes * kBoxBytes;
  const uint32_t sk = base, sv = sk + kTileBytes, sq = sv + kTileBytes, sdo = sq + kStages * kTileBytes;
  const uint32_t vec0 = sdo + kStages * kTileBytes;  // a stage's [2][128]: lse, delta
  float* vec = reinterpret_cast<float*>(smem_raw + (vec0 - raw));
  const uint32_t bar0 = vec0 + kStages * 1024;
  uint8_t* misc = smem_raw + (bar0 - raw) + 8 * A_COUNT;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(misc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 4);
  const auto bar = [&](int i) { return bar0 + 8u * i; };
  const int warp = warp_uniform(static_cast<int>(threadIdx.x >> 5)), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < A_COUNT; ++i) {
      const bool rows = i == A_PREADY || i == A_DSREADY || i == A_OEMPTY || (i >= A_VECEMPTY && i < A_VECEMPTY + kStages);
      mbar_init(bar(i), rows ? kRowWarps : 1);
    }
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == kMmaWarp) {
    tmem_alloc(smem_u32(tmem_slot), 512);
    tmem_relinquish();
  }
  if (warp == kTmaWarp && lane == 0) {
    tma_prefetch_desc(&map_q);
    tma_prefetch_desc(&map_k);
    tma_prefetch_desc(&map_v);
    tma_prefetch_desc(&map_do);
  }
  zero_behind(p, const_cast<void*>(p.dk.x), p.dk.token_stride, p.dk.head_stride, p.Hk);
  zero_behind(p, const_cast<void*>(p.dv.x), p.dv.token_stride, p.dv.head_stride, p.Hk);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = warp_uniform(*tmem_slot);
  const uint32_t t_s = tmem, t_dp = tmem + 128, t_dv = tmem + 256, t_dk = tmem + 384;
  const WaitCtl ctl{abort_flag, p.wait_limit_ns};
  KvItem it;
  int head, q0;

  if (warp >= kTmaWarp) {
    regs_dec<kRegsRest>();
    if (warp == kTmaWarp) {
      const bool leader = elect_one();
      uint32_t n_kv = 0, n_q = 0;
      bool ok = true;
      for (int64_t i = blockIdx.x; ok && i < items; i += gridDim.x) {
        if (!kv_item(p, i, it)) continue;
        if (!(ok = mbar_wait_warp(bar(A_KVEMPTY), (n_kv++ & 1) ^ 1, ctl))) break;
        if (leader) {
          mbar_arrive_expect_tx(bar(A_KVFULL), 2 * kTileBytes);
          load_tile(sk, &map_k, bar(A_KVFULL), kBoxes, p.k.head_stride ? it.kv_head : 0, it.q.start + it.k0);
          load_tile(sv, &map_v, bar(A_KVFULL), kBoxes, p.v.head_stride ? it.kv_head : 0, it.q.start + it.k0);
        }
        for (int t = 0; t < it.steps; ++t, ++n_q) {
          const int s = n_q % kStages;
          kv_step(p, it, t, head, q0);
          if (!(ok = mbar_wait_warp(bar(A_QEMPTY + s), (n_q / kStages & 1) ^ 1, ctl))) break;
          if (leader) {
            mbar_arrive_expect_tx(bar(A_QFULL + s), 2 * kTileBytes);
            load_tile(sq + s * kTileBytes, &map_q, bar(A_QFULL + s), kBoxes, p.q.head_stride ? head : 0, it.q.start + q0);
            load_tile(sdo + s * kTileBytes, &map_do, bar(A_QFULL + s), kBoxes, p.d_o.head_stride ? head : 0, it.q.start + q0);
          }
          // the sequence's last rows: what follows them up to whole K steps is zeroed
          const int rows = it.q.n - q0;
          if (rows < 128 && rows % 16 != 0) {
            if (!(ok = mbar_wait_warp(bar(A_QFULL + s), n_q / kStages & 1, ctl))) break;
            zero_rows(sq + s * kTileBytes, kBoxes, rows, up16(rows));
            zero_rows(sdo + s * kTileBytes, kBoxes, rows, up16(rows));
            fence_proxy_async_shared();
            __syncwarp();
            if (leader) mbar_arrive(bar(A_FIX + s));
          }
        }
      }
      if (!ok) let_copies_land();
      __syncwarp();
    } else if (warp == kMmaWarp) {
      const bool leader = elect_one();
      const int steps = (p.D + 15) / 16;
      const uint32_t id_out = idesc_bf16(128, 16 * steps, false, true);
      uint32_t n_kv = 0, n_q = 0, fixed = 0, n = 0;
      bool ok = true;
      for (int64_t i = blockIdx.x; ok && i < items; i += gridDim.x) {
        if (!kv_item(p, i, it)) continue;
        if (!(ok = mbar_wait_warp(bar(A_KVFULL), n_kv & 1, ctl))) break;
        // (the last rows' tile is shorter)
        const auto rows_of = [&](int t) {
          kv_step(p, it, t, head, q0);
          return min(128, it.q.n - q0);
        };
        const auto scores = [&](int t) {
          const int s = (n_q + t) % kStages;
          if (!mbar_wait_warp(bar(A_QFULL + s), (n_q + t) / kStages & 1, ctl)) return false;
          tc_fence_after();
          const uint32_t id = idesc_bf16(128, up16(rows_of(t)), false, false);
          if (leader) {
            mma_rows(t_s, sk, sq + s * kTileBytes, id, steps);
            umma_commit(bar(A_SFULL));
          }
          return true;
        };
        if (!(ok = scores(0))) break;
        for (int t = 0; t < it.steps; ++t, ++n) {
          const int s = (n_q + t) % kStages, rows = rows_of(t);
          if (leader) {
            mma_rows(t_dp, sv, sdo + s * kTileBytes, idesc_bf16(128, up16(rows), false, false), steps);
            umma_commit(bar(A_DPFULL));
          }
          if (rows % 16 != 0) {
            if (!(ok = mbar_wait_warp(bar(A_FIX + s), fixed >> s & 1, ctl))) break;
            fixed ^= 1u << s;
          }
          if (t == 0 && !(ok = mbar_wait_warp(bar(A_OEMPTY), (n_kv & 1) ^ 1, ctl))) break;
          if (!(ok = mbar_wait_warp(bar(A_PREADY), n & 1, ctl))) break;
          tc_fence_after();
          if (leader) mma_cols(t_dv, t_s, 64, sdo + s * kTileBytes, id_out, up16(rows) / 16, t > 0);
          if (t + 1 < it.steps && !(ok = scores(t + 1))) break;
          if (!(ok = mbar_wait_warp(bar(A_DSREADY), n & 1, ctl))) break;
          tc_fence_after();
          if (leader) {
            mma_cols(t_dk, t_dp, 64, sq + s * kTileBytes, id_out, up16(rows) / 16, t > 0);
            umma_commit(bar(A_QEMPTY + s));
          }
        }
        if (!ok) break;
        n_q += it.steps;
        ++n_kv;
        if (leader) {
          umma_commit(bar(A_OFULL));
          umma_commit(bar(A_KVEMPTY));
        }
      }
      drain_mmas(bar(A_DRAIN), leader, p.wait_limit_ns);
    } else if (warp == kVecWarp) {
      uint32_t n_q = 0;
      bool ok = true;
      for (int64_t i = blockIdx.x; ok && i < items; i += gridDim.x) {
        if (!kv_item(p, i, it)) continue;
        for (int t = 0; t < it.steps; ++t, ++n_q) {
          const int s = n_q % kStages;
          kv_step(p, it, t, head, q0);
          float2 got[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = min(q0 + lane + 32 * e, it.q.n - 1);
            got[e] = stats[static_cast<int64_t>(head) * p.T + it.q.start + r];
          }
          if (!(ok = mbar_wait_warp(bar(A_VECEMPTY + s), (n_q / kStages & 1) ^ 1, ctl))) break;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            vec[s * 256 + lane + 32 * e] = got[e].x;
            vec[s * 256 + 128 + lane + 32 * e] = got[e].y;
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(A_VECFULL + s));
        }
      }
    }
  } else {
    regs_inc<kRegsRows>();
    const int half = warp >> 2;  // of the tile's query columns
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const float scale2 = p.scale * kAttLog2e;
    uint32_t n_q = 0, n_o = 0;
    bool ok = true;
    for (int64_t i = blockIdx.x; ok && i < items; i += gridDim.x) {
      if (!kv_item(p, i, it)) continue;
      const int key = it.k0 + (warp & 3) * 32 + lane;
      const bool alone = first_row_alone(p, it.q);
      for (int t = 0; t < it.steps; ++t, ++n_q) {
        const int s = n_q % kStages;
        kv_step(p, it, t, head, q0);
        // columns [lo, hi) of this half see the key
        const int at = q0 + 64 * half;
        const int lo = key >= it.q.n ? 64 : p.causal && key >= it.q.prefix ? key - at : 0, hi = it.q.n - at;
        const bool masked = __any_sync(0xffffffffu, lo > 0 || hi < 64);
        const float slope2 = kExtra && p.slopes ? p.slopes[head] * kAttLog2e : 0.f;
        if (!(ok = mbar_wait_warp(bar(A_VECFULL + s), n_q / kStages & 1, ctl))) break;
        if (!(ok = mbar_wait_warp(bar(A_SFULL), n_q & 1, ctl))) break;
        tc_fence_after();
        float pr[64];
        [[maybe_unused]] float bend[kExtra ? 64 : 1];
        {
          uint32_t a[2][32];
          tmem_ld_32x32b_x32(t_s + lanes + 64 * half, a[0]);
          tmem_ld_32x32b_x32(t_s + lanes + 64 * half + 32, a[1]);
          tmem_ld_wait();
          const float4* lse = reinterpret_cast<const float4*>(vec + s * 256 + 64 * half);
#pragma unroll
          for (int c = 0; c < 16; ++c) {
            const float4 l4 = lse[c];
            const float l[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int k = 4 * c + e;
              float x = __uint_as_float(a[k >> 5][k & 31]);
              if constexpr (kExtra) {
                x = score2(p, x, slope2, fabsf(static_cast<float>(at + k - key)), bend[k]) - l[e];
              } else {
                x = fmaf(x, scale2, -l[e]);
              }
              pr[k] = fast_exp2(x);
            }
          }
          if (masked) {
#pragma unroll
            for (int k = 0; k < 64; ++k) pr[k] = k >= lo && k < hi ? pr[k] : 0.f;
          }
          uint32_t w[32];
#pragma unroll
          for (int k = 0; k < 32; ++k) w[k] = pack_bf16x2(pr[2 * k], pr[2 * k + 1]);
          tmem_st_32x32b_x32(t_s + lanes + 64 * half, w);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(A_PREADY));
        if (!(ok = mbar_wait_warp(bar(A_DPFULL), n_q & 1, ctl))) break;
        tc_fence_after();
        {
          uint32_t a[2][32], w[32];
          tmem_ld_32x32b_x32(t_dp + lanes + 64 * half, a[0]);
          tmem_ld_32x32b_x32(t_dp + lanes + 64 * half + 32, a[1]);
          tmem_ld_wait();
          const float4* del = reinterpret_cast<const float4*>(vec + s * 256 + 128 + 64 * half);
#pragma unroll
          for (int c = 0; c < 16; ++c) {
            const float4 d4 = del[c];
            const float d[4] = {d4.x, d4.y, d4.z, d4.w};
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int k = 4 * c + e;
              x[e] = pr[k] * (__uint_as_float(a[k >> 5][k & 31]) - d[e]);
              if constexpr (kExtra) x[e] *= bend[k];
              if (masked) x[e] = k >= lo && k < hi && !(alone && at + k == 0) ? x[e] : 0.f;
            }
            w[2 * c] = pack_bf16x2(x[0], x[1]);
            w[2 * c + 1] = pack_bf16x2(x[2], x[3]);
          }
          tmem_st_32x32b_x32(t_dp + lanes + 64 * half, w);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bar(A_DSREADY));
          mbar_arrive(bar(A_VECEMPTY + s));
        }
      }
      if (!ok) break;
      // dv by the first four warps, dk by the others
      if (!(ok = mbar_wait_warp(bar(A_OFULL), n_o++ & 1, ctl))) break;
      tc_fence_after();
      const HeadsView& dst = half ? p.dk : p.dv;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(const_cast<void*>(dst.x)) +
                           static_cast<int64_t>(it.q.start + key) * dst.token_stride + it.kv_head * dst.head_stride;
      for (int c = 0; c < p.D; c += 32)
        store_cols((half ? t_dk : t_dv) + lanes, out, key < it.q.n, c, p.D, half ? p.scale : 1.f);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(A_OEMPTY));
    }
  }

  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag && p.dev_status) atomicOr(p.dev_status, kStatusTimeout);
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// --------------------------------------------------------------------- dq ---
// tensor memory: S, two of dP (then dS), dQ.  Order of the MMAs: dP_j, S_{j+1}, dQ_j.
enum { C_QFULL = 0, C_QEMPTY, C_KVFULL, C_KVEMPTY = C_KVFULL + kStages, C_FIX = C_KVEMPTY + kStages,
       C_SFULL = C_FIX + kStages, C_SEMPTY, C_DPFULL, C_DSREADY, C_OFULL, C_OEMPTY, C_DRAIN, C_COUNT };

constexpr int dq_smem(int boxes) { return 1024 + (2 + 2 * kStages) * boxes * kBoxBytes + 8 * C_COUNT + 16; }

struct QItem {
  Seq q;
  int head, q0, seen, tiles;
};
__device__ __forceinline__ bool q_item(const AttArgs& p, int64_t i, QItem& it) {
  it.q = seq_of_slot<128>(p, static_cast<int>(i / p.Hq));
  if (it.q.tile < 0) return false;
  it.head = static_cast<int>(i % p.Hq);
  // the longest rows first
  it.q0 = 128 * (p.causal ? (it.q.n + 127) / 128 - 1 - it.q.tile : it.q.tile);
  it.seen = keys_seen(p, it.q, min(it.q0 + 128, it.q.n) - 1);
  it.tiles = (it.seen + 127) / 128;
  return true;
}

template <int kBoxes, bool kExtra>
__global__ void __launch_bounds__(kThreads, 1)
    att_dq_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                  const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do, const AttArgs p,
                  const float2* stats, int64_t items) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  constexpr uint32_t kTileBytes = kBoxes * kBoxBytes;
  const uint32_t sq = base, sdo = sq + kTileBytes, sk = sdo + kTileBytes, sv = sk + kStages * kTileBytes;
  const uint32_t bar0 = sv + kStages * kTileBytes;
  uint8_t* misc = smem_raw + (bar0 - raw) + 8 * C_COUNT;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(misc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 4);
  const auto bar = [&](int i) { return bar0 + 8u * i; };
  const int warp = warp_uniform(static_cast<int>(threadIdx.x >> 5)), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < C_COUNT; ++i) mbar_init(bar(i), i == C_SEMPTY || i == C_DSREADY || i == C_OEMPTY ? kRowWarps : 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == kMmaWarp) {
    tmem_alloc(smem_u32(tmem_slot), 512);
    tmem_relinquish();
  }
  if (warp == kTmaWarp && lane == 0) {
    tma_prefetch_desc(&map_q);
    tma_prefetch_desc(&map_k);
    tma_prefetch_desc(&map_v);
    tma_prefetch_desc(&map_do);
  }
  check_offsets(p);
  zero_behind(p, const_cast<void*>(p.dq.x), p.dq.token_stride, p.dq.head_stride, p.Hq);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = warp_uniform(*tmem_slot);
  const auto t_dp = [&](uint32_t n) { return tmem + 128u + 128u * (n & 1); };
  const uint32_t t_s = tmem, t_dq = tmem + 384;
  const WaitCtl ctl{abort_flag, p.wait_limit_ns};
  QItem it;

  if (warp >= kTmaWarp) {
    regs_dec<kRegsRest>();
    if (warp == kTmaWarp) {
      const bool leader = elect_one();
      uint32_t n_q = 0, n_kv = 0;
      bool ok = true;
      for (int64_t i = blockIdx.x; ok && i < items; i += gridDim.x) {
        if (!q_item(p, i, it)) continue;
        const int kv = it.head / (p.Hq / p.Hk);
        if (!(ok = mbar_wait_warp(bar(C_QEMPTY), (n_q++ & 1) ^ 1, ctl))) break;
        if (leader) {
          mbar_arrive_expect_tx(bar(C_QFULL), 2 * kTileBytes);
          load_tile(sq, &map_q, bar(C_QFULL), kBoxes, p.q.head_stride ? it.head : 0, it.q.start + it.q0);
          load_tile(sdo, &map_do, bar(C_QFULL), kBoxes, p.d_o.head_stride ? it.head : 0, it.q.start + it.q0);
        }
        for (int j = 0; j < it.tiles; ++j, ++n_kv) {
          const int s = n_kv % kStages;
          if (!(ok = mbar_wait_warp(bar(C_KVEMPTY + s), (n_kv / kStages & 1) ^ 1, ctl))) break;
          if (leader) {
            mbar_arrive_expect_tx(bar(C_KVFULL + s), 2 * kTileBytes);
            load_tile(sk + s * kTileBytes, &map_k, bar(C_KVFULL + s), kBoxes, p.k.head_stride ? kv : 0, it.q.start + 128 * j);
            load_tile(sv + s * kTileBytes, &map_v, bar(C_KVFULL + s), kBoxes, p.v.head_stride ? kv : 0, it.q.start + 128 * j);
          }
          const int rows = it.seen - 128 * j;
          if (rows < 128 && rows % 16 != 0) {
            if (!(ok = mbar_wait_warp(bar(C_KVFULL + s), n_kv / kStages & 1, ctl))) break;
            zero_rows(sk + s * kTileBytes, kBoxes, rows, up16(rows));
            fence_proxy_async_shared();
            __syncwarp();
            if (leader) mbar_arrive(bar(C_FIX + s));
          }
        }
      }
      if (!ok) let_copies_land();
      __syncwarp();
    } else if (warp == kMmaWarp) {
      const bool leader = elect_one();
      const int steps = (p.D + 15) / 16;
      const uint32_t id_out = idesc_bf16(128, 16 * steps, false, true);
      uint32_t n_q = 0, n_kv = 0, fixed = 0;
      bool ok = true;
      for (int64_t i = blockIdx.x; ok && i < items; i += gridDim.x) {
        if (!q_item(p, i, it)) continue;
        if (!(ok = mbar_wait_warp(bar(C_QFULL), n_q & 1, ctl))) break;
        const auto cols_of = [&](int j) { return up16(min(128, it.seen - 128 * j)); };
        const auto scores = [&](int j) {
          const uint32_t n = n_kv + j;
          if (!mbar_wait_warp(bar(C_KVFULL + n % kStages), n / kStages & 1, ctl)) return false;
          if (!mbar_wait_warp(bar(C_SEMPTY), (n & 1) ^ 1, ctl)) return false;
          tc_fence_after();
          const uint32_t id = idesc_bf16(128, cols_of(j), false, false);
          if (leader) {
            mma_rows(t_s, sq, sk + n % kStages * kTileBytes, id, steps);
            umma_commit(bar(C_SFULL));
          }
          return true;
        };
        if (!(ok = scores(0))) break;
        for (int j = 0; j < it.tiles; ++j) {
          const uint32_t n = n_kv + j;
          const int s = n % kStages, cols = cols_of(j);
          if (leader) {
            mma_rows(t_dp(n), sdo, sv + s * kTileBytes, idesc_bf16(128, cols, false, false), steps);
            umma_commit(bar(C_DPFULL));
          }
          if (j + 1 < it.tiles && !(ok = scores(j + 1))) break;
          const int rows = it.seen - 128 * j;
          if (rows < 128 && rows % 16 != 0) {
            if (!(ok = mbar_wait_warp(bar(C_FIX + s), fixed >> s & 1, ctl))) break;
            fixed ^= 1u << s;
          }
          if (j == 0 && !(ok = mbar_wait_warp(bar(C_OEMPTY), (n_q & 1) ^ 1, ctl))) break;
          if (!(ok = mbar_wait_warp(bar(C_DSREADY), n & 1, ctl))) break;
          tc_fence_after();
          if (leader) {
            mma_cols(t_dq, t_dp(n), 64, sk + s * kTileBytes, id_out, cols / 16, j > 0);
            umma_commit(bar(C_KVEMPTY + s));
          }
        }
        if (!ok) break;
        n_kv += it.tiles;
        ++n_q;
        if (leader) {
          umma_commit(bar(C_OFULL));
          umma_commit(bar(C_QEMPTY));
        }
      }
      drain_mmas(bar(C_DRAIN), leader, p.wait_limit_ns);
    }
  } else {
    regs_inc<kRegsRows>();
    const int half = warp >> 2;  // of the tile's key columns
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const float scale2 = p.scale * kAttLog2e;
    uint32_t n_kv = 0, n_o = 0;
    bool ok = true;
    for (int64_t i = blockIdx.x; ok && i < items; i += gridDim.x) {
      if (!q_item(p, i, it)) continue;
      const int pos = it.q0 + (warp & 3) * 32 + lane, real = min(pos, it.q.n - 1);
      const float2 st = stats[static_cast<int64_t>(it.head) * p.T + it.q.start + real];
      const int lim = keys_seen(p, it.q, real);
      const bool alone = pos == 0 && first_row_alone(p, it.q);
      const float slope2 = kExtra && p.slopes ? p.slopes[it.head] * kAttLog2e : 0.f;
      for (int j = 0; j < it.tiles; ++j, ++n_kv) {
        const int at = 128 * j + 64 * half, here = lim - at;
        const bool masked = __any_sync(0xffffffffu, here < 64);
        if (!(ok = mbar_wait_warp(bar(C_SFULL), n_kv & 1, ctl))) break;
        tc_fence_after();
        float pr[64];
        {
          uint32_t a[2][32];
          tmem_ld_32x32b_x32(t_s + lanes + 64 * half, a[0]);
          tmem_ld_32x32b_x32(t_s + lanes + 64 * half + 32, a[1]);
          tmem_ld_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(C_SEMPTY));
#pragma unroll
          for (int k = 0; k < 64; ++k) {
            float x = __uint_as_float(a[k >> 5][k & 31]);
            if constexpr (kExtra) {
              float bend;
              x = score2(p, x, slope2, fabsf(static_cast<float>(pos - at - k)), bend) - st.x;
              pr[k] = fast_exp2(x) * bend;  // (p itself is not needed here)
            } else {
              pr[k] = fast_exp2(fmaf(x, scale2, -st.x));
            }
          }
        }
        if (!(ok = mbar_wait_warp(bar(C_DPFULL), n_kv & 1, ctl))) break;
        tc_fence_after();
        {
          uint32_t a[2][32], w[32];
          const uint32_t td = t_dp(n_kv) + lanes + 64 * half;
          tmem_ld_32x32b_x32(td, a[0]);
          tmem_ld_32x32b_x32(td + 32, a[1]);
          tmem_ld_wait();
#pragma unroll
          for (int k = 0; k < 64; k += 2) {
            float x = pr[k] * (__uint_as_float(a[k >> 5][k & 31]) - st.y);
            float y = pr[k + 1] * (__uint_as_float(a[k >> 5][(k & 31) + 1]) - st.y);
            if (masked) {
              x = k < here && !alone ? x : 0.f;
              y = k + 1 < here && !alone ? y : 0.f;
            }
            w[k / 2] = pack_bf16x2(x, y);
          }
          tmem_st_32x32b_x32(td, w);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C_DSREADY));
      }
      if (!ok) break;
      if (!(ok = mbar_wait_warp(bar(C_OFULL), n_o++ & 1, ctl))) break;
      tc_fence_after();
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(const_cast<void*>(p.dq.x)) +
                           static_cast<int64_t>(it.q.start + pos) * p.dq.token_stride + it.head * p.dq.head_stride;
      for (int c = 32 * half; c < p.D; c += 64) store_cols(t_dq + lanes, out, pos < it.q.n, c, p.D, p.scale);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C_OEMPTY));
    }
  }

  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag && p.dev_status) atomicOr(p.dev_status, kStatusTimeout);
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <int kBoxes, bool kExtra>
olive_status run_bwd(const Ctx& c, const AttArgs& a) {
  CUtensorMap mq, mk, mv, mdo;
  if (!encode_heads(&mq, a.q, a.T, a.Hq, a.D) || !encode_heads(&mk, a.k, a.T, a.Hk, a.D) ||
      !encode_heads(&mv, a.v, a.T, a.Hk, a.D) || !encode_heads(&mdo, a.d_o, a.T, a.Hq, a.D))
    return OLIVE_ERR_CUDA;
  static std::atomic<int> done_kv[kMaxDevices], done_q[kMaxDevices];
  const auto dkdv = att_dkdv_kernel<kBoxes, kExtra>;
  const auto dq = att_dq_kernel<kBoxes, kExtra>;
  constexpr int kSmemKv = kv_smem(kBoxes), kSmemQ = dq_smem(kBoxes);
  static_assert(kSmemKv <= 227 * 1024 && kSmemQ <= 227 * 1024, "shared memory");
  if (!set_smem_once(reinterpret_cast<const void*>(dkdv), kSmemKv, c.device, done_kv) ||
      !set_smem_once(reinterpret_cast<const void*>(dq), kSmemQ, c.device, done_q))
    return OLIVE_ERR_CUDA;
  float2* stats = static_cast<float2*>(a.ws);
  const int64_t slots = att_slots(a.T, a.S, 128);
  const auto grid = [&](int64_t items) { return static_cast<unsigned>(std::min<int64_t>(items, c.num_sms)); };
  att_delta_kernel<<<static_cast<unsigned>(slots * a.Hq), kDeltaThreads, 0, c.stream>>>(a, stats);
  dkdv<<<grid(slots * a.Hk), kThreads, kSmemKv, c.stream>>>(mq, mk, mv, mdo, a, stats, slots * a.Hk);
  dq<<<grid(slots * a.Hq), kThreads, kSmemQ, c.stream>>>(mq, mk, mv, mdo, a, stats, slots * a.Hq);
  return cudaGetLastError() == cudaSuccess ? OLIVE_OK : OLIVE_ERR_CUDA;
}

template <int kBoxes>
olive_status by_form(const Ctx& c, const AttArgs& a) {
  return a.cap > 0.f || a.slopes ? run_bwd<kBoxes, true>(c, a) : run_bwd<kBoxes, false>(c, a);
}

}  // namespace

size_t att_bwd_ws_bytes(int64_t T, int64_t Hq) { return align_up(8ull * T * Hq, kWsAlign); }

olive_status launch_att_bwd(const Ctx& c, const AttArgs& a) {
  return a.D <= 64 ? by_form<1>(c, a) : by_form<2>(c, a);
}

}  // namespace olive
