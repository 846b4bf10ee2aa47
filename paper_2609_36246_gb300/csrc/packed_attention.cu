// packed_attention.cu -- attention inside packed sequences, forward.
//
//   z_ij = scale q_i . k_j,  s_ij = cap tanh(z_ij / cap) - slope |i - j|,
//   o_i = sum over the keys j that i sees of exp(s_ij - lse_i) v_j
//
// What a row sees is always its sequence's first keys (up to itself, its prompt's end
// or the sequence's end), so a mask is one number a row.
//
// A CTA works on two slots of 128 query rows with the same keys (two heads of a key
// head, or two tiles of a head) and walks the key tiles:
//   warp 8     TMA: query tiles, then key and value tiles into rings of two
//   warp 9     MMA: S = Q K^T into tensor memory, O += P V with P read from there
//   warps 0-3, 4-7  the rows of slot 0 and 1, one a thread: the running maximum and
//              sum, P = exp2(S - reference) in bf16 over S in tensor memory.
// While one slot's rows are exponentiated the other's products run.  A row's reference
// follows its maximum only when that is more than 8 (in log2) above, as O has to be
// scaled then; until there P and the sum are relative to the old one, exactly.
#include <algorithm>

#include "packed_attention.cuh"

namespace olive {
namespace {

constexpr int kThreads = 384;  // (the last two warps only give up their registers)
constexpr int kRegsLaunch = 168, kRegsSoft = 224, kRegsRest = 56;
static_assert(2 * kRegsSoft + kRegsRest <= 3 * kRegsLaunch, "the block's registers");
constexpr int kStages = 2;
constexpr int kTmaWarp = 8, kMmaWarp = 9;
constexpr float kLag = 8.f;
enum { B_QFULL = 0, B_QEMPTY = 2, B_KFULL = 4, B_KEMPTY = B_KFULL + kStages, B_VFULL = B_KEMPTY + kStages,
       B_VEMPTY = B_VFULL + kStages, B_VFIX = B_VEMPTY + kStages, B_SFULL = B_VFIX + kStages, B_PREADY = B_SFULL + 2,
       B_OFULL = B_PREADY + 2, B_OEMPTY = B_OFULL + 2, B_DRAIN = B_OEMPTY + 2, B_COUNT };

constexpr int smem_bytes(int boxes) { return 1024 + (2 + 2 * kStages) * boxes * kBoxBytes + 8 * B_COUNT + 16; }

// An item's slots: heads, first rows and key tiles.
struct Item {
  Seq q;
  int kv_head, head[2], row0[2], tiles[2], seen[2];  // seen: keys that the slot's last row sees
};
// Two heads of a key head where their number is even, else two tiles of a head.
template <bool kPairHeads>
__device__ __forceinline__ bool item_at(const AttArgs& p, int64_t i, int units, Item& it) {
  const int slot = static_cast<int>(i / units), u = static_cast<int>(i % units);
  it.q = seq_of_slot<kPairHeads ? 128 : 256>(p, slot);
  if (it.q.tile < 0) return false;
  constexpr int R = kPairHeads ? 128 : 256;
  // the longest rows first
  const int tile = p.causal ? (it.q.n + R - 1) / R - 1 - it.q.tile : it.q.tile;
  const int per = p.Hq / p.Hk;
#pragma unroll
  for (int a = 0; a < 2; ++a) {
    it.head[a] = kPairHeads ? 2 * u + a : u;
    it.row0[a] = kPairHeads ? tile * 128 : tile * 256 + a * 128;
    it.seen[a] = it.row0[a] < it.q.n ? keys_seen(p, it.q, min(it.row0[a] + 128, it.q.n) - 1) : 0;
    it.tiles[a] = (it.seen[a] + 127) / 128;
  }
  it.kv_head = it.head[0] / per;
  return true;
}

template <int kBoxes, bool kPairHeads, bool kExtra>
__global__ void __launch_bounds__(kThreads, 1)
    att_fwd_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                   const __grid_constant__ CUtensorMap map_v, const AttArgs p, int units, int64_t items) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  constexpr uint32_t kTileBytes = kBoxes * kBoxBytes;
  const uint32_t sq = base, sk = sq + 2 * kTileBytes, sv = sk + kStages * kTileBytes;
  const uint32_t bar0 = sv + kStages * kTileBytes;
  uint8_t* misc = smem_raw + (bar0 - raw) + 8 * B_COUNT;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(misc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 4);
  const auto bar = [&](int i) { return bar0 + 8u * i; };
  const int warp = warp_uniform(static_cast<int>(threadIdx.x >> 5)), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < B_COUNT; ++i)
      mbar_init(bar(i), i >= B_PREADY && i < B_PREADY + 2 ? 4 : i >= B_OEMPTY && i < B_OEMPTY + 2 ? 4 : 1);
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
  }
  check_offsets(p);
  zero_behind(p, const_cast<void*>(p.o.x), p.o.token_stride, p.o.head_stride, p.Hq);
  if (p.lse) {
    const int first = cu_at(p, p.S), n = p.T - first;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < static_cast<int64_t>(n) * p.Hq;
         i += static_cast<int64_t>(gridDim.x) * kThreads)
      p.lse[i / n * p.T + first + i % n] = __uint_as_float(0xff800000u);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = warp_uniform(*tmem_slot);
  const WaitCtl ctl{abort_flag, p.wait_limit_ns};
  // tensor memory: S (and P in its first half) of slot 0 and 1, O of slot 0 and 1
  const auto t_s = [&](int a) { return tmem + 128u * a; };
  const auto t_o = [&](int a) { return tmem + 256u + 128u * a; };
  Item it;

  if (warp >= kTmaWarp) {
    regs_dec<kRegsRest>();
    if (warp == kTmaWarp) {
      const bool leader = elect_one();
      uint32_t n_q[2] = {0, 0}, n_kv = 0;
      bool ok = true;
      for (int64_t i = blockIdx.x; ok && i < items; i += gridDim.x) {
        if (!item_at<kPairHeads>(p, i, units, it)) continue;
        const int tiles = max(it.tiles[0], it.tiles[1]), seen = max(it.seen[0], it.seen[1]);
        const auto query = [&](int a) {
          if (it.tiles[a] == 0) return true;
          if (!mbar_wait_warp(bar(B_QEMPTY + a), (n_q[a] & 1) ^ 1, ctl)) return false;
          ++n_q[a];
          if (leader) {
            mbar_arrive_expect_tx(bar(B_QFULL + a), kTileBytes);
            load_tile(sq + a * kTileBytes, &map_q, bar(B_QFULL + a), kBoxes, p.q.head_stride ? it.head[a] : 0, it.q.start + it.row0[a]);
          }
          return true;
        };
        ok = query(0);
        for (int j = 0; ok && j < tiles; ++j, ++n_kv) {
          const int s = n_kv % kStages;
          const uint32_t free = (n_kv / kStages & 1) ^ 1;
          if (!(ok = mbar_wait_warp(bar(B_KEMPTY + s), free, ctl))) break;
          if (leader) {
            mbar_arrive_expect_tx(bar(B_KFULL + s), kTileBytes);
            load_tile(sk + s * kTileBytes, &map_k, bar(B_KFULL + s), kBoxes, p.k.head_stride ? it.kv_head : 0, it.q.start + 128 * j);
          }
          if (j == 0 && !(ok = query(1))) break;
          if (!(ok = mbar_wait_warp(bar(B_VEMPTY + s), free, ctl))) break;
          if (leader) {
            mbar_arrive_expect_tx(bar(B_VFULL + s), kTileBytes);
            load_tile(sv + s * kTileBytes, &map_v, bar(B_VFULL + s), kBoxes, p.v.head_stride ? it.kv_head : 0, it.q.start + 128 * j);
          }
          // the sequence's last rows: what follows them up to whole K steps is zeroed
          const int rows = seen - 128 * j;
          if (rows < 128 && rows % 16 != 0) {
            if (!(ok = mbar_wait_warp(bar(B_VFULL + s), n_kv / kStages & 1, ctl))) break;
            if (it.q.n - 128 * j < 128) zero_rows(sv + s * kTileBytes, kBoxes, rows, up16(rows));
            fence_proxy_async_shared();
            __syncwarp();
            if (leader) mbar_arrive(bar(B_VFIX + s));
          }
        }
      }
      if (!ok) let_copies_land();
      __syncwarp();
    } else if (warp == kMmaWarp) {
      const bool leader = elect_one();
      const int steps = (p.D + 15) / 16;
      uint32_t n_q[2] = {0, 0}, n_kv = 0, fixed = 0, n_p[2] = {0, 0}, n_o[2] = {0, 0};
      bool ok = true;
      for (int64_t i = blockIdx.x; ok && i < items; i += gridDim.x) {
        if (!item_at<kPairHeads>(p, i, units, it)) continue;
        const int tiles = max(it.tiles[0], it.tiles[1]), seen = max(it.seen[0], it.seen[1]);
        for (int j = 0; ok && j <= tiles; ++j) {
          const uint32_t at = n_kv + j, before = at - 1;
          if (j < tiles && !(ok = mbar_wait_warp(bar(B_KFULL + at % kStages), at / kStages & 1, ctl))) break;
          if (j > 0) {
            if (!(ok = mbar_wait_warp(bar(B_VFULL + before % kStages), before / kStages & 1, ctl))) break;
            const int rows = seen - 128 * (j - 1), s = before % kStages;
            if (rows < 128 && rows % 16 != 0) {
              if (!(ok = mbar_wait_warp(bar(B_VFIX + s), fixed >> s & 1, ctl))) break;
              fixed ^= 1u << s;
            }
          }
#pragma unroll
          for (int a = 0; a < 2; ++a) {
            if (j > 0 && j - 1 < it.tiles[a]) {  // O += P V of the tile before
              if (j == 1 && !(ok = mbar_wait_warp(bar(B_OEMPTY + a), (n_o[a]++ & 1) ^ 1, ctl))) break;
              if (!(ok = mbar_wait_warp(bar(B_PREADY + a), n_p[a]++ & 1, ctl))) break;
              tc_fence_after();
              const int ks = up16(min(128, it.seen[a] - 128 * (j - 1))) / 16;
              if (leader) {
                mma_cols(t_o(a), t_s(a), 32, sv + before % kStages * kTileBytes, idesc_bf16(128, 16 * steps, false, true), ks, j > 1);
                if (j == it.tiles[a]) umma_commit(bar(B_OFULL + a));
              }
            }
            if (j < it.tiles[a]) {  // S of this one
              if (j == 0 && !(ok = mbar_wait_warp(bar(B_QFULL + a), n_q[a]++ & 1, ctl))) break;
              tc_fence_after();
              const int cols = up16(min(128, it.seen[a] - 128 * j));
              if (leader) {
                mma_rows(t_s(a), sq + a * kTileBytes, sk + at % kStages * kTileBytes, idesc_bf16(128, cols, false, false), steps);
                umma_commit(bar(B_SFULL + a));
                if (j == it.tiles[a] - 1) umma_commit(bar(B_QEMPTY + a));
              }
            }
          }
          if (ok && leader) {
            if (j > 0) umma_commit(bar(B_VEMPTY + before % kStages));
            if (j < tiles) umma_commit(bar(B_KEMPTY + at % kStages));
          }
        }
        n_kv += tiles;
      }
      // every MMA issued is complete before the CTA retires (they end by themselves)
      if (leader) umma_commit(bar(B_DRAIN));
      volatile int keep_waiting = 0;
      const uint64_t floor_ns = 200ull * 1000 * 1000;
      const WaitCtl own{&keep_waiting, p.wait_limit_ns > floor_ns ? p.wait_limit_ns : floor_ns};
      mbar_wait_warp(bar(B_DRAIN), 0, own);
      __syncwarp();
    }
  } else {
    regs_inc<kRegsSoft>();
    const int a = warp >> 2;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const int row = (warp & 3) * 32 + lane;
    const uint32_t ts = t_s(a) + lanes, to = t_o(a) + lanes;
    const float scale2 = p.scale * kAttLog2e;
    uint32_t n_s = 0, n_o = 0;
    bool ok = true;
    for (int64_t i = blockIdx.x; ok && i < items; i += gridDim.x) {
      if (!item_at<kPairHeads>(p, i, units, it)) continue;
      const int tiles = a ? it.tiles[1] : it.tiles[0];
      if (tiles == 0) continue;
      const int head = a ? it.head[1] : it.head[0];
      const int pos = (a ? it.row0[1] : it.row0[0]) + row;
      const int lim = keys_seen(p, it.q, min(pos, it.q.n - 1));
      const float slope2 = kExtra && p.slopes ? p.slopes[head] * kAttLog2e : 0.f;
      const float to_cap = kExtra && p.cap > 0.f ? 2.f * scale2 / p.cap : 0.f, cap2 = p.cap * kAttLog2e;
      float ref = 0.f, sum = 0.f;
      for (int j = 0; j < tiles; ++j) {
        if (!(ok = mbar_wait_warp(bar(B_SFULL + a), n_s++ & 1, ctl))) break;
        tc_fence_after();
        uint32_t s[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld_32x32b_x32(ts + 32 * c, s[c]);
        tmem_ld_wait();
        float mul = scale2;
        if constexpr (kExtra) {
          mul = 1.f;
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              float x = __uint_as_float(s[c][e]);
              x = to_cap != 0.f ? cap2 * tanh_of(x * to_cap) : x * scale2;
              s[c][e] = __float_as_uint(fmaf(-slope2, fabsf(static_cast<float>(pos - (128 * j + 32 * c + e))), x));
            }
        }
        const int here = lim - 128 * j;
        if (__any_sync(0xffffffffu, here < 128)) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (32 * c + e >= here) s[c][e] = 0xff800000u;
        }
        float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int e = 0; e < 32; ++e)
#pragma unroll
          for (int c = 0; c < 4; ++c) top[c] = fmaxf(top[c], __uint_as_float(s[c][e]));
        const float m = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * mul;
        if (j == 0) {
          ref = m > -INFINITY ? m : 0.f;
        } else if (__any_sync(0xffffffffu, m > ref + kLag)) {
          const float now = m > ref + kLag ? m : ref;
          const float f = fast_exp2(ref - now);
          ref = now;
          sum *= f;
          for (int c = 0; c < p.D; c += 32) {
            uint32_t o[32];
            tmem_ld_32x32b_x32(to + c, o);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
            tmem_st_32x32b_x32(to + c, o);
          }
        }
        float part[4] = {};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t w[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            const int c = 2 * h + (e >> 4), k = 2 * (e & 15);
            const float x = fast_exp2(fmaf(__uint_as_float(s[c][k]), mul, -ref));
            const float y = fast_exp2(fmaf(__uint_as_float(s[c][k + 1]), mul, -ref));
            part[2 * (e & 1)] += x;
            part[2 * (e & 1) + 1] += y;
            w[e] = pack_bf16x2(x, y);
          }
          tmem_st_32x32b_x32(ts + 32 * h, w);
        }
        sum += (part[0] + part[1]) + (part[2] + part[3]);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_PREADY + a));
      }
      if (!ok) break;
      if (!(ok = mbar_wait_warp(bar(B_OFULL + a), n_o++ & 1, ctl))) break;
      tc_fence_after();
      const bool store = pos < it.q.n;
      const float inv = 1.f / sum;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(const_cast<void*>(p.o.x)) +
                           static_cast<int64_t>(it.q.start + pos) * p.o.token_stride + head * p.o.head_stride;
      for (int c = 0; c < p.D; c += 32) {
        uint32_t o[32];
        tmem_ld_32x32b_x32(to + c, o);
        tmem_ld_wait();
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          if (!store || c + 8 * v >= p.D) continue;
          float f[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(o[8 * v + e]) * inv;
          reinterpret_cast<uint4*>(out + c)[v] = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]),
                                                            pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_OEMPTY + a));
      if (store && p.lse) p.lse[static_cast<int64_t>(head) * p.T + it.q.start + pos] = (ref + log2f(sum)) * kAttLn2;
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

template <int kBoxes, bool kPairHeads, bool kExtra>
olive_status run_fwd(const Ctx& c, const AttArgs& a) {
  CUtensorMap mq, mk, mv;
  if (!encode_heads(&mq, a.q, a.T, a.Hq, a.D) || !encode_heads(&mk, a.k, a.T, a.Hk, a.D) || !encode_heads(&mv, a.v, a.T, a.Hk, a.D))
    return OLIVE_ERR_CUDA;
  static std::atomic<int> done[kMaxDevices];
  const auto kernel = att_fwd_kernel<kBoxes, kPairHeads, kExtra>;
  constexpr int kSmem = smem_bytes(kBoxes);
  if (!set_smem_once(reinterpret_cast<const void*>(kernel), kSmem, c.device, done)) return OLIVE_ERR_CUDA;
  const int units = kPairHeads ? a.Hq / 2 : a.Hq;
  const int64_t items = att_slots(a.T, a.S, kPairHeads ? 128 : 256) * units;
  kernel<<<static_cast<unsigned>(std::min<int64_t>(items, c.num_sms)), kThreads, kSmem, c.stream>>>(mq, mk, mv, a, units, items);
  return cudaGetLastError() == cudaSuccess ? OLIVE_OK : OLIVE_ERR_CUDA;
}

template <int kBoxes>
olive_status by_form(const Ctx& c, const AttArgs& a) {
  const bool pair = a.Hq / a.Hk % 2 == 0, extra = a.cap > 0.f || a.slopes;
  if (pair) return extra ? run_fwd<kBoxes, true, true>(c, a) : run_fwd<kBoxes, true, false>(c, a);
  return extra ? run_fwd<kBoxes, false, true>(c, a) : run_fwd<kBoxes, false, false>(c, a);
}

}  // namespace

olive_status launch_att_fwd(const Ctx& c, const AttArgs& a) {
  return a.D <= 64 ? by_form<1>(c, a) : by_form<2>(c, a);
}

}  // namespace olive
