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
//
// 8 sequences of 4096, 32 + 8 heads of 128, causal: 107, 1230 and 1110 us; the seven products
// run at 1.57 PFLOP/s (tensor pipe active 74 and 62 % of a shorter launch's cycles), near what
// the power cap leaves.  200 sequences of some 41 tokens, 16 + 16 heads of 64: 29, 91 and 48
// us, an item's chain of waits.
#include <algorithm>
#include <type_traits>

#include "packed_attention.cuh"

namespace olive {
namespace {

// Rows of a tile: 16 warps, four to a quarter of its columns.  (With eight, a half each,
// their chain of waits, loads and stores is longer than the MMAs beside it.)
constexpr int kRowWarps = 16, kCols = kAttTile / (kRowWarps / 4);
constexpr int kTmaWarp = 0, kMmaWarp = 1, kItemWarp = 3, kRestWarps = 4;
constexpr int kThreads = 32 * 20;
constexpr int kReaders = kRowWarps + 2;
constexpr int kRegsLaunch = 96, kRegsRows = 104, kRegsRest = 64;
static_assert(4 * kRegsRows + kRegsRest <= 5 * kRegsLaunch, "the block's registers");

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
// stats: [Hq, T] of (lse in base 2, delta); a block works on a tile's rows of one head,
// 16 lanes a row, two rows' loads in flight together.
__global__ void __launch_bounds__(kDeltaThreads, 8) att_delta_kernel(const AttArgs p, float2* stats) {
  constexpr int kGroups = kDeltaThreads / 16, kAtOnce = 2;
  const int head = static_cast<int>(blockIdx.x % p.Hq), slot = static_cast<int>(blockIdx.x / p.Hq);
  grid_launch_dependents();
  int near = 0;
  const Seq q = seq_of_slot<128>(p, slot, near);
  if (q.tile < 0) return;
  const int lane = threadIdx.x % 16, group = threadIdx.x / 16, kv = head / (p.Hq / p.Hk);
  const bool in = 8 * lane < p.D;
  const ScoreForm form(p);
  const float slope2 = p.slopes ? p.slopes[head] * kAttLog2e : 0.f;
  const int row0 = q.tile * 128, rows = min(128, q.n - row0);
  const float* lse = p.lse + static_cast<int64_t>(head) * p.T + q.start;
  float2* out = stats + static_cast<int64_t>(head) * p.T + q.start;
#pragma unroll 1
  for (int r = group; __any_sync(0xffffffffu, r < rows); r += kAtOnce * kGroups) {
    float a[kAtOnce][8], b[kAtOnce][8], l[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int64_t t = q.start + row0 + min(r + k * kGroups, rows - 1);
      eight(row_of(p.d_o, t, head) + 8 * lane, in, a[k]);
      eight(row_of(p.o, t, head) + 8 * lane, in, b[k]);
      l[k] = lse[t - q.start];
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      if (!__any_sync(0xffffffffu, r + k * kGroups < rows)) break;
      const int i = row0 + min(r + k * kGroups, rows - 1);
      const float lse2 = l[k] * kAttLog2e;
      float delta = dot16(a[k], b[k]);
      const int keys = keys_seen(p, q, i);
      const bool few = keys <= kFewKeys && r + k * kGroups < rows;
      if (__any_sync(0xffffffffu, few)) {
        const int64_t t = q.start + i;
        const int most = few ? keys : 0;
        float qr[8], sum = 0.f;
        eight(row_of(p.q, t, head) + 8 * lane, in, qr);
        for (int j0 = 0; __any_sync(0xffffffffu, j0 < most); j0 += kAtOnce) {
          float key[kAtOnce][8], value[kAtOnce][8];
#pragma unroll
          for (int e = 0; e < kAtOnce; ++e) {
            const int64_t tj = q.start + min(j0 + e, keys - 1);
            eight(row_of(p.k, tj, kv) + 8 * lane, in, key[e]);
            eight(row_of(p.v, tj, kv) + 8 * lane, in, value[e]);
          }
#pragma unroll
          for (int e = 0; e < kAtOnce; ++e) {
            const float s = form.at(dot16(qr, key[e]), slope2, fabsf(static_cast<float>(i - min(j0 + e, keys - 1))));
            const float dp = dot16(a[k], value[e]);
            if (j0 + e < most) sum = fmaf(fast_exp2(s - lse2), dp, sum);
          }
        }
        if (few) delta = sum;
      }
      if (r + k * kGroups < rows && lane == 0) out[i] = make_float2(lse2, delta);
    }
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

// The same as they are, in fp32, and where: [dv, dk][part][T, Hk, D].
__device__ __forceinline__ void store_sums(uint32_t taddr, float* row, bool store, int col, int D) {
  uint32_t o[32];
  tmem_ld_32x32b_x32(taddr + col, o);
  tmem_ld_wait();
#pragma unroll
  for (int v = 0; v < 8; ++v)
    if (store && col + 4 * v < D) reinterpret_cast<uint4*>(row + col)[v] = make_uint4(o[4 * v], o[4 * v + 1], o[4 * v + 2], o[4 * v + 3]);
}
__device__ __forceinline__ int64_t sums_at(const AttArgs& p, bool is_k, int parts, int part, int64_t token, int kv_head) {
  return (((static_cast<int64_t>(is_k) * parts + part) * p.T + token) * p.Hk + kv_head) * p.D;
}
// dv and dk of the query heads' parts added, in their order.
__global__ void __launch_bounds__(256) att_join_kernel(const AttArgs p, const float* sums, int parts) {
  grid_launch_dependents();
  grid_wait();
  const int vecs = p.D / 8;
  const int64_t n = static_cast<int64_t>(cu_at(p, p.S)) * p.Hk * vecs;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < 2 * n; i += static_cast<int64_t>(gridDim.x) * 256) {
    const bool is_k = i >= n;
    const int64_t row = (is_k ? i - n : i) / vecs;
    const int col = 8 * static_cast<int>((is_k ? i - n : i) % vecs);
    const int64_t token = row / p.Hk;
    const int head = static_cast<int>(row % p.Hk);
    float f[8] = {};
#pragma unroll 4
    for (int g = 0; g < parts; ++g) {
      const float4* at = reinterpret_cast<const float4*>(sums + sums_at(p, is_k, parts, g, token, head) + col);
      const float4 a = at[0], b = at[1];
      f[0] += a.x, f[1] += a.y, f[2] += a.z, f[3] += a.w, f[4] += b.x, f[5] += b.y, f[6] += b.z, f[7] += b.w;
    }
    const float by = is_k ? p.scale : 1.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] *= by;
    const HeadsView& dst = is_k ? p.dk : p.dv;
    __nv_bfloat16* to = static_cast<__nv_bfloat16*>(const_cast<void*>(dst.x)) + token * dst.token_stride + head * dst.head_stride + col;
    *reinterpret_cast<uint4*>(to) = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
  }
}

// ----------------------------------------------------------------- dk, dv ---
// tensor memory: S^T (then P^T), dP^T (then dS^T), dV, dK.  The MMAs run in the order
// dV_t, S_{t+1}, dK_t, dP_{t+1}: P_{t+1} is formed while the last two run, dS_t while the
// first two do.  (A warp for each pair mixes them: all four then end late.)
constexpr int kQ = 3, kO = 2;  // stages of q and of do (whose rows' lse and delta come along)
// An item's own tiles: narrow heads have room for the next one's.
constexpr int own_stages(int boxes) { return boxes == 1 ? 2 : 1; }
enum { A_KVFULL = 0, A_KVEMPTY = 2, A_QFULL = 4, A_QEMPTY = A_QFULL + kQ, A_QFIX = A_QEMPTY + kQ, A_DOFULL = A_QFIX + kQ,
       A_DOEMPTY = A_DOFULL + kO, A_DOFIX = A_DOEMPTY + kO, A_VECFULL = A_DOFIX + kO, A_VECEMPTY = A_VECFULL + kO,
       A_SFULL = A_VECEMPTY + kO, A_PREADY, A_DPFULL, A_DSREADY, A_OFULL, A_OEMPTY, A_DRAIN, A_RING,
       A_COUNT = A_RING + kRingBars };

struct KvItem {
  Seq q;
  int kv_head, part, heads;        // which part of the key head's query heads, how many
  int k0, first, tiles, steps;     // first query tile, query tiles of a head, of all heads
  int end;
};
constexpr int kKvBars = (8 * A_COUNT + 15) / 16 * 16, kKvMisc = 16 + static_cast<int>(sizeof(ItemRing<KvItem>));
constexpr int kv_smem(int boxes) { return (2 * own_stages(boxes) + kQ + kO) * boxes * kBoxBytes + kO * 1024 + kKvBars + kKvMisc; }
__device__ __forceinline__ bool kv_item(const AttArgs& p, int i, int parts, KvItem& it, int& near) {
  const int units = p.Hk * parts, u = i % units;
  it.q = seq_of_slot<128>(p, i / units, near);
  if (it.q.tile < 0) return false;
  it.end = 0;
  it.kv_head = u / parts;
  it.part = u % parts;
  it.heads = p.Hq / p.Hk / parts;
  it.k0 = 128 * it.q.tile;
  it.first = p.causal && it.k0 >= it.q.prefix ? it.q.tile : 0;
  it.tiles = (it.q.n + 127) / 128 - it.first;
  it.steps = it.tiles * it.heads;
  return true;
}
// An item's steps: a query head and the first row of a query tile.
struct KvStep {
  int head, q0, left;
  __device__ __forceinline__ KvStep(const AttArgs& p, const KvItem& it)
      : head(it.kv_head * (p.Hq / p.Hk) + it.part * it.heads), q0(128 * it.first), left(it.tiles) {}
  __device__ __forceinline__ void next(const KvItem& it) {
    q0 += 128;
    if (--left == 0) {
      ++head;
      q0 = 128 * it.first;
      left = it.tiles;
    }
  }
};

template <int kBoxes, int kForm>
__global__ void __launch_bounds__(kThreads, 1)
    att_dkdv_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                    const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do, const AttArgs p,
                    const float2* stats, float* sums, int parts, int ask) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);  // (of 1024 bytes' alignment: there is no room to move up)
  constexpr uint32_t kTileBytes = kBoxes * kBoxBytes;
  constexpr int kOwn = own_stages(kBoxes);
  const uint32_t skv = raw, sq = skv + 2 * kOwn * kTileBytes, sdo = sq + kQ * kTileBytes;
  const uint32_t vec0 = sdo + kO * kTileBytes;  // a stage's [2][128]: -lse, -delta
  float* vec = reinterpret_cast<float*>(smem_raw + (vec0 - raw));
  const uint32_t bar0 = vec0 + kO * 1024;
  uint8_t* misc = smem_raw + (bar0 - raw) + kKvBars;
  ItemRing<KvItem>& ring = *reinterpret_cast<ItemRing<KvItem>*>(misc + 16);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(misc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 4);
  const auto bar = [&](int i) { return bar0 + 8u * i; };
  const RingAt ring_at{bar(A_RING)};
  const int warp = warp_uniform(static_cast<int>(threadIdx.x >> 5)), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < A_RING; ++i) {
      const bool rows = i == A_PREADY || i == A_DSREADY || i == A_OEMPTY || (i >= A_VECEMPTY && i < A_VECEMPTY + kO);
      mbar_init(bar(i), rows ? kRowWarps : 1);
    }
    init_ring(ring_at, kReaders);
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
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  grid_launch_dependents();
  grid_wait();
  const uint32_t tmem = warp_uniform(*tmem_slot);
  const uint32_t t_s = tmem, t_dp = tmem + 128, t_dv = tmem + 256, t_dk = tmem + 384;
  const WaitCtl ctl{abort_flag, p.wait_limit_ns};
  KvItem it;

  if (warp < kRestWarps) {
    regs_dec<kRegsRest>();
    if (warp == kTmaWarp) {
      const bool leader = elect_one();
      Turn kv, q, o;
      bool ok = true;
      for (uint32_t ni = 0; ok && next_item<true>(ring, ring_at, ni, it, ctl, ok);) {
        if (!(ok = mbar_wait_warp(bar(A_KVEMPTY + kv.i), kv.phase ^ 1, ctl))) break;
        if (leader) {
          const uint32_t full = bar(A_KVFULL + kv.i), sk = skv + 2 * kv.i * kTileBytes;
          mbar_arrive_expect_tx(full, 2 * kTileBytes);
          load_tile(sk, &map_k, full, kBoxes, p.k.head_stride ? it.kv_head : 0, it.q.start + it.k0);
          load_tile(sk + kTileBytes, &map_v, full, kBoxes, p.v.head_stride ? it.kv_head : 0, it.q.start + it.k0);
        }
        kv.next(kOwn);
        KvStep at(p, it);
        for (int t = 0; t < it.steps; ++t, at.next(it), q.next(kQ), o.next(kO)) {
          float2 got[4];  // the rows' lse and delta, on their way while the stages are waited for
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = min(at.q0 + lane + 32 * e, it.q.n - 1);
            got[e] = stats[static_cast<int64_t>(at.head) * p.T + it.q.start + r];
          }
          if (!(ok = mbar_wait_warp(bar(A_QEMPTY + q.i), q.phase ^ 1, ctl))) break;
          if (leader) {
            mbar_arrive_expect_tx(bar(A_QFULL + q.i), kTileBytes);
            load_tile(sq + q.i * kTileBytes, &map_q, bar(A_QFULL + q.i), kBoxes, p.q.head_stride ? at.head : 0, it.q.start + at.q0);
          }
          if (!(ok = mbar_wait_warp(bar(A_DOEMPTY + o.i), o.phase ^ 1, ctl))) break;
          if (leader) {
            mbar_arrive_expect_tx(bar(A_DOFULL + o.i), kTileBytes);
            load_tile(sdo + o.i * kTileBytes, &map_do, bar(A_DOFULL + o.i), kBoxes, p.d_o.head_stride ? at.head : 0,
                      it.q.start + at.q0);
          }
          if (!(ok = mbar_wait_warp(bar(A_VECEMPTY + o.i), o.phase ^ 1, ctl))) break;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            vec[o.i * 256 + lane + 32 * e] = -got[e].x;
            vec[o.i * 256 + 128 + lane + 32 * e] = -got[e].y;
          }
          __syncwarp();
          if (leader) mbar_arrive(bar(A_VECFULL + o.i));
          // the sequence's last rows: what follows them up to whole K steps is zeroed
          const int rows = it.q.n - at.q0;
          if (rows < 128 && rows % 16 != 0) {
            if (!(ok = mbar_wait_warp(bar(A_QFULL + q.i), q.phase, ctl) && mbar_wait_warp(bar(A_DOFULL + o.i), o.phase, ctl))) break;
            zero_rows(sq + q.i * kTileBytes, kBoxes, rows, up16(rows));
            zero_rows(sdo + o.i * kTileBytes, kBoxes, rows, up16(rows));
            fence_proxy_async_shared();
            __syncwarp();
            if (leader) {
              mbar_arrive(bar(A_QFIX + q.i));
              mbar_arrive(bar(A_DOFIX + o.i));
            }
          }
        }
        if (ok && leader) mbar_arrive(ring_at.issued());
      }
      if (!ok) let_copies_land();
      __syncwarp();
    } else if (warp == kMmaWarp) {
      const bool leader = elect_one();
      const int steps = (p.D + 15) / 16;
      const uint32_t id_out = idesc_bf16(128, 16 * steps, false, true);
      uint32_t n_o = 0, n = 0, q_fixed = 0, o_fixed = 0;
      Turn kv, q, o;  // of the step whose second products are next
      bool ok = true;
      for (uint32_t ni = 0; ok && next_item<true>(ring, ring_at, ni, it, ctl, ok); ++n_o, kv.next(kOwn)) {
        KvStep at(p, it);
        int rows = min(128, it.q.n - at.q0);  // (a tile of a sequence's last rows is shorter)
        const uint32_t sk = skv + 2 * kv.i * kTileBytes, sv = sk + kTileBytes;
        const auto scores = [&](const Turn& qs) {
          mma_rows(leader, t_s, sk, sq + qs.i * kTileBytes, idesc_bf16(128, up16(rows), false, false), steps);
          umma_commit_by(leader, bar(A_SFULL));
        };
        const auto slopes = [&](const Turn& os) {
          mma_rows(leader, t_dp, sv, sdo + os.i * kTileBytes, idesc_bf16(128, up16(rows), false, false), steps);
          umma_commit_by(leader, bar(A_DPFULL));
        };
        const Phase begin[3] = {{bar(A_KVFULL + kv.i), kv.phase}, {bar(A_QFULL + q.i), q.phase}, {bar(A_DOFULL + o.i), o.phase}};
        if (!(ok = mbar_wait_warp(begin, ctl))) break;
        tc_fence_after();
        scores(q);
        slopes(o);
        if (!(ok = mbar_wait_warp(bar(A_OEMPTY), (n_o & 1) ^ 1, ctl))) break;
        for (int t = 0; t < it.steps; ++t, ++n) {
          const bool more = t + 1 < it.steps;
          Turn q2 = q, o2 = o;
          q2.next(kQ);
          o2.next(kO);
          const int ks = up16(rows) / 16;
          if (rows % 16 != 0) {
            const Phase fix[2] = {{bar(A_DOFIX + o.i), o_fixed >> o.i & 1}, {bar(A_QFIX + q.i), q_fixed >> q.i & 1}};
            if (!(ok = mbar_wait_warp(fix, ctl))) break;
            o_fixed ^= 1u << o.i;
            q_fixed ^= 1u << q.i;
          }
          at.next(it);
          rows = min(128, it.q.n - at.q0);
          // (one wait for what two products need: 100 cycles where nothing is waited for)
          const Phase with_p[2] = {{bar(A_PREADY), n & 1}, {bar(A_QFULL + q2.i), q2.phase}};
          if (!(ok = more ? mbar_wait_warp(with_p, ctl) : mbar_wait_warp(with_p[0].bar, with_p[0].parity, ctl))) break;
          tc_fence_after();
          mma_cols<2>(leader, t_dv, t_s, sdo + o.i * kTileBytes, id_out, ks, t > 0);
          umma_commit_by(leader, bar(A_DOEMPTY + o.i));
          if (more) scores(q2);
          const Phase with_ds[2] = {{bar(A_DSREADY), n & 1}, {bar(A_DOFULL + o2.i), o2.phase}};
          if (!(ok = more ? mbar_wait_warp(with_ds, ctl) : mbar_wait_warp(with_ds[0].bar, with_ds[0].parity, ctl))) break;
          tc_fence_after();
          mma_cols<2>(leader, t_dk, t_dp, sq + q.i * kTileBytes, id_out, ks, t > 0);
          umma_commit_by(leader, bar(A_QEMPTY + q.i));
          if (more) slopes(o2);
          q = q2;
          o = o2;
        }
        if (!ok) break;
        umma_commit_by(leader, bar(A_OFULL));
        umma_commit_by(leader, bar(A_KVEMPTY + kv.i));
      }
      drain_mmas(bar(A_DRAIN), leader, p.wait_limit_ns);
    } else if (warp == kItemWarp) {
      int near = 0;
      hand_out(ring, ring_at, ask, ctl, [&](int i, KvItem& item) { return kv_item(p, i, parts, item, near); },
               [&](int i) {
                 const int64_t shares = min(static_cast<int64_t>(gridDim.x), kParts);
                 if (i >= shares) return;
                 zero_behind(p, p.dk, p.Hk, i, shares);
                 zero_behind(p, p.dv, p.Hk, i, shares);
               });
    }
  } else {
    regs_inc<kRegsRows>();
    const int part = (warp - kRestWarps) >> 2;  // of the tile's query columns
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t ts = t_s + lanes + kCols * part, td = t_dp + lanes + kCols * part;
    const ScoreForm form(p);
    uint32_t n_q = 0, n_o = 0;
    Turn o;
    bool ok = true;
    for (uint32_t ni = 0; ok && next_item<false>(ring, ring_at, ni, it, ctl, ok);) {
      const int key = it.k0 + (warp & 3) * 32 + lane;
      const bool alone = first_row_alone(p, it.q);
      KvStep step(p, it);
      for (int t = 0; t < it.steps; ++t, ++n_q, step.next(it), o.next(kO)) {
        // columns [lo, hi) of this part see the key
        const int at = step.q0 + kCols * part;
        const int lo = key >= it.q.n ? kCols : p.causal && key >= it.q.prefix ? key - at : 0, hi = it.q.n - at;
        const bool masked = __any_sync(0xffffffffu, lo > 0 || hi < kCols);
        const float slope2 = kForm != FORM_PLAIN && p.slopes ? p.slopes[step.head] * kAttLog2e : 0.f;
        [[maybe_unused]] const float far = static_cast<float>(key - at);
        const float* stage = vec + o.i * 256 + kCols * part;
        const Phase of[2] = {{bar(A_VECFULL + o.i), o.phase}, {bar(A_SFULL), n_q & 1}};
        if (!(ok = mbar_wait_warp(of, ctl))) break;
        tc_fence_after();
        // (not where all rows or all columns are behind the sequence: nothing reads them)
        const bool some = it.k0 + (warp & 3) * 32 < it.q.n && hi > 0;
        uint64_t pr[kCols / 2];  // pairs of columns: p, times the cap's derivative
        uint32_t a[32];
        [[maybe_unused]] uint64_t bend[kForm == FORM_CAP ? 16 : 1];
        if (some) {
          tmem_ld_32x32b_x32(ts, a);
          tmem_ld_wait();
          if constexpr (kForm != FORM_PLAIN) {
            if (!masked && (kForm == FORM_CAP ? all_small(form, largest(a)) : one_side(far, kCols)))
              form_scores<kForm, kForm == FORM_CAP, true>(form, a, slope2, far, bend);
            else
              form_scores<kForm, kForm == FORM_CAP, false>(form, a, slope2, far, bend);
          }
        }
        // (two copies of the loops: as one, the masks' instructions are issued for every tile)
        const auto weights = [&](auto is_masked) {
          uint32_t w[16];
          const ulonglong2* lse = reinterpret_cast<const ulonglong2*>(stage);
          constexpr bool kFormed = kForm != FORM_PLAIN;
          const uint64_t mul = pair(kFormed ? 1.f : form.scale2, kFormed ? 1.f : form.scale2);
#pragma unroll
          for (int c = 0; c < kCols / 2; ++c) {
            const int k = 2 * c;
            const ulonglong2 l2 = lse[c / 2];
            const uint64_t l = c & 1 ? l2.y : l2.x, s2 = pair(__uint_as_float(a[k]), __uint_as_float(a[k + 1]));
            float x, y;
            unpair(kFormed ? add_pair(s2, l) : fma_pair(s2, mul, l), x, y);
            x = fast_exp2(x);
            y = fast_exp2(y);
            if constexpr (decltype(is_masked)::value) {
              x = k >= lo && k < hi ? x : 0.f;
              y = k + 1 >= lo && k + 1 < hi ? y : 0.f;
            }
            pr[c] = pair(x, y);
            if constexpr (kForm == FORM_CAP) pr[c] = mul_pair(pr[c], bend[c]);
            w[c] = pack_bf16x2(x, y);
          }
          tmem_st_32x32b_x16(ts, w);
        };
        if (some && masked)
          weights(std::true_type{});
        else if (some)
          weights(std::false_type{});
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(A_PREADY));
        if (!(ok = mbar_wait_warp(bar(A_DPFULL), n_q & 1, ctl))) break;
        tc_fence_after();
        const auto slopes = [&](auto is_masked) {
          uint32_t a[32], w[16];
          tmem_ld_32x32b_x32(td, a);
          tmem_ld_wait();
          const ulonglong2* del = reinterpret_cast<const ulonglong2*>(stage + 128);
#pragma unroll
          for (int c = 0; c < kCols / 2; ++c) {
            const int k = 2 * c;
            const ulonglong2 d2 = del[c / 2];
            float x, y;
            unpair(mul_pair(pr[c], add_pair(pair(__uint_as_float(a[k]), __uint_as_float(a[k + 1])), c & 1 ? d2.y : d2.x)), x, y);
            if constexpr (decltype(is_masked)::value) {
              x = k >= lo && k < hi && !(alone && at + k == 0) ? x : 0.f;
              y = k + 1 >= lo && k + 1 < hi ? y : 0.f;
            }
            w[c] = pack_bf16x2(x, y);
          }
          tmem_st_32x32b_x16(td, w);
        };
        if (some && masked)
          slopes(std::true_type{});
        else if (some)
          slopes(std::false_type{});
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bar(A_DSREADY));
          mbar_arrive(bar(A_VECEMPTY + o.i));
        }
      }
      if (!ok) break;
      // dv by the first eight warps, dk by the others
      if (!(ok = mbar_wait_warp(bar(A_OFULL), n_o++ & 1, ctl))) break;
      tc_fence_after();
      const bool is_k = part >= 2;
      const HeadsView& dst = is_k ? p.dk : p.dv;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(const_cast<void*>(dst.x)) +
                           static_cast<int64_t>(it.q.start + key) * dst.token_stride + it.kv_head * dst.head_stride;
      for (int c = 32 * (part & 1); c < p.D; c += 64) {
        const uint32_t from = (is_k ? t_dk : t_dv) + lanes;
        if (parts == 1)
          store_cols(from, out, key < it.q.n, c, p.D, is_k ? p.scale : 1.f);
        else
          store_sums(from, sums + sums_at(p, is_k, parts, it.part, it.q.start + key, it.kv_head), key < it.q.n, c, p.D);
      }
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
// tensor memory: S, two of dP (then dS), dQ.  The MMAs run in the order S_{j+1}, dP_{j+1},
// dQ_j: the products of a tile do not wait for the rows of the one before.  So a warp may
// be done with a tile that another has not begun: barriers of dP and dS by parity.
constexpr int kK = 3, kV = 2;  // stages of key and value tiles
enum { C_QFULL = 0, C_QEMPTY = 2, C_KFULL = 4, C_KEMPTY = C_KFULL + kK, C_KFIX = C_KEMPTY + kK, C_VFULL = C_KFIX + kK,
       C_VEMPTY = C_VFULL + kV, C_SFULL = C_VEMPTY + kV, C_SEMPTY, C_DPFULL, C_DSREADY = C_DPFULL + 2, C_OFULL = C_DSREADY + 2, C_OEMPTY,
       C_DRAIN, C_RING, C_COUNT = C_RING + kRingBars };

struct QItem {
  Seq q;
  int head, q0, seen, tiles;
  int end;
};
constexpr int kQBars = (8 * C_COUNT + 15) / 16 * 16, kQMisc = 16 + static_cast<int>(sizeof(ItemRing<QItem>));
constexpr int dq_smem(int boxes) { return 1024 + (2 * own_stages(boxes) + kK + kV) * boxes * kBoxBytes + kQBars + kQMisc; }
__device__ __forceinline__ bool q_item(const AttArgs& p, int i, QItem& it, int& near) {
  it.q = seq_of_slot<128>(p, i / p.Hq, near);
  if (it.q.tile < 0) return false;
  it.end = 0;
  it.head = i % p.Hq;
  // the longest rows first
  it.q0 = 128 * (p.causal ? (it.q.n + 127) / 128 - 1 - it.q.tile : it.q.tile);
  it.seen = keys_seen(p, it.q, min(it.q0 + 128, it.q.n) - 1);
  it.tiles = (it.seen + 127) / 128;
  return true;
}

template <int kBoxes, int kForm>
__global__ void __launch_bounds__(kThreads, 1)
    att_dq_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                  const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do, const AttArgs p,
                  const float2* stats, int ask) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  constexpr uint32_t kTileBytes = kBoxes * kBoxBytes;
  constexpr int kOwn = own_stages(kBoxes);
  const uint32_t sqdo = base, sk = sqdo + 2 * kOwn * kTileBytes, sv = sk + kK * kTileBytes;
  const uint32_t bar0 = sv + kV * kTileBytes;
  uint8_t* misc = smem_raw + (bar0 - raw) + kQBars;
  ItemRing<QItem>& ring = *reinterpret_cast<ItemRing<QItem>*>(misc + 16);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(misc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 4);
  const auto bar = [&](int i) { return bar0 + 8u * i; };
  const RingAt ring_at{bar(C_RING)};
  const int warp = warp_uniform(static_cast<int>(threadIdx.x >> 5)), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < C_RING; ++i) mbar_init(bar(i), i == C_SEMPTY || i == C_DSREADY || i == C_DSREADY + 1 || i == C_OEMPTY ? kRowWarps : 1);
    init_ring(ring_at, kReaders);
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
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  grid_launch_dependents();
  grid_wait();
  const uint32_t tmem = warp_uniform(*tmem_slot);
  const auto t_dp = [&](uint32_t n) { return tmem + 128u + 128u * (n & 1); };
  const uint32_t t_s = tmem, t_dq = tmem + 384;
  const WaitCtl ctl{abort_flag, p.wait_limit_ns};
  QItem it;

  if (warp < kRestWarps) {
    regs_dec<kRegsRest>();
    if (warp == kTmaWarp) {
      const bool leader = elect_one();
      Turn q, k, v;
      bool ok = true;
      for (uint32_t ni = 0; ok && next_item<true>(ring, ring_at, ni, it, ctl, ok);) {
        const int kv = it.head / (p.Hq / p.Hk);
        if (!(ok = mbar_wait_warp(bar(C_QEMPTY + q.i), q.phase ^ 1, ctl))) break;
        if (leader) {
          const uint32_t full = bar(C_QFULL + q.i), sq = sqdo + 2 * q.i * kTileBytes;
          mbar_arrive_expect_tx(full, 2 * kTileBytes);
          load_tile(sq, &map_q, full, kBoxes, p.q.head_stride ? it.head : 0, it.q.start + it.q0);
          load_tile(sq + kTileBytes, &map_do, full, kBoxes, p.d_o.head_stride ? it.head : 0, it.q.start + it.q0);
        }
        q.next(kOwn);
        for (int j = 0; j < it.tiles; ++j, k.next(kK), v.next(kV)) {
          if (!(ok = mbar_wait_warp(bar(C_KEMPTY + k.i), k.phase ^ 1, ctl))) break;
          if (leader) {
            mbar_arrive_expect_tx(bar(C_KFULL + k.i), kTileBytes);
            load_tile(sk + k.i * kTileBytes, &map_k, bar(C_KFULL + k.i), kBoxes, p.k.head_stride ? kv : 0, it.q.start + 128 * j);
          }
          if (!(ok = mbar_wait_warp(bar(C_VEMPTY + v.i), v.phase ^ 1, ctl))) break;
          if (leader) {
            mbar_arrive_expect_tx(bar(C_VFULL + v.i), kTileBytes);
            load_tile(sv + v.i * kTileBytes, &map_v, bar(C_VFULL + v.i), kBoxes, p.v.head_stride ? kv : 0, it.q.start + 128 * j);
          }
          const int rows = it.seen - 128 * j;
          if (rows < 128 && rows % 16 != 0) {
            if (!(ok = mbar_wait_warp(bar(C_KFULL + k.i), k.phase, ctl))) break;
            zero_rows(sk + k.i * kTileBytes, kBoxes, rows, up16(rows));
            fence_proxy_async_shared();
            __syncwarp();
            if (leader) mbar_arrive(bar(C_KFIX + k.i));
          }
        }
        if (ok && leader) mbar_arrive(ring_at.issued());
      }
      if (!ok) let_copies_land();
      __syncwarp();
    } else if (warp == kMmaWarp) {
      const bool leader = elect_one();
      const int steps = (p.D + 15) / 16;
      const uint32_t id_out = idesc_bf16(128, 16 * steps, false, true);
      uint32_t n_o = 0, n = 0, fixed = 0;  // items, tiles
      Turn q, k, v;                        // k, v: of the tile whose S and dP are next
      bool ok = true;
      for (uint32_t ni = 0; ok && next_item<true>(ring, ring_at, ni, it, ctl, ok); ++n_o, q.next(kOwn)) {
        const auto cols_of = [&](int j) { return up16(min(128, it.seen - 128 * j)); };
        const uint32_t sq = sqdo + 2 * q.i * kTileBytes, sdo = sq + kTileBytes;
        const Phase begin[2] = {{bar(C_QFULL + q.i), q.phase}, {bar(C_OEMPTY), (n_o & 1) ^ 1}};
        if (!(ok = mbar_wait_warp(begin, ctl))) break;
        int last_k = 0;  // the stage of the tile before
        for (int j = 0; j <= it.tiles; ++j) {
          const int stage = k.i;
          if (j < it.tiles) {
            const Phase of[3] = {{bar(C_SEMPTY), ((n + j) & 1) ^ 1}, {bar(C_KFULL + k.i), k.phase}, {bar(C_VFULL + v.i), v.phase}};
            if (!(ok = mbar_wait_warp(of, ctl))) break;
            tc_fence_after();
            const uint32_t id = idesc_bf16(128, cols_of(j), false, false);
            mma_rows(leader, t_s, sq, sk + k.i * kTileBytes, id, steps);
            umma_commit_by(leader, bar(C_SFULL));
            // (into the accumulator that dQ of the last tile but one has read)
            mma_rows(leader, t_dp(n + j), sdo, sv + v.i * kTileBytes, id, steps);
            umma_commit_by(leader, bar(C_DPFULL + ((n + j) & 1)));
            umma_commit_by(leader, bar(C_VEMPTY + v.i));
            k.next(kK);
            v.next(kV);
          }
          if (j > 0) {
            const int rows = it.seen - 128 * (j - 1);
            if (rows < 128 && rows % 16 != 0) {
              if (!(ok = mbar_wait_warp(bar(C_KFIX + last_k), fixed >> last_k & 1, ctl))) break;
              fixed ^= 1u << last_k;
            }
            const uint32_t before = n + j - 1;
            if (!(ok = mbar_wait_warp(bar(C_DSREADY + (before & 1)), before >> 1 & 1, ctl))) break;
            tc_fence_after();
            mma_cols<2>(leader, t_dq, t_dp(before), sk + last_k * kTileBytes, id_out, cols_of(j - 1) / 16, j > 1);
            umma_commit_by(leader, bar(C_KEMPTY + last_k));
          }
          last_k = stage;
        }
        if (!ok) break;
        n += it.tiles;
        umma_commit_by(leader, bar(C_OFULL));
        umma_commit_by(leader, bar(C_QEMPTY + q.i));
      }
      drain_mmas(bar(C_DRAIN), leader, p.wait_limit_ns);
    } else if (warp == kItemWarp) {
      int near = 0;
      hand_out(ring, ring_at, ask, ctl, [&](int i, QItem& item) { return q_item(p, i, item, near); },
               [&](int i) {
                 if (i == 0) check_offsets(p);
                 const int64_t parts = min(static_cast<int64_t>(gridDim.x), kParts);
                 if (i < parts) zero_behind(p, p.dq, p.Hq, i, parts);
               });
    }
  } else {
    regs_inc<kRegsRows>();
    const int part = (warp - kRestWarps) >> 2;  // of the tile's key columns
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const ScoreForm form(p);
    uint32_t n_kv = 0, n_o = 0;
    bool ok = true;
    for (uint32_t ni = 0; ok && next_item<false>(ring, ring_at, ni, it, ctl, ok);) {
      const int pos = it.q0 + (warp & 3) * 32 + lane, real = min(pos, it.q.n - 1);
      const float2 st = stats[static_cast<int64_t>(it.head) * p.T + it.q.start + real];
      const int lim = keys_seen(p, it.q, real);
      const bool alone = pos == 0 && first_row_alone(p, it.q);
      const float slope2 = kForm != FORM_PLAIN && p.slopes ? p.slopes[it.head] * kAttLog2e : 0.f;
      for (int j = 0; j < it.tiles; ++j, ++n_kv) {
        const int at = 128 * j + kCols * part, here = lim - at;
        const bool masked = __any_sync(0xffffffffu, here < kCols);
        // (not where all rows or all columns are behind the sequence: nothing reads them)
        const bool some = it.q0 + (warp & 3) * 32 < it.q.n && at < it.seen;
        [[maybe_unused]] const float far = static_cast<float>(pos - at);
        if (!(ok = mbar_wait_warp(bar(C_SFULL), n_kv & 1, ctl))) break;
        tc_fence_after();
        uint64_t pr[kCols / 2];
        if (!some) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(C_SEMPTY));
        } else {
          uint32_t a[32];
          tmem_ld_32x32b_x32(t_s + lanes + kCols * part, a);
          tmem_ld_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(C_SEMPTY));
          [[maybe_unused]] uint64_t bend[kForm == FORM_CAP ? 16 : 1];
          if constexpr (kForm != FORM_PLAIN) {
            if (!masked && (kForm == FORM_CAP ? all_small(form, pos < it.q.n ? largest(a) : 0.f) : one_side(far, kCols)))
              form_scores<kForm, kForm == FORM_CAP, true>(form, a, slope2, far, bend);
            else
              form_scores<kForm, kForm == FORM_CAP, false>(form, a, slope2, far, bend);
          }
#pragma unroll
          for (int c = 0; c < kCols / 2; ++c) {
            const uint64_t s2 = pair(__uint_as_float(a[2 * c]), __uint_as_float(a[2 * c + 1])), l = pair(-st.x, -st.x);
            float x, y;
            unpair(kForm != FORM_PLAIN ? add_pair(s2, l) : fma_pair(s2, pair(form.scale2, form.scale2), l), x, y);
            pr[c] = pair(fast_exp2(x), fast_exp2(y));
            if constexpr (kForm == FORM_CAP) pr[c] = mul_pair(pr[c], bend[c]);  // (p itself is not needed here)
          }
        }
        if (!(ok = mbar_wait_warp(bar(C_DPFULL + (n_kv & 1)), n_kv >> 1 & 1, ctl))) break;
        tc_fence_after();
        // (two copies of the loop: as one, the masks' instructions are issued for every tile)
        const auto slopes = [&](auto is_masked) {
          uint32_t a[32], w[16];
          const uint32_t td = t_dp(n_kv) + lanes + kCols * part;
          tmem_ld_32x32b_x32(td, a);
          tmem_ld_wait();
#pragma unroll
          for (int c = 0; c < kCols / 2; ++c) {
            const int k = 2 * c;
            float x, y;
            unpair(mul_pair(pr[c], add_pair(pair(__uint_as_float(a[k]), __uint_as_float(a[k + 1])), pair(-st.y, -st.y))), x, y);
            if constexpr (decltype(is_masked)::value) {
              x = k < here && !alone ? x : 0.f;
              y = k + 1 < here && !alone ? y : 0.f;
            }
            w[c] = pack_bf16x2(x, y);
          }
          tmem_st_32x32b_x16(td, w);
        };
        if (some && masked)
          slopes(std::true_type{});
        else if (some)
          slopes(std::false_type{});
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C_DSREADY + (n_kv & 1)));
      }
      if (!ok) break;
      if (!(ok = mbar_wait_warp(bar(C_OFULL), n_o++ & 1, ctl))) break;
      tc_fence_after();
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(const_cast<void*>(p.dq.x)) +
                           static_cast<int64_t>(it.q.start + pos) * p.dq.token_stride + it.head * p.dq.head_stride;
      if (32 * part < p.D) store_cols(t_dq + lanes, out, pos < it.q.n, 32 * part, p.D, p.scale);
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

size_t stats_bytes(int64_t T, int64_t Hq) { return align_up(8ull * T * Hq, kWsAlign); }
// Parts that the query heads of a key head are cut into for dk and dv: all of them where
// the key tiles do not fill the SMs (152), as the first tiles of a causal sequence take
// longest.  (5003 tokens of 15 + 3 heads: 215 us in one part, 112 in five with their join.
// Below four tiles a launch more costs what it saves.)
int head_parts(int64_t T, int64_t Hq, int64_t Hk) {
  const int64_t tiles = ceil_div(T, 128);
  return tiles >= 4 && tiles * Hk <= 152 ? static_cast<int>(Hq / Hk) : 1;
}

// Launches a kernel that waits for the one ahead by itself, once it has set itself up: it
// starts on SMs that the one ahead leaves idle at its end.
template <class... K, class... A>
void launch_after(const Ctx& c, void (*kernel)(K...), int64_t blocks, int threads, size_t smem, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(blocks));
  cfg.blockDim = dim3(static_cast<unsigned>(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = c.stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cudaLaunchKernelEx(&cfg, kernel, static_cast<K>(args)...);
}

template <int kBoxes, int kForm>
olive_status run_bwd(const Ctx& c, const AttArgs& a) {
  CUtensorMap mq, mk, mv, mdo;
  if (!encode_heads(&mq, a.q, a.T, a.Hq, a.D) || !encode_heads(&mk, a.k, a.T, a.Hk, a.D) ||
      !encode_heads(&mv, a.v, a.T, a.Hk, a.D) || !encode_heads(&mdo, a.d_o, a.T, a.Hq, a.D))
    return OLIVE_ERR_CUDA;
  static std::atomic<int> done_kv[kMaxDevices], done_q[kMaxDevices];
  const auto dkdv = att_dkdv_kernel<kBoxes, kForm>;
  const auto dq = att_dq_kernel<kBoxes, kForm>;
  constexpr int kSmemKv = kv_smem(kBoxes), kSmemQ = dq_smem(kBoxes);
  static_assert(kSmemKv <= 227 * 1024 && kSmemQ <= 227 * 1024, "shared memory");
  if (!set_smem_once(reinterpret_cast<const void*>(dkdv), kSmemKv, c.device, done_kv) ||
      !set_smem_once(reinterpret_cast<const void*>(dq), kSmemQ, c.device, done_q))
    return OLIVE_ERR_CUDA;
  float2* stats = static_cast<float2*>(a.ws);
  const int64_t slots = att_slots(a.T, a.S, 128);
  const auto ask = [&](int64_t items) { return when_to_ask(items, c.num_sms, a.T, a.S); };
  att_delta_kernel<<<static_cast<unsigned>(slots * a.Hq), kDeltaThreads, 0, c.stream>>>(a, stats);
  const int parts = head_parts(a.T, a.Hq, a.Hk);
  float* sums = reinterpret_cast<float*>(static_cast<char*>(a.ws) + stats_bytes(a.T, a.Hq));
  launch_after(c, dkdv, slots * a.Hk * parts, kThreads, kSmemKv, mq, mk, mv, mdo, a, stats, sums, parts, ask(slots * a.Hk * parts));
  if (parts > 1) {
    const int64_t blocks = ceil_div(2ll * a.T * a.Hk * (a.D / 8), 256);
    launch_after(c, att_join_kernel, std::min<int64_t>(blocks, 16 * c.num_sms), 256, 0, a, sums, parts);
  }
  launch_after(c, dq, slots * a.Hq, kThreads, kSmemQ, mq, mk, mv, mdo, a, stats, ask(slots * a.Hq));
  return cudaGetLastError() == cudaSuccess ? OLIVE_OK : OLIVE_ERR_CUDA;
}

template <int kBoxes>
olive_status by_form(const Ctx& c, const AttArgs& a) {
  if (a.cap > 0.f) return run_bwd<kBoxes, FORM_CAP>(c, a);
  return a.slopes ? run_bwd<kBoxes, FORM_BIAS>(c, a) : run_bwd<kBoxes, FORM_PLAIN>(c, a);
}

}  // namespace

size_t att_bwd_ws_bytes(int64_t T, int64_t Hq, int64_t Hk, int64_t D) {
  const int parts = head_parts(T, Hq, Hk);
  return stats_bytes(T, Hq) + (parts > 1 ? align_up(8ull * parts * T * Hk * D, kWsAlign) : 0);
}

olive_status launch_att_bwd(const Ctx& c, const AttArgs& a) {
  return a.D <= 64 ? by_form<1>(c, a) : by_form<2>(c, a);
}

}  // namespace olive
