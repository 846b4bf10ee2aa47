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
// 8 sequences of 4096, 32 + 8 heads of 128, causal: 88, 1235 and 1130 us; the seven products
// run at 1.55 PFLOP/s (tensor pipe active 74 and 62 % of a shorter launch's cycles), near what
// the power cap leaves.  200 sequences of some 41 tokens, 16 + 16 heads of 64: 9, 95 and 59
// us (with what each waits for the one ahead), an item's chain of waits.  Each launch starts
// under the one ahead (225 us forward and backward at that step, 236 without).
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
// They are among the first so many of a sequence.  (Up to 128 keys: the error of short
// sequences' dq and dk 2.6e-3 -> 2.4e-3 of their norm, this launch 9 -> 49 us.)
constexpr int kFewKeys = 16;
constexpr int kDeltaThreads = 128;

__device__ __forceinline__ const __nv_bfloat16* row_of(const HeadsView& x, int64_t t, int h) {
  return static_cast<const __nv_bfloat16*>(x.x) + t * x.token_stride + h * x.head_stride;
}
// s + <a, b>, even and odd entries apart.
__device__ __forceinline__ uint64_t dot8(const uint4& a, const uint4& b, uint64_t s) {
  const auto two = [](uint32_t w) { return pair(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); };
  s = fma_pair(two(a.x), two(b.x), s);
  s = fma_pair(two(a.y), two(b.y), s);
  s = fma_pair(two(a.z), two(b.z), s);
  return fma_pair(two(a.w), two(b.w), s);
}
// 16 x 8 += 16 x 16 times 16 x 8 of a warp's registers.
__device__ __forceinline__ void mma_16x8(float (&d)[4], const uint32_t (&a)[4], const uint32_t (&b)[2]) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
// A warp: stats of a sequence's first 16 rows that see up to 16 keys, for one head: two
// products of 16 x 16, too small for tensor memory.  (By dot products of 16 lanes the 200
// sequences' launch took 29 us, of which 18 for these.)
__device__ __forceinline__ void few_keys(const AttArgs& p, float2* stats, int s, int head) {
  const int lane = threadIdx.x & 31;
  Seq q;
  q.start = cu_at(p, s);
  q.n = max(q.start, cu_at(p, s + 1)) - q.start;
  q.prefix = prefix_of(p, s, q);
  if (q.n == 0 || keys_seen(p, q, 0) > kFewKeys) return;
  const int kv = head / (p.Hq / p.Hk), r = lane / 4, last = q.n - 1;
  const __nv_bfloat16 *q0 = row_of(p.q, q.start + min(r, last), head), *q1 = row_of(p.q, q.start + min(r + 8, last), head);
  const __nv_bfloat16 *d0 = row_of(p.d_o, q.start + min(r, last), head), *d1 = row_of(p.d_o, q.start + min(r + 8, last), head);
  const __nv_bfloat16 *k0 = row_of(p.k, q.start + min(r, last), kv), *k1 = row_of(p.k, q.start + min(r + 8, last), kv);
  const __nv_bfloat16 *v0 = row_of(p.v, q.start + min(r, last), kv), *v1 = row_of(p.v, q.start + min(r + 8, last), kv);
  float z[2][4] = {}, dp[2][4] = {};
#pragma unroll 4
  for (int c = 2 * (lane % 4); c < p.D; c += 16) {  // (D is a multiple of 8: only the second half may be behind it)
    const bool both = c + 8 < p.D;
    const auto low = [&](const __nv_bfloat16* x) { return *reinterpret_cast<const uint32_t*>(x + c); };
    const auto high = [&](const __nv_bfloat16* x) { return both ? *reinterpret_cast<const uint32_t*>(x + c + 8) : 0u; };
    const uint32_t aq[4] = {low(q0), low(q1), high(q0), high(q1)}, ad[4] = {low(d0), low(d1), high(d0), high(d1)};
    const uint32_t bk[2][2] = {{low(k0), high(k0)}, {low(k1), high(k1)}}, bv[2][2] = {{low(v0), high(v0)}, {low(v1), high(v1)}};
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      mma_16x8(z[t], aq, bk[t]);
      mma_16x8(dp[t], ad, bv[t]);
    }
  }
  const ScoreForm form(p);
  const float slope2 = p.slopes ? p.slopes[head] * kAttLog2e : 0.f;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = r + 8 * h, keys = i < q.n ? keys_seen(p, q, i) : 0;
    const bool few = keys > 0 && keys <= kFewKeys;
    const int64_t at = static_cast<int64_t>(head) * p.T + q.start + i;
    const float lse2 = few ? p.lse[at] * kAttLog2e : 0.f;
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int t = e / 2, x = e % 2, j = 8 * t + 2 * (lane % 4) + x;
      const float w = fast_exp2(form.at(z[t][2 * h + x], slope2, fabsf(static_cast<float>(i - j))) - lse2);
      if (few && j < keys) sum = fmaf(w, dp[t][2 * h + x], sum);
    }
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    if (few && lane % 4 == 0) stats[at] = make_float2(lse2, sum);
  }
}
// The last sequence that begins at or before token t (a warp; the first where none does).
__device__ __forceinline__ int seq_of_token(const AttArgs& p, int t) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = p.S;
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32, s = lo + step * lane;
    const uint32_t before = __ballot_sync(0xffffffffu, s < hi && cu_at(p, s) <= t);
    lo += step * (before ? 31 - __clz(before) : 0);
    hi = min(hi, lo + step);
  }
  return lo;
}
// stats: [Hq, T] of (lse in base 2, delta).  The first blocks: few_keys, a warp a sequence
// and head.  The others: L = 8 or 16 lanes work on four tokens of a head, whose rows are on
// their way while the sequence is looked up.  Bound by memory: 32768 tokens of 32 heads of
// 128, 537 MB, 88 us (6.1 TB/s; 107 by tiles of 128 rows of a head).
template <int L>
__global__ void __launch_bounds__(kDeltaThreads, 8) att_delta_kernel(const AttArgs p, float2* stats, int64_t few_blocks) {
  constexpr int kGroups = kDeltaThreads / L, kAtOnce = 4;
  grid_launch_dependents();
  if (blockIdx.x < few_blocks) {
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * (kDeltaThreads / 32) + threadIdx.x / 32;
    const int s = static_cast<int>(unit / p.Hq);
    if (s < p.S) few_keys(p, stats, s, static_cast<int>(unit % p.Hq));
    return;
  }
  const int lane = threadIdx.x % L;
  const bool in = 8 * lane < p.D;
  const int64_t units = (static_cast<int64_t>(p.T) + kAtOnce - 1) / kAtOnce * p.Hq;
  const int64_t first = (blockIdx.x - few_blocks) * kGroups + threadIdx.x / 32 * (32 / L);  // the warp's
  for (int64_t u0 = first; u0 < units; u0 += (gridDim.x - few_blocks) * kGroups) {
    const int64_t unit = min(u0 + (threadIdx.x % 32) / L, units - 1);  // (the last one more than once, to the same bits)
    const int quad = unit >> 32 ? static_cast<int>(unit / p.Hq) : static_cast<int>(static_cast<uint32_t>(unit) / static_cast<uint32_t>(p.Hq));
    const int head = static_cast<int>(unit - static_cast<int64_t>(quad) * p.Hq), t0 = quad * kAtOnce;
    const int64_t at = static_cast<int64_t>(head) * p.T;
    uint4 a[kAtOnce] = {}, b[kAtOnce] = {};
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int t = min(t0 + k, p.T - 1);
      if (in) a[k] = reinterpret_cast<const uint4*>(row_of(p.d_o, t, head))[lane];
      if (in) b[k] = reinterpret_cast<const uint4*>(row_of(p.o, t, head))[lane];
    }
    // lane k of a group writes token k's
    const int t = t0 + lane;
    const bool mine = lane < kAtOnce && t < p.T;
    const float lse2 = mine ? p.lse[at + t] * kAttLog2e : 0.f;
    int s = seq_of_token(p, __shfl_sync(0xffffffffu, t0, 0));
    // (mostly that sequence or the next; with any number of empty ones between: one after the
    // other, 4096 of them took 290 us)
    if (mine) {
      const auto begun = [&](int later) { return s + later < p.S && cu_at(p, s + later) <= t; };
      int step = 1;
      for (; begun(step); step *= 2) s += step;
      while ((step /= 2) > 0)
        if (begun(step)) s += step;
    }
    Seq q;
    q.start = cu_at(p, s);
    q.n = max(q.start, cu_at(p, s + 1)) - q.start;
    q.prefix = prefix_of(p, s, q);
    const int i = t - q.start;
    const bool live = mine && i >= 0 && i < q.n && keys_seen(p, q, i) > kFewKeys;
    __syncwarp();
    float delta = 0.f;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      float x, y;
      unpair(dot8(a[k], b[k], 0), x, y);
      x += y;
#pragma unroll
      for (int o = L / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
      if (lane == k) delta = x;
    }
    if (live) stats[at + t] = make_float2(lse2, delta);
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
  int kv_head, part, head;         // which part of the key head's query heads, the first of them
  int k0, first, tiles, steps;     // first query tile, query tiles of a head, of all heads
  int end;
  __device__ __forceinline__ int length() const { return steps; }
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
  const int per = p.Hq / p.Hk, each = (per + parts - 1) / parts;  // (the last part may be smaller)
  it.head = it.kv_head * per + it.part * each;
  it.k0 = 128 * it.q.tile;
  it.first = p.causal && it.k0 >= it.q.prefix ? it.q.tile : 0;
  it.tiles = (it.q.n + 127) / 128 - it.first;
  it.steps = it.tiles * min(each, per - it.part * each);
  return true;
}
// An item's steps: a query head and the first row of a query tile.
struct KvStep {
  int head, q0, left;
  __device__ __forceinline__ explicit KvStep(const KvItem& it) : head(it.head), q0(128 * it.first), left(it.tiles) {}
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
        KvStep at(it);
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
        KvStep at(it);
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
      KvStep step(it);
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
        [[maybe_unused]] uint64_t bend[is_capped(kForm) ? 16 : 1];
        if (some) {
          tmem_ld_32x32b_x32(ts, a);
          tmem_ld_wait();
          if constexpr (kForm != FORM_PLAIN) {
            bool even = !masked || kForm == FORM_WIDE;
            if (even) even = is_capped(kForm) ? all_small(form, key < it.q.n ? largest(a) : 0.f) : one_side(far, kCols);
            if (even)
              form_scores<kForm, is_capped(kForm), true>(form, a, slope2, far, bend);
            else
              form_scores<kForm, is_capped(kForm), false>(form, a, slope2, far, bend);
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
            if constexpr (is_capped(kForm)) pr[c] = mul_pair(pr[c], bend[c]);
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
  __device__ __forceinline__ int length() const { return tiles; }
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
          [[maybe_unused]] uint64_t bend[is_capped(kForm) ? 16 : 1];
          if constexpr (kForm != FORM_PLAIN) {
            bool even = !masked || kForm == FORM_WIDE;
            if (even) even = is_capped(kForm) ? all_small(form, pos < it.q.n ? largest(a) : 0.f) : one_side(far, kCols);
            if (even)
              form_scores<kForm, is_capped(kForm), true>(form, a, slope2, far, bend);
            else
              form_scores<kForm, is_capped(kForm), false>(form, a, slope2, far, bend);
          }
#pragma unroll
          for (int c = 0; c < kCols / 2; ++c) {
            const uint64_t s2 = pair(__uint_as_float(a[2 * c]), __uint_as_float(a[2 * c + 1])), l = pair(-st.x, -st.x);
            float x, y;
            unpair(kForm != FORM_PLAIN ? add_pair(s2, l) : fma_pair(s2, pair(form.scale2, form.scale2), l), x, y);
            pr[c] = pair(fast_exp2(x), fast_exp2(y));
            if constexpr (is_capped(kForm)) pr[c] = mul_pair(pr[c], bend[c]);  // (p itself is not needed here)
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
// Parts that the query heads of a key head are cut into for dk and dv: where the key tiles
// do not fill the SMs (152), as the first tiles of a causal sequence take longest, as many
// as give some four items an SM, with as few heads in the largest as these allow.  Their
// sums, 1024 D bytes of a key head's tile and part, are so at most 100 MB whatever the
// heads' number.  (dk, dv and join, us.  5003 tokens of 15 + 3 heads of 96: 112 in five
// parts, 215 in one; 16384 of 64 + 1 heads of 128: 4770 + 130 in five, 5290 + 205 and 1.1 GB
// in 64; 4096 of 32 + 4: 181 + 24 in four, 215 + 42 in eight.  Three items an SM in place of
// four: 16384 of 64 + 1 heads 5010 + 460, 2048 of 32 + 1 71 + 22 for 89 + 32.  Below four
// tiles a launch more costs what it saves.)
int head_parts(int64_t T, int64_t Hq, int64_t Hk) {
  const int64_t items = ceil_div(T, 128) * Hk, per = Hq / Hk;
  if (items < 4 * Hk || items > 152) return 1;
  const int64_t each = ceil_div(per, std::min(per, ceil_div(4 * 152, items)));
  return static_cast<int>(ceil_div(per, each));
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
  constexpr int kLanes = kBoxes == 1 ? 8 : 16;
  const int64_t few = ceil_div(static_cast<int64_t>(a.S) * a.Hq, kDeltaThreads / 32);
  const int64_t rest = std::min<int64_t>(ceil_div(ceil_div(a.T, 4) * a.Hq, kDeltaThreads / kLanes), 1 << 30);
  att_delta_kernel<kLanes><<<static_cast<unsigned>(few + rest), kDeltaThreads, 0, c.stream>>>(a, stats, few);
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
  if (a.cap > 0.f) return a.cap > kWideCap ? run_bwd<kBoxes, FORM_WIDE>(c, a) : run_bwd<kBoxes, FORM_CAP>(c, a);
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
