// gated_mlp_few.cu -- the gated feed-forward block on few rows (single tokens, a
// batch's next tokens): the forward in two launches that read the weights once, and
// the backward's products of the same shape, dh and dx, in two more.
//
// Few rows make the weights the wide operand: they are A (M = 128 of their rows or
// columns in the lanes), the tokens B (N = 16 to 128 columns), so one MMA shape
// serves any count of tokens and the accumulator's columns are the tokens.
//   FEW_UP    a CTA takes `rows` rows of W_gate and the same of W_up, into two
//             accumulators, so that a thread has g and u of its row; h = act(g) u
//   FEW_DOWN  a CTA takes `rows` rows of W_down; y = h W_down^T (+ residual)
//   FEW_DH    a CTA takes `rows` columns of W_down, read MN-major as they lie;
//             dh = dy W_down, and from g and u dg, du and h
//   FEW_DX    a CTA takes `rows` columns of W_gate, then the same of W_up, into one
//             accumulator; dx = dg W_gate + du W_up
// MMAs always cover 128 lanes: where a CTA has fewer rows the others read what
// lies behind the tile in shared memory and their lanes are not read back.
//
// What bounds it: HBM, the weights' 6 d f bytes; so the CTAs are made small and
// many (two to an SM, up to 108 KB each in flight).  Where there are too few
// rows for that, the CTAs of a cluster share a tile's K steps and add their
// accumulators up through distributed shared memory, every CTA for a part of the
// tokens, in the cluster's order.  The second launch starts while the first runs
// (programmatic dependent launch) and fills its stages with weights before it waits
// for the first one's results.
//
// Measured, us, the weights in HBM: one token 53 at d = 4096, f = 12288 (5.7 TB/s
// over 302 MB), 21 at 2048, 6144; 64 tokens 63 and 29; 128 tokens 75 and 37.  (In
// gated_mlp.cu's form: one 138 and 49, 64 77 and 37, 128 79 and 38.)  Backward, with
// the weights' gradients: one row 152 at 4096, 12288, 52 of them dh and dx (5.8 TB/s);
// 16 rows 50 and 64 rows 56 at 2048, 6144 (200, 70 and 69 in gated_mlp.cu's form).
#include <algorithm>
#include <atomic>

#include "gated_mlp.cuh"
#include "sm103.cuh"

namespace olive {
namespace {

constexpr int kBK = 64;
constexpr int kMaxStages = 24;
constexpr int kEpiWarps = 8, kProducerWarp = 8, kMmaWarp = 9;
constexpr int kThreads = 32 * 10;
constexpr int kTile = 128 * 128;      // bytes the MMA reads of an A tile
// shared memory of a CTA: two to an SM, or one where the tokens' tile is large
constexpr int budget(int n) { return (n <= 64 ? 108 : 210) * 1024; }

enum { FEW_UP = 0, FEW_DOWN = 1, FEW_DH = 2, FEW_DX = 3 };

struct FewMaps {
  CUtensorMap a0, a1;  // W_gate and W_up, or W_down
  CUtensorMap b0, b1;  // tokens (FEW_DX: dg, du)
};
struct FewParams {
  int T, rows_all, K;     // tokens, weight rows (columns of the result), inner width
  int rows, stages;
  int ld, out_f32;        // FEW_DH: pitch of its results; FEW_DX: type of dx
  void* out;              // h, y, h again or dx
  const __nv_bfloat16* residual;
  uint16_t *saved_g, *saved_u;  // [T, rows_all], written by FEW_UP, read by FEW_DH
  __nv_bfloat16 *out_g, *out_u; // FEW_DH: dg, du
  int32_t* dev_status;
  uint64_t wait_limit_ns;
};

__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(r));
  return r;
}

__device__ __forceinline__ void st_cluster_v2(uint32_t addr, uint32_t x, uint32_t y) {
  asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void st_cluster_v4(uint32_t addr, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(x), "r"(y), "r"(z), "r"(w)
               : "memory");
}

template <int kMode, int kN, int kAct>
__global__ void __launch_bounds__(kThreads) few_kernel(const __grid_constant__ FewMaps maps, const FewParams p) {
  constexpr bool kUp = kMode == FEW_UP;
  constexpr bool kFirst = kMode == FEW_UP || kMode == FEW_DH;  // of its call
  constexpr bool kMn = kMode == FEW_DH || kMode == FEW_DX;     // A is MN-major
  constexpr int kAcc = kUp ? 2 : 1;
  constexpr uint32_t kCols = kAcc * kN < 32 ? 32 : kAcc * kN;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t base = smem_u32(smem_raw);
  const int a_bytes = p.rows * 128;
  const int stage_bytes = kAcc * a_bytes + kN * 128;
  // barriers first (1 KB), then the stages, then what the last one's MMAs read past it
  auto full_bar = [&](int s) { return base + 8u * s; };
  auto empty_bar = [&](int s) { return base + 8u * (kMaxStages + s); };
  const uint32_t done_bar = base + 8u * (2 * kMaxStages);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem_raw + 8 * (2 * kMaxStages + 1));
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem_raw + 8 * (2 * kMaxStages + 1) + 4);
  const uint32_t ring = base + 1024;
  float* recv = reinterpret_cast<float*>(smem_raw + 1024);

  const int warp = warp_uniform(static_cast<int>(threadIdx.x >> 5));
  const int lane = threadIdx.x & 31;
  const int c = static_cast<int>(cluster_size()), rank = static_cast<int>(cluster_rank());
  const int row0 = static_cast<int>(blockIdx.x) / c * p.rows;
  const int t0 = static_cast<int>(blockIdx.y) * kN;
  const int nt = min(kN, p.T - t0);
  const int ks_half = (p.K + kBK - 1) / kBK, ks_all = kMode == FEW_DX ? 2 * ks_half : ks_half;
  const int ks0 = ks_all * rank / c, ks1 = ks_all * (rank + 1) / c;

  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    mbar_init(done_bar, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == kProducerWarp && lane == 0) {
    tma_prefetch_desc(&maps.a0);
    if (kUp || kMode == FEW_DX) tma_prefetch_desc(&maps.a1);
    tma_prefetch_desc(&maps.b0);
    if (kMode == FEW_DX) tma_prefetch_desc(&maps.b1);
  }
  if (warp == kMmaWarp) {
    tmem_alloc(smem_u32(tmem_slot), kCols);
    tmem_relinquish();
    // (not before this CTA has its tensor memory: the next launch's CTAs take theirs
    // and keep it while they wait for this grid)
    grid_launch_dependents();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const WaitCtl ctl{abort_flag, p.wait_limit_ns};
  bool ok = true;

  if (warp == kProducerWarp) {
    const bool leader = elect_one();
    auto weights = [&](int s, int ks) {
      const uint32_t at = ring + s * stage_bytes;
      mbar_arrive_expect_tx(full_bar(s), stage_bytes);
      if constexpr (kMn) {
        const bool second = kMode == FEW_DX && ks >= ks_half;
        for (int i = 0; i < p.rows; i += 64)
          tma_load_2d(at + i * 128, second ? &maps.a1 : &maps.a0, full_bar(s), row0 + i, (second ? ks - ks_half : ks) * kBK);
      } else {
        tma_load_2d(at, &maps.a0, full_bar(s), ks * kBK, row0);
        if (kUp) tma_load_2d(at + a_bytes, &maps.a1, full_bar(s), ks * kBK, row0);
      }
    };
    auto tokens = [&](int s, int ks) {
      const bool second = kMode == FEW_DX && ks >= ks_half;
      tma_load_2d(ring + s * stage_bytes + kAcc * a_bytes, second ? &maps.b1 : &maps.b0, full_bar(s),
                  (second ? ks - ks_half : ks) * kBK, t0);
    };
    const int first = min(p.stages, ks1 - ks0);
    if (leader) {
      for (int s = 0; s < first; ++s) weights(s, ks0 + s);
      // the weights do not depend on the launch before this one; h, dg and du do
      if (!kFirst) {
        grid_wait();
        fence_proxy_async_global();
      }
      for (int s = 0; s < first; ++s) tokens(s, ks0 + s);
    }
    __syncwarp();
    int s = 0;
    uint32_t phase = 0;
    for (int ks = ks0 + first; ks < ks1; ++ks) {
      if (!mbar_wait_warp(empty_bar(s), phase, ctl)) { ok = false; break; }
      if (leader) {
        weights(s, ks);
        tokens(s, ks);
      }
      if (++s == p.stages) { s = 0; phase ^= 1u; }
    }
    __syncwarp();
  } else if (warp == kMmaWarp) {
    const bool leader = elect_one();
    const uint32_t acc = warp_uniform(tmem_base);
    const uint32_t id = idesc_bf16(128, kN, kMn, false);
    int s = 0;
    uint32_t phase = 0;
    for (int ks = ks0; ks < ks1; ++ks) {
      if (!mbar_wait_warp(full_bar(s), phase, ctl)) { ok = false; break; }
      tc_fence_after();
      // (MN-major: 16 K elements are 16 rows of 128 bytes, 64-element blocks 8 KB apart)
      const uint64_t da = sdesc_sw128(ring + s * stage_bytes, kMn ? 64 * kBK * 2 : 16, 1024);
      constexpr int kStepA = kMn ? 128 : 2;
      const uint64_t db = sdesc_sw128(ring + s * stage_bytes + kAcc * a_bytes, 16, 1024);
      if (leader) {
#pragma unroll
        for (int kk = 0; kk < kBK / 16; ++kk) {
          const uint32_t go = ks > ks0 || kk > 0 ? 1u : 0u;
          umma_bf16(acc, da + kStepA * kk, db + 2 * kk, id, go);
          if (kUp) umma_bf16(acc + kN, da + (a_bytes >> 4) + 2 * kk, db + 2 * kk, id, go);
        }
        umma_commit(empty_bar(s));
      }
      if (++s == p.stages) { s = 0; phase ^= 1u; }
    }
    // every MMA issued above has completed before the accumulators are read or
    // freed (a bounded wait that ignores the abort flag: it is for work in flight)
    if (leader) umma_commit(done_bar);
    volatile int keep_waiting = 0;
    const uint64_t floor_ns = 200ull * 1000 * 1000;
    const WaitCtl own{&keep_waiting, p.wait_limit_ns > floor_ns ? p.wait_limit_ns : floor_ns};
    mbar_wait_warp(done_bar, 0, own);
  } else {
    // (the MMA warp commits to it in any case; its own waits are bounded.  This one
    // lasts as long as the products, so looking at the limit each time costs nothing,
    // and a limit that is shorter than they take is noticed)
    ok = mbar_wait_warp<1>(done_bar, 0, ctl);
    tc_fence_after();
  }

  __syncthreads();
  if (*abort_flag) let_copies_land();  // a wait ran out: the stages may still be written
  // epilogue warp w: weight rows 32 (w % 4).. of the accumulators and half w / 4
  // of the tokens, 8 at a time
  const uint32_t lane_addr = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16);
  const int row = (warp & 3) * 32 + lane;
  const int tb = (warp >> 2) * (kN / 2), te = min(tb + kN / 2, nt);
  const bool epi = warp < kEpiWarps && ok && (warp & 3) * 32 < p.rows;
  __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out);
  const int ld = kMode == FEW_DH ? p.ld : p.rows_all;  // pitch of the results
  // g and u of FEW_DH, read ahead of a group's stores
  auto before = [&](size_t at, uint32_t& g, uint32_t& u) {
    if (kMode == FEW_DH) {
      g = p.saved_g[at];
      u = p.saved_u[at];
    }
  };
  // one result from its sums; at: in the results, in: in what is saved
  auto store = [&](float a, float b, uint32_t g, uint32_t u, size_t at, size_t in) {
    if constexpr (kUp) {
      out[at] = __float2bfloat16_rn(activate<kAct>(a) * b);
      if (p.saved_g) {
        p.saved_g[in] = static_cast<uint16_t>(saved_bits(a));
        p.saved_u[in] = static_cast<uint16_t>(saved_bits(b));
      }
    } else if constexpr (kMode == FEW_DH) {
      float ag, slope;
      activate_both<kAct>(saved_lo(g), ag, slope);
      float uf = saved_lo(u);
      if ((saved_nan(g) | saved_nan(u)) & 0x8000u) ag = slope = uf = __uint_as_float(0x7fffffffu);
      p.out_g[at] = __float2bfloat16_rn(a * uf * slope);
      p.out_u[at] = __float2bfloat16_rn(a * ag);
      out[at] = __float2bfloat16_rn(ag * uf);
    } else if constexpr (kMode == FEW_DX) {
      if (p.out_f32)
        static_cast<float*>(p.out)[at] = a;
      else
        out[at] = __float2bfloat16_rn(a);
    } else {
      out[at] = __float2bfloat16_rn(p.residual ? a + __bfloat162float(p.residual[at]) : a);
    }
  };
  if (c == 1) {
    const bool mine = epi && row < p.rows && row0 + row < p.rows_all;
    size_t at = static_cast<size_t>(t0 + tb) * ld + row0 + row;
    size_t in = kMode == FEW_DH ? static_cast<size_t>(t0 + tb) * p.rows_all + row0 + row : 0;
#pragma unroll 1
    for (int t = tb; epi && t < te; t += 8) {
      uint32_t a[8], b[8], g[8] = {}, u[8] = {};
#pragma unroll
      for (int i = 0; kMode == FEW_DH && i < 8; ++i)
        if (mine && t + i < te) before(in + static_cast<size_t>(i) * p.rows_all, g[i], u[i]);
      tmem_ld_32x32b_x8(lane_addr + t, a);
      if (kUp) tmem_ld_32x32b_x8(lane_addr + kN + t, b);
      tmem_ld_wait();
#pragma unroll
      for (int i = 0; i < 8; ++i, at += ld, in += p.rows_all)
        if (mine && t + i < te) store(__uint_as_float(a[i]), kUp ? __uint_as_float(b[i]) : 0.f, g[i], u[i], at, kMode == FEW_DH ? in : at);
    }
  } else {
    // CTA q of the cluster finishes tokens [q per, (q + 1) per): every CTA sends
    // it its sums of them, recv[sender][accumulator][row][token]
    const int per = kN / c;
    cluster_sync_all();  // all MMAs of the cluster are done: the stages are free
#pragma unroll 1
    for (int t = tb; epi && t < te; t += 8) {
      uint32_t a[8], b[8];
      tmem_ld_32x32b_x8(lane_addr + t, a);
      if (kUp) tmem_ld_32x32b_x8(lane_addr + kN + t, b);
      tmem_ld_wait();
      if (row >= p.rows) continue;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int q = (t + 2 * v) / per, j = t + 2 * v - q * per;
        const uint32_t at = ring + 4u * ((rank * kAcc * p.rows + row) * per + j);
        const uint32_t au = at + 4u * p.rows * per;
        if (per == 2) {
          st_cluster_v2(map_shared(at, q), a[2 * v], a[2 * v + 1]);
          if (kUp) st_cluster_v2(map_shared(au, q), b[2 * v], b[2 * v + 1]);
        } else if (v % 2 == 0) {
          st_cluster_v4(map_shared(at, q), a[2 * v], a[2 * v + 1], a[2 * v + 2], a[2 * v + 3]);
          if (kUp) st_cluster_v4(map_shared(au, q), b[2 * v], b[2 * v + 1], b[2 * v + 2], b[2 * v + 3]);
        }
      }
    }
    cluster_sync_all();
    const int my = min(per, nt - rank * per);
    for (int i = threadIdx.x; i < (my + 1) / 2 * p.rows; i += kThreads) {
      const int j = i / p.rows * 2, r = i - j / 2 * p.rows;
      if (row0 + r >= p.rows_all) continue;
      float2 a = {0.f, 0.f}, b = {0.f, 0.f};
      const size_t t = t0 + rank * per + j;
      const size_t at = t * ld + row0 + r, in = kMode == FEW_DH ? t * p.rows_all + row0 + r : at;
      uint32_t g0 = 0, u0 = 0, g1 = 0, u1 = 0;
      before(in, g0, u0);
      if (j + 1 < my) before(in + p.rows_all, g1, u1);
      for (int q = 0; q < c; ++q) {
        const float* f = recv + (q * kAcc * p.rows + r) * per + j;
        const float2 x = *reinterpret_cast<const float2*>(f);
        a.x += x.x;
        a.y += x.y;
        if (kUp) {
          const float2 y = *reinterpret_cast<const float2*>(f + p.rows * per);
          b.x += y.x;
          b.y += y.y;
        }
      }
      store(a.x, b.x, g0, u0, at, in);
      if (j + 1 < my) store(a.y, b.y, g1, u1, at + ld, in + p.rows_all);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag && p.dev_status) atomicOr(p.dev_status, 1 << OLIVE_ERR_TIMEOUT);
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem_base, kCols);
  }
}

// Weight rows of a CTA and CTAs of a cluster for `rows_all` rows, `ks` K steps
// and `tiles` tiles of n tokens.
//
// Long tiles (many rows, K steps shared by a cluster) read each token's values
// fewer times; the exchange of accumulators, 4 rows n bytes each, is what they
// cost.  So: as many rows as keep a CTA's exchange within 16 KB (32 KB from n =
// 128 on), and clusters that fill the slots.  Measured, us a call: d = 2048,
// f = 6144 at n = 16 15.2 with 128 rows by 4 and 8 CTAs, 20.5 with 48 rows by 1
// and 2; at n = 64 in the second launch 23.2 with 64 rows by 4, 25.6 with 128 rows
// by 8.  The first launch has two accumulators to exchange and from n = 64 on is
// quicker with whole K steps (23.2 us with 64 rows by 1, 27.5 by 2; n = 128, d =
// 4096, f = 12288: 73.6 with 88 rows by 1, 93.0 by 2).
// MN-major weights come in blocks of 64 (`least`).
struct FewShape {
  int rows, c;
};
FewShape few_shape(int rows_all, int ks, int tiles, int n, int sms, bool up, int least) {
  const int slots = n <= 64 ? 2 * sms : sms;  // CTAs that run at once
  const int most = (n < 128 ? 16 : 32) * 1024 / (4 * n * (up ? 2 : 1));
  FewShape s{std::min(128, std::max(64, most)), 1};
  const auto ctas = [&] { return ceil_div(rows_all, s.rows) * s.c * tiles; };
  if (up && n >= 128) {
    // one CTA a slot where that is one wave
    const int64_t even = align_up(ceil_div(static_cast<int64_t>(rows_all) * tiles, slots), 8);
    s.rows = static_cast<int>(std::min<int64_t>(128, std::max<int64_t>(64, even)));
  }
  // fewer rows where there are few: in the first launch, from n = 64 on, rather
  // than a larger cluster (64 tokens, d = 1024, f = 2816: 17.2 us with 32 rows by 1,
  // 18.6 with 64 by 2)
  const int enough = up && n >= 64 ? sms / 2 : sms / 8;
  while (s.rows > least && ctas() < enough) s.rows = s.rows > 64 ? 64 : 32;
  const int c_most = up && n >= 64 && 2 * ctas() >= sms ? 1 : 8;
  while (s.c < c_most && 2 * ctas() <= slots && ks >= 8 * s.c) s.c *= 2;
  return s;
}

template <int kMode, int kN, int kAct>
olive_status launch_few(const Ctx& c, const FewMaps& maps, FewParams p, const FewShape& s) {
  constexpr bool kUp = kMode == FEW_UP, kFirst = kUp || kMode == FEW_DH;
  constexpr int kAcc = kUp ? 2 : 1;
  const int stage = kAcc * p.rows * 128 + kN * 128;
  // the MMAs read 128 rows from the last stage's last A
  const int past = std::max(0, (kAcc - 1) * p.rows * 128 + kTile - stage);
  const int ks = static_cast<int>(ceil_div((kMode == FEW_DX ? 2 : 1) * ceil_div(p.K, kBK), s.c));
  p.stages = std::min({(budget(kN) - 1024 - past) / stage, kMaxStages, ks});
  const int exchange = s.c > 1 ? 4 * kAcc * p.rows * kN : 0;
  const int smem = 1024 + std::max(p.stages * stage + past, exchange);
  p.wait_limit_ns = c.wait_limit_ns;
  static std::atomic<int> done[kMaxDevices];
  if (!set_smem_once(reinterpret_cast<const void*>(few_kernel<kMode, kN, kAct>), 227 * 1024, c.device, done))
    return OLIVE_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(ceil_div(p.rows_all, p.rows) * s.c), static_cast<unsigned>(ceil_div(p.T, kN)));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = c.stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = s.c;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = kFirst ? 1 : 2;  // (only the second launch may start before the one ahead of it ends)
  if (cudaLaunchKernelEx(&cfg, few_kernel<kMode, kN, kAct>, maps, p) != cudaSuccess) {
    cudaGetLastError();
    return OLIVE_ERR_CUDA;
  }
  return OLIVE_OK;
}

template <int kMode, int kAct>
olive_status by_tokens(const Ctx& c, const FewMaps& maps, const FewParams& p, int n, const FewShape& s) {
  switch (n) {
    case 16: return launch_few<kMode, 16, kAct>(c, maps, p, s);
    case 32: return launch_few<kMode, 32, kAct>(c, maps, p, s);
    case 64: return launch_few<kMode, 64, kAct>(c, maps, p, s);
    default: break;
  }
  if constexpr (kMode == FEW_UP || kMode == FEW_DOWN) return launch_few<kMode, 128, kAct>(c, maps, p, s);
  return OLIVE_ERR_SHAPE;
}

}  // namespace

olive_status launch_mlp_few(const Ctx& c, const void* x, const void* W_gate, const void* W_up,
                            const void* W_down, const void* residual, int32_t T, int32_t d,
                            int32_t f, int act, void* y, void* saved, void* h,
                            int32_t* dev_status) {
  const int n = T <= 16 ? 16 : T <= 32 ? 32 : T <= 64 ? 64 : 128;
  const int tiles = static_cast<int>(ceil_div(T, n));
  FewMaps m = {};
  FewParams p = {};
  p.T = T;
  p.dev_status = dev_status;

  FewShape s = few_shape(f, static_cast<int>(ceil_div(d, kBK)), tiles, n, c.num_sms, true, 32);
  p.rows_all = f;
  p.K = d;
  p.rows = s.rows;
  p.out = h;
  p.saved_g = static_cast<uint16_t*>(saved);
  p.saved_u = saved ? p.saved_g + static_cast<size_t>(T) * f : nullptr;
  if (!encode_bf16_2d(&m.a0, W_gate, d, f, 2ull * d, kBK, s.rows) ||
      !encode_bf16_2d(&m.a1, W_up, d, f, 2ull * d, kBK, s.rows) ||
      !encode_bf16_2d(&m.b0, x, d, T, 2ull * d, kBK, n))
    return OLIVE_ERR_CUDA;
  const olive_status st = act == OLIVE_ACT_SILU ? by_tokens<FEW_UP, OLIVE_ACT_SILU>(c, m, p, n, s)
                                                : by_tokens<FEW_UP, OLIVE_ACT_GELU_TANH>(c, m, p, n, s);
  if (st != OLIVE_OK) return st;

  s = few_shape(d, static_cast<int>(ceil_div(f, kBK)), tiles, n, c.num_sms, false, 32);
  p.rows_all = d;
  p.K = f;
  p.rows = s.rows;
  p.out = y;
  p.residual = static_cast<const __nv_bfloat16*>(residual);
  p.saved_g = p.saved_u = nullptr;
  if (!encode_bf16_2d(&m.a0, W_down, f, d, 2ull * f, kBK, s.rows) ||
      !encode_bf16_2d(&m.b0, h, f, T, 2ull * f, kBK, n))
    return OLIVE_ERR_CUDA;
  return by_tokens<FEW_DOWN, 0>(c, m, p, n, s);
}

olive_status launch_mlp_few_bwd(const Ctx& c, const void* dy, const void* W_gate, const void* W_up,
                                const void* W_down, const void* saved, int32_t T, int32_t d,
                                int32_t f, int act, const MlpWs& w, void* dx, int grad_dtype,
                                int32_t* dev_status) {
  const int n = T <= 16 ? 16 : T <= 32 ? 32 : 64;
  const int fp = static_cast<int>(mlp_pitch(f));
  FewMaps m = {};
  FewParams p = {};
  p.T = T;
  p.dev_status = dev_status;

  FewShape s = few_shape(f, static_cast<int>(ceil_div(d, kBK)), 1, n, c.num_sms, false, 64);
  p.rows_all = f;
  p.K = d;
  p.rows = s.rows;
  p.out = w.h;
  p.out_g = static_cast<__nv_bfloat16*>(w.dg);
  p.out_u = static_cast<__nv_bfloat16*>(w.du);
  p.ld = fp;
  p.saved_g = static_cast<uint16_t*>(const_cast<void*>(saved));
  p.saved_u = p.saved_g + static_cast<size_t>(T) * f;
  if (!encode_bf16_2d(&m.a0, W_down, f, d, 2ull * f, 64, kBK) || !encode_bf16_2d(&m.b0, dy, d, T, 2ull * d, kBK, n))
    return OLIVE_ERR_CUDA;
  const olive_status st = act == OLIVE_ACT_SILU ? by_tokens<FEW_DH, OLIVE_ACT_SILU>(c, m, p, n, s)
                                                : by_tokens<FEW_DH, OLIVE_ACT_GELU_TANH>(c, m, p, n, s);
  if (st != OLIVE_OK || !dx) return st;

  s = few_shape(d, 2 * static_cast<int>(ceil_div(f, kBK)), 1, n, c.num_sms, false, 64);
  p.rows_all = d;
  p.K = f;
  p.rows = s.rows;
  p.out = dx;
  p.out_f32 = grad_dtype == OLIVE_DTYPE_F32;
  if (!encode_bf16_2d(&m.a0, W_gate, d, f, 2ull * d, 64, kBK) ||
      !encode_bf16_2d(&m.a1, W_up, d, f, 2ull * d, 64, kBK) ||
      !encode_bf16_2d(&m.b0, w.dg, f, T, 2ull * fp, kBK, n) || !encode_bf16_2d(&m.b1, w.du, f, T, 2ull * fp, kBK, n))
    return OLIVE_ERR_CUDA;
  return by_tokens<FEW_DX, 0>(c, m, p, n, s);
}

}  // namespace olive
