// gated_mlp.cu -- the gated feed-forward block of a decoder layer on many rows,
// forward and backward (olive_gated_mlp_fwd, olive_gated_mlp_bwd):
//   g = x Wg^T, u = x Wu^T, h = act(g) u, y = h Wd^T (+ residual)
//   dh = dy Wd, dg = dh u act'(g), du = dh act(g)
//   dx = dg Wg + du Wu, dWg = dg^T x, dWu = du^T x, dWd = dy^T h
// as four kinds of one persistent tcgen05 kernel:
//   MM_UP     g and u of the same columns side by side in one accumulator; h
//             (and, for a backward, g and u) in the epilogue
//   MM_DOWN   h Wd^T, the residual added in the epilogue
//   MM_DH     dy Wd; the epilogue reads g and u and writes dg, du and h
//   MM_GRADS  the four products that are left, in one launch
// Few rows take gated_mlp_few.cu's form, except for the weights' gradients.
//
// CTA pairs (clusters of two, tcgen05.mma.cta_group::2, M = 256): each CTA
// stages its 128 rows of A and its half of the B rows (256 or 128 wide tiles), and
// receives its 128 rows of the fp32 accumulator in its own TMEM, twice, so that
// the epilogue of a tile runs under the next tile's MMAs.  An operand is
// read K-major or MN-major as it lies in memory; nothing is transposed or
// copied.  Results are turned in shared memory so that a warp's store covers whole
// 64-byte rows.  Wide tiles read each operand less often (64 KB a K step of 512 MMA
// cycles); narrow ones are for small problems, whose epilogues and last waves are
// then shorter (512 rows, d = 256, f = 704, us: forward 13.4, backward 18.5; 19.3 and
// 35.3 with wide tiles; 2777 rows, 2048, 5504: 150 and 314; 137 and 260 with wide
// ones); plan_tiles below chooses.
//
// What bounds it: the tensor pipe in the products with long K steps and light
// epilogues, the epilogue's loads and stores in MM_UP and MM_DH at small d.
// Measured: 8192 rows, d = 4096, f = 12288, forward and backward 4.5 ms, 1.64
// PFLOP/s, under the power cap; 2777 rows, d = 2048, f = 5504, launch by launch from
// empty caches, us: up 83, down 52, dh 68, gradients 175 (1.8 PFLOP/s; 91 % of the
// tensor pipe's cycles on 2816 rows); d = 2040, f = 5464, whose rows are not whole
// 128-byte lines: 109, 53, 91, 187.
//
// Rounding: g and u are used from the fp32 accumulators; h, dg and du are rounded
// to bf16 once, as operands of the next product; g and u are saved with 10
// significant bits (pack_saved).
#include <algorithm>
#include <atomic>

#include "gated_mlp.cuh"
#include "sm103.cuh"

namespace olive {
namespace {

constexpr int kBM = 128;             // rows of a CTA's tile
constexpr int kWide = 256, kNarrow = 128;  // columns of a tile (half of them g, half u in MM_UP)
constexpr int kBK = 64;
constexpr int kSA = kBM * kBK * 2;   // this CTA's 128 rows of A
constexpr int kEpiWarps = 8;
constexpr int kProducerWarp = 8, kMmaWarp = 9;
constexpr int kThreads = 32 * 10;
constexpr int kOutBuf = 32 * 64;     // a warp's 32 rows of 64 bytes of a result
constexpr int kSlots = 8;            // a finisher warp's pieces in flight
constexpr int kSlotBytes = 16 * 32 * 4;
enum { MM_UP = 0, MM_DOWN = 1, MM_DH = 2, MM_GRADS = 3 };
// An output buffer a warp for each result of a tile.
template <int kMode, int kBN>
struct Layout {
  static constexpr bool kThree = kMode == MM_UP || kMode == MM_DH;
  static constexpr int kOutBufs = kThree ? 3 : 1;
  static constexpr int kSB = kBN / 2 * kBK * 2;  // this CTA's half of B
  static constexpr int kStageBytes = kSA + kSB;
  static constexpr int kStages = kBN == kNarrow ? 7 : kThree ? 5 : 6;
  static constexpr int kOut = kStages * kStageBytes;
  static constexpr int kBars = kOut + kEpiWarps * kOutBufs * kOutBuf;
  static constexpr int kBarCount = 2 * kStages + 5 + kEpiWarps * kSlots;
  static constexpr int kMisc = kBars + 8 * kBarCount;
  static constexpr int kSmem = kMisc + 64;
  static_assert(kSmem <= 227 * 1024, "shared memory budget");
  static_assert(kEpiWarps * kSlots * kSlotBytes <= kStages * kStageBytes, "pieces pass through the stages");
};
constexpr int kRaster = 8;           // row tiles of a raster group (L2 reuse)
constexpr int kMaxProbs = 4;
constexpr int kStatusTimeout = 1 << OLIVE_ERR_TIMEOUT;

// One product out[M, N] = A . B of a launch; maps are indices into MlpMaps.
struct MlpProb {
  int16_t a0, a1, b0, b1;  // operands before and from K step ks_half on (MM_UP: b0, b1 by CTA)
  int a_mn;                // MN-major A
  void* out;               // row-major, pitch ld
  int M, N, ld;
  int mt, nt;              // pair tiles (256 rows), column tiles
  int ks_half, ks;         // K steps
};

// The first whole[i] tiles of each product are dealt to the pairs in turn; the K
// steps of the others (fewer than there are pairs, of each product) are laid end
// to end and cut into runs of `run` steps, one a pair.
struct MlpSplit {
  int n_whole;             // sum of whole
  int whole[kMaxProbs];
  int steps;               // K steps of the tiles that are cut
  int run;
  int off[kMaxProbs];      // offset in steps of each product's cut tiles
};

struct MlpMaps {
  CUtensorMap m[10];
};

struct MlpParams {
  MlpProb pr[kMaxProbs];
  int n_prob;
  int n_maps;
  MlpSplit cut;
  float* part;             // [pairs][2 CTAs][8 warps][kBN / 2 columns][32 rows] partial accumulators
  uint32_t* flag;          // [pairs][2 CTAs] warps that have stored theirs
  uint32_t* clear;         // words the next launch of the call wants zero
  int n_clear;
  const __nv_bfloat16* residual;  // MM_DOWN
  const uint16_t* saved_g;        // MM_DH: [T, f]
  const uint16_t* saved_u;
  int save, out_f32;
  void *out_g, *out_u;     // MM_UP: saved g, u (pitch N); MM_DH: dg, du (pitch ld)
  int32_t* dev_status;
  uint64_t wait_limit_ns;
};

struct Unit {
  int prob, m0, n0;        // the pair's first row, first column (MM_UP: of h)
  int k0, k1;              // K steps
  int ks;                  // of the whole tile
  int from;                // first pair that holds a part of the tile (k1 == ks: it is this pair's to finish)
};

// The units of one pair, in order: its whole tiles, then its run from the end
// to the beginning.  So a run's piece that another pair finishes comes first,
// and a pair that waits for pieces waits for runs whose first unit they are:
// no chain of waits.
struct UnitWalk {
  int t, pos, lo, pairs, pair;
  __device__ UnitWalk(const MlpParams& p, int pair_, int pairs_) {
    pair = pair_;
    pairs = pairs_;
    t = pair;
    lo = min(pair * p.cut.run, p.cut.steps);
    pos = min(lo + p.cut.run, p.cut.steps);
  }
  __device__ void place(const MlpParams& p, int i, int tile, Unit& u) const {
    const MlpProb& q = p.pr[i];
    Raster ra{q.mt, q.nt, kRaster};
    int mi, nj;
    ra.tile(tile, mi, nj);
    u.prob = i;
    u.m0 = mi * 2 * kBM;
    u.n0 = nj;
    u.ks = q.ks;
  }
  __device__ bool next(const MlpParams& p, Unit& u) {
    if (t < p.cut.n_whole) {
      int i = 0, at = t;
      while (i + 1 < p.n_prob && at >= p.cut.whole[i]) at -= p.cut.whole[i++];
      place(p, i, at, u);
      u.k0 = 0;
      u.k1 = u.ks;
      u.from = pair;
      t += pairs;
      return true;
    }
    if (pos <= lo) return false;
    int i = 0;
    while (i + 1 < p.n_prob && pos - 1 >= p.cut.off[i + 1]) ++i;
    const int ks = p.pr[i].ks;
    const int w = (pos - 1 - p.cut.off[i]) / ks;
    const int start = p.cut.off[i] + w * ks;
    place(p, i, p.cut.whole[i] + w, u);
    u.k1 = pos - start;
    u.k0 = max(lo - start, 0);
    u.from = u.k0 > 0 ? start / p.cut.run : pair;
    pos = start + u.k0;
    return true;
  }
};

// 16-byte piece `c` of row `row` of a warp's output buffer: written by rows and
// read by pieces without bank conflicts.
__device__ __forceinline__ uint32_t out_piece(uint32_t buf, int row, int c) {
  return buf + row * 64 + ((c ^ ((row >> 1) & 3)) << 4);
}
// The buffer to rows y.. and the columns of 64 bytes from x on of an [M, N] array
// of elt-byte values, pitch ld.
__device__ __forceinline__ void put_rows(void* out, uint32_t buf, int lane, int x, int y, int M, int N, int ld, int elt) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = i * 8 + (lane >> 2), c = lane & 3;
    const int col = x + c * (16 / elt);
    if (y + row < M && col < N)
      *reinterpret_cast<uint4*>(static_cast<char*>(out) + (static_cast<size_t>(y + row) * ld + col) * elt) =
          ld_shared_v4(out_piece(buf, row, c));
  }
}

// Untiled bulk copy global -> shared, completion counted on the mbarrier.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(bar)
      : "memory");
}

template <int kMode, int kAct, int kBN>
__global__ void __launch_bounds__(kThreads, 1)
    mlp_gemm_kernel(const __grid_constant__ MlpMaps maps, const __grid_constant__ MlpParams p) {
  using L = Layout<kMode, kBN>;
  constexpr int kStages = L::kStages, kStageBytes = L::kStageBytes;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t base = smem_u32(smem_raw);
  const uint32_t stages = base;
  const uint32_t bar0 = base + L::kBars;
  auto full_bar = [&](int st) { return bar0 + 8u * st; };
  auto empty_bar = [&](int st) { return bar0 + 8u * (kStages + st); };
  auto tfull = [&](int b) { return bar0 + 8u * (2 * kStages + b); };
  auto tempty = [&](int b) { return bar0 + 8u * (2 * kStages + 2 + b); };
  const uint32_t drain = bar0 + 8u * (2 * kStages + 4);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem_raw + L::kMisc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem_raw + L::kMisc + 4);

  const int warp = warp_uniform(static_cast<int>(threadIdx.x >> 5));
  const int lane = threadIdx.x & 31;
  const uint32_t rank = warp_uniform(cluster_rank());
  const int pair = static_cast<int>(blockIdx.x >> 1), pairs = static_cast<int>(gridDim.x >> 1);

  if (threadIdx.x == 0) {
    for (int st = 0; st < kStages; ++st) {
      mbar_init(full_bar(st), 1);   // the even CTA's producer (both CTAs' bytes)
      mbar_init(empty_bar(st), 1);  // the even CTA's MMA commit (multicast)
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(tfull(b), 1);
      mbar_init(tempty(b), 2 * kEpiWarps);  // the epilogue warps of both CTAs
    }
    mbar_init(drain, 1);
    for (int i = 0; i < kEpiWarps * kSlots; ++i) mbar_init(drain + 8u * (1 + i), 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == kProducerWarp && lane < p.n_maps) tma_prefetch_desc(&maps.m[lane]);
  if (warp == kMmaWarp) {
    tmem_alloc_pair(smem_u32(tmem_slot), 2 * kBN);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  cluster_sync_all();
  tc_fence_after();
  // The launch ahead may still be running (programmatic dependent launch): up to
  // here nothing of it was needed, and this launch's successor may do the same.
  grid_launch_dependents();
  grid_wait();
  fence_proxy_async_global();
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < p.n_clear; i += kThreads) p.clear[i] = 0;
  const uint32_t tmem_base = *tmem_slot;
  const WaitCtl ctl{abort_flag, p.wait_limit_ns};
  // Every role walks the pair's units by itself, and finds the next one while it
  // has work in flight: the walk's divisions take about 1000 cycles, a short tile's
  // MMAs 2000.
  UnitWalk walk(p, pair, pairs);
  Unit u, ahead;
  bool more = walk.next(p, u);

  if (warp == kProducerWarp) {
    const bool leader = elect_one();
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (; ok && more; u = ahead) {
      const MlpProb& q = p.pr[u.prob];
      const int mrow = u.m0 + static_cast<int>(rank) * kBM;
      // MM_UP: the even CTA holds the tile's rows of Wg, the odd one those of Wu
      const int nrow = kMode == MM_UP ? u.n0 * (kBN / 2) : u.n0 * kBN + static_cast<int>(rank) * (kBN / 2);
      for (int ks = u.k0; ks < u.k1; ++ks) {
        if (!mbar_wait_warp(empty_bar(stage), phase ^ 1u, ctl)) { ok = false; break; }
        const uint32_t sA = stages + stage * kStageBytes;
        const uint32_t fb = map_shared(full_bar(stage), 0);
        const bool second = kMode != MM_UP && ks >= q.ks_half;
        const int k = (second ? ks - q.ks_half : ks) * kBK;
        const CUtensorMap* ma = &maps.m[second ? q.a1 : q.a0];
        const CUtensorMap* mb = &maps.m[(kMode == MM_UP ? rank != 0 : second) ? q.b1 : q.b0];
        if (leader) {
          if (rank == 0) mbar_arrive_expect_tx(full_bar(stage), 2 * kStageBytes);
          if (kMode == MM_GRADS && q.a_mn) {
            tma_load_2d_pair(sA, ma, fb, mrow, k);
            tma_load_2d_pair(sA + kSA / 2, ma, fb, mrow + 64, k);
          } else {
            tma_load_2d_pair(sA, ma, fb, k, mrow);
          }
          if (kMode == MM_GRADS || kMode == MM_DH) {
            tma_load_2d_pair(sA + kSA, mb, fb, nrow, k);
            if (kBN == kWide) tma_load_2d_pair(sA + kSA + L::kSB / 2, mb, fb, nrow + 64, k);
          } else {
            tma_load_2d_pair(sA + kSA, mb, fb, k, nrow);
          }
        }
        if (ks == u.k0) more = walk.next(p, ahead);
        if (++stage == kStages) { stage = 0; phase ^= 1u; }
      }
    }
    __syncwarp();
  } else if (warp == kMmaWarp) {
    if (rank == 0) {
      const bool leader = elect_one();
      int stage = 0, n = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (; ok && more; u = ahead) {
        const MlpProb& q = p.pr[u.prob];
        const bool a_mn = kMode == MM_GRADS && q.a_mn;
        constexpr bool b_mn = kMode == MM_GRADS || kMode == MM_DH;
        const uint32_t id = idesc_bf16(2 * kBM, kBN, a_mn, b_mn);
        // K-major: 16 K elements are 32 bytes along the swizzled row; MN-major:
        // 16 rows of 128 bytes, 64-element blocks 8 KB apart
        const uint64_t dA = sdesc_sw128(stages, a_mn ? 64 * kBK * 2 : 16, 1024);
        const uint64_t dB = sdesc_sw128(stages + kSA, b_mn ? 64 * kBK * 2 : 16, 1024);
        const uint32_t stepA = a_mn ? 128 : 2, stepB = b_mn ? 128 : 2;
        const int b = n & 1;
        if (!mbar_wait_warp(tempty(b), ((n >> 1) & 1) ^ 1, ctl)) { ok = false; break; }
        tc_fence_after();
        const uint32_t acc = warp_uniform(tmem_base) + b * kBN;
        for (int ks = u.k0; ks < u.k1; ++ks) {
          if (!mbar_wait_warp(full_bar(stage), phase, ctl)) { ok = false; break; }
          tc_fence_after();
          const uint32_t so = static_cast<uint32_t>(stage) * (kStageBytes >> 4);
          if (leader) {
#pragma unroll
            for (int kk = 0; kk < kBK / 16; ++kk)
              umma_bf16_pair(acc, dA + (so + kk * stepA), dB + (so + kk * stepB), id, kk > 0 || ks > u.k0 ? 1u : 0u);
            umma_commit_pair(empty_bar(stage));
          }
          if (ks == u.k0) more = walk.next(p, ahead);
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
        if (!ok) break;
        if (leader) umma_commit_pair(tfull(b));
        ++n;
      }
      // every MMA issued above has completed before TMEM is freed (a bounded
      // wait that ignores the abort flag: it is for work already in flight)
      if (leader) umma_commit_pair(drain);
      volatile int keep_waiting = 0;
      const uint64_t floor_ns = 200ull * 1000 * 1000;
      const WaitCtl own{&keep_waiting, p.wait_limit_ns > floor_ns ? p.wait_limit_ns : floor_ns};
      mbar_wait_warp(drain, 0, own);
    }
    __syncwarp();
  } else {
    // epilogue warp w: rows 32 (w % 4).. of the CTA's tile (TMEM lanes, one row
    // a thread) and half w / 4 of its columns, 16 columns at a time.  The loops
    // are rolled: a tile's epilogue runs once in several microseconds, and code
    // that is unrolled over the columns is fetched from the L2 each time.
    const int half = warp >> 2;
    const uint32_t lane_addr = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const uint32_t out0 = base + L::kOut + warp * L::kOutBufs * kOutBuf;
    int n = 0;
    bool ok = true;
    constexpr int kCols = kMode == MM_UP ? kBN / 2 : kBN;  // result columns of a tile
    // What the epilogue reads from memory (MM_DH: g and u, MM_DOWN: the residual), a
    // chunk of 32 columns ahead of its use, in whole 64-byte rows as put_rows stores
    // them; the chunk goes through the results' buffers.  (Each thread reading its
    // own row from memory, 32 rows an instruction, took the dh launch 75 us in place
    // of 68 at 2816 rows, d = 2048, f = 5632, and 66 in place of 54 at d = 512.)
    constexpr bool kReads = kMode == MM_DH || kMode == MM_DOWN;
    const bool reads = kMode == MM_DH || (kMode == MM_DOWN && p.residual);
    uint4 e0[4], e1[4];
    auto fetch = [&](const Unit& w, int chunk, bool valid) {
      const MlpProb& q = p.pr[0];
      const int y = w.m0 + static_cast<int>(rank) * kBM + (warp & 3) * 32 + (lane >> 2);
      const int x = w.n0 * kCols + half * (kCols / 2) + chunk * 32 + (lane & 3) * 8;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool in = valid && reads && y + 8 * i < q.M && x < q.N;
        const size_t at = static_cast<size_t>(y + 8 * i) * q.N + x;
        e0[i] = e1[i] = make_uint4(0, 0, 0, 0);
        if (in && kMode == MM_DH) {
          e0[i] = __ldg(reinterpret_cast<const uint4*>(p.saved_g + at));
          e1[i] = __ldg(reinterpret_cast<const uint4*>(p.saved_u + at));
        } else if (in) {
          e0[i] = *reinterpret_cast<const uint4*>(p.residual + at);
        }
      }
    };
    if (kReads && more) fetch(u, 0, u.k1 == u.ks);

    for (; ok && more; u = ahead) {
      const MlpProb& q = p.pr[u.prob];
      const int b = n & 1;
      const uint32_t acc = lane_addr + b * kBN;
      const int y = u.m0 + static_cast<int>(rank) * kBM + (warp & 3) * 32;  // the warp's first row
      constexpr int kSteps = kCols / 32;                     // of 16 columns, this warp's half
      const int x0 = u.n0 * kCols + half * (kCols / 2);
      // TMEM column of step s (MM_UP: g; u is kBN / 2 columns on)
      auto col = [&](int s) { return half * (kCols / 2) + s * 16; };
      // this warp's part of a pair's partial accumulator: [kBN / 32 steps][16 columns][32 rows]
      auto part_of = [&](int pr) {
        return p.part + (static_cast<size_t>(pr * 2 + static_cast<int>(rank)) * kEpiWarps + warp) * (kBN / 2 * 32);
      };
      auto release = [&] {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(map_shared(tempty(b), 0));
      };
      const bool whole = u.k1 == u.ks;
      more = walk.next(p, ahead);
      if (!mbar_wait_warp(tfull(b), (n >> 1) & 1, ctl)) break;
      tc_fence_after();
      ++n;

      if (!whole) {
        // a piece of a tile that another pair finishes
        float* to = part_of(pair) + lane;
#pragma unroll 1
        for (int s = 0; s < kBN / 32; ++s) {
          uint32_t r[16];
          tmem_ld_32x32b_x16(acc + (kMode == MM_UP ? s / kSteps * (kBN / 2) + col(s % kSteps) : col(s)), r);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 16; ++i) __stcg(to + (s * 16 + i) * 32, __uint_as_float(r[i]));
        }
        release();
        __threadfence();
        __syncwarp();
        if (lane == 0) red_release_add(p.flag + pair * 2 + rank, 1u);
        if (kReads) fetch(ahead, 0, more && ahead.k1 == ahead.ks);
        continue;
      }
      // A tile that is finished from pieces is the pair's last unit: its MMAs are
      // done, so the pieces pass through the stages, kSlots steps of them in flight
      // (plain loads held 16 KB in flight and took 8 us a 128 KB piece).  Step i of
      // the sequence is columns step_of(i / pieces) of pair u.from + i % pieces.
      const int pieces = pair - u.from;
      constexpr int kAll = kBN / 32;
      auto step_of = [&](int k) { return kMode == MM_UP ? (k & 1) * kSteps + (k >> 1) : k; };
      const uint32_t slot0 = stages + warp * (kSlots * kSlotBytes);
      const uint32_t slot_bar = drain + 8u * (1 + warp * kSlots);
      auto request = [&](int i) {
        if (lane == 0 && i < kAll * pieces) {
          const uint32_t bar = slot_bar + 8u * (i % kSlots);
          mbar_arrive_expect_tx(bar, kSlotBytes);
          bulk_load(slot0 + i % kSlots * kSlotBytes,
                    part_of(u.from + i % pieces) + step_of(i / pieces) * (16 * 32), kSlotBytes, bar);
        }
      };
      int taken = 0;
      if (pieces > 0) {
        for (int o = u.from; ok && o < pair; ++o) ok = wait_counter(p.flag + o * 2 + rank, kEpiWarps, ctl);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        fence_proxy_async_global();
        for (int i = 0; i < kSlots; ++i) request(i);
      }
      // the next 16 columns of the finished accumulator: the pair's own sum and the pieces'
      auto load = [&](int tcol, uint32_t(&r)[16]) {
        tmem_ld_32x32b_x16(acc + tcol, r);
        tmem_ld_wait();
        for (int o = 0; o < pieces; ++o, ++taken) {
          const int slot = taken % kSlots;
          ok = ok && mbar_wait_warp(slot_bar + 8u * slot, (taken / kSlots) & 1, ctl);
          if (!ok) return;
          const uint32_t f = slot0 + slot * kSlotBytes + 4 * lane;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float v;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(f + i * 128) : "memory");
            r[i] = __float_as_uint(__uint_as_float(r[i]) + v);
          }
          __syncwarp();
          request(taken + kSlots);
        }
      };
#pragma unroll 1
      for (int s = 0; s < kSteps; ++s) {
        const int x = x0 + (s & ~1) * 16;  // first column of the 64-byte output rows
        // (fp32 results fill a buffer in one step)
        const bool f32 = kMode == MM_GRADS && p.out_f32;
        const bool opens = f32 || (s & 1) == 0, closes = f32 || (s & 1) == 1;
        uint32_t r[16], v[16];
        load(col(s), r);
        if constexpr (kMode == MM_UP) load(kBN / 2 + col(s), v);
        if (!ok) break;
        if (s == kSteps - 1) release();
        const uint32_t buf = out0;
        if (opens) {
          __syncwarp();  // the buffers' last contents have been read
          if (kReads && reads) {
            // MM_DH: g where dg will be, u where du will be; MM_DOWN: the residual
            // where y will be, each thread's row by the thread that replaces it
            constexpr int kFirst = kMode == MM_DH ? kOutBuf : 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              st_shared_v4(out_piece(buf + kFirst, i * 8 + (lane >> 2), lane & 3), e0[i]);
              if (kMode == MM_DH) st_shared_v4(out_piece(buf + 2 * kOutBuf, i * 8 + (lane >> 2), lane & 3), e1[i]);
            }
            if (s + 2 < kSteps)
              fetch(u, (s >> 1) + 1, true);
            else
              fetch(ahead, 0, more && ahead.k1 == ahead.ks);
            __syncwarp();
          }
        }
        const int c0 = f32 ? 0 : (s & 1) * 2;  // 16-byte pieces of the row

        if constexpr (kMode == MM_UP) {
          uint32_t hw[8], gw[8], uw[8], wide = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float g0 = __uint_as_float(r[2 * i]), g1 = __uint_as_float(r[2 * i + 1]);
            const float u0 = __uint_as_float(v[2 * i]), u1 = __uint_as_float(v[2 * i + 1]);
            hw[i] = pack_bf16x2(activate<kAct>(g0) * u0, activate<kAct>(g1) * u1);
            gw[i] = pack_saved(g0, g1, wide);
            uw[i] = pack_saved(u0, u1, wide);
          }
          if (wide & kSavedWide) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              gw[i] = saved_bits(__uint_as_float(r[2 * i])) | saved_bits(__uint_as_float(r[2 * i + 1])) << 16;
              uw[i] = saved_bits(__uint_as_float(v[2 * i])) | saved_bits(__uint_as_float(v[2 * i + 1])) << 16;
            }
          }
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            st_shared_v4(out_piece(buf, lane, c0 + c), make_uint4(hw[4 * c], hw[4 * c + 1], hw[4 * c + 2], hw[4 * c + 3]));
            st_shared_v4(out_piece(buf + kOutBuf, lane, c0 + c),
                         make_uint4(gw[4 * c], gw[4 * c + 1], gw[4 * c + 2], gw[4 * c + 3]));
            st_shared_v4(out_piece(buf + 2 * kOutBuf, lane, c0 + c),
                         make_uint4(uw[4 * c], uw[4 * c + 1], uw[4 * c + 2], uw[4 * c + 3]));
          }
        } else if constexpr (kMode == MM_DH) {
          const uint4 ga = ld_shared_v4(out_piece(buf + kOutBuf, lane, c0)), gb = ld_shared_v4(out_piece(buf + kOutBuf, lane, c0 + 1));
          const uint4 ua = ld_shared_v4(out_piece(buf + 2 * kOutBuf, lane, c0)),
                      ub = ld_shared_v4(out_piece(buf + 2 * kOutBuf, lane, c0 + 1));
          const uint32_t gs[8] = {ga.x, ga.y, ga.z, ga.w, gb.x, gb.y, gb.z, gb.w};
          const uint32_t us[8] = {ua.x, ua.y, ua.z, ua.w, ub.x, ub.y, ub.z, ub.w};
          uint32_t hw[8], gw[8], uw[8], bad = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            float a0, a1, d0, d1;
            activate_both<kAct>(saved_lo(gs[i]), a0, d0);
            activate_both<kAct>(saved_hi(gs[i]), a1, d1);
            const float u0 = saved_lo(us[i]), u1 = saved_hi(us[i]);
            const float h0 = __uint_as_float(r[2 * i]), h1 = __uint_as_float(r[2 * i + 1]);
            gw[i] = pack_bf16x2(h0 * u0 * d0, h1 * u1 * d1);
            uw[i] = pack_bf16x2(h0 * a0, h1 * a1);
            hw[i] = pack_bf16x2(a0 * u0, a1 * u1);
            bad |= saved_nan(gs[i]) | saved_nan(us[i]);
          }
          if (bad) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              // (0x7fff is NaN in bf16 as well)
              const uint32_t m = saved_nan(gs[i]) | saved_nan(us[i]);
              const uint32_t nan = (m >> 15) * 0x7fffu;
              gw[i] |= nan;
              uw[i] |= nan;
              hw[i] |= nan;
            }
          }
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            st_shared_v4(out_piece(buf, lane, c0 + c), make_uint4(hw[4 * c], hw[4 * c + 1], hw[4 * c + 2], hw[4 * c + 3]));
            st_shared_v4(out_piece(buf + kOutBuf, lane, c0 + c),
                         make_uint4(gw[4 * c], gw[4 * c + 1], gw[4 * c + 2], gw[4 * c + 3]));
            st_shared_v4(out_piece(buf + 2 * kOutBuf, lane, c0 + c),
                         make_uint4(uw[4 * c], uw[4 * c + 1], uw[4 * c + 2], uw[4 * c + 3]));
          }
        } else if (f32) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
            st_shared_v4(out_piece(buf, lane, c), make_uint4(r[4 * c], r[4 * c + 1], r[4 * c + 2], r[4 * c + 3]));
        } else {
          if (kMode == MM_DOWN && reads) {
            const uint4 ra = ld_shared_v4(out_piece(buf, lane, c0)), rb = ld_shared_v4(out_piece(buf, lane, c0 + 1));
            const uint32_t rs[8] = {ra.x, ra.y, ra.z, ra.w, rb.x, rb.y, rb.z, rb.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              r[2 * i] = __float_as_uint(__uint_as_float(r[2 * i]) + __uint_as_float(rs[i] << 16));
              r[2 * i + 1] = __float_as_uint(__uint_as_float(r[2 * i + 1]) + __uint_as_float(rs[i] & 0xffff0000u));
            }
          }
          uint32_t w[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) w[i] = pack_bf16x2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1]));
#pragma unroll
          for (int c = 0; c < 2; ++c)
            st_shared_v4(out_piece(buf, lane, c0 + c), make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]));
        }

        if (closes) {
          __syncwarp();
          const int elt = f32 ? 4 : 2;
          const int xo = f32 ? x0 + s * 16 : x;
          put_rows(q.out, buf, lane, xo, y, q.M, q.N, q.ld, elt);
          if (kMode == MM_DH || (kMode == MM_UP && p.save)) {
            const int ld = kMode == MM_UP ? q.N : q.ld;
            put_rows(p.out_g, buf + kOutBuf, lane, xo, y, q.M, q.N, ld, 2);
            put_rows(p.out_u, buf + 2 * kOutBuf, lane, xo, y, q.M, q.N, ld, 2);
          }
        }
      }
    }
    __syncwarp();
  }

  tc_fence_before();
  __syncthreads();
  // a wait ran out: copies in flight, to this CTA or counted on its peer's
  // barriers, land before either retires
  if (*abort_flag) let_copies_land();
  // the pair's MMAs are complete and every access to the peer's barriers is
  // over before either CTA frees its TMEM
  cluster_sync_all();
  if (threadIdx.x == 0 && *abort_flag && p.dev_status) atomicOr(p.dev_status, kStatusTimeout);
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc_pair(tmem_base, 2 * kBN);
  }
}

// ------------------------------------------------------------------- host ---

// Collects a launch's tensor maps.
struct MapSet {
  MlpMaps maps;
  int n = 0;
  bool ok = true;
  int16_t add(bool good) {
    ok = ok && good;
    return static_cast<int16_t>(n++);
  }
  // operand [rows, cols] bf16 with K along the columns: boxes of `box` rows x 64
  int16_t k_major(const void* a, int64_t rows, int64_t cols, int64_t pitch, int box) {
    return add(encode_bf16_2d(&maps.m[n], a, cols, rows, 2 * pitch, kBK, box));
  }
  // operand [rows, cols] bf16 with K along the rows: boxes of 64 rows x 64
  int16_t mn_major(const void* a, int64_t rows, int64_t cols, int64_t pitch) {
    return add(encode_bf16_2d(&maps.m[n], a, cols, rows, 2 * pitch, 64, kBK));
  }
};

// Pairs of CTAs the device holds at once (at most one for two SMs): runs of cut
// tiles wait for one another, so the grid is never larger.
template <int kMode, int kAct, int kBN>
int resident_pairs(const Ctx& c) {
  static std::atomic<int> held[kMaxDevices];
  const bool cached = c.device >= 0 && c.device < kMaxDevices;
  int n = cached ? held[c.device].load(std::memory_order_acquire) - 1 : -1;
  if (n >= 0) return n;
  static std::atomic<int> done[kMaxDevices];
  constexpr int kSmem = Layout<kMode, kBN>::kSmem;
  if (!set_smem_once(reinterpret_cast<const void*>(mlp_gemm_kernel<kMode, kAct, kBN>), kSmem, c.device, done)) return 0;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * (c.num_sms / 2));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaOccupancyMaxActiveClusters(&n, mlp_gemm_kernel<kMode, kAct, kBN>, &cfg) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  n = std::min({n, c.num_sms / 2, kMlpMaxPairs});
  if (cached) held[c.device].store(n + 1, std::memory_order_release);
  return n;
}

// How a launch is cut up: tile width, tiles dealt whole or cut, pairs.
struct Plan {
  int bn, pairs;
  MlpSplit cut;
  double ns;  // estimate
};

// The estimate's terms, ns, by tile width: by mode, a K step of a pair, the least
// that a tile takes while all pairs' epilogues load and store, and the last tile's
// epilogue; the store of a piece and the wait for it, and each piece that a
// finisher adds.
struct Cost {
  double step[4], tile[4], tail[4], cut, piece;
};
constexpr Cost kCostWide{{290, 290, 290, 290}, {7000, 3300, 13000, 3300}, {4500, 3300, 6500, 3300}, 2500, 1800};
constexpr Cost kCostNarrow{{165, 165, 165, 185}, {4000, 1900, 7000, 2100}, {2500, 1900, 3500, 1900}, 2000, 1000};
constexpr double kClear = 3500;  // zeroing the flags, where no launch of the call has

// Deals the tiles to the pairs, whole ones, every product's last ones cut, or those
// of the products with long K steps only, by what is estimated to end first.  A run
// of short tiles takes as many epilogues (the backward of 7 rows, d = 1376, f = 3864,
// whose weight gradients have one K step a tile: 101 us where the estimate counted
// a run's K steps alone, 45 with the epilogues, both with dx in the launch).
Plan plan_tiles(const MlpParams& p, int mode, int bn, int pairs) {
  const Cost& k = bn == kWide ? kCostWide : kCostNarrow;
  const double step = k.step[mode];
  const int cols = mode == MM_UP ? bn / 2 : bn;
  int tiles[kMaxProbs], all = 0;
  double ns[kMaxProbs];  // of a whole tile
  for (int i = 0; i < p.n_prob; ++i) {
    tiles[i] = p.pr[i].mt * static_cast<int>(ceil_div(p.pr[i].N, cols));
    ns[i] = std::max(p.pr[i].ks * step, k.tile[mode]);
    all += tiles[i];
  }
  // The time of whole tiles dealt in turn: of the pair with the most to do.  A
  // product's last tiles go to neighbouring pairs, one each, from the pair on that
  // its first tile went to; so the most is found at one of those pairs.
  const auto in_turn = [&](const int* whole) {
    double most = 0;
    for (int j = 0, from = 0; j < p.n_prob; from = (from + whole[j++]) % pairs) {
      double load = 0;
      for (int i = 0, first = 0; i < p.n_prob; first = (first + whole[i++]) % pairs) {
        const int skip = from >= first ? from - first : from - first + pairs;
        load += (whole[i] / pairs + (skip < whole[i] % pairs ? 1 : 0)) * ns[i];
      }
      most = std::max(most, load);
    }
    return most;
  };
  Plan w{bn, std::min(pairs, all), {}, in_turn(tiles) + k.tail[mode]};
  w.cut.run = 1;
  for (int i = 0; i < p.n_prob; ++i) w.cut.whole[i] = tiles[i];
  w.cut.n_whole = all;
  // the last tiles cut: of every product, of those that are not bound by epilogues
  for (int some = 0; some < 2; ++some) {
    MlpSplit s = {};
    int64_t steps = 0;
    int longest = 0;
    double slow = step;  // a step of the shortest tiles
    for (int i = 0; i < p.n_prob; ++i) {
      const int rest = some && p.pr[i].ks * step <= k.tile[mode] ? 0 : tiles[i] % pairs;
      s.whole[i] = tiles[i] - rest;
      s.n_whole += s.whole[i];
      s.off[i] = static_cast<int>(steps);
      steps += static_cast<int64_t>(rest) * p.pr[i].ks;
      if (steps > (1 << 30)) return w;
      if (rest > 0) {
        longest = std::max(longest, p.pr[i].ks);
        slow = std::max(slow, ns[i] / p.pr[i].ks);
      }
    }
    if (steps == 0) continue;
    s.steps = static_cast<int>(steps);
    const double before = in_turn(s.whole);
    for (int m = 1; m <= 8; ++m) {  // longer runs on fewer pairs: fewer pieces
      s.run = static_cast<int>(ceil_div(steps * m, pairs));
      const double pieces = static_cast<double>(longest) / s.run;
      // the run that adds another tile's pieces, or the one of short tiles
      double t = before + k.tail[mode] + std::max(s.run * step + k.cut + k.piece * pieces, s.run * slow);
      if (mode == MM_UP || mode == MM_DH) t += kClear;
      if (t < w.ns) w = Plan{bn, s.n_whole > 0 ? pairs : static_cast<int>(ceil_div(steps, s.run)), s, t};
    }
  }
  return w;
}

// `zeroed`: an earlier launch of the call clears this one's flags.
template <int kMode, int kAct, int kBN>
olive_status launch_tiles(const Ctx& c, const MlpMaps& maps, MlpParams& p, const Plan& plan, bool zeroed) {
  p.cut = plan.cut;
  for (int i = 0; i < p.n_prob; ++i)
    p.pr[i].nt = static_cast<int>(ceil_div(p.pr[i].N, kMode == MM_UP ? kBN / 2 : kBN));
  if (p.cut.steps > 0 && !zeroed &&
      cudaMemsetAsync(p.flag, 0, 4 * mlp_flag_words(), c.stream) != cudaSuccess) {
    cudaGetLastError();
    return OLIVE_ERR_CUDA;
  }
  p.wait_limit_ns = c.wait_limit_ns;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * plan.pairs);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Layout<kMode, kBN>::kSmem;
  cfg.stream = c.stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  if (cudaLaunchKernelEx(&cfg, mlp_gemm_kernel<kMode, kAct, kBN>, maps, p) != cudaSuccess) {
    cudaGetLastError();
    return OLIVE_ERR_CUDA;
  }
  return OLIVE_OK;
}

// `fill(bn)` sets the launch's tensor maps for tiles of bn columns.
template <int kMode, int kAct = 0, class Fill>
olive_status launch(const Ctx& c, MlpParams& p, bool zeroed, Fill&& fill) {
  const int pairs = std::min(resident_pairs<kMode, kAct, kWide>(c), resident_pairs<kMode, kAct, kNarrow>(c));
  if (pairs < 1) return OLIVE_ERR_UNSUPPORTED_DEVICE;
  const Plan wide = plan_tiles(p, kMode, kWide, pairs);
  const Plan narrow = plan_tiles(p, kMode, kNarrow, pairs);
  const bool w = wide.ns <= narrow.ns;
  MapSet s;
  fill(s, w ? kWide : kNarrow);
  if (!s.ok) return OLIVE_ERR_CUDA;
  p.n_maps = s.n;
  return w ? launch_tiles<kMode, kAct, kWide>(c, s.maps, p, wide, zeroed)
           : launch_tiles<kMode, kAct, kNarrow>(c, s.maps, p, narrow, zeroed);
}

MlpProb problem(int M, int N, int K, int halves, void* out, int ld) {
  MlpProb q = {};
  q.out = out;
  q.M = M;
  q.N = N;
  q.ld = ld;
  q.mt = static_cast<int>(ceil_div(M, 2 * kBM));
  q.ks_half = static_cast<int>(ceil_div(K, kBK));
  q.ks = halves * q.ks_half;
  return q;
}

}  // namespace

size_t mlp_part_bytes() { return 4ull * kMlpMaxPairs * 2 * kEpiWarps * (kWide / 2 * 32); }
size_t mlp_flag_words() { return 2ull * kMlpMaxPairs; }

olive_status launch_mlp_fwd(const Ctx& c, const void* x, const void* W_gate, const void* W_up,
                            const void* W_down, const void* residual, int32_t T, int32_t d,
                            int32_t f, int act, void* y, void* saved, void* ws,
                            int32_t* dev_status) {
  const MlpWs w = carve_mlp(ws, T, f, false);
  if (mlp_few(T, f))
    return launch_mlp_few(c, x, W_gate, W_up, W_down, residual, T, d, f, act, y, saved, w.h, dev_status);
  const int fp = static_cast<int>(mlp_pitch(f));
  MlpParams p = {};
  p.n_prob = 1;
  p.part = w.part;
  p.dev_status = dev_status;

  p.pr[0] = problem(T, f, d, 1, w.h, fp);
  p.flag = w.flag;
  p.clear = w.flag + mlp_flag_words();
  p.n_clear = static_cast<int>(mlp_flag_words());
  p.save = saved != nullptr;
  p.out_g = saved;
  p.out_u = saved ? static_cast<uint16_t*>(saved) + static_cast<size_t>(T) * f : nullptr;
  auto up = [&](MapSet& s, int bn) {
    MlpProb& q = p.pr[0];
    q.a0 = q.a1 = s.k_major(x, T, d, d, kBM);
    q.b0 = s.k_major(W_gate, f, d, d, bn / 2);
    q.b1 = s.k_major(W_up, f, d, d, bn / 2);
  };
  const olive_status st = act == OLIVE_ACT_SILU ? launch<MM_UP, OLIVE_ACT_SILU>(c, p, false, up)
                                                : launch<MM_UP, OLIVE_ACT_GELU_TANH>(c, p, false, up);
  if (st != OLIVE_OK) return st;

  p.pr[0] = problem(T, d, f, 1, y, d);
  p.flag = w.flag + mlp_flag_words();
  p.n_clear = 0;
  p.residual = static_cast<const __nv_bfloat16*>(residual);
  return launch<MM_DOWN>(c, p, true, [&](MapSet& s, int bn) {
    MlpProb& q = p.pr[0];
    q.a0 = q.a1 = s.k_major(w.h, T, f, fp, kBM);
    q.b0 = q.b1 = s.k_major(W_down, d, f, f, bn / 2);
  });
}

olive_status launch_mlp_bwd(const Ctx& c, const void* dy, const void* x, const void* W_gate,
                            const void* W_up, const void* W_down, const void* saved, int32_t T,
                            int32_t d, int32_t f, int act, void* dx, void* dW_gate, void* dW_up,
                            void* dW_down, int grad_dtype, void* ws, int32_t* dev_status) {
  const MlpWs w = carve_mlp(ws, T, f, true);
  const int fp = static_cast<int>(mlp_pitch(f));
  MlpParams p = {};
  p.part = w.part;
  p.dev_status = dev_status;

  const bool few = T <= kMlpFewRows;
  olive_status st;
  if (few) {
    st = launch_mlp_few_bwd(c, dy, W_gate, W_up, W_down, saved, T, d, f, act, w, dx, grad_dtype, dev_status);
    dx = nullptr;  // (done)
    if (!dW_gate) return st;
  } else {
    p.n_prob = 1;
    p.pr[0] = problem(T, f, d, 1, w.h, fp);
    p.flag = w.flag;
    p.clear = w.flag + mlp_flag_words();
    p.n_clear = static_cast<int>(mlp_flag_words());
    p.saved_g = static_cast<const uint16_t*>(saved);
    p.saved_u = p.saved_g + static_cast<size_t>(T) * f;
    p.out_g = w.dg;
    p.out_u = w.du;
    auto dh = [&](MapSet& s, int) {
      MlpProb& q = p.pr[0];
      q.a0 = q.a1 = s.k_major(dy, T, d, d, kBM);
      q.b0 = q.b1 = s.mn_major(W_down, d, f, f);
    };
    st = act == OLIVE_ACT_SILU ? launch<MM_DH, OLIVE_ACT_SILU>(c, p, false, dh)
                               : launch<MM_DH, OLIVE_ACT_GELU_TANH>(c, p, false, dh);
  }
  if (st != OLIVE_OK) return st;

  p.n_prob = 0;
  p.flag = w.flag + mlp_flag_words();
  p.n_clear = 0;
  p.out_f32 = grad_dtype == OLIVE_DTYPE_F32;
  if (dx) p.pr[p.n_prob++] = problem(T, d, f, 2, dx, d);
  const int first = p.n_prob;
  if (dW_gate) {
    p.pr[p.n_prob++] = problem(f, d, T, 1, dW_gate, d);
    p.pr[p.n_prob++] = problem(f, d, T, 1, dW_up, d);
    p.pr[p.n_prob++] = problem(d, f, T, 1, dW_down, f);
  }
  return launch<MM_GRADS>(c, p, !few, [&](MapSet& s, int) {
    if (dx) {
      MlpProb& q = p.pr[0];
      q.a0 = s.k_major(w.dg, T, f, fp, kBM);
      q.a1 = s.k_major(w.du, T, f, fp, kBM);
      q.b0 = s.mn_major(W_gate, f, d, d);
      q.b1 = s.mn_major(W_up, f, d, d);
    }
    if (dW_gate) {
      const int16_t xm = s.mn_major(x, T, d, d);
      for (int i = 0; i < 2; ++i) {
        MlpProb& q = p.pr[first + i];
        q.a0 = q.a1 = s.mn_major(i ? w.du : w.dg, T, f, fp);
        q.b0 = q.b1 = xm;
        q.a_mn = 1;
      }
      MlpProb& q = p.pr[first + 2];
      q.a0 = q.a1 = s.mn_major(dy, T, d, d);
      q.b0 = q.b1 = s.mn_major(w.h, T, f, fp);
      q.a_mn = 1;
    }
  });
}

}  // namespace olive
