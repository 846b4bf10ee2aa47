// packed_attention.cu -- attention inside packed sequences, forward.
//
//   z_ij = scale q_i . k_j,  s_ij = cap tanh(z_ij / cap) - slope |i - j|,
//   o_i = sum over the keys j that i sees of exp(s_ij - lse_i) v_j
//
// What a row sees is always its sequence's first keys (up to itself, its prompt's end
// or the sequence's end), so a mask is one number a row.
//
// A CTA works on two slots of 128 query rows, two heads of a key head or two tiles of a
// head (or two heads each with its own keys, where sequences are short), and walks the key tiles from the last that a row sees to
// the first (scores that a bias lowers with the distance are largest at its beginning, so
// a row's reference stays):
//   warp 0     TMA: query tiles, then key and value tiles into rings of three and two
//   warp 1     MMA: S = Q K^T into tensor memory, O += P V with P read from there, the
//              slots in turn (a warp for each: their products mix, both slots' rows then
//              wait at once; 922 us in place of 833 at that step, sizes as below)
//   warp 3     hands out items
//   warps 4-7, 8-11  the rows of slot 0 and 1, one a thread: the running maximum and
//              sum, P = exp2(S - reference) in bf16 over S in tensor memory.
// While one slot's rows are exponentiated the other's products run.  A row's reference
// follows its maximum only when that is more than 32 (in log2) above, as O has to be
// scaled then; until there P and the sum are relative to the old one, exactly (bf16 and
// fp32 hold 2^32 times a row's length), so a tile's exponentials do not wait for its maximum.
//
// Bound by the chain S, rows, P V of a slot and, in long runs, by the power cap: 8 sequences
// of 4096, 32 + 8 heads of 128, causal: 760 us, 1.45 PFLOP/s counted (tensor pipe active 58 %
// of a shorter launch's cycles).  One sequence of 20011, 8 + 2 heads, with a bias: 575 us,
// 1.43 PFLOP/s (704 from the first key tile to the last, where every tile raises the
// reference; 770 with two and a half instructions more a score).  200 sequences of some 41
// tokens, 16 + 16 heads of 64: 51 us, latency, and two thirds of a tile's rows nobody's.
// 5003 tokens in 7 sequences, 15 + 3 heads of 96, capped: 73 us, 47 without the cap: tiles
// that some row does not see whole go through tensor memory once more, and capped scores
// there take three special functions each.
#include <algorithm>
#include <type_traits>

#include "packed_attention.cuh"

namespace olive {
namespace {

constexpr int kThreads = 384;
constexpr int kRegsLaunch = 168, kRegsSoft = 208, kRegsRest = 88;
static_assert(2 * kRegsSoft + kRegsRest <= 3 * kRegsLaunch, "the block's registers");
constexpr int kK = 3, kV = 2;  // stages of key and value tiles
constexpr int kTmaWarp = 0, kMmaWarp = 1, kItemWarp = 3, kRestWarps = 4;
constexpr int kReaders = 10;
constexpr float kLag = 32.f;
enum { B_QFULL = 0, B_QEMPTY = 2, B_KFULL = 4, B_KEMPTY = B_KFULL + kK, B_VFULL = B_KEMPTY + kK, B_VEMPTY = B_VFULL + kV,
       B_VFIX = B_VEMPTY + kV, B_SFULL = B_VFIX + kV, B_PREADY = B_SFULL + 2, B_OFULL = B_PREADY + 4, B_OEMPTY = B_OFULL + 2,
       B_DRAIN = B_OEMPTY + 2, B_RING, B_COUNT = B_RING + kRingBars };

// What an item's two slots are: two tiles of a head, two heads of a key head, or two heads
// whose keys and values are loaded apart.
enum { PAIR_TILES = 0, PAIR_HEADS = 1, PAIR_APART = 2 };
constexpr int rows_of(int pair) { return pair == PAIR_TILES ? 256 : 128; }
// An item's slots: heads, first rows and key tiles.
struct Item {
  Seq q;
  int kv_head[2], head[2], row0[2], tiles[2], seen[2];  // seen: keys that the slot's last row sees
  int end;
  __device__ __forceinline__ int length() const { return max(tiles[0], tiles[1]); }
};
constexpr int kMisc = 16 + static_cast<int>(sizeof(ItemRing<Item>));
constexpr int smem_bytes(int boxes) {
  return 1024 + (2 + kK + kV) * boxes * kBoxBytes + (8 * B_COUNT + 15) / 16 * 16 + kMisc;
}
template <int kPair>
__device__ __forceinline__ bool item_at(const AttArgs& p, int i, int units, Item& it, int& near) {
  const int slot = i / units, u = i % units;
  constexpr int R = rows_of(kPair);
  it.q = seq_of_slot<R>(p, slot, near);
  if (it.q.tile < 0) return false;
  // the longest rows first
  const int tile = p.causal ? (it.q.n + R - 1) / R - 1 - it.q.tile : it.q.tile;
  const int per = p.Hq / p.Hk;
#pragma unroll
  for (int a = 0; a < 2; ++a) {
    it.head[a] = kPair == PAIR_TILES ? u : 2 * u + a;
    it.row0[a] = kPair == PAIR_TILES ? tile * 256 + a * 128 : tile * 128;
    const bool there = it.row0[a] < it.q.n && (kPair != PAIR_APART || it.head[a] < p.Hq);
    it.seen[a] = there ? keys_seen(p, it.q, min(it.row0[a] + 128, it.q.n) - 1) : 0;
    it.tiles[a] = (it.seen[a] + 127) / 128;
    it.kv_head[a] = it.head[a] / per;
  }
  it.end = 0;
  return true;
}

template <int kBoxes, int kPair, int kForm>
__global__ void __launch_bounds__(kThreads, 1)
    att_fwd_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                   const __grid_constant__ CUtensorMap map_v, const AttArgs p, int units, int ask) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  constexpr uint32_t kTileBytes = kBoxes * kBoxBytes;
  const uint32_t sq = base, sk = sq + 2 * kTileBytes, sv = sk + kK * kTileBytes;
  const uint32_t bar0 = sv + kV * kTileBytes;
  uint8_t* misc = smem_raw + (bar0 - raw) + (8 * B_COUNT + 15) / 16 * 16;
  ItemRing<Item>& ring = *reinterpret_cast<ItemRing<Item>*>(misc + 16);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(misc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 4);
  const auto bar = [&](int i) { return bar0 + 8u * i; };
  const RingAt ring_at{bar(B_RING)};
  const int warp = warp_uniform(static_cast<int>(threadIdx.x >> 5)), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < B_RING; ++i) {
      const auto among = [&](int first, int n) { return i >= first && i < first + n; };
      mbar_init(bar(i), among(B_PREADY, 4) || among(B_OEMPTY, 2) ? 4 : 1);
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

  if (warp < kRestWarps) {
    regs_dec<kRegsRest>();
    if (warp == kTmaWarp) {
      const bool leader = elect_one();
      uint32_t n_q[2] = {0, 0};
      Turn k, v;
      bool ok = true;
      for (uint32_t n = 0; ok && next_item<true>(ring, ring_at, n, it, ctl, ok);) {
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
        const auto first_key = [&](int j) { return 128 * (tiles - 1 - j); };
        const auto keys = [&](int j, int a) {
          if (!mbar_wait_warp(bar(B_KEMPTY + k.i), k.phase ^ 1, ctl)) return false;
          if (leader) {
            mbar_arrive_expect_tx(bar(B_KFULL + k.i), kTileBytes);
            load_tile(sk + k.i * kTileBytes, &map_k, bar(B_KFULL + k.i), kBoxes, p.k.head_stride ? it.kv_head[a] : 0, it.q.start + first_key(j));
          }
          k.next(kK);
          return true;
        };
        const auto values = [&](const Turn& to, int j, int a) {
          if (!mbar_wait_warp(bar(B_VEMPTY + to.i), to.phase ^ 1, ctl)) return false;
          if (leader) {
            mbar_arrive_expect_tx(bar(B_VFULL + to.i), kTileBytes);
            load_tile(sv + to.i * kTileBytes, &map_v, bar(B_VFULL + to.i), kBoxes, p.v.head_stride ? it.kv_head[a] : 0, it.q.start + first_key(j));
          }
          return true;
        };
        // the sequence's last rows: what follows them up to whole K steps is zeroed
        const auto last_values = [&](const Turn& at, int j) {
          const int rows = seen - first_key(j);
          if (rows < 128 && rows % 16 != 0) {
            if (!mbar_wait_warp(bar(B_VFULL + at.i), at.phase, ctl)) return false;
            if (it.q.n - first_key(j) < 128) zero_rows(sv + at.i * kTileBytes, kBoxes, rows, up16(rows));
            fence_proxy_async_shared();
            __syncwarp();
            if (leader) mbar_arrive(bar(B_VFIX + at.i));
          }
          return true;
        };
        if constexpr (kPair == PAIR_APART) {
          const bool two = it.tiles[1] > 0;
          if (!(ok = query(0) && keys(0, 0) && (!two || (query(1) && keys(0, 1))))) break;
          for (int j = 0; j < tiles; ++j) {
            if (j + 1 < tiles && !(ok = keys(j + 1, 0) && (!two || keys(j + 1, 1)))) break;
            const Turn v0 = v;
            v.next(kV);
            const Turn v1 = v;
            if (two) v.next(kV);
            if (!(ok = values(v0, j, 0) && (!two || values(v1, j, 1)) && last_values(v0, j) && (!two || last_values(v1, j)))) break;
          }
        } else {
          if (!(ok = query(0) && keys(0, 0) && query(1))) break;
          for (int j = 0; j < tiles; ++j, v.next(kV)) {
            // (keys a tile ahead: V's stage is free only after the round before)
            if (j + 1 < tiles && !(ok = keys(j + 1, 0))) break;
            if (!(ok = values(v, j, 0) && last_values(v, j))) break;
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
      uint32_t n_q[2] = {0, 0}, n_p[2] = {0, 0}, n_o[2] = {0, 0}, fixed = 0;
      Turn k, v;
      bool ok = true;
      for (uint32_t n = 0; ok && next_item<true>(ring, ring_at, n, it, ctl, ok);) {
        const int tiles = max(it.tiles[0], it.tiles[1]), seen = max(it.seen[0], it.seen[1]);
        if constexpr (kPair == PAIR_APART) {  // (short sequences: most have one tile)
          const int left = up16(min(128, seen - 128 * (tiles - 1)));  // of the first round's tile, the sequence's last
          for (int j = 0; ok && j <= tiles; ++j) {
            const auto keys_at = [&](int i) { return i == 0 ? left : 128; };
#pragma unroll
            for (int a = 0; a < 2; ++a) {
              if (it.tiles[a] == 0) continue;
              if (j > 0) {
                if (j == 1 && !(ok = mbar_wait_warp(bar(B_OEMPTY + a), (n_o[a]++ & 1) ^ 1, ctl))) break;
                const Phase of[2] = {{bar(B_PREADY + 2 * a + 1), n_p[a]++ & 1}, {bar(B_VFULL + v.i), v.phase}};
                if (!(ok = mbar_wait_warp(of, ctl))) break;
                if (j == 1 && seen % 16 != 0) {
                  if (!(ok = mbar_wait_warp(bar(B_VFIX + v.i), fixed >> v.i & 1, ctl))) break;
                  fixed ^= 1u << v.i;
                }
                tc_fence_after();
                mma_cols<8>(leader, t_o(a), t_s(a), sv + v.i * kTileBytes, id_out, keys_at(j - 1) / 16, j > 1);
                umma_commit_by(leader, bar(B_VEMPTY + v.i));
                v.next(kV);
                if (j == tiles) umma_commit_by(leader, bar(B_OFULL + a));
              }
              if (j < tiles) {
                if (j == 0 && !(ok = mbar_wait_warp(bar(B_QFULL + a), n_q[a]++ & 1, ctl))) break;
                if (!(ok = mbar_wait_warp(bar(B_KFULL + k.i), k.phase, ctl))) break;
                tc_fence_after();
                mma_rows(leader, t_s(a), sq + a * kTileBytes, sk + k.i * kTileBytes, idesc_bf16(128, keys_at(j), false, false), steps);
                umma_commit_by(leader, bar(B_SFULL + a));
                umma_commit_by(leader, bar(B_KEMPTY + k.i));
                k.next(kK);
                if (j == tiles - 1) umma_commit_by(leader, bar(B_QEMPTY + a));
              }
            }
          }
          continue;
        }
        // A round: O += P V of the tile before and S of this one, slot 0, then slot 1.
        // (A wait takes some 100 cycles where nothing is waited for, and what is queued
        // for the tensor pipe lasts 300: so tiles are waited for together with the rows,
        // and P's second half while the first one's products run.)
        if (!(ok = mbar_wait_warp(bar(B_KFULL + k.i), k.phase, ctl))) break;
        // a slot's first round; those from `even` on: both slots have whole tiles
        const int begin[2] = {tiles - it.tiles[0], tiles - it.tiles[1]}, even = tiles - min(it.seen[0], it.seen[1]) / 128;
        const auto keys_of = [&](int a, int j) { return up16(min(128, it.seen[a] - 128 * (tiles - 1 - j))); };
        const auto whole_rounds = [&](auto s_steps, int& j) {
          constexpr int kS = decltype(s_steps)::value;
          constexpr uint32_t id_s = idesc_bf16(128, 128, false, false);
          const uint64_t dq[2] = {sdesc_sw128(sq, 16, 1024), sdesc_sw128(sq + kTileBytes, 16, 1024)};
          for (; j < tiles; ++j) {
            const uint64_t dk = sdesc_sw128(sk + k.i * kTileBytes, 16, 1024), dv = sdesc_sw128(sv + v.i * kTileBytes, kBoxBytes, 1024);
            Turn next_k = k;
            next_k.next(kK);
#pragma unroll
            for (int a = 0; a < 2; ++a) {
              const uint32_t more = j - 1 > begin[a] ? 1u : 0u;
              const Phase of[2] = {{bar(B_PREADY + 2 * a), n_p[a] & 1},
                                   a == 0 ? Phase{bar(B_VFULL + v.i), v.phase} : Phase{bar(B_KFULL + next_k.i), next_k.phase}};
              if (a == 0 || j + 1 < tiles ? !mbar_wait_warp(of, ctl) : !mbar_wait_warp(of[0].bar, of[0].parity, ctl)) return false;
              tc_fence_after();
              mma_cols_of<8, 0, 4>(leader, t_o(a), t_s(a), dv, id_out, more);
              if (!mbar_wait_warp(bar(B_PREADY + 2 * a + 1), n_p[a]++ & 1, ctl)) return false;
              tc_fence_after();
              mma_cols_of<8, 4, 8>(leader, t_o(a), t_s(a), dv, id_out, 1u);
              mma_rows_of<kS>(leader, t_s(a), dq[a], dk, id_s);
              umma_commit_by(leader, bar(B_SFULL + a));
              if (j == tiles - 1) umma_commit_by(leader, bar(B_QEMPTY + a));
            }
            umma_commit_by(leader, bar(B_VEMPTY + v.i));
            umma_commit_by(leader, bar(B_KEMPTY + k.i));
            v.next(kV);
            k = next_k;
          }
          return true;
        };
        for (int j = 0; ok && j <= tiles; ++j) {
          if (j > even && j < tiles && steps >= 4) {
#pragma unroll
            for (int a = 0; ok && a < 2; ++a)
              if (j - 1 == begin[a]) ok = mbar_wait_warp(bar(B_OEMPTY + a), (n_o[a]++ & 1) ^ 1, ctl);
            if (!ok) break;
            if constexpr (kBoxes == 1)
              ok = whole_rounds(std::integral_constant<int, 4>{}, j);
            else
              ok = steps == 8   ? whole_rounds(std::integral_constant<int, 8>{}, j)
                   : steps == 6 ? whole_rounds(std::integral_constant<int, 6>{}, j)
                   : steps == 5 ? whole_rounds(std::integral_constant<int, 5>{}, j)
                                : whole_rounds(std::integral_constant<int, 7>{}, j);
            if (!ok) break;
          }
          Turn next_k = k;
          if (j < tiles) next_k.next(kK);
          bool have_v = false, have_k = j + 1 >= tiles;
#pragma unroll
          for (int a = 0; a < 2; ++a) {
            if (j > begin[a]) {
              if (j - 1 == begin[a] && !(ok = mbar_wait_warp(bar(B_OEMPTY + a), (n_o[a]++ & 1) ^ 1, ctl))) break;
              const Phase rows = {bar(B_PREADY + 2 * a + 1), n_p[a]++ & 1};  // (P's second half: then the first is there too)
              if (!have_v) {
                const Phase of[2] = {rows, {bar(B_VFULL + v.i), v.phase}};
                if (!(ok = mbar_wait_warp(of, ctl))) break;
                const int left = seen - 128 * (tiles - j);
                if (left < 128 && left % 16 != 0) {
                  if (!(ok = mbar_wait_warp(bar(B_VFIX + v.i), fixed >> v.i & 1, ctl))) break;
                  fixed ^= 1u << v.i;
                }
                have_v = true;
              } else if (!have_k) {
                const Phase of[2] = {rows, {bar(B_KFULL + next_k.i), next_k.phase}};
                if (!(ok = mbar_wait_warp(of, ctl))) break;
                have_k = true;
              } else if (!(ok = mbar_wait_warp(rows.bar, rows.parity, ctl))) {
                break;
              }
              tc_fence_after();
              mma_cols<8>(leader, t_o(a), t_s(a), sv + v.i * kTileBytes, id_out, keys_of(a, j - 1) / 16, j - 1 > begin[a]);
              if (j == tiles) umma_commit_by(leader, bar(B_OFULL + a));
            }
            if (j >= begin[a] && j < tiles) {
              if (j == begin[a] && !(ok = mbar_wait_warp(bar(B_QFULL + a), n_q[a]++ & 1, ctl))) break;
              tc_fence_after();
              const uint32_t id = idesc_bf16(128, keys_of(a, j), false, false);
              mma_rows(leader, t_s(a), sq + a * kTileBytes, sk + k.i * kTileBytes, id, steps);
              umma_commit_by(leader, bar(B_SFULL + a));
              if (j == tiles - 1) umma_commit_by(leader, bar(B_QEMPTY + a));
            }
          }
          if (!ok) break;
          if (j > 0) umma_commit_by(leader, bar(B_VEMPTY + v.i));
          if (j < tiles) umma_commit_by(leader, bar(B_KEMPTY + k.i));
          if (j > 0) v.next(kV);
          k = next_k;
          if (!have_k && !(ok = mbar_wait_warp(bar(B_KFULL + k.i), k.phase, ctl))) break;
        }
      }
      drain_mmas(bar(B_DRAIN), leader, p.wait_limit_ns);
    } else if (warp == kItemWarp) {
      int near = 0;
      hand_out(ring, ring_at, ask, ctl, [&](int i, Item& item) { return item_at<kPair>(p, i, units, item, near); },
               [&](int i) {
                 if (i == 0) check_offsets(p);
                 const int64_t parts = min(static_cast<int64_t>(gridDim.x), kParts);
                 if (i >= parts) return;
                 zero_behind(p, p.o, p.Hq, i, parts);
                 const int first = cu_at(p, p.S), rows = p.T - first;
                 if (p.lse)
                   for (int64_t e = static_cast<int64_t>(i) * 32 + lane; e < static_cast<int64_t>(rows) * p.Hq; e += parts * 32)
                     p.lse[e / rows * p.T + first + e % rows] = __uint_as_float(0xff800000u);
               });
    }
  } else {
    regs_inc<kRegsSoft>();
    const int a = (warp - kRestWarps) >> 2;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const int row = (warp & 3) * 32 + lane;
    const uint32_t ts = t_s(a) + lanes, to = t_o(a) + lanes;
    const ScoreForm form(p);
    uint32_t n_s = 0, n_o = 0;
    bool ok = true;
    for (uint32_t n = 0; ok && next_item<false>(ring, ring_at, n, it, ctl, ok);) {
      const int tiles = a ? it.tiles[1] : it.tiles[0];
      if (tiles == 0) {  // (the other slot's rows are worked on: all of them, before the next item is out)
        ok = mbar_wait_warp(ring_at.full(n), n / kItems & 1, for_steps(ctl, it.length()));
        continue;
      }
      const int head = a ? it.head[1] : it.head[0];
      const int pos = (a ? it.row0[1] : it.row0[0]) + row;
      const int lim = keys_seen(p, it.q, min(pos, it.q.n - 1));
      const float slope2 = kForm != FORM_PLAIN && p.slopes ? p.slopes[head] * kAttLog2e : 0.f;
      const int my_seen = a ? it.seen[1] : it.seen[0];
      // keys that all the warp's rows see; whether it has any
      const int whole = warp_uniform(keys_seen(p, it.q, min(pos - lane, it.q.n - 1)));
      const bool live = warp_uniform(static_cast<int>(pos - lane < it.q.n));
      const float mul = kForm == FORM_PLAIN ? form.scale2 : 1.f;
      float ref = 0.f, sum = 0.f;
      for (int j = tiles - 1; j >= 0; --j) {
        if (!(ok = mbar_wait_warp(bar(B_SFULL + a), n_s++ & 1, ctl))) break;
        tc_fence_after();
        const auto arrive = [&](int h) {  // P's half h is there
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(B_PREADY + 2 * a + h));
        };
        const int here = lim - 128 * j;
        const float far = static_cast<float>(pos - 128 * j);
        // the reference follows the maximum m
        const auto follow = [&](float m) {
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
        };
        if (!live) {  // (rows behind the sequence: nobody's)
          arrive(0);
          arrive(1);
          continue;
        }
        uint32_t s[4][32];
        bool at_once = 128 * (j + 1) <= whole;
        if constexpr (kForm == FORM_BIAS) at_once = at_once && one_side(far, 128);
        if (at_once) {
#pragma unroll
          for (int c = 0; c < 4; ++c) tmem_ld_32x32b_x32(ts + 32 * c, s[c]);
          tmem_ld_wait();
          if constexpr (is_capped(kForm))
            at_once = all_small(form, pos < it.q.n ? fmaxf(fmaxf(largest(s[0]), largest(s[1])), fmaxf(largest(s[2]), largest(s[3]))) : 0.f);
        }
        if (at_once) {
          if constexpr (kForm != FORM_PLAIN) {
            uint64_t none[1];
#pragma unroll
            for (int c = 0; c < 4; ++c) form_scores<kForm, false, true>(form, s[c], slope2, far - 32 * c, none);
          }
          float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int e = 0; e < 32; ++e)
#pragma unroll
            for (int c = 0; c < 4; ++c) top[c] = fmaxf(top[c], __uint_as_float(s[c][e]));
          const float m = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * mul;
          if (j == tiles - 1) ref = m > -INFINITY ? m : 0.f;
          uint64_t part[2];
          uint32_t w[2][32];
          const auto weights = [&](int h) {  // of half the columns
            const uint64_t mul2 = pair(mul, mul), off2 = pair(-ref, -ref);
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const int c = 2 * h + (e >> 4), k = 2 * (e & 15);
              float x, y;
              unpair(fma_pair(pair(__uint_as_float(s[c][k]), __uint_as_float(s[c][k + 1])), mul2, off2), x, y);
              x = fast_exp2(x);
              y = fast_exp2(y);
              part[e & 1] = add_pair(part[e & 1], pair(x, y));
              w[h][e] = pack_bf16x2(x, y);
            }
          };
          const auto begin = [&] {
            part[0] = pair(sum, 0.f);
            part[1] = pair(0.f, 0.f);
            weights(0);
          };
          begin();
          if (__any_sync(0xffffffffu, m > ref + kLag)) {
            follow(m);
            begin();
          }
          tmem_st_32x32b_x32(ts, w[0]);
          arrive(0);
          weights(1);
          tmem_st_32x32b_x32(ts + 32, w[1]);
          arrive(1);
          float x, y;
          unpair(add_pair(part[0], part[1]), x, y);
          sum = x + y;
        } else {
          // A tile that some row does not see whole (or some score is near its cap), 32
          // columns at a time and only those that some row of the slot sees: scores as they are formed and masked go back
          // to tensor memory, P follows them there.  (A loop: sequences of some forty
          // tokens run this once an item, where unrolled code takes as long to fetch.)
          const int chunks = min(4, (my_seen - 128 * j + 31) / 32);
          float m = -INFINITY;
#pragma unroll 1
          for (int c = 0; c < chunks; ++c) {
            uint32_t s[32];
            tmem_ld_32x32b_x32(ts + 32 * c, s);
            tmem_ld_wait();
            const int seen = here - 32 * c;
            uint64_t none[1];
            bool small = false;
            if constexpr (kForm == FORM_WIDE) {
              float top = 0.f;
#pragma unroll
              for (int e = 0; e < 32; ++e) top = fmaxf(top, e < seen ? fabsf(__uint_as_float(s[e])) : 0.f);
              small = all_small(form, pos < it.q.n ? top : 0.f);
              if (small) form_scores<kForm, false, true>(form, s, slope2, far - 32 * c, none);
            }
            if constexpr (kForm != FORM_PLAIN)
              if (!small) form_scores<kForm, false, false>(form, s, slope2, far - 32 * c, none);
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const float x = e < seen ? __uint_as_float(s[e]) : -INFINITY;
              m = fmaxf(m, x);
              s[e] = __float_as_uint(x);
            }
            tmem_st_32x32b_x32(ts + 32 * c, s);
          }
          tmem_st_wait();
          m *= mul;
          if (j == tiles - 1) ref = m > -INFINITY ? m : 0.f;
          if (__any_sync(0xffffffffu, m > ref + kLag)) follow(m);
          const uint64_t mul2 = pair(mul, mul), off2 = pair(-ref, -ref);
          uint64_t part = pair(sum, 0.f);
#pragma unroll 1
          for (int c = 0; c < chunks; ++c) {
            uint32_t s[32], w[16];
            tmem_ld_32x32b_x32(ts + 32 * c, s);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              float x, y;
              unpair(fma_pair(pair(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1])), mul2, off2), x, y);
              x = fast_exp2(x);
              y = fast_exp2(y);
              part = add_pair(part, pair(x, y));
              w[e] = pack_bf16x2(x, y);
            }
            tmem_st_32x32b_x16(ts + 16 * c, w);
          }
          float x, y;
          unpair(part, x, y);
          sum = x + y;
          arrive(0);
          arrive(1);
        }
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

template <int kBoxes, int kPair, int kForm>
olive_status run_fwd(const Ctx& c, const AttArgs& a) {
  CUtensorMap mq, mk, mv;
  if (!encode_heads(&mq, a.q, a.T, a.Hq, a.D) || !encode_heads(&mk, a.k, a.T, a.Hk, a.D) || !encode_heads(&mv, a.v, a.T, a.Hk, a.D))
    return OLIVE_ERR_CUDA;
  static std::atomic<int> done[kMaxDevices];
  const auto kernel = att_fwd_kernel<kBoxes, kPair, kForm>;
  constexpr int kSmem = smem_bytes(kBoxes);
  if (!set_smem_once(reinterpret_cast<const void*>(kernel), kSmem, c.device, done)) return OLIVE_ERR_CUDA;
  const int units = kPair == PAIR_TILES ? a.Hq : (a.Hq + 1) / 2;
  const int64_t items = att_slots(a.T, a.S, rows_of(kPair)) * units;
  kernel<<<static_cast<unsigned>(items), kThreads, kSmem, c.stream>>>(mq, mk, mv, a, units,
                                                                     when_to_ask(items, c.num_sms, a.T, a.S));
  return cudaGetLastError() == cudaSuccess ? OLIVE_OK : OLIVE_ERR_CUDA;
}

template <int kBoxes, int kPair>
olive_status by_form(const Ctx& c, const AttArgs& a) {
  if (a.cap > 0.f) return a.cap > kWideCap ? run_fwd<kBoxes, kPair, FORM_WIDE>(c, a) : run_fwd<kBoxes, kPair, FORM_CAP>(c, a);
  return a.slopes ? run_fwd<kBoxes, kPair, FORM_BIAS>(c, a) : run_fwd<kBoxes, kPair, FORM_PLAIN>(c, a);
}

// Two heads of a key head where their number is even: K and V are loaded once for both.
// Else two tiles of a head, or two heads apart where sequences are so short that the second
// tile is mostly empty, or causal and so short that items of 256 rows end too unevenly.
// (8192 tokens, two tiles and apart, us.  16 + 16 heads of 64 in sequences of 41: 59 and 45;
// of 128 in 128 that see all: 49 and 53, 1024: 77 and 86; causal 256: 64 and 53, 384: 57 and
// 49, 1024: 66 and 67.)
bool heads_apart(const AttArgs& a) { return a.Hq > 1 && a.T / a.S < (a.causal ? 512 : 128); }
template <int kBoxes>
olive_status by_heads(const Ctx& c, const AttArgs& a) {
  if (a.Hq / a.Hk % 2 == 0) return by_form<kBoxes, PAIR_HEADS>(c, a);
  return heads_apart(a) ? by_form<kBoxes, PAIR_APART>(c, a) : by_form<kBoxes, PAIR_TILES>(c, a);
}

}  // namespace

olive_status launch_att_fwd(const Ctx& c, const AttArgs& a) {
  return a.D <= 64 ? by_heads<1>(c, a) : by_heads<2>(c, a);
}

}  // namespace olive
