// packed_attention.cuh -- what the forward and backward of attention inside packed
// sequences share: the work's tiles, the scores' forms and the operands in shared memory.
#pragma once

#include <type_traits>

#include "internal.h"
#include "sm103.cuh"

namespace olive {

constexpr int kAttTile = 128;                   // rows of a query or key tile
constexpr int kBoxBytes = kAttTile * 64 * 2;    // a tile's 64 columns in shared memory
constexpr int kStatusOffsets = 1 << OLIVE_ERR_OFFSETS;
constexpr int kStatusTimeout = 1 << OLIVE_ERR_TIMEOUT;
constexpr float kAttLog2e = 1.4426950408889634f;
constexpr float kAttLn2 = 0.6931471805599453f;

// Offsets as they may be used: inside [0, T] and not falling.
__device__ __forceinline__ int cu_at(const AttArgs& p, int s) { return min(max(p.cu[s], 0), p.T); }

// The sequence of a tile slot.  With tiles of R rows sequence s has its slots from
// cu[s] / R + s on: one more than R divides its length into, at least as many as it
// has tiles.  So a slot's sequence is found without a sum over those before it.  All
// lanes of a warp search together, 32 sequences a step.
struct Seq {
  int start, n, prefix, tile;  // first token, tokens, those seen by all, tile in it
};
// Keys of a sequence that all its rows see: none where the end given is before it, all where
// it is behind.  (Compared before it is subtracted from: an end near -2^31 must not wrap.)
__device__ __forceinline__ int prefix_of(const AttArgs& p, int s, const Seq& q) {
  return p.prefix_end ? min(max(p.prefix_end[s], q.start) - q.start, q.n) : 0;
}
// `near`: a sequence at or before it, looked from first (items come in rising order), so
// that one load, of 32 sequences' offsets, does for most.
template <int R>
__device__ __forceinline__ Seq seq_of_slot(const AttArgs& p, int slot, int& near) {
  const int lane = threadIdx.x & 31;
  int cu, first;
  uint32_t got;
  const auto look = [&](int from) {  // which of the 32 sequences from there on begin at or before the slot
    first = from;
    cu = cu_at(p, min(first + lane, p.S));
    got = __ballot_sync(0xffffffffu, first + lane < p.S && cu / R + first + lane <= slot);
  };
  look(near);
  if (got == 0 || (got >> 31) != 0) {
    int lo = 0, hi = p.S;  // the last s in [lo, hi) whose slots begin at or before this one
    while (hi - lo > 1) {
      const int step = (hi - lo + 31) / 32;
      const int s = lo + step * lane;
      const uint32_t before = __ballot_sync(0xffffffffu, s < hi && cu_at(p, s) / R + s <= slot);
      // (offsets that fall set a status bit; the highest lane keeps the search going)
      lo = lo + step * (before ? 31 - __clz(before) : 0);
      hi = min(hi, lo + step);
    }
    look(lo);
    got = 1;
  }
  const int last = 31 - __clz(got);
  near = first + last;
  Seq q;
  q.start = __shfl_sync(0xffffffffu, cu, last);
  const int end = max(q.start, __shfl_sync(0xffffffffu, cu, last + 1));
  q.n = end - q.start;
  q.prefix = prefix_of(p, near, q);
  q.tile = slot - (q.start / R + near);
  if (q.tile < 0 || static_cast<int64_t>(q.tile) * R >= q.n) q.tile = -1;
  return q;
}
inline int64_t att_slots(int64_t T, int64_t S, int R) { return T / R + S; }

// Keys that row i of a sequence sees: always its first ones.
__device__ __forceinline__ int keys_seen(const AttArgs& p, const Seq& q, int i) {
  return p.causal ? min(max(i + 1, q.prefix), q.n) : q.n;
}

// Offsets that do not describe the batch (a warp).
__device__ __forceinline__ void check_offsets(const AttArgs& p) {
  const int lane = threadIdx.x & 31;
  bool bad = lane == 0 && p.cu[0] != 0;
  for (int s = lane; s < p.S; s += 32) {
    const int a = p.cu[s], b = p.cu[s + 1];
    bad |= a < 0 || b < a || b > p.T;
  }
  if (bad && p.dev_status) atomicOr(p.dev_status, kStatusOffsets);
}
// Part `part` of `parts` of the rows behind the last sequence, zeroed (a warp).
__device__ __forceinline__ void zero_behind(const AttArgs& p, const HeadsView& x, int heads, int64_t part, int64_t parts) {
  const int first = cu_at(p, p.S), vecs = p.D / 8;
  const int64_t n = static_cast<int64_t>(p.T - first) * heads * vecs;
  for (int64_t i = part * 32 + (threadIdx.x & 31); i < n; i += parts * 32) {
    const int64_t row = i / vecs;
    __nv_bfloat16* at = static_cast<__nv_bfloat16*>(const_cast<void*>(x.x)) + (first + row / heads) * x.token_stride +
                        (row % heads) * x.head_stride;
    reinterpret_cast<uint4*>(at)[i % vecs] = make_uint4(0, 0, 0, 0);
  }
}

// The items of a launch, one a block; a block that is done takes over blocks that have
// not started.  One warp asks, finds the item's sequence and hands it to the others
// through a ring in shared memory.  What is claimed early cannot be taken by blocks that
// run dry, so a block asks when the copies of its last item are issued (two tiles before
// its end); where items are so short that asking and searching would show, it asks while
// the ring of kItems has room; and where there is an SM for every item it does not ask.
enum { ASK_NEVER = 0, ASK_LATE = 2, ASK_EARLY = 4 };  // and the entries of the ring in use
constexpr int kItems = 4;
constexpr int64_t kParts = 1024;  // items that also zero a part of the rows behind the last sequence
template <class Item>
struct ItemRing {
  alignas(16) uint32_t answer[4];
  Item item[kItems];
};
// Barriers: `taken`, `issued` (an item's copies), full [kItems], empty [kItems].
constexpr int kRingBars = 2 + 2 * kItems;
struct RingAt {
  uint32_t bars;
  __device__ __forceinline__ uint32_t taken() const { return bars; }
  __device__ __forceinline__ uint32_t issued() const { return bars + 8; }
  __device__ __forceinline__ uint32_t full(uint32_t n) const { return bars + 16 + 8 * (n % kItems); }
  __device__ __forceinline__ uint32_t empty(uint32_t n) const { return bars + 16 + 8 * kItems + 8 * (n % kItems); }
};
__device__ __forceinline__ void init_ring(const RingAt& r, int readers) {
  mbar_init(r.taken(), 1);
  mbar_init(r.issued(), 1);
  for (int i = 0; i < kItems; ++i) {
    mbar_init(r.full(i), 1);
    mbar_init(r.empty(i), readers);
  }
}
// A wait's limit is that of a tile, a microsecond or two of work: who waits for an item of
// `steps` tiles as a whole has as many.  (Where the work itself is stuck, those who do it
// give up after one, and everybody sees their flag.)
__device__ __forceinline__ WaitCtl for_steps(const WaitCtl& ctl, int steps) {
  const uint64_t n = 1 + static_cast<uint64_t>(steps);
  return {ctl.abort, __umul64hi(ctl.limit_ns, n) == 0 ? ctl.limit_ns * n : ~0ull};  // (a limit that means none stays one)
}
// The warp that hands out items.  find(i, item) says whether item i exists; rest(i) is
// what else is done for every i, after the item is out.
template <class Item, class Find, class Rest>
__device__ __forceinline__ void hand_out(ItemRing<Item>& ring, const RingAt& at, int ask, const WaitCtl& ctl, Find find, Rest rest) {
  const int lane = threadIdx.x & 31;
  const uint32_t answer = smem_u32(ring.answer);
  uint32_t n = 0, asked = 0;
  int most = 0;  // steps of an item so far
  bool ok = true, pending = false;
  const auto put_question = [&] {
    if (lane == 0) {
      fence_proxy_async_shared();
      mbar_arrive_expect_tx(at.taken(), 16);
      take_block(answer, at.taken());
    }
    __syncwarp();
    pending = true;
  };
  int i = blockIdx.x;
  while (i >= 0) {
    // (early: the next answer is on its way while this item's sequence is looked up)
    if (ask == ASK_EARLY) put_question();
    Item it;
    const bool there = find(i, it);
    if (there) {
      if (!(ok = mbar_wait_warp(at.empty(n), (n / kItems & 1) ^ 1, for_steps(ctl, most)))) break;
      most = max(most, it.length());
      if (lane == 0) ring.item[n % kItems] = it;
      __syncwarp();
      if (lane == 0) mbar_arrive(at.full(n));
      ++n;
    }
    rest(i);
    if (ask == ASK_NEVER) break;
    if (ask == ASK_LATE) {
      if (there && !(ok = mbar_wait_warp(at.issued(), (n - 1) & 1, for_steps(ctl, most)))) break;
      put_question();
    }
    if (!(ok = mbar_wait_warp(at.taken(), asked++ & 1, ctl))) break;
    pending = false;
    i = warp_uniform(taken_block(answer));
  }
  if (pending) let_copies_land();
  if (ok && mbar_wait_warp(at.empty(n), (n / kItems & 1) ^ 1, for_steps(ctl, most)) && lane == 0) {
    ring.item[n % kItems].end = 1;
    mbar_arrive(at.full(n));
  }
  __syncwarp();
}
// A reader's next item; false: there is none (or the block gives up, ok = false).
// kUniform: for a warp that issues copies or MMAs, whose operands follow from it.  (The
// exchange by which the compiler learns that takes some 30 cycles a word.)
template <bool kUniform, class Item>
__device__ __forceinline__ bool next_item(const ItemRing<Item>& ring, const RingAt& at, uint32_t& n, Item& it,
                                          const WaitCtl& ctl, bool& ok) {
  if (!(ok = mbar_wait_warp(at.full(n), n / kItems & 1, ctl))) return false;
  if constexpr (kUniform)
    it = warp_uniform_copy(&ring.item[n % kItems]);
  else
    it = ring.item[n % kItems];
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(at.empty(n));
  ++n;
  return it.end == 0;
}
inline int when_to_ask(int64_t items, int sms, int64_t T, int64_t S) {
  return items <= sms ? ASK_NEVER : T / S <= 256 ? ASK_EARLY : ASK_LATE;
}

// tanh(x) = 1 - 2 / (1 + e^2x), x in units of ln 2 / 2: off by some 2^-23 (2^-21 at
// most), which is times the cap in a score: up to kWideCap as little as a product's own
// fp32 sum.
constexpr float kWideCap = 64.f;
__device__ __forceinline__ float tanh_of(float x2) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + fast_exp2(x2)));
  return fmaf(-2.f, r, 1.f);
}
// Two at once for |x| <= kSmallTanh: x times a polynomial in x^2, fitted to tanh(x) / x at
// Chebyshev nodes of [0, 0.5] (off by 2^-25 of it at most, before rounding).  A score as
// most are takes half the time: the exact form's three special functions an element, four
// cycles each, are what bounds a capped tile.
constexpr float kSmallTanh = 0.7f;
__device__ __forceinline__ uint64_t small_tanh_pair(uint64_t x) {
  const uint64_t y = mul_pair(x, x);
  const auto k = [](float v) { return pair(v, v); };
  uint64_t r = fma_pair(y, k(-0.005041549913585186f), k(0.019973110407590866f));
  r = fma_pair(y, r, k(-0.05350660905241966f));
  r = fma_pair(y, r, k(0.13328121602535248f));
  r = fma_pair(y, r, k(-0.3333311676979065f));
  return mul_pair(x, fma_pair(y, r, k(1.f)));
}
// Two for wide caps, each by its own size: off by a part of itself, however small it is.
// (Both forms are computed and one is selected: as a condition it became a branch an
// element, a tenth slower where most scores are near the cap.  With the exact form for
// small ones too a cap of 1e6 was off by 0.09 in the tiles that it took, one of 1e9 by the
// score.)
__device__ __forceinline__ float select_above(float size, float than, float yes, float no) {
  float r;
  asm("{\n\t.reg .pred p;\n\tsetp.gt.f32 p, %1, %2;\n\tselp.f32 %0, %3, %4, p;\n\t}" : "=f"(r) : "f"(size), "f"(than), "f"(yes), "f"(no));
  return r;
}
__device__ __forceinline__ uint64_t wide_tanh_pair(uint64_t x) {
  float a, b, s, t;
  unpair(x, a, b);
  unpair(small_tanh_pair(x), s, t);
  return pair(select_above(fabsf(a), kSmallTanh, tanh_of(a * (2.f * kAttLog2e)), s),
              select_above(fabsf(b), kSmallTanh, tanh_of(b * (2.f * kAttLog2e)), t));
}
// How scores are formed from products: as they are, lowered with the distance, or
// capped (and lowered, by a slope that may be 0), by a cap up to kWideCap or a wider one.
// In base 2.  (The wide caps' form in place of the other, forward, us.  A cap of 1, 8
// sequences of 4096, 32 + 8 heads of 128: 3235 and 1812.  All scores small: these 1392 and
// 1338; 200 sequences of 41, 16 + 16 heads of 64: 63 and 55.)
enum { FORM_PLAIN = 0, FORM_BIAS = 1, FORM_CAP = 2, FORM_WIDE = 3 };
constexpr bool is_capped(int form) { return form == FORM_CAP || form == FORM_WIDE; }
struct ScoreForm {
  float scale2, in_cap, cap2;
  // (a cap above 1e30 bends no score that one of 1e30 does not, but its reciprocal loses
  // bits; that of one near 0 must not be infinite, as 0 times it is a NaN)
  __device__ __forceinline__ explicit ScoreForm(const AttArgs& p)
      : scale2(p.scale * kAttLog2e), in_cap(p.cap > 0.f ? fminf(p.scale / fminf(p.cap, 1e30f), 1e37f) : 0.f),
        cap2(fminf(p.cap, 1e30f) * kAttLog2e) {}
  // One score of a product at a distance.
  __device__ __forceinline__ float at(float s, float slope2, float dist) const {
    float x = s * scale2;
    if (cap2 > kWideCap * kAttLog2e) {
      float t, same;
      unpair(wide_tanh_pair(pair(s * in_cap, s * in_cap)), t, same);
      x = cap2 * t;
    } else if (cap2 > 0.f) {
      x = cap2 * tanh_of(s * (2.f * kAttLog2e * in_cap));
    }
    return fmaf(-slope2, dist, x);
  }
};
__device__ __forceinline__ float largest(const uint32_t (&s)[32]) {
  float top = 0.f;
#pragma unroll
  for (int e = 0; e < 32; ++e) top = fmaxf(top, fabsf(__uint_as_float(s[e])));
  return top;
}
// Whether a warp's products, none larger than `top`, take the small form.  Asked of whole
// tiles and of a sequence's own rows alone: what lies behind it must not decide in which
// form, so with which rounding, its scores are formed.  (With a wide cap a score's form is
// its own, and this only a shorter way to the same bits.)
__device__ __forceinline__ bool all_small(const ScoreForm& f, float top) { return __all_sync(0xffffffffu, top * f.in_cap <= kSmallTanh); }
// Whether each of a warp's rows has `cols` columns on one side of its own, before it or
// behind: then the distance is linear in the column, one instruction a score in place of
// two and half of one.
__device__ __forceinline__ bool one_side(float far, int cols) {
  return __all_sync(0xffffffffu, far <= 0.f || far >= static_cast<float>(cols - 1));
}
// 32 products to scores, column e at the distance |far - e| (kEven: all on one side, or all
// capped ones small); with kBend the derivatives of the cap, in pairs.
template <int kForm, bool kBend, bool kEven>
__device__ __forceinline__ void form_scores(const ScoreForm& f, uint32_t (&s)[32], float slope2, float far, uint64_t (&bend)[kBend ? 16 : 1]) {
  if constexpr (is_capped(kForm)) {
    if constexpr (kEven || kForm == FORM_WIDE) {
      const uint64_t in = pair(f.in_cap, f.in_cap), out = pair(f.cap2, f.cap2), one = pair(1.f, 1.f), minus = pair(-1.f, -1.f);
#pragma unroll
      for (int e = 0; e < 32; e += 2) {
        const uint64_t x2 = mul_pair(pair(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), in);
        const uint64_t t = kEven ? small_tanh_pair(x2) : wide_tanh_pair(x2);
        if constexpr (kBend) bend[e / 2] = fma_pair(mul_pair(t, minus), t, one);
        float x, y;
        unpair(mul_pair(t, out), x, y);
        s[e] = __float_as_uint(x);
        s[e + 1] = __float_as_uint(y);
      }
    } else {
      const float in = 2.f * kAttLog2e * f.in_cap;
#pragma unroll
      for (int e = 0; e < 32; e += 2) {
        const float t = tanh_of(__uint_as_float(s[e]) * in), u = tanh_of(__uint_as_float(s[e + 1]) * in);
        if constexpr (kBend) bend[e / 2] = pair(fmaf(-t, t, 1.f), fmaf(-u, u, 1.f));
        s[e] = __float_as_uint(f.cap2 * t);
        s[e + 1] = __float_as_uint(f.cap2 * u);
      }
    }
  }
  // (a bias is there in FORM_BIAS: scaled and lowered in one instruction)
  if constexpr (kForm == FORM_BIAS && kEven) {
    const float per = far > 0.f ? slope2 : -slope2, first = -per * far;
    const uint64_t scale = pair(f.scale2, f.scale2);
#pragma unroll
    for (int e = 0; e < 32; e += 2) {
      float x, y;
      unpair(fma_pair(pair(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), scale, pair(fmaf(per, e, first), fmaf(per, e + 1, first))), x, y);
      s[e] = __float_as_uint(x);
      s[e + 1] = __float_as_uint(y);
    }
  } else if constexpr (kForm == FORM_BIAS) {
#pragma unroll
    for (int e = 0; e < 32; ++e) s[e] = __float_as_uint(fmaf(-slope2, fabsf(far - e), __uint_as_float(s[e]) * f.scale2));
  } else if (slope2 != 0.f) {
#pragma unroll
    for (int e = 0; e < 32; ++e) s[e] = __float_as_uint(fmaf(-slope2, fabsf(far - e), __uint_as_float(s[e])));
  }
}

// A tile of up to 128 columns into shared memory: boxes of 64 columns.
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, uint32_t bar, int boxes, int head, int token) {
  for (int b = 0; b < boxes; ++b) tma_load_3d(dst + b * kBoxBytes, map, bar, 64 * b, head, token);
}

// Rows [from, to) of a tile in shared memory zeroed by a warp.  Rows behind a sequence
// are another's (or nobody's, uninitialised): their weight is 0, but 0 times a NaN is one.
__device__ __forceinline__ void zero_rows(uint32_t tile, int boxes, int from, int to) {
  const int lane = threadIdx.x & 31;
  for (int b = 0; b < boxes; ++b)
    for (int i = from * 8 + lane; i < to * 8; i += 32) st_shared_v4(tile + b * kBoxBytes + i * 16, make_uint4(0, 0, 0, 0));
}

// A place in a ring of barriers and its phase.
struct Turn {
  int i = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next(int n) {
    if (++i == n) {
      i = 0;
      phase ^= 1;
    }
  }
};

// The end of an MMA warp: what it issued is complete before the CTA retires (a wait that
// ignores the abort flag: MMAs in flight end by themselves).
__device__ __forceinline__ void drain_mmas(uint32_t bar, bool leader, uint64_t limit_ns) {
  if (leader) umma_commit(bar);
  volatile int keep_waiting = 0;
  const uint64_t floor_ns = 200ull * 1000 * 1000;
  const WaitCtl own{&keep_waiting, limit_ns > floor_ns ? limit_ns : floor_ns};
  mbar_wait_warp(bar, 0, own);
  __syncwarp();
}

__device__ __forceinline__ int up16(int n) { return (n + 15) & ~15; }

// The products of a whole warp, `leader` the lane that issues: with the loop and the
// operands the warp's they stay in uniform registers (sm103.cuh, mbar_wait_warp).  An MMA
// takes some 33 cycles to issue and 65 to run; a bound that is looked at before each
// doubles the first, so every number of K steps has its own copy.
//
// S = A B^T over a head's width: both operands tiles of rows (K-major).
template <int kSteps>
__device__ __forceinline__ void mma_rows_of(bool leader, uint32_t d, uint64_t da, uint64_t db, uint32_t idesc) {
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
    const uint32_t at = (k >> 2) * (kBoxBytes >> 4) + (k & 3) * 2;
    umma_bf16_by(leader, d, da + at, db + at, idesc, k > 0 ? 1u : 0u);
  }
}
// f of a number of K steps, 1 to 8, as a constant.
template <class F>
__device__ __forceinline__ void by_steps(int steps, F f) {
  if (steps == 8) return f(std::integral_constant<int, 8>{});
  switch (steps) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 3: return f(std::integral_constant<int, 3>{});
    case 4: return f(std::integral_constant<int, 4>{});
    case 5: return f(std::integral_constant<int, 5>{});
    case 6: return f(std::integral_constant<int, 6>{});
    case 7: return f(std::integral_constant<int, 7>{});
  }
}
__device__ __forceinline__ void mma_rows(bool leader, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, int steps) {
  const uint64_t da = sdesc_sw128(a, 16, 1024), db = sdesc_sw128(b, 16, 1024);
  by_steps(steps, [&](auto n) { mma_rows_of<decltype(n)::value>(leader, d, da, db, idesc); });
}
// D (+)= A B with A [128, rows of B] in tensor memory and B a tile of rows (MN-major).  kRun K steps of A are side by side, the next run 16 kRun columns on.
template <int kRun>
__device__ __forceinline__ uint32_t a_step(int k) { return (k / kRun) * (16 * kRun) + (k % kRun) * 8; }
template <int kRun, int kFrom, int kTo>
__device__ __forceinline__ void mma_cols_of(bool leader, uint32_t d, uint32_t a, uint64_t db, uint32_t idesc, uint32_t first) {
#pragma unroll
  for (int k = kFrom; k < kTo; ++k)
    umma_bf16_ta_by(leader, d, a + a_step<kRun>(k), db + k * 128, idesc, k > 0 ? 1u : first);
}
template <int kRun>
__device__ __forceinline__ void mma_cols(bool leader, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, int steps, bool more) {
  const uint64_t db = sdesc_sw128(b, kBoxBytes, 1024);
  const uint32_t first = more ? 1u : 0u;
  by_steps(steps, [&](auto n) { mma_cols_of<kRun, 0, decltype(n)::value>(leader, d, a, db, idesc, first); });
}

}  // namespace olive
