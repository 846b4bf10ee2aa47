// packed_attention.cuh -- what the forward and backward of attention inside packed
// sequences share: the work's tiles, the scores' forms and the operands in shared memory.
#pragma once

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
template <int R>
__device__ __forceinline__ Seq seq_of_slot(const AttArgs& p, int slot) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = p.S;  // the last s in [lo, hi) whose slots begin at or before this one
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32;
    const int s = lo + step * lane;
    const bool before = s < hi && cu_at(p, s) / R + s <= slot;
    const uint32_t got = __ballot_sync(0xffffffffu, before);
    // (offsets that fall set a status bit; the highest lane keeps the search going)
    const int last = got ? 31 - __clz(got) : 0;
    lo = lo + step * last;
    hi = min(hi, lo + step);
  }
  Seq q;
  q.start = cu_at(p, lo);
  const int end = max(q.start, cu_at(p, lo + 1));
  q.n = end - q.start;
  q.prefix = p.prefix_end ? min(max(p.prefix_end[lo] - q.start, 0), q.n) : 0;
  q.tile = slot - (q.start / R + lo);
  if (q.tile < 0 || static_cast<int64_t>(q.tile) * R >= q.n) q.tile = -1;
  return q;
}
inline int64_t att_slots(int64_t T, int64_t S, int R) { return T / R + S; }

// Keys that row i of a sequence sees: always its first ones.
__device__ __forceinline__ int keys_seen(const AttArgs& p, const Seq& q, int i) {
  return p.causal ? min(max(i + 1, q.prefix), q.n) : q.n;
}

// Offsets that do not describe the batch, and outputs behind the last sequence.
__device__ __forceinline__ void check_offsets(const AttArgs& p) {
  if (blockIdx.x != 0) return;
  bool bad = threadIdx.x == 0 && p.cu[0] != 0;
  for (int s = threadIdx.x; s < p.S; s += blockDim.x) {
    const int a = p.cu[s], b = p.cu[s + 1];
    bad |= a < 0 || b < a || b > p.T;
  }
  if (bad && p.dev_status) atomicOr(p.dev_status, kStatusOffsets);
}
__device__ __forceinline__ void zero_behind(const AttArgs& p, void* x, int64_t token_stride, int64_t head_stride, int heads) {
  const int first = cu_at(p, p.S), vecs = p.D / 8;
  const int64_t n = static_cast<int64_t>(p.T - first) * heads * vecs;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * blockDim.x) {
    const int64_t row = i / vecs;
    __nv_bfloat16* at = static_cast<__nv_bfloat16*>(x) + (first + row / heads) * token_stride + (row % heads) * head_stride;
    reinterpret_cast<uint4*>(at)[i % vecs] = make_uint4(0, 0, 0, 0);
  }
}

// tanh(x) = 1 - 2 / (1 + e^2x), x in units of ln 2 / 2: off by some 2^-23, which is
// times the cap in a score.
__device__ __forceinline__ float tanh_of(float x2) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + fast_exp2(x2)));
  return fmaf(-2.f, r, 1.f);
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

__device__ __forceinline__ int up16(int n) { return (n + 15) & ~15; }

// S = A B^T over a head's width: both operands tiles of rows (K-major).
__device__ __forceinline__ void mma_rows(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, int steps) {
  const uint64_t da = sdesc_sw128(a, 16, 1024), db = sdesc_sw128(b, 16, 1024);
#pragma unroll 1
  for (int k = 0; k < steps; ++k) {
    const uint32_t at = (k >> 2) * (kBoxBytes >> 4) + (k & 3) * 2;
    umma_bf16(d, da + at, db + at, idesc, k > 0 ? 1u : 0u);
  }
}
// D (+)= A B with A [128, rows of B] in tensor memory and B a tile of rows (MN-major);
// A's second 64 columns lie `half` tensor memory columns behind its first.
__device__ __forceinline__ void mma_cols(uint32_t d, uint32_t a, int half, uint32_t b, uint32_t idesc, int steps, bool more) {
  const uint64_t db = sdesc_sw128(b, kBoxBytes, 1024);
#pragma unroll 1
  for (int k = 0; k < steps; ++k)
    umma_bf16_ta(d, a + (k >> 2) * half + (k & 3) * 8, db + k * 128, idesc, more || k > 0 ? 1u : 0u);
}

}  // namespace olive
