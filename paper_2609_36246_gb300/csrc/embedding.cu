// embedding.cu -- rows of the embedding looked up by packed ids and scaled, and the
// gradient of the embedding by sorted tokens.
//
// The gradient of row v is the sum of the output's gradients at the tokens that name
// v.  So that the sum has a fixed order, the tokens are sorted by id (a stable radix
// sort, 9 bits a pass: two passes up to a vocabulary of 2^18) and the sorted list is
// cut into units of equal size whatever the ids' frequencies.  A warp walks a unit for
// 256 columns and adds up runs of equal ids; a run inside the unit is a row's whole
// gradient, and what belongs to a run that crosses a unit's ends is stored in fp32 and
// added in the units' order by a last launch.  Rows that no token names are zeroed by
// blocks of the same launch, found in a bitmap that the sort leaves.
//
// Bound by memory.  32768 tokens of a vocabulary of 151936, rows of 4096 in bf16: look-up 64
// us, gradient 262 us (5.8 TB/s over dy and dW), of which the sort is some 25 (its launches,
// and the counts that every block reads) and the joins 10 to 20.  9001 tokens, 4097 rows of
// 1000 in fp32: 13 and 39 us, six launches in a chain, each starting under the one ahead
// (51 us where each waits for the last one's end).
#include <algorithm>

#include "internal.h"
#include "sm103.cuh"

namespace olive {
namespace {

constexpr int kStatusToken = 1 << OLIVE_ERR_TOKEN_RANGE;
constexpr int kDigit = 9, kBins = 1 << kDigit;
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kLookThreads = 256;
constexpr int kSumThreads = 128, kSumCols = 8 * kSumThreads;  // columns of a block
constexpr int kJoinThreads = 256;

// Eight values.
template <typename T>
struct Run;
template <>
struct Run<__nv_bfloat16> {
  using Raw = uint4;
  static __device__ __forceinline__ void get(const Raw& r, float (&v)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ Raw put(const float (&v)[8]) {
    return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                      pack_bf16x2(v[6], v[7]));
  }
};
template <>
struct Run<float> {
  struct alignas(16) Raw {
    float4 a, b;
  };
  static __device__ __forceinline__ void get(const Raw& r, float (&v)[8]) {
    v[0] = r.a.x, v[1] = r.a.y, v[2] = r.a.z, v[3] = r.a.w;
    v[4] = r.b.x, v[5] = r.b.y, v[6] = r.b.z, v[7] = r.b.w;
  }
  static __device__ __forceinline__ Raw put(const float (&v)[8]) {
    return {make_float4(v[0], v[1], v[2], v[3]), make_float4(v[4], v[5], v[6], v[7])};
  }
};

__device__ __forceinline__ int ids_in_use(const EmbArgs& p) {
  return p.n_ids ? min(max(*p.n_ids, 0), p.T) : p.T;
}

// Forward: a thread copies kLookVecs vectors of eight, a block's width apart.
constexpr int kLookVecs = 4;
template <typename T>
__global__ void __launch_bounds__(kLookThreads) look_up_kernel(const EmbArgs p) {
  using V = Run<T>;
  using Raw = typename V::Raw;
  const int nv = p.d / 8;
  const int64_t all = static_cast<int64_t>(p.T) * nv;
  const int64_t i0 = static_cast<int64_t>(blockIdx.x) * (kLookThreads * kLookVecs) + threadIdx.x;
  const int n = ids_in_use(p);
  Raw raw[kLookVecs];
  int state[kLookVecs];  // 0: zeros, 1: a row, 2: none of that id
#pragma unroll
  for (int k = 0; k < kLookVecs; ++k) {
    const int64_t i = i0 + k * kLookThreads;
    state[k] = 0;
    if (i >= all) continue;
    const int t = i >> 32 ? static_cast<int>(i / nv) : static_cast<int>(static_cast<uint32_t>(i) / static_cast<uint32_t>(nv));
    const int at = static_cast<int>(i - static_cast<int64_t>(t) * nv);
    if (t >= n) continue;
    const int id = p.ids[t];
    const bool fine = id >= 0 && id < p.V;
    state[k] = fine ? 1 : 2;
    if (fine) raw[k] = static_cast<const Raw*>(p.W)[static_cast<size_t>(id) * nv + at];
    if (!fine && at == 0 && p.dev_status) atomicOr(p.dev_status, kStatusToken);
  }
#pragma unroll
  for (int k = 0; k < kLookVecs; ++k) {
    const int64_t i = i0 + k * kLookThreads;
    if (i >= all) continue;
    float v[8] = {};
    if (state[k] == 1) V::get(raw[k], v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = state[k] == 2 ? __uint_as_float(0x7fffffffu) : v[e] * p.scale;
    static_cast<Raw*>(p.out)[i] = V::put(v);
  }
}

// A token's sort key: its id, or V (behind all ids) where it has none.
__device__ __forceinline__ uint32_t first_key(const EmbArgs& p, int n, int t, bool report) {
  if (t >= n) return p.V;
  const int id = p.ids[t];
  const bool fine = id >= 0 && id < p.V;
  if (!fine && report && p.dev_status) atomicOr(p.dev_status, kStatusToken);
  return fine ? id : p.V;
}

// How often each digit occurs in a block's tile, and (first pass) the bitmap cleared.
template <bool kFirst>
__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(const EmbArgs p, EmbSort s, const uint32_t* keys, int shift, int tile) {
  __shared__ uint32_t count[kBins];
  grid_launch_dependents();
  if (threadIdx.x < kBins) count[threadIdx.x] = 0;
  if (!kFirst) grid_wait();
  if constexpr (kFirst) {
    const int words = (p.V - 1) / 32 + 1;
    for (int w = blockIdx.x * kSortThreads + threadIdx.x; w < words; w += gridDim.x * kSortThreads) s.named[w] = 0;
  }
  const int n = kFirst ? ids_in_use(p) : 0;
  __syncthreads();
  const int64_t first = static_cast<int64_t>(blockIdx.x) * tile;
  const int64_t end = min(first + tile, static_cast<int64_t>(p.T));
  for (int64_t i = first + threadIdx.x; i < end; i += kSortThreads) {
    const uint32_t key = kFirst ? first_key(p, n, static_cast<int>(i), true) : keys[i];
    atomicAdd(&count[(key >> shift) & (kBins - 1)], 1u);
  }
  __syncthreads();
  if (threadIdx.x < kBins) s.table[static_cast<size_t>(blockIdx.x) * kBins + threadIdx.x] = count[threadIdx.x];
}

// Marks the rows of a warp's keys, one atomic a word of the bitmap.  (One a key: the words
// of the frequent tokens took 8 us.)
__device__ __forceinline__ void name_rows(const EmbArgs& p, const EmbSort& s, uint32_t key) {
  const bool real = key < static_cast<uint32_t>(p.V);
  const uint32_t word = real ? key >> 5 : 0xffffffffu;
  const uint32_t same = __match_any_sync(0xffffffffu, word);
  const uint32_t bits = __reduce_or_sync(same, 1u << (key & 31));
  if (real && (same & ((1u << (threadIdx.x & 31)) - 1)) == 0) atomicOr(&s.named[word], bits);
}

// A block moves its tile: an entry goes behind all of lower digits, those of its digit
// in earlier blocks, in earlier warps of this one, and earlier ones of its warp.
template <bool kFirst, bool kLast>
__global__ void __launch_bounds__(kSortThreads) sort_move_kernel(const EmbArgs p, EmbSort s, const uint32_t* keys, const int32_t* pos,
                                                                 uint32_t* keys_out, int32_t* pos_out, int shift, int tile) {
  extern __shared__ uint32_t per_warp[];  // [kSortWarps][kBins]
  __shared__ uint32_t base[kBins];
  __shared__ uint32_t warp_total[kBins / 32];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  grid_launch_dependents();
  for (int i = threadIdx.x; i < kSortWarps * kBins; i += kSortThreads) per_warp[i] = 0;
  grid_wait();
  uint32_t total = 0, before = 0;
  if (threadIdx.x < kBins) {
#pragma unroll 4
    for (int b = 0; b < static_cast<int>(gridDim.x); ++b) {
      const uint32_t c = s.table[static_cast<size_t>(b) * kBins + threadIdx.x];
      before += b < static_cast<int>(blockIdx.x) ? c : 0;
      total += c;
    }
    uint32_t sum = total;  // up to this digit
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += v;
    }
    if (lane == 31) warp_total[warp] = sum;
    base[threadIdx.x] = sum - total + before;
  }
  __syncthreads();
  if (threadIdx.x < kBins) {
    uint32_t more = 0;
    for (int w = 0; w < warp; ++w) more += warp_total[w];
    base[threadIdx.x] += more;
  }
  // each warp a run of the tile, 32 entries at a time
  const int n = kFirst ? ids_in_use(p) : 0;
  const int run = tile / kSortWarps;
  const int64_t first = static_cast<int64_t>(blockIdx.x) * tile + static_cast<int64_t>(warp) * run;
  uint32_t* mine = per_warp + warp * kBins;
  for (int r = 0; r < run; r += 32) {
    const int64_t i = first + r + lane;
    const bool in = i < p.T;
    const uint32_t key = !in ? 0u : kFirst ? first_key(p, n, static_cast<int>(i), false) : keys[i];
    const uint32_t d = in ? (key >> shift) & (kBins - 1) : kBins;
    const uint32_t same = __match_any_sync(0xffffffffu, d);
    if (in && (same & ((1u << lane) - 1)) == 0) mine[d] += __popc(same);
    __syncwarp();
  }
  __syncthreads();
  if (threadIdx.x < kBins) {
    uint32_t sum = base[threadIdx.x];
#pragma unroll 4
    for (int w = 0; w < kSortWarps; ++w) {
      const uint32_t c = per_warp[w * kBins + threadIdx.x];
      per_warp[w * kBins + threadIdx.x] = sum;
      sum += c;
    }
  }
  __syncthreads();
  for (int r = 0; r < run; r += 32) {
    const int64_t i = first + r + lane;
    const bool in = i < p.T;
    const uint32_t key = !in ? 0u : kFirst ? first_key(p, n, static_cast<int>(i), false) : keys[i];
    const uint32_t d = in ? (key >> shift) & (kBins - 1) : kBins;
    const uint32_t same = __match_any_sync(0xffffffffu, d);
    const uint32_t at = in ? mine[d] + __popc(same & ((1u << lane) - 1)) : 0;
    __syncwarp();
    if (in && (same & ((1u << lane) - 1)) == 0) mine[d] += __popc(same);
    __syncwarp();
    if (in) {
      keys_out[at] = key;
      pos_out[at] = kFirst ? static_cast<int32_t>(i) : pos[i];
    }
    if (kLast) name_rows(p, s, in ? key : 0xffffffffu);
  }
}

// Up to kOneBlock tokens: all passes in one block, keys and tokens in shared memory; a
// thread takes its entries (a warp a run of the list, 32 at a time) into registers and
// puts them where they belong.
constexpr int kOneBlock = 4096;  // (9001 in one block: 26 us, in four launches 21)
constexpr int kOneSmem = 8 * kOneBlock + 4 * kSortWarps * kBins;
template <int kItems>
__global__ void __launch_bounds__(kSortThreads) sort_one_kernel(const EmbArgs p, EmbSort s, int passes) {
  extern __shared__ uint32_t one_smem[];
  uint32_t* keys = one_smem;
  int32_t* pos = reinterpret_cast<int32_t*>(one_smem + kItems * kSortThreads);
  uint32_t* per_warp = one_smem + 2 * kItems * kSortThreads;  // [kSortWarps][kBins]
  __shared__ uint32_t warp_total[kBins / 32];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  grid_launch_dependents();
  const int n = ids_in_use(p);
  uint32_t key[kItems];
  int32_t at[kItems];
  const int first = warp * 32 * kItems + lane;
  for (int w = threadIdx.x; w < (p.V - 1) / 32 + 1; w += kSortThreads) s.named[w] = 0;
#pragma unroll
  for (int r = 0; r < kItems; ++r) {
    at[r] = first + 32 * r;
    key[r] = at[r] < p.T ? first_key(p, n, at[r], true) : 0xffffffffu;  // (behind all: the last of every digit)
  }
  uint32_t* mine = per_warp + warp * kBins;
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * kDigit;
    for (int i = threadIdx.x; i < kSortWarps * kBins; i += kSortThreads) per_warp[i] = 0;
    __syncthreads();
    uint32_t rank[kItems];
#pragma unroll
    for (int r = 0; r < kItems; ++r) {
      const uint32_t d = (key[r] >> shift) & (kBins - 1);
      const uint32_t same = __match_any_sync(0xffffffffu, d);
      rank[r] = mine[d] + __popc(same & ((1u << lane) - 1));
      __syncwarp();
      if ((same & ((1u << lane) - 1)) == 0) mine[d] += __popc(same);
      __syncwarp();
    }
    __syncthreads();
    // before each warp's entries of a digit: those of lower digits and of earlier warps
    uint32_t sum = 0;
    if (threadIdx.x < kBins) {
#pragma unroll 8
      for (int w = 0; w < kSortWarps; ++w) {
        const uint32_t c = per_warp[w * kBins + threadIdx.x];
        per_warp[w * kBins + threadIdx.x] = sum;
        sum += c;
      }
      uint32_t up = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(0xffffffffu, up, o);
        if (lane >= o) up += v;
      }
      if (lane == 31) warp_total[warp] = up;
      sum = up - sum;
    }
    __syncthreads();
    if (threadIdx.x < kBins) {
      for (int w = 0; w < warp; ++w) sum += warp_total[w];
#pragma unroll 8
      for (int w = 0; w < kSortWarps; ++w) per_warp[w * kBins + threadIdx.x] += sum;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kItems; ++r) {
      const uint32_t to = mine[(key[r] >> shift) & (kBins - 1)] + rank[r];
      keys[to] = key[r];
      pos[to] = at[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kItems; ++r) {
      key[r] = keys[first + 32 * r];
      at[r] = pos[first + 32 * r];
    }
  }
#pragma unroll
  for (int r = 0; r < kItems; ++r) {
    const int i = first + 32 * r;
    if (i >= p.T) continue;
    s.buf_keys[0][i] = key[r];
    s.buf_pos[0][i] = at[r];
    if (i == 0 || keys[i - 1] != key[r]) {
      if (key[r] < static_cast<uint32_t>(p.V)) atomicOr(&s.named[key[r] >> 5], 1u << (key[r] & 31));
    }
  }
}

// acc (scaled) into eight columns of a row of the gradient.
template <typename O>
__device__ __forceinline__ void put_row(const EmbArgs& p, uint32_t row, int col, const float (&acc)[8]) {
  using V = Run<O>;
  typename V::Raw* at = static_cast<typename V::Raw*>(p.dW) + (static_cast<size_t>(row) * p.d + col) / 8;
  float v[8] = {};
  if (p.accumulate) V::get(*at, v);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = fmaf(acc[e], p.scale, v[e]);
  *at = V::put(v);
}

__device__ __forceinline__ void put_part(float* part, const float (&acc)[8]) {
  reinterpret_cast<float4*>(part)[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
  reinterpret_cast<float4*>(part)[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
}

// Blocks below `sums`: a unit's runs for kSumCols columns.  The others: 32 rows each,
// those that no token names zeroed.
template <typename T, typename O>
__global__ void __launch_bounds__(kSumThreads) sum_runs_kernel(const EmbArgs p, EmbSort s, int unit, int units, int64_t sums) {
  constexpr int kAhead = 8;
  using V = Run<T>;
  using Raw = typename V::Raw;
  const int64_t block = blockIdx.x;
  grid_launch_dependents();
  grid_wait();
  if (block >= sums) {
    const int word = static_cast<int>(block - sums);
    const uint32_t named = s.named[word];
    const int rows = min(32, p.V - 32 * word);
    const float none[8] = {};
    for (int r = 0; r < rows; ++r) {
      if (named >> r & 1) continue;
      typename Run<O>::Raw* at = static_cast<typename Run<O>::Raw*>(p.dW) + (static_cast<size_t>(word) * 32 + r) * (p.d / 8);
      for (int k = threadIdx.x; k < p.d / 8; k += kSumThreads) at[k] = Run<O>::put(none);
    }
    return;
  }
  const int u = static_cast<int>(block % units);
  const int col = static_cast<int>(block / units) * kSumCols + 8 * static_cast<int>(threadIdx.x);
  const int lane = threadIdx.x % 32;
  const bool in = col < p.d;
  const uint32_t none = p.V;
  const int64_t begin = static_cast<int64_t>(u) * unit, end = min(begin + unit, static_cast<int64_t>(p.T));
  uint32_t run = s.keys[begin];
  bool open = begin > 0 && s.keys[begin - 1] == run;  // the run began in an earlier unit
  const uint32_t after = end < p.T ? s.keys[end] : none;
  float* part = s.part + static_cast<size_t>(u) * 2 * p.d + col;  // [unit][of an open run, of the last run][d]
  float acc[8] = {};
  const Raw* dy = static_cast<const Raw*>(p.dy) + col / 8;
  for (int64_t i = begin; i < end; i += 32) {
    const uint32_t my_key = i + lane < end ? s.keys[i + lane] : none;
    const int32_t my_pos = i + lane < end ? s.pos[i + lane] : 0;
    const int here = static_cast<int>(min(static_cast<int64_t>(32), end - i));
    for (int j = 0; j < here; j += kAhead) {
      Raw raw[kAhead];
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        const uint32_t key = __shfl_sync(0xffffffffu, my_key, j + a);
        const int32_t t = __shfl_sync(0xffffffffu, my_pos, j + a);
        if (in && key != none) raw[a] = dy[static_cast<size_t>(t) * (p.d / 8)];
      }
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        const uint32_t key = __shfl_sync(0xffffffffu, my_key, j + a);
        if (j + a < here && key != run) {  // the run ends here
          if (in && run != none) {
            if (open)
              put_part(part, acc);
            else
              put_row<O>(p, run, col, acc);
          }
          open = false;
          run = key;
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] = 0.f;
        }
        if (in && key != none) {
          float v[8];
          V::get(raw[a], v);
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] += v[e];
        }
      }
    }
  }
  if (!in || run == none) return;
  if (open)
    put_part(part, acc);
  else if (after == run)
    put_part(part + p.d, acc);
  else
    put_row<O>(p, run, col, acc);
}

// Rows whose runs cross units: the unit that a run begins in adds up what it and the
// units behind it stored, four columns a thread, with a running compensation (a run may
// be all tokens).
template <typename O>
__global__ void __launch_bounds__(kJoinThreads) join_runs_kernel(const EmbArgs p, EmbSort s, int unit, int units) {
  const int u = static_cast<int>(blockIdx.x), lane = threadIdx.x % 32;
  const int col = static_cast<int>(blockIdx.y) * (4 * kJoinThreads) + 4 * static_cast<int>(threadIdx.x);
  const int64_t begin = static_cast<int64_t>(u) * unit, end = begin + unit;
  if (end >= p.T) return;
  grid_wait();
  const uint32_t run = s.keys[end - 1], behind = s.keys[end], ahead = begin > 0 ? s.keys[begin - 1] : ~run;
  if (run == static_cast<uint32_t>(p.V) || behind != run || ahead == run) return;
  // the last unit that begins with the run, a warp looking at 32 places at a time
  int lo = u + 1, hi = units;  // unit lo begins with it, unit hi does not (or is none)
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32, w = lo + step * lane;
    const uint32_t got = __ballot_sync(0xffffffffu, w < hi && s.keys[static_cast<int64_t>(w) * unit] == run);
    lo += step * (31 - __clz(got));
    hi = min(hi, lo + step);
  }
  if (col >= p.d) return;
  float4 acc = *reinterpret_cast<const float4*>(s.part + (static_cast<size_t>(u) * 2 + 1) * p.d + col), low = make_float4(0.f, 0.f, 0.f, 0.f);
  const auto add = [](float& a, float& c, float v) {
    const float y = v - c, t = a + y;
    c = (t - a) - y;
    a = t;
  };
#pragma unroll 8
  for (int w = u + 1; w <= lo; ++w) {
    const float4 v = *reinterpret_cast<const float4*>(s.part + static_cast<size_t>(w) * 2 * p.d + col);
    add(acc.x, low.x, v.x);
    add(acc.y, low.y, v.y);
    add(acc.z, low.z, v.z);
    add(acc.w, low.w, v.w);
  }
  O* at = static_cast<O*>(p.dW) + static_cast<size_t>(run) * p.d + col;
  const float v[4] = {acc.x, acc.y, acc.z, acc.w};
  if constexpr (sizeof(O) == 4) {
    float4 was = make_float4(0.f, 0.f, 0.f, 0.f);
    if (p.accumulate) was = *reinterpret_cast<const float4*>(at);
    *reinterpret_cast<float4*>(at) = make_float4(fmaf(v[0], p.scale, was.x), fmaf(v[1], p.scale, was.y),
                                                 fmaf(v[2], p.scale, was.z), fmaf(v[3], p.scale, was.w));
  } else {
    uint2 was = make_uint2(0, 0);
    if (p.accumulate) was = *reinterpret_cast<const uint2*>(at);
    const float w[4] = {__uint_as_float(was.x << 16), __uint_as_float(was.x & 0xffff0000u), __uint_as_float(was.y << 16),
                        __uint_as_float(was.y & 0xffff0000u)};
    *reinterpret_cast<uint2*>(at) = make_uint2(pack_bf16x2(fmaf(v[0], p.scale, w[0]), fmaf(v[1], p.scale, w[1])),
                                               pack_bf16x2(fmaf(v[2], p.scale, w[2]), fmaf(v[3], p.scale, w[3])));
  }
}

// Launches a kernel that waits for the one ahead by itself (grid_wait, before it touches
// what that one reads or writes), so that it is on the SMs when that ends.
template <class... K, class... A>
void launch_after(const Ctx& c, void (*kernel)(K...), dim3 grid, int threads, size_t smem, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
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

// Tokens of a sort's block: every block reads all blocks' counts, so larger ones where there
// are many.  (The last of the sort's launches, us, tiles of 2048, 4096 and 8192, rows of
// 4096: 65537 tokens 23, 33, 57; 131072 30, 35, 58.  The call, rows of 64: 2^18 tokens 145,
// 139, 150; 2^20 555, 481, 489; 2^21 1200, 918, 861.  The order is the same with all.)
int sort_tile(int64_t T) { return T <= 131072 ? 2048 : T <= 1 << 20 ? 4096 : 8192; }
// Tokens of a unit: short ones spread frequent ids over more blocks, but their joins and the
// workspace grow with the units' number.  (Sums and joins, us, units of 32 and 128, rows of
// 4096: 65537 tokens 278 + 63, 295 + 41; 131072 371 + 102, 380 + 49.)
int sum_unit(int64_t T) { return T <= 65536 ? 32 : 128; }

template <typename T, typename O>
void run_sums(const Ctx& c, const EmbArgs& a, const EmbSort& s) {
  const int unit = sum_unit(a.T), units = static_cast<int>(ceil_div(a.T, unit));
  const int cols = static_cast<int>(ceil_div(a.d, kSumCols));
  const int64_t sums = static_cast<int64_t>(units) * cols;
  const int64_t blocks = sums + (a.accumulate ? 0 : ceil_div(a.V, 32));
  launch_after(c, sum_runs_kernel<T, O>, dim3(static_cast<unsigned>(blocks)), kSumThreads, 0, a, s, unit, units, sums);
  if (units > 1)
    launch_after(c, join_runs_kernel<O>, dim3(units, static_cast<unsigned>(ceil_div(a.d, 4 * kJoinThreads))), kJoinThreads, 0, a, s, unit, units);
}

}  // namespace

static EmbSort carve_emb_impl(void* ws, int64_t T, int64_t d, int64_t V, size_t* total) {
  size_t off = 0;
  const auto take = [&](size_t bytes) {
    void* p = ws ? static_cast<char*>(ws) + off : nullptr;
    off = align_up(off + bytes, kWsAlign);
    return p;
  };
  EmbSort s;
  for (int i = 0; i < 2; ++i) {
    s.buf_keys[i] = static_cast<uint32_t*>(take(4ull * T));
    s.buf_pos[i] = static_cast<int32_t*>(take(4ull * T));
  }
  s.table = static_cast<uint32_t*>(take(4ull * kBins * ceil_div(T, sort_tile(T))));
  s.named = static_cast<uint32_t*>(take(4ull * ceil_div(V, 32)));
  s.part = static_cast<float*>(take(8ull * ceil_div(T, sum_unit(T)) * d));
  s.keys = nullptr;
  s.pos = nullptr;
  if (total) *total = off;
  return s;
}
size_t emb_bwd_ws_bytes(int64_t T, int64_t d, int64_t V) {
  size_t n = 0;
  carve_emb_impl(nullptr, T, d, V, &n);
  return n;
}

olive_status launch_emb_fwd(const Ctx& c, const EmbArgs& a) {
  const int64_t blocks = ceil_div(static_cast<int64_t>(a.T) * (a.d / 8), kLookThreads * kLookVecs);
  if (a.dtype == OLIVE_DTYPE_BF16)
    look_up_kernel<__nv_bfloat16><<<static_cast<unsigned>(blocks), kLookThreads, 0, c.stream>>>(a);
  else
    look_up_kernel<float><<<static_cast<unsigned>(blocks), kLookThreads, 0, c.stream>>>(a);
  return cudaGetLastError() == cudaSuccess ? OLIVE_OK : OLIVE_ERR_CUDA;
}

olive_status launch_emb_bwd(const Ctx& c, const EmbArgs& a, void* ws) {
  EmbSort s = carve_emb_impl(ws, a.T, a.d, a.V, nullptr);
  const int tile = sort_tile(a.T);
  const unsigned blocks = static_cast<unsigned>(ceil_div(a.T, tile));
  constexpr int kSmem = 4 * kSortWarps * kBins;
  static std::atomic<int> done[3][kMaxDevices];
  if (!set_smem_once(reinterpret_cast<const void*>(sort_move_kernel<true, true>), kSmem, c.device, done[0]) ||
      !set_smem_once(reinterpret_cast<const void*>(sort_move_kernel<true, false>), kSmem, c.device, done[1]) ||
      !set_smem_once(reinterpret_cast<const void*>(sort_move_kernel<false, true>), kSmem, c.device, done[2]))
    return OLIVE_ERR_CUDA;
  static std::atomic<int> done_mid[kMaxDevices];
  if (!set_smem_once(reinterpret_cast<const void*>(sort_move_kernel<false, false>), kSmem, c.device, done_mid))
    return OLIVE_ERR_CUDA;
  // keys up to V itself
  int bits = 1;
  while (bits < 32 && (static_cast<uint64_t>(a.V) >> bits) != 0) ++bits;
  const int passes = (bits + kDigit - 1) / kDigit;
  const uint32_t* keys = s.buf_keys[0];
  const int32_t* pos = s.buf_pos[0];
  if (a.T <= kOneBlock) {
    static std::atomic<int> done_one[2][kMaxDevices];
    const bool few = a.T <= kSortThreads;
    const auto one = few ? sort_one_kernel<1> : sort_one_kernel<kOneBlock / kSortThreads>;
    if (!set_smem_once(reinterpret_cast<const void*>(one), kOneSmem, c.device, done_one[few])) return OLIVE_ERR_CUDA;
    one<<<1, kSortThreads, kOneSmem, c.stream>>>(a, s, passes);
  }
  for (int i = 0; a.T > kOneBlock && i < passes; ++i) {
    const int shift = i * kDigit;
    uint32_t* ko = s.buf_keys[i & 1];
    int32_t* po = s.buf_pos[i & 1];
    const bool last = i == passes - 1;
    if (i == 0)
      sort_count_kernel<true><<<blocks, kSortThreads, 0, c.stream>>>(a, s, keys, shift, tile);
    else
      launch_after(c, sort_count_kernel<false>, dim3(blocks), kSortThreads, 0, a, s, keys, shift, tile);
    const auto move = i == 0 ? (last ? sort_move_kernel<true, true> : sort_move_kernel<true, false>)
                             : (last ? sort_move_kernel<false, true> : sort_move_kernel<false, false>);
    launch_after(c, move, dim3(blocks), kSortThreads, kSmem, a, s, keys, pos, ko, po, shift, tile);
    keys = ko;
    pos = po;
  }
  s.keys = keys;
  s.pos = pos;
  const bool bf = a.dtype == OLIVE_DTYPE_BF16, obf = a.grad_dtype == OLIVE_DTYPE_BF16;
  if (bf && obf)
    run_sums<__nv_bfloat16, __nv_bfloat16>(c, a, s);
  else if (bf)
    run_sums<__nv_bfloat16, float>(c, a, s);
  else if (obf)
    run_sums<float, __nv_bfloat16>(c, a, s);
  else
    run_sums<float, float>(c, a, s);
  return cudaGetLastError() == cudaSuccess ? OLIVE_OK : OLIVE_ERR_CUDA;
}

}  // namespace olive
