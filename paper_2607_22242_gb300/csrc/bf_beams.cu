// bf_beams.cu -- a step of beam search: the best continuations over beams and
// vocabulary, and the reordering of the beams' states.
//
// A row's continuations have the totals score + (x_v - m) / tau - ln s, with m the
// row's largest logit and s = sum e^((x_v - m) / tau): within a row they are ranked by the logits alone, so a row's `keep`
// largest logits are all that a group has to look at.  Rows are read once, a
// chunk of a row to a block (row_kernel); a block leaves its chunk's maximum and
// sum of exponentials and its `keep` largest logits.  A block per group
// (group_kernel) joins the sums and chooses.  Ranks are compared in two 32-bit parts, so
// a group's order is that of the real numbers up to what the 32-bit sums are off by
// (below 1e-6), and two equal rows tie exactly wherever they lie.
#include "bf_answer.h"
#include "bf_blackwell.cuh"
#include "bf_elem.cuh"
#include "bf_launches.cuh"

namespace bfk {

namespace {

constexpr float kMinusInf = -__builtin_huge_valf();

__device__ __forceinline__ float exp2_of(float t) {
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t));
  return e;
}

// Whole numbers in the order of the values; -0 counts as 0.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_order(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
constexpr uint32_t kOrderMinusInf = 0x007FFFFFu;

// A continuation that may be among the best: what it is ranked by, and ties.
template <typename Key>
struct Entry {
  Key key;
  uint64_t tie;
};
constexpr uint32_t kList = 1024, kRowList = 2048;  // entries of a group's list, and of a chunk's

// The sum of a block's counts (all threads get it); `sums` has two words.
__device__ __forceinline__ uint32_t block_count(uint32_t mine, uint32_t* sums) {
  mine = __reduce_add_sync(~0u, mine);
  __syncthreads();
  if (threadIdx.x == 0) *sums = 0;
  __syncthreads();
  if (threadIdx.x % 32 == 0 && mine) atomicAdd(sums, mine);
  __syncthreads();
  return *sums;
}

// Bounds that at least `keep` of a block's threads' values reach (keep <= threads), and mostly not many more; above -inf.
//
// Where the values of the `full` warps that have some are alike: each finds its ceil(2 keep / full)-th
// largest, and the one of those that enough warps reach is the bound.  One barrier.
// `warps` holds a word for each warp.
// The need-th largest of the warps' values (the same in all of a warp's lanes).
__device__ __forceinline__ uint32_t bound_of_warps(uint32_t value, uint32_t need, uint32_t* warps) {
  const uint32_t count = blockDim.x / 32, lane = threadIdx.x % 32;
  if (lane == 0) warps[threadIdx.x / 32] = value;
  __syncthreads();
  const uint32_t w = lane < count ? warps[lane] : 0;
  uint32_t above = 0;
  for (uint32_t i = 0; i < count; ++i) {
    const uint32_t o = __shfl_sync(~0u, w, i);
    above += o > w || (o == w && i < lane);
  }
  const uint32_t bound = __reduce_max_sync(~0u, lane < count && above == need - 1 ? w : 0);
  return max(bound, kOrderMinusInf + 1);
}
__device__ __forceinline__ uint32_t bound_of(uint32_t mine, uint32_t keep, uint32_t full, uint32_t* warps) {
  const uint32_t each = min(32u, (2 * keep + full - 1) / full), lane = threadIdx.x % 32;
  uint32_t most = 0;
  for (uint32_t i = 0; i < each; ++i) {
    most = __reduce_max_sync(~0u, mine);
    if (lane == __ffs(__ballot_sync(~0u, mine == most)) - 1u) mine = 0;
  }
  return bound_of_warps(most, (keep + each - 1) / each, warps);
}
// The same from N values of each thread (N times as many: for a `keep` that is large
// beside the threads), the warps' by bisection.
template <int N>
__device__ __forceinline__ uint32_t bound_of_all(const uint32_t (&mine)[N], uint32_t keep, uint32_t full, uint32_t* warps) {
  const uint32_t each = min(32u * N, (2 * keep + full - 1) / full);
  uint32_t lo = 0, hi = 0xFFFFFFFFu;
  while (hi - lo > 1) {
    const uint32_t mid = lo + (hi - lo) / 2;
    uint32_t n = 0;
#pragma unroll
    for (int k = 0; k < N; ++k) n += mine[k] >= mid;
    n = __reduce_add_sync(~0u, n);
    if (n >= each) {
      lo = mid;
      if (n <= each + each / 8) break;
    } else {
      hi = mid;
    }
  }
  return bound_of_warps(lo, (keep + each - 1) / each, warps);
}
// Where one warp's may be far above another's (beams of different scores): the keep-th
// largest of the first `some` threads' values itself, by counting.  `all` holds a word for each thread.
__device__ __forceinline__ uint32_t exact_of(uint32_t mine, uint32_t keep, uint32_t some, uint32_t* all, uint32_t* bound) {
  const uint32_t t = threadIdx.x;
  all[t] = t < some ? mine : 0;
  if (t == 0) *bound = kOrderMinusInf + 1;
  __syncthreads();
  if (t < some && mine > kOrderMinusInf) {  // the bound is above -inf
    uint32_t above = 0;
#pragma unroll 4
    for (uint32_t i = 0; i < some; i += 4) {
      const uint4 o = *reinterpret_cast<const uint4*>(all + i);
      const uint32_t least = i < t / 4 * 4 ? mine : mine + 1;  // of those ahead, equal ones are above
      above += (o.x >= least) + (o.y >= least) + (o.z >= least) + (o.w >= least);
    }
    for (uint32_t i = t / 4 * 4; i < t; ++i) above += all[i] == mine;
    if (above == keep - 1) *bound = mine;
  }
  __syncthreads();
  return *bound;
}

// Where a list would overflow (many equal values): the exact keep-th largest of
// all (key, tie), by counting.  each(f) calls f(key, tie) for all of a thread's
// candidates.  Candidates of at least `key`, and of a tie below `tie` where they have
// just that key, are the best; there are `keep` of them or, with fewer in all, all.
// All ties are from `below` on, and below `upto`.
template <typename Key, typename Each>
__device__ __noinline__ void exact_bound(Each each, Key least, uint64_t below, uint64_t upto, uint32_t keep, uint32_t* sums, Key* key,
                                         uint64_t* tie) {
  const auto count = [&](Key k, uint64_t t) {  // candidates above (k, t): better keys, or k and a lower tie
    uint32_t n = 0;
    each([&](Key c, uint64_t at) { n += c > k || (c == k && at < t); });
    return block_count(n, sums);
  };
  Key lo = least, hi = ~(Key)0;  // the largest key that `keep` candidates reach
  *key = least;
  *tie = ~0ull;
  if (count(lo, ~0ull) <= keep) return;
  while (hi - lo > 1) {
    const Key mid = lo + (hi - lo) / 2;
    if (count(mid, ~0ull) >= keep) lo = mid;
    else hi = mid;
  }
  // the lowest tie that makes it `keep`
  while (upto - below > 1) {
    const uint64_t mid = below + (upto - below) / 2;
    if (count(lo, mid) >= keep) upto = mid;
    else below = mid;
  }
  *key = lo;
  *tie = upto;
}

// Puts a list of n (and room for the next power of two) in order, the best first, by
// exchanges of pairs; `none` is behind all others.
template <typename T, typename Above>
__device__ __forceinline__ void sort_list(T* list, uint32_t n, T none, Above above) {
  uint32_t size = 1;
  while (size < n) size *= 2;
  for (uint32_t i = n + threadIdx.x; i < size; i += blockDim.x) list[i] = none;
  __syncthreads();
  for (uint32_t run = 2; run <= size; run *= 2)
    for (uint32_t apart = run / 2; apart; apart /= 2) {
      for (uint32_t i = threadIdx.x; i < size / 2; i += blockDim.x) {
        const uint32_t lo = i / apart * 2 * apart + i % apart, hi = lo + apart;
        const T x = list[lo], y = list[hi];
        if (above(y, x) == ((lo & run) == 0)) {
          list[lo] = y;
          list[hi] = x;
        }
      }
      __syncthreads();
    }
}
// How many of a list of n are above `mine`.
template <typename T, typename Above>
__device__ __forceinline__ uint32_t rank_of(const T* list, uint32_t n, const T& mine, Above above) {
  uint32_t rank = 0, j = 0;
  if constexpr (sizeof(T) == 4)  // plain numbers, four a read
    for (; j + 4 <= n; j += 4) {
      const uint4 o = *reinterpret_cast<const uint4*>(list + j);
      rank += (o.x > mine) + (o.y > mine) + (o.z > mine) + (o.w > mine);
    }
  for (; j < n; ++j) rank += above(list[j], mine);
  return rank;
}
// Up to so many entries (twice as many of one word) are ranked by all others, which takes their square; more are
// sorted.  (Rows of 50,001 f16 logits, 32 kept, 100 to 250 entries a chunk: 31.5 us against 32.6 with 200 for both.)
constexpr uint32_t kRanked = 200;

// Calls put(rank, entry) for the best `keep` of a list of n.
template <bool kFew, typename T, typename Above, typename Put>
__device__ __forceinline__ void best_of(T* list, uint32_t n, uint32_t keep, T none, Above above, Put put) {
  if (kFew || n <= (sizeof(T) == 4 ? 2 : 1) * kRanked) {
    for (uint32_t i = threadIdx.x; i < n; i += blockDim.x) {
      const T mine = list[i];
      const uint32_t rank = rank_of(list, n, mine, above);
      if (rank < keep) put(rank, mine);
    }
  } else {
    sort_list(list, n, none, above);
    for (uint32_t i = threadIdx.x; i < min(n, keep); i += blockDim.x) put(i, list[i]);
  }
}

// ---- rows -------------------------------------------------------------------

struct Candidate {
  float x;  // -inf: none
  uint32_t token;
};

struct Chunks {
  uint32_t per_row, elements, tiles, threads;
  float2* heads;    // [rows][per_row]: maximum, sum of e^((x - maximum) / tau)
  Candidate* best;  // [rows][per_row][keep]
};

constexpr uint32_t kThreads = 256;

__device__ __forceinline__ bool is_alive(const BeamArgs& a, uint64_t row) {
  const float score = __ldg(a.scores + row);
  return !(score == kMinusInf) && !(a.finished && __ldg(a.finished + row));
}

// The largest element of a vector, as one word: of 32 bits, or of either half.
__device__ __forceinline__ uint32_t most_of(const uint4& u, float) {
  return __float_as_uint(fmaxf(fmaxf(__uint_as_float(u.x), __uint_as_float(u.y)), fmaxf(__uint_as_float(u.z), __uint_as_float(u.w))));
}
template <typename E2>
__device__ __forceinline__ uint32_t most_of_pairs(const uint4& u) {
  const auto pair = [](uint32_t v) { return *reinterpret_cast<const E2*>(&v); };
  const E2 m = __hmax2(__hmax2(pair(u.x), pair(u.y)), __hmax2(pair(u.z), pair(u.w)));
  return *reinterpret_cast<const uint32_t*>(&m);
}
__device__ __forceinline__ uint32_t most_of(const uint4& u, __nv_bfloat16) { return most_of_pairs<__nv_bfloat162>(u); }
__device__ __forceinline__ uint32_t most_of(const uint4& u, __half) { return most_of_pairs<__half2>(u); }
__device__ __forceinline__ float value_of(uint32_t word, float) { return __uint_as_float(word); }
template <typename E>
__device__ __forceinline__ float value_of(uint32_t word, E) {
  const float2 f = unpack2(word, E());
  return fmaxf(f.x, f.y);
}
// What a chunk's candidates are ranked by: the order of the logit, then of the element's
// place in the chunk the other way round; for 16 bits in one word (ranking was a fifth of the kernel's time with two).
template <typename E>
struct Ranks {
  using Key = uint32_t;
  static __device__ __forceinline__ Key key(float v, uint32_t place) {
    const E e = from_f32<E>(v + 0.0f);
    const uint32_t u = *reinterpret_cast<const uint16_t*>(&e);
    return (u & 0x8000u ? ~u : u | 0x8000u) << 16 | (0xFFFFu - place);
  }
  static __device__ __forceinline__ float value(Key k) {
    const uint16_t u = (uint16_t)(k >> 31 ? k >> 16 ^ 0x8000u : ~(k >> 16));
    return to_f32(*reinterpret_cast<const E*>(&u));
  }
  static __device__ __forceinline__ uint32_t place(Key k) { return 0xFFFFu - (k & 0xFFFFu); }
};
template <>
struct Ranks<float> {
  using Key = uint64_t;
  static __device__ __forceinline__ Key key(float v, uint32_t place) { return (uint64_t)order_of(v) << 32 | ~place; }
  static __device__ __forceinline__ float value(Key k) { return from_order((uint32_t)(k >> 32)); }
  static __device__ __forceinline__ uint32_t place(Key k) { return ~(uint32_t)k; }
};
constexpr uint32_t kHits = 1024;  // vectors of a chunk that have a candidate

// The exponentials of V vectors against m, summed.  (x - m) c2 as x c2 - r, r = m c2
// rounded, and what r is off by put back into the sum; where m c2 is far from ordinary
// (nothing but the type's lowest values, a very small temperature), as it stands.
template <typename E, int V, bool fits>
__device__ __forceinline__ float sum_of(const uint4 (&u)[V], float m, float c2) {
  const float r = fits ? -m * c2 : 0.0f, base = m == kMinusInf ? 0.0f : -m;
  float2 s2 = make_float2(0.0f, 0.0f);
#pragma unroll
  for (int k = 0; k < V; ++k) {
    float2 f[Vec<E>::kWidth / 2];
    unpack<E>(u[k], f);
#pragma unroll
    for (uint32_t i = 0; i < Vec<E>::kWidth / 2; ++i) {
      if (!fits) f[i] = __fadd2_rn(f[i], make_float2(base, base));
      const float2 e = __ffma2_rn(f[i], make_float2(c2, c2), make_float2(r, r));
      s2 = __fadd2_rn(s2, make_float2(exp2_of(e.x), exp2_of(e.y)));
    }
  }
  const float s = s2.x + s2.y, rest = fits ? fmaf(-m, c2, m * c2) * 0.693147180559945309f : 0.0f;
  return fmaf(s, rest, s);
}

// V aligned vectors of each lane, which follow one another over a warp's lanes and then its turns, shifted down by
// `off` bytes, of which W are whole words; `tail` is what follows the last one (lane 0's).  A lane has its next words from its neighbour.
template <int V, int W>
__device__ __forceinline__ void shift_by(uint4 (&u)[V], const uint4& tail, uint32_t off) {
  const uint32_t lane = threadIdx.x % 32, r = off % 4 * 8;
#pragma unroll
  for (int k = 0; k < V; ++k) {
    const uint4 next = k + 1 < V ? u[k + 1 < V ? k + 1 : k] : tail;
    uint32_t w[8] = {u[k].x, u[k].y, u[k].z, u[k].w, 0, 0, 0, 0};
    const uint32_t n[4] = {next.x, next.y, next.z, next.w};
#pragma unroll
    for (int i = 0; i <= W; ++i) w[4 + i] = __shfl_sync(~0u, lane == 0 ? n[i] : w[i], (lane + 1) % 32);
    u[k] = make_uint4(__funnelshift_r(w[W], w[W + 1], r), __funnelshift_r(w[W + 1], w[W + 2], r), __funnelshift_r(w[W + 2], w[W + 3], r),
                      __funnelshift_r(w[W + 3], w[W + 4], r));
  }
}

// Lists what reaches `least` of a row's elements [cut, end).
template <typename E, bool kAligned, uint32_t T, uint32_t kMost, typename Key>
__device__ __forceinline__ void list_again(const E* x, uint32_t cut, uint32_t end, float least, Key* list, uint32_t* count) {
  constexpr uint32_t kW = Vec<E>::kWidth;
  const auto look = [=](uint32_t i) {
    const float v = to_f32(x[i]);
    if (v >= least) {
      const uint32_t to = atomicAdd(count, 1u);
      if (to < kMost) list[to] = Ranks<E>::key(v, i - cut);
    }
  };
  const uint32_t whole = kAligned ? (end - cut) / kW * kW : 0;
  if constexpr (kAligned)
#pragma unroll 4
    for (uint32_t j = cut + threadIdx.x * kW; j < cut + whole; j += T * kW)
      if (value_of(most_of(__ldg(reinterpret_cast<const uint4*>(x + j)), E()), E()) >= least)
#pragma unroll 1
        for (uint32_t i = 0; i < kW; ++i) look(j + i);
#pragma unroll 4
  for (uint32_t i = cut + whole + threadIdx.x; i < end; i += T) look(i);
}

// Out of line for rows at any alignment, whose kernel has no registers for it (2 % of a step).
template <typename E, uint32_t T, uint32_t kMost, typename Key>
__device__ __noinline__ void list_again_apart(const E* x, uint32_t cut, uint32_t end, float least, Key* list, uint32_t* count) {
  list_again<E, false, T, kMost>(x, cut, end, least, list, count);
}

// A chunk of a row, `tiles` times V vectors a thread, cut by the row's elements and not
// by addresses, so that equal rows have equal sums.  kAligned: rows start at 16 bytes.
// What reaches a bound that `keep` of the threads' maxima in the first tile (that has so many not banned) reach may be
// among the chunk's best: a few more than `keep` in each tile.
//
// 107 MB of 131,072 bf16 logits a row in 31 us, 3.5 TB/s.  Neither the memory nor the issue slots are full (55 % of them over the
// kernel's time, 63 % of a busy SM's cycles; 12 instructions an element, of which the exponential and its sum are 4):
// a block's reads, bound, notes and ranks follow one another, and four blocks an SM, 3.4 waves of them, do not cover that;
// rows at any alignment take a quarter more (512 of 131,071: 57 us a step, 45 of 131,072),
// and took two thirds more when each thread read both vectors that hold its elements.
template <typename E, int V, bool kAligned, uint32_t T>
__global__ void __launch_bounds__(T, 1024 / T) row_kernel(const __grid_constant__ BeamArgs a, const __grid_constant__ Chunks ch) {
  constexpr uint32_t kW = Vec<E>::kWidth;
  constexpr uint32_t kRowList = T == 256 ? bfk::kRowList : 512, kHits = T == 256 ? bfk::kHits : 128;
  using Key = typename Ranks<E>::Key;
  __shared__ __align__(16) Key list[kRowList];
  __shared__ uint4 hit[kHits];
  __shared__ uint32_t hit_token[kHits];
  __shared__ uint32_t count, hits, sums, warp_bound[T / 32];
  __shared__ float warp_max[T / 32], warp_sum[T / 32];
  let_next_start();
  const uint32_t row = blockIdx.x / ch.per_row, chunk = blockIdx.x - row * ch.per_row, t = threadIdx.x;
  if (!is_alive(a, row)) return;
  if (t == 0) count = hits = 0;
  const E* x = static_cast<const E*>(a.x) + (uint64_t)row * a.ldx;
  const uint32_t cut = chunk * ch.elements, end = min(cut + ch.elements, a.vocab);
  const uint32_t none = minus_inf_bits(E());
  float m = kMinusInf, s = 0.0f, least = 0.0f;
  uint32_t bound = 0;
#pragma unroll 1
  for (uint32_t tile = 0; tile < ch.tiles; ++tile) {
    // A thread's vectors are `step` elements apart.  Unaligned, a warp's vectors follow one another, up to V times 32,
    // and all warps have some where a tile is short (44 us for 512 aligned rows of 131,072 as they are, 47 so).
    const uint32_t tile0 = cut + tile * V * T * kW, last = min(tile0 + V * T * kW, end);
    const uint32_t turns = tile0 < last ? (last - tile0 + T * kW - 1) / (T * kW) : 0;
    constexpr uint32_t step = (kAligned ? T : 32) * kW;
    const uint32_t first = tile0 + (kAligned ? t : t / 32 * turns * 32 + t % 32) * kW;
    uint4 u[V];
    if constexpr (kAligned) {
#pragma unroll
      for (uint32_t k = 0; k < V; ++k) {
        const uint32_t j = first + k * step;
        u[k] = make_uint4(none, none, none, none);
        if (j + kW <= last) u[k] = __ldcs(reinterpret_cast<const uint4*>(x + j));
        else if (j < last) u[k] = load_ends<E>(x + j, 0, (int32_t)(last - j), none);
      }
    } else {
      const Extent matrix(static_cast<const E*>(a.x), (uint64_t)a.groups * a.beams, a.ldx, a.vocab);
      // Each aligned vector is read once, and those behind the row's end but one are not, where all of that lies inside the matrix.
      const uintptr_t at = (uintptr_t)x, off = at % 16, base = at - off;
      if (base + (uint64_t)tile0 * sizeof(E) >= matrix.begin && base + ((uint64_t)last + 2 * kW) * sizeof(E) <= matrix.end) {
        const uint4* p = reinterpret_cast<const uint4*>(base) + first / kW;
        uint4 tail = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (uint32_t k = 0; k < V; ++k) {
          u[k] = make_uint4(none, none, none, none);
          if (k < turns + (t % 32 == 0) && first + k * step < last + kW) u[k] = __ldg(p + k * 32);
        }
        if (t % 32 == 0 && turns == V && first + V * step < last + kW) tail = __ldg(p + V * 32);
        if (off >= 12) shift_by<V, 3>(u, tail, off);
        else if (off >= 8) shift_by<V, 2>(u, tail, off);
        else if (off >= 4) shift_by<V, 1>(u, tail, off);
        else if (off) shift_by<V, 0>(u, tail, off);
        if (last == end) {  // (in all other tiles every vector is whole)
#pragma unroll
          for (uint32_t k = 0; k < V; ++k) {
            const uint32_t j = first + k * step;
            if (k >= turns || j >= last) u[k] = make_uint4(none, none, none, none);
            else if (j + kW > last) u[k] = load_ends<E>(x + j, 0, (int32_t)(last - j), none);
          }
        }
      } else {
#pragma unroll
        for (int k = 0; k < V; ++k) u[k] = make_uint4(none, none, none, none);
#pragma unroll 1
        for (uint32_t k = 0; k < turns; ++k) {
          const uint32_t j = first + k * step;
          uint4 v = make_uint4(none, none, none, none);
          if (j + kW <= last) {
            Unaligned<E> raw;
            raw.load(x, a.vocab, (int64_t)j, matrix);
            v = raw.take();
          } else if (j < last) {
            v = load_ends<E>(x + j, 0, (int32_t)(last - j), none);
          }
#pragma unroll
          for (uint32_t i = 0; i < V; ++i)
            if (i == k) u[i] = v;
        }
      }
    }
    uint32_t most[V];
    float tmax = kMinusInf;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      most[k] = most_of(u[k], E());
      tmax = fmaxf(tmax, value_of(most[k], E()));
    }
    // The thread's sum, against its own maximum so far.
    const float now = fmaxf(m, tmax);
    if (now > m) s *= m == kMinusInf ? 1.0f : exp2_of((m - now) * a.c2);  // (s is 0, or NaN, before the first number)
    m = now;
    s += fabsf(m) * a.c2 < 1024.0f ? sum_of<E, V, true>(u, m, a.c2) : sum_of<E, V, false>(u, m, a.c2);
    if (bound <= kOrderMinusInf + 1 && tile0 < last) {  // the first tile, or all so far are banned
      if (tile != 0) __syncthreads();  // the tile before's words of the warps have been read
      // Warps that have vectors; half of them are enough to count on all.
      const uint32_t each = kAligned ? 32 : turns * 32, some = ((last - tile0 + kW - 1) / kW + each - 1) / each;
      const uint32_t full = 2 * some >= T / 32 ? T / 32 : some;
      if (8 * a.keep <= 3 * T && a.keep <= 16 * full) {
        bound = bound_of(order_of(tmax), a.keep, full, warp_bound);
      } else {
        uint32_t keys[V];
#pragma unroll
        for (int k = 0; k < V; ++k) keys[k] = order_of(value_of(most[k], E()));
        bound = bound_of_all<V>(keys, a.keep, full, warp_bound);
      }
      least = from_order(bound);
    }
    // First the vectors that have any, then their elements, one to a thread: few threads
    // have a vector, and a warp that went through its own took twice the instructions.
    if (tmax >= least) {
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (value_of(most[k], E()) >= least) {
          const uint32_t at = atomicAdd(&hits, 1u);
          if (at < kHits) {
            hit[at] = u[k];
            hit_token[at] = first + (uint32_t)k * step;
          }
        }
    }
  }
  {
    const float top = from_order(__reduce_max_sync(~0u, order_of(m)));
    s *= m == top ? 1.0f : exp2_of((m - top) * a.c2);
#pragma unroll
    for (int d = 16; d; d /= 2) s += __shfl_xor_sync(~0u, s, d);
    if (t % 32 == 0) {
      warp_max[t / 32] = top;
      warp_sum[t / 32] = s;
    }
  }
  __syncthreads();
  uint32_t found = hits;
  // Where the first tile lies below the rest, the threads' maxima over all tiles give a better bound; the chunk is read again.
  // (512 rows of 131,072 that ascend, or whose chunks' first tiles are banned, took 7 ms by exact bounds, and 45 us if
  // alike all along.)
  if (found > kHits && ch.tiles > 1) {  // (so few kept that bound_of has them)
    const uint32_t here = bound_of(order_of(m), a.keep, T / 32, warp_bound);
    if (here > bound) {
      bound = here;
      least = from_order(bound);
      found = 0;
      if constexpr (kAligned) list_again<E, true, T, kRowList>(x, cut, end, least, list, &count);
      else list_again_apart<E, T, kRowList>(x, cut, end, least, list, &count);
    }
  }
  for (uint32_t i = t; i < min(found, kHits) * kW; i += T) {
    const uint32_t at = i / kW, j = i % kW;
    const float v = to_f32(reinterpret_cast<const E*>(&hit[at])[j]);
    if (v >= least) {
      const uint32_t to = atomicAdd(&count, 1u);
      if (to < kRowList) list[to] = Ranks<E>::key(v, hit_token[at] - cut + j);
    }
  }
  __syncthreads();
  uint32_t n = count;
  if (n > kRowList || found > kHits) {
    const uint32_t some = end - cut;
    const auto each = [=](auto f) {
      for (uint32_t i = t; i < some; i += T) {
        const float v = to_f32(x[cut + i]);
        if (v >= least) f(order_of(v), (uint64_t)(cut + i));
      }
    };
    uint32_t key;
    uint64_t tie;
    exact_bound<uint32_t>(each, bound, cut, end, a.keep, &sums, &key, &tie);
    __syncthreads();
    if (t == 0) count = 0;
    __syncthreads();
    each([&](uint32_t c, uint64_t at) {
      if (c > key || (c == key && at < tie)) list[atomicAdd(&count, 1u)] = Ranks<E>::key(from_order(c), (uint32_t)at - cut);
    });
    __syncthreads();
    n = count;
  }
  const uint64_t record = (uint64_t)row * ch.per_row + chunk;
  Candidate* best = ch.best + record * a.keep;
  best_of<false, Key>(
      list, n, a.keep, 0, [](Key x, Key y) { return x > y; },
      [&](uint32_t rank, Key e) { best[rank] = {Ranks<E>::value(e), cut + Ranks<E>::place(e)}; });
  for (uint32_t i = min(n, a.keep) + t; i < a.keep; i += T) best[i] = {kMinusInf, 0};
  if (t < 32) {
    const float wm = t < T / 32 ? warp_max[t] : kMinusInf, ws = t < T / 32 ? warp_sum[t] : 0.0f;
    const float top = from_order(__reduce_max_sync(~0u, order_of(wm)));
    float total = wm == top ? ws : ws * exp2_of((wm - top) * a.c2);
#pragma unroll
    for (int d = T / 64; d; d /= 2) total += __shfl_xor_sync(~0u, total, d);
    if (t == 0) ch.heads[record] = make_float2(top, total);
  }
}

__device__ __forceinline__ void prefetch(const void* p) { asm volatile("prefetch.global.L1 [%0];" ::"l"(p)); }

// ---- groups -----------------------------------------------------------------

enum BeamState : uint32_t { kDead, kAlive, kFinished };

// Numbers in two parts, the second at most half a last place of the first: their
// order is that of the parts, and 64-bit units are few.
struct Two {
  float hi, lo;
};
__device__ __forceinline__ Two two_sum(float a, float b) {
  const float s = a + b, t = s - a;
  return {s, (a - (s - t)) + (b - t)};
}
__device__ __forceinline__ Two quick_two(float a, float b) {  // |a| >= |b|, or either infinite
  const float s = a + b;
  return {s, b - (s - a)};
}
__device__ __forceinline__ uint64_t order_of(const Two& v) { return (uint64_t)order_of(v.hi) << 32 | order_of(v.lo); }
// ln v of a normal v as k ln 2 + ln f, f in [3/4, 3/2): Cody and Waite's ln 2 = 355/512 - 2.12e-4.
__device__ __forceinline__ Two log_of(float v) {
  const int bits = __float_as_int(v), k = (bits - __float_as_int(0.75f)) >> 23;
  return quick_two((float)k * 0.693359375f, fmaf((float)k, -2.12194440054690583e-4f, logf(__int_as_float(bits - k * (1 << 23)))));
}

// What a beam's continuations are made from: total = base + (x - most) / tau, rank = total * weight / 2^down.
struct Beam {
  Two base, weight;  // score - ln sum (a finished beam's score); 2^down / max(1, length)^penalty
  float most;        // the row's largest logit
  uint32_t state;    // and 256 times `down`, which is not 0 where length^penalty is above e^80
};

// Ranks in 32-bit numbers are right while length^penalty is at most e^80: theirs end in steps of 2^-149, 2^-34 of a total then.
// No length is above 2^63, so penalties up to 80 / ln 2^63 = 1.83 need nothing else, and their kernels have nothing else
// (it took 4 % of a step of 4,096 groups of 16 x 100).
constexpr float kNearWeights = 80.0f, kNearPenalty = 1.8f;
// n^-penalty as weight / 2^down, weight in [0.7, 1.5); `penalty` is up to 2^16, so down is below 2^22 and the
// 64-bit exponent off by less than 2^-30.
__device__ __noinline__ Two far_weight(float penalty, int64_t n, uint32_t* down) {
  const double y = (double)penalty * log2((double)n), whole = rint(y), w = exp2(whole - y);
  *down = (uint32_t)whole;
  const float hi = (float)w;
  return {hi, (float)(w - (double)hi)};
}
// Whole numbers in the order of r / 2^down: sign, exponent (23 bits), r.hi's 23 bits and r.lo in 2^-16 of r.hi's last place; 0 is
// none of them.
__device__ __noinline__ uint64_t far_order_of(Two r, int32_t down) {
  if (r.hi == 0.0f) return 1ull << 63;
  if (!(fabsf(r.hi) < -kMinusInf)) return r.hi < 0.0f ? 1 : ~0ull;
  if (fabsf(r.hi) < 0x1p-64f) {
    r = {r.hi * 0x1p64f, r.lo * 0x1p64f};
    down += 64;
  }
  const uint32_t u = __float_as_uint(fabsf(r.hi));
  const int32_t e = (int32_t)(u >> 23), rest = (int32_t)rintf(ldexpf(r.hi < 0.0f ? -r.lo : r.lo, 166 - e));
  const uint64_t size = ((uint64_t)(uint32_t)(e - down + (1 << 22)) << 40) + ((uint64_t)(u & 0x7FFFFFu) << 17) + (uint32_t)(rest + (1 << 15));
  return r.hi < 0.0f ? (1ull << 63) - 1 - size : (1ull << 63) + 1 + size;
}

__device__ __forceinline__ Two total_of(const Beam& b, float x, float tau, float inv_tau) {
  const float d = x - b.most, z = d * inv_tau;
  if (!(fabsf(z) < -kMinusInf)) return {z, 0.0f};  // the lowest values under a small temperature
  const Two s = two_sum(b.base.hi, z);
  return quick_two(s.hi, s.lo + fmaf(fmaf(-z, tau, d), inv_tau, b.base.lo));
}
__device__ __forceinline__ Two times(const Two& a, const Two& b) {
  const float p = a.hi * b.hi;
  if (!(fabsf(p) < -kMinusInf)) return {p, 0.0f};
  return quick_two(p, fmaf(a.hi, b.hi, -p) + (a.hi * b.lo + a.lo * b.hi));
}

// Dynamic shared memory of a group: its beams, its list, and its logits or the numbers of its lists.
__host__ __device__ __forceinline__ uint32_t list_of(uint64_t slots) {  // a power of two: lists are sorted
  uint32_t n = 32;
  while (n < slots && n < kList) n *= 2;
  return n;
}
__host__ __device__ __forceinline__ uint64_t group_bytes(uint32_t beams, uint64_t slots, uint64_t more) {
  return (beams * sizeof(Beam) + 15) / 16 * 16 + list_of(slots) * sizeof(Entry<uint64_t>) + more * 4;
}

// A group's block: beams, list and what both kernels below do with them.  kFar: weights may be beyond 32-bit numbers.
template <bool kFar>
struct Group {
  const BeamArgs& a;
  Beam* beam;
  Entry<uint64_t>* list;
  uint32_t most_listed;
  uint64_t row0;
  float inv_tau;
  uint32_t *count, *odd, *far;  // `far`: some beam's weight is beyond

  __device__ __forceinline__ Group(const BeamArgs& args, unsigned char* raw, uint64_t slots, uint32_t* words)
      : a(args), beam(reinterpret_cast<Beam*>(raw)),
        list(reinterpret_cast<Entry<uint64_t>*>(raw + (args.beams * sizeof(Beam) + 15) / 16 * 16)), most_listed(list_of(slots)),
        row0((uint64_t)blockIdx.x * args.beams), inv_tau(1.0f / args.tau), count(words), odd(words + 1), far(words + 2) {
    if (threadIdx.x == 0) *count = *odd = *far = 0;
  }
  __device__ __forceinline__ uint32_t state_of(uint32_t b) const {
    const float score = __ldg(a.scores + row0 + b);
    return score == kMinusInf ? kDead : a.finished && __ldg(a.finished + row0 + b) ? kFinished : kAlive;
  }
  __device__ __forceinline__ static uint32_t kind(const Beam& o) { return kFar ? o.state & 255 : o.state; }
  // From the maximum and sum of a row's exponentials.
  __device__ __forceinline__ void put(uint32_t b, uint32_t state, float m, float s) {
    const float score = __ldg(a.scores + row0 + b);
    Beam o;
    if (state == kAlive && m == kMinusInf && s == s) state = kDead;
    o.state = state;
    o.most = state == kAlive ? m : 0.0f;
    o.base = {score, 0.0f};
    if (state == kAlive) {
      const Two l = log_of(s), d = two_sum(score, -l.hi);
      o.base = quick_two(d.hi, d.lo - l.lo);
    }
    o.weight = {1.0f, 0.0f};
    if (a.penalty != 0.0f) {  // n^-penalty = e^(-penalty ln n), ln n and the product in two parts
      int64_t n = __ldg(a.lengths + row0 + b) + (state != kFinished);
      if (n < 1) n = 1;
      const Two l = log_of((float)n);
      const float p = a.penalty * l.hi;
      if (!kFar || p <= kNearWeights) {
        const float w = expf(-p);
        o.weight = quick_two(w, -w * fmaf(a.penalty, l.lo, fmaf(a.penalty, l.hi, -p)));
      } else {
        uint32_t down;
        o.weight = far_weight(a.penalty, n, &down);
        o.state |= down << 8;
        *far = 1;
      }
    }
    beam[b] = o;
    if (score != score || score == -kMinusInf || s != s) *odd = 1;
  }
  __device__ __forceinline__ uint64_t key_of(uint32_t b, float x) const {
    const Beam& o = beam[b];
    const Two total = kind(o) == kFinished ? o.base : total_of(o, x, a.tau, inv_tau);
    if (kFar && *far) return far_order_of(times(total, o.weight), (int32_t)(o.state >> 8));
    return order_of(a.penalty != 0.0f ? times(total, o.weight) : total);
  }
  // Equal in both parts: the lower beam, in it the larger logit, then the lower token (8, 32 and 24 bits).
  static __device__ __forceinline__ uint64_t tie_of(uint32_t b, float x, uint32_t token) {
    return (uint64_t)b << 56 | (uint64_t)~order_of(x) << 24 | token;
  }
  __device__ __forceinline__ void push(uint64_t key, uint64_t tie) const {
    const uint32_t at = atomicAdd(count, 1u);
    if (at < most_listed) list[at] = {key, tie};
  }
  // The best of the list, of all candidates each(f) -> f(key, tie) where they did not fit in (kFew: they do).
  template <bool kFew, typename Each>
  __device__ __forceinline__ void finish(Each each, uint32_t* sums) const {
    __syncthreads();
    uint32_t n = *odd ? 0 : *count;
    if (!kFew && n > most_listed) {
      uint64_t key, tie;
      exact_bound<uint64_t>(each, (uint64_t)0, 0, ~0ull, a.keep, sums, &key, &tie);
      __syncthreads();
      if (threadIdx.x == 0) *count = 0;
      __syncthreads();
      each([&](uint64_t c, uint64_t at) {
        if (c > key || (c == key && at < tie)) list[atomicAdd(count, 1u)] = {c, at};
      });
      __syncthreads();
      n = *count;
    }
    const uint64_t out = (uint64_t)blockIdx.x * a.keep;
    const auto above = [](const Entry<uint64_t>& x, const Entry<uint64_t>& y) { return x.key > y.key || (x.key == y.key && x.tie < y.tie); };
    best_of<kFew, Entry<uint64_t>>(list, n, a.keep, Entry<uint64_t>{0, ~0ull}, above, [&](uint32_t rank, const Entry<uint64_t>& e) {
      const uint32_t b = (uint32_t)(e.tie >> 56);
      const Beam& o = beam[b];
      const bool was = kind(o) == kFinished;
      const int64_t token = was ? a.end_token : (int64_t)(e.tie & 0xFFFFFFu);
      a.out_scores[out + rank] = was ? o.base.hi : total_of(o, from_order(~(uint32_t)(e.tie >> 24)), a.tau, inv_tau).hi;
      a.out_tokens[out + rank] = token;
      a.out_parents[out + rank] = (int64_t)(row0 + b);
      if (a.out_finished) a.out_finished[out + rank] = was || token == a.end_token;
      if (a.out_lengths) a.out_lengths[out + rank] = __ldg(a.lengths + row0 + b) + !was;
    });
    for (uint32_t i = min(n, a.keep) + threadIdx.x; i < a.keep; i += blockDim.x) {
      a.out_scores[out + i] = *odd ? __int_as_float(0x7FC00000) : kMinusInf;
      a.out_tokens[out + i] = -1;
      a.out_parents[out + i] = (int64_t)(row0 + i % a.beams);
      if (a.out_finished) a.out_finished[out + i] = 0;
      if (a.out_lengths) a.out_lengths[out + i] = 0;
    }
  }
};

constexpr uint32_t kFewSlots = 128;

// Few logits in a group: all of it in shared memory.  4,096 groups of 16 x 3 are 12.6 us, of 16 x 17 42: latency and
// the ranking of all by all.  kFew: so few that all of them are ranked (code that is not there
// is not fetched, which is most of the time of thousands of such groups).
template <typename E, bool kFew, bool kFar>
__global__ void __launch_bounds__(kThreads) direct_kernel(const __grid_constant__ BeamArgs a) {
  extern __shared__ __align__(16) unsigned char raw[];
  __shared__ uint32_t words[3], sums, bound_word;
  __shared__ __align__(16) uint32_t all[kThreads];
  const uint32_t t = threadIdx.x, slots = a.beams * a.vocab, warp = t / 32, lane = t % 32;
  Group<kFar> g(a, raw, slots, words);
  float* logits = reinterpret_cast<float*>(g.list + g.most_listed);
  // Lanes to a row of logits: as many as a short row has.
  const uint32_t row_lanes = a.vocab >= 32 ? 32 : 1u << (31 - __clz(a.vocab)), rows = blockDim.x / row_lanes;
  const uint32_t my_row = t / row_lanes, my_lane = t % row_lanes;
  for (uint32_t b = my_row; b < a.beams; b += rows)
    for (uint32_t j = my_lane; j < a.vocab; j += row_lanes)
      logits[b * a.vocab + j] = to_f32(static_cast<const E*>(a.x)[(g.row0 + b) * a.ldx + j]);
  __syncthreads();
  // The beams' maxima and sums: a warp to a beam, or a thread where rows are short.
  const bool by_thread = a.vocab <= 16;
  const uint32_t mine = by_thread ? 0 : lane, step = by_thread ? 1 : 32;
  for (uint32_t b = by_thread ? t : warp; b < a.beams; b += by_thread ? blockDim.x : blockDim.x / 32) {
    const uint32_t state = g.state_of(b);
    const float* x = logits + b * a.vocab;
    float m = kMinusInf, s = 0.0f;
    if (state == kAlive) {
      for (uint32_t i = mine; i < a.vocab; i += step) m = fmaxf(m, x[i]);
      if (!by_thread)
#pragma unroll
        for (int d = 16; d; d /= 2) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
      const float base = m == kMinusInf ? 0.0f : m;
      for (uint32_t i = mine; i < a.vocab; i += step) s += expf((x[i] - base) * g.inv_tau);
      if (!by_thread)
#pragma unroll
        for (int d = 16; d; d /= 2) s += __shfl_xor_sync(~0u, s, d);
    }
    if (mine == 0) g.put(b, state, m, s);
  }
  __syncthreads();
  // All candidates of a thread: f(beam, token, x), x the logit (0 for a finished beam).
  const auto each = [=](auto f) {
    for (uint32_t b = my_row; b < a.beams; b += rows) {
      const uint32_t state = g.kind(g.beam[b]);
      if (state == kAlive) {
        for (uint32_t j = my_lane; j < a.vocab; j += row_lanes) {
          const float x = logits[b * a.vocab + j];
          if (x > kMinusInf) f(b, j, x);
        }
      } else if (state == kFinished && my_lane == 0) {
        f(b, 0u, 0.0f);
      }
    }
  };
  uint64_t least = 0;
  if (!kFew && slots > 2 * a.keep && a.keep <= blockDim.x) {
    uint32_t most = 0;
    each([&](uint32_t b, uint32_t, float x) { most = max(most, (uint32_t)(g.key_of(b, x) >> 32)); });
    const uint32_t bound = exact_of(most, a.keep, blockDim.x, all, &bound_word);
    least = bound == kOrderMinusInf + 1 ? 0 : (uint64_t)bound << 32;
  }
  const auto each_key = [=](auto f) {
    each([&](uint32_t b, uint32_t token, float x) {
      const uint64_t key = g.key_of(b, x);
      if (key >= least) f(key, g.tie_of(b, x, token));
    });
  };
  each_key([&](uint64_t key, uint64_t tie) { g.push(key, tie); });
  g.template finish<kFew>(each_key, &sums);
}

constexpr uint32_t kLists = 4096;  // of a group that are noted as gone through

// The chunks' sums and sorted lists; a chain of reads that follow one another, 8 to 10 us behind the rows
// (64 groups of 8 beams, 16 kept).  A bound that `keep` continuations reach comes
// from one of each list, the depth-th; only lists whose first reaches it are gone through,
// eight lanes to a list, up to their first that does not.
template <bool kFar>
__global__ void __launch_bounds__(kThreads) group_kernel(const __grid_constant__ BeamArgs a, const __grid_constant__ Chunks ch) {
  extern __shared__ __align__(16) unsigned char raw[];
  __shared__ uint32_t words[3], sums, going, bound_word;
  __shared__ __align__(16) uint32_t tops[kThreads];
  const uint32_t t = threadIdx.x, chunks = a.beams * ch.per_row;
  Group<kFar> g(a, raw, (uint64_t)chunks * a.keep, words);
  uint32_t* lists = reinterpret_cast<uint32_t*>(g.list + g.most_listed);  // those that are gone through
  if (t == 0) going = 0;
  // The beams' sums: as many lanes to a beam as its row has chunks, up to 32.
  uint32_t lanes = 1;
  while (lanes < 32 && lanes < ch.per_row) lanes *= 2;
  const uint32_t mine = t % lanes;
  for (uint32_t b = t / lanes; b < a.beams; b += kThreads / lanes) {  // into the cache while the rows are worked on
    prefetch(a.scores + g.row0 + b);
    if (a.finished) prefetch(a.finished + g.row0 + b);
  }
  __syncthreads();  // the group's words are 0 before any beam is found odd
  wait_for_previous();
  for (uint32_t b0 = 0; b0 < a.beams; b0 += kThreads / lanes) {
    const uint32_t b = b0 + t / lanes;
    const uint32_t state = b < a.beams ? g.state_of(b) : (uint32_t)kDead;
    const float2* heads = ch.heads + (g.row0 + b) * ch.per_row;
    float m = kMinusInf, s = 0.0f;
    float2 part = make_float2(kMinusInf, 0.0f);
    if (state == kAlive) {
      if (mine < ch.per_row) part = __ldca(heads + mine);
      m = part.x;
      for (uint32_t i = mine + lanes; i < ch.per_row; i += lanes) m = fmaxf(m, __ldca(heads + i).x);
    }
    for (uint32_t d = lanes / 2; d; d /= 2) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
    const float base = m == kMinusInf ? 0.0f : m;
    const auto add = [&](float2 p) { s += p.y == 0.0f ? 0.0f : p.y * expf((p.x - base) * g.inv_tau); };
    add(part);
    if (state == kAlive)
      for (uint32_t i = mine + lanes; i < ch.per_row; i += lanes) add(__ldca(heads + i));
    for (uint32_t d = lanes / 2; d; d /= 2) s += __shfl_xor_sync(~0u, s, d);
    if (mine == 0 && b < a.beams) g.put(b, state, m, s);
  }
  __syncthreads();
  const uint2* best = reinterpret_cast<const uint2*>(ch.best) + g.row0 * ch.per_row * a.keep;
  // A list's i-th continuation, as key and tie; 0: none.
  const auto key_at = [=](uint32_t b, uint32_t list, uint32_t i, uint64_t* tie) -> uint64_t {
    const uint32_t state = g.kind(g.beam[b]);
    uint2 c = make_uint2(0, 0);
    if (state == kAlive) {
      c = __ldca(best + (uint64_t)list * a.keep + i);
      if (!(__uint_as_float(c.x) > kMinusInf)) return 0;
    } else if (state == kDead || i != 0 || list != b * ch.per_row) {
      return 0;
    }
    *tie = g.tie_of(b, __uint_as_float(c.x), c.y);
    return g.key_of(b, __uint_as_float(c.x));
  };
  // Of as many lists as are needed, the depth-th continuation: `keep` reach the least of them.  So deep that
  // a quarter of the lists is enough; deeper where the list overflows, because few lists hold most of the best.
  uint32_t depth = min(a.keep, (4 * a.keep + chunks - 1) / chunks);
  uint64_t least = 0, tie;
  const auto raise = [&](uint32_t mine, uint32_t need) {
    const uint32_t bound = exact_of(mine, need, min(chunks, kThreads), tops, &bound_word);
    if (bound > kOrderMinusInf + 1) least = max(least, (uint64_t)bound << 32);
  };
  if (chunks <= kThreads) {
    raise(t < chunks ? (uint32_t)(key_at(t / ch.per_row, t, depth - 1, &tie) >> 32) : 0, (a.keep + depth - 1) / depth);
  } else {  // several lists to a thread: the best of each thread's is one of a list
    uint32_t best_top = 0;
    for (uint32_t l = t; l < chunks; l += kThreads) best_top = max(best_top, (uint32_t)(key_at(l / ch.per_row, l, 0, &tie) >> 32));
    raise(best_top, a.keep);
  }
  const auto each_from = [=](uint64_t from, uint32_t all, bool some, auto f) {
    for (uint32_t n = t / 8; n < all; n += kThreads / 8) {
      const uint32_t l = some ? lists[n] : n, b = l / ch.per_row;
      uint64_t at_tie;
      for (uint32_t i = t % 8; i < a.keep; i += 8) {
        const uint64_t key = key_at(b, l, i, &at_tie);
        if (key == 0 || key < from) break;  // and so are all behind it
        f(key, at_tie);
      }
    }
  };
  for (;;) {
    for (uint32_t l = t; l < chunks; l += kThreads) {
      const uint64_t key = key_at(l / ch.per_row, l, 0, &tie);
      if (key == 0 || key < least) continue;
      const uint32_t at = atomicAdd(&going, 1u);
      if (at < kLists) lists[at] = l;
    }
    __syncthreads();
    const bool some = going <= kLists;  // else equal logits all over: all lists are gone through
    const uint32_t all = some ? going : chunks;
    each_from(least, all, some, [&](uint64_t key, uint64_t at_tie) { g.push(key, at_tie); });
    __syncthreads();
    if (*g.count <= g.most_listed || depth == a.keep || *g.odd) {
      g.finish<false>([=](auto f) { each_from(least, all, some, f); }, &sums);
      return;
    }
    depth = min(a.keep, 4 * depth);
    raise(t < chunks ? (uint32_t)(key_at(t / ch.per_row, t, depth - 1, &tie) >> 32) : 0, (a.keep + depth - 1) / depth);
    if (t == 0) *g.count = going = 0;
    __syncthreads();
  }
}

// Logits of a group that one block takes as they are: what fits into its shared memory beside the list.  (4,096
// groups of 16 x 100 and 16 x 250: 84 and 120 us so, 240 and 170 by rows; 64 groups of 16 x 250: 16.4 and 13.0.)
constexpr uint64_t kDirectMost = 4096;

// How rows are cut: 8 vectors a thread, twice
// where there are blocks enough all the same (what a block does once takes as long as a tile),
// 2 where there would be too few for two on each of 152 SMs.  Rows that 64 threads hold in
// two vectors each have blocks of 64.  (512 rows of 131,072 bf16, 16 kept: 45 us so, 54 with one
// tile, 60 with 4 vectors; 16,000 rows of 300 and 1,000: 49 and 52 us, 294 and 110 with blocks of 256.)
// A row's chunks are equally long: 512 rows of 50,000 f16, 32 kept, 40 us, and 43 with all but the last full.
constexpr uint32_t kShort = 64;
Chunks chunks_of(uint32_t groups, uint32_t beams, uint64_t vocab, uint32_t keep, uint32_t width, void* workspace,
                 uint32_t* vectors, uint64_t* bytes) {
  Chunks c = {};
  *bytes = 0;
  if (beams * vocab <= kDirectMost) return c;
  const uint64_t rows = (uint64_t)groups * beams;
  c.tiles = 1;
  c.threads = vocab <= 2 * kShort * width && keep <= kShort * 3 / 8 ? kShort : kThreads;
  const auto per_row = [&](uint32_t v) { return (vocab + c.threads * v * width - 1) / (c.threads * v * width); };
  *vectors = 8;
  if (per_row(2) == 1 || rows * per_row(*vectors) < 304) *vectors = 2;
  else if (keep <= 96 && rows * per_row(2 * *vectors) >= 1216 && per_row(*vectors) > 1) c.tiles = 2;  // (the lists would overflow)
  c.per_row = (uint32_t)per_row(c.tiles * *vectors);
  c.elements = (uint32_t)((vocab + (uint64_t)c.per_row * width - 1) / ((uint64_t)c.per_row * width)) * width;  // evenly
  c.per_row = (uint32_t)((vocab + c.elements - 1) / c.elements);
  c.heads = static_cast<float2*>(workspace);
  const uint64_t records = rows * c.per_row, heads = (records * sizeof(float2) + 255) / 256 * 256;
  c.best = reinterpret_cast<Candidate*>(static_cast<char*>(workspace) + heads);
  *bytes = heads + records * keep * sizeof(Candidate);
  return c;
}

template <typename E>
cudaError_t launch_step(const BeamArgs& a, void* workspace, cudaStream_t st) {
  uint32_t vectors = 0;
  uint64_t bytes = 0;
  const bool aligned = ((uintptr_t)a.x | (a.ldx * sizeof(E))) % 16 == 0;
  const Chunks c = chunks_of(a.groups, a.beams, a.vocab, a.keep, Vec<E>::kWidth, workspace, &vectors, &bytes);
  const bool direct = c.per_row == 0, far = a.penalty > kNearPenalty;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute after;
  cfg.gridDim = dim3(a.groups);
  cfg.stream = st;
  cfg.attrs = &after;
  if (direct) {
    const uint32_t n = a.beams * a.vocab;
    uint32_t threads = (n / 2 + 31) / 32 * 32;
    threads = threads < 32 ? 32 : threads > kThreads ? kThreads : threads;
    if (threads < a.keep && n > kFewSlots) threads = (a.keep + 31) / 32 * 32;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = group_bytes(a.beams, n, n);
    if (far) return cudaLaunchKernelEx(&cfg, n <= kFewSlots ? direct_kernel<E, true, true> : direct_kernel<E, false, true>, a);
    return cudaLaunchKernelEx(&cfg, n <= kFewSlots ? direct_kernel<E, true, false> : direct_kernel<E, false, false>, a);
  }
  const uint64_t blocks = (uint64_t)a.groups * a.beams * c.per_row;
  const auto rows = [&](auto kernel) { return launch_plain(kernel, blocks, c.threads, st, a, c); };
  cudaError_t e;
  if (c.threads == kShort) e = aligned ? rows(row_kernel<E, 2, true, kShort>) : rows(row_kernel<E, 2, false, kShort>);
  else if (aligned) e = vectors == 8 ? rows(row_kernel<E, 8, true, kThreads>) : rows(row_kernel<E, 2, true, kThreads>);
  else e = vectors == 8 ? rows(row_kernel<E, 8, false, kThreads>) : rows(row_kernel<E, 2, false, kThreads>);
  if (e != cudaSuccess) return e;
  cfg.blockDim = dim3(kThreads);
  const uint64_t chunks = (uint64_t)a.beams * c.per_row;  // beams, list and lists fit into 48 KB
  cfg.dynamicSmemBytes = group_bytes(a.beams, chunks * a.keep, chunks < kLists ? chunks : kLists);
  after.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  after.val.programmaticStreamSerializationAllowed = 1;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, far ? group_kernel<true> : group_kernel<false>, a, c);
}

// ---- states -----------------------------------------------------------------

// Rows' tiles by way of shared memory: a block reads a tile of every row that is
// somebody's parent, once, and then writes the tile of every row, so that rows
// may change places.
struct Tiles {
  uint32_t units;          // of a tile and row
  uint32_t run;            // units of a token (and head, where heads are apart)
  uint32_t per_row, heads; // tiles; heads that are apart
};

// What a block's tile is made of.
struct Moves {
  int32_t parent[BF_MAX_BEAMS];       // of each row; -1: stays
  uint32_t limit[BF_MAX_BEAMS];       // units of the tile that the row's parent has
  uint32_t needed[BF_MAX_BEAMS / 32]; // rows that are parents
  uint32_t from[BF_MAX_BEAMS];        // slot -> row
  uint32_t have[BF_MAX_BEAMS];        // slot -> units
  uint32_t many;

  __device__ __forceinline__ uint32_t slot_of(uint32_t p) const {
    uint32_t n = __popc(needed[p / 32] & ((1u << p % 32) - 1));
    for (uint32_t w = 0; w < p / 32; ++w) n += __popc(needed[w]);
    return n;
  }
};

// Units of a tile at `first` that a row of `n` tokens has.
__device__ __forceinline__ uint32_t units_of(int64_t n, uint64_t tokens, uint64_t first, const Tiles& tl) {
  const uint64_t end = n <= 0 ? 0 : min((uint64_t)n, tokens) * tl.run;
  return end > first ? (uint32_t)min(end - first, (uint64_t)tl.units) : 0;
}

// By all threads of a block.
__device__ __forceinline__ void find_moves(const ReorderArgs& a, const Tiles& tl, uint64_t row0, uint64_t first, Moves& mv) {
  const uint32_t t = threadIdx.x;
  if (t < BF_MAX_BEAMS / 32) mv.needed[t] = 0;
  __syncthreads();
  for (uint32_t b = t; b < a.beams; b += blockDim.x) {
    const int64_t p = __ldg(a.parents + row0 + b) - (int64_t)row0;
    int32_t from = p >= 0 && p < (int64_t)a.beams && !(a.in_place && p == (int64_t)b) ? (int32_t)p : -1;
    const uint32_t mine = from < 0 ? 0 : units_of(a.lengths ? __ldg(a.lengths + row0 + from) : (int64_t)a.tokens, a.tokens, first, tl);
    if (mine == 0) from = -1;
    mv.parent[b] = from;
    mv.limit[b] = mine;
    if (from >= 0) atomicOr(&mv.needed[from / 32], 1u << from % 32);
  }
  __syncthreads();
  for (uint32_t b = t; b < a.beams; b += blockDim.x)
    if (mv.parent[b] >= 0) {
      const uint32_t s = mv.slot_of(mv.parent[b]);  // the same for all rows of a parent
      mv.from[s] = mv.parent[b];
      mv.have[s] = mv.limit[b];
    }
  if (t == 0) {
    uint32_t many = 0;
    for (uint32_t w = 0; w < (a.beams + 31) / 32; ++w) many += __popc(mv.needed[w]);
    mv.many = many;
  }
  __syncthreads();
}

// A block's place: array, head, first row of its group, first unit of its tile.
struct TilePlace {
  uint32_t array, head;
  uint64_t row0, first;
  __device__ __forceinline__ TilePlace(const ReorderArgs& a, const Tiles& tl) {
    uint32_t i = blockIdx.x;
    first = (uint64_t)(i % tl.per_row) * tl.units;
    i /= tl.per_row;
    head = i % tl.heads;
    i /= tl.heads;
    array = i % a.count;
    row0 = (uint64_t)(i / a.count) * a.beams;
  }
};

// Rows whose valid part is one run of 16-byte units: a warp has the copying done, three
// blocks of up to 64 KB an SM on their way.  4.15 GB in 631 us, 6.6 TB/s: the memory.  (By
// loads and stores of 256 threads, two of each on their way: 3.7 TB/s.)
__global__ void __launch_bounds__(32) reorder_runs_kernel(const __grid_constant__ ReorderArgs a, const __grid_constant__ Tiles tl) {
  extern __shared__ __align__(16) unsigned char held[];
  __shared__ Moves mv;
  __shared__ uint64_t full;
  __shared__ uint32_t gave_up;
  const uint32_t lane = threadIdx.x;
  const TilePlace at(a, tl);
  find_moves(a, tl, at.row0, at.first, mv);
  const uint32_t many = mv.many;
  if (many == 0) return;
  uint32_t bytes = 0;
  for (uint32_t s = lane; s < many; s += 32) bytes += mv.have[s] * 16;
  bytes = __reduce_add_sync(~0u, bytes);
  if (lane == 0) {
    gave_up = 0;
    barrier_init(&full, 1);
    fence_barriers();
    barrier_expect(&full, bytes);
  }
  __syncwarp();
  for (uint32_t s = lane; s < many; s += 32)
    copy_run(held + s * tl.units * 16, a.from[at.array] + (at.row0 + mv.from[s]) * a.from_row + at.head * a.from_head + at.first * 16,
             mv.have[s] * 16, &full);
  bool come = barrier_wait(&full, 0, &gave_up);
  if (!come) {  // once more: no copy is on its way to this block's memory when it ends, if the GPU does anything still
    __syncwarp();
    if (lane == 0) gave_up = 0;
    __syncwarp();
    come = barrier_wait(&full, 0, &gave_up);
  }
  if (!come) {  // rows of two beams in one would show nowhere; bytes of 255 do: NaN, or -1
    for (uint32_t b = 0; b < a.beams; ++b)
      for (uint32_t u = lane; mv.parent[b] >= 0 && u < mv.limit[b]; u += 32)
        reinterpret_cast<uint4*>(a.to[at.array] + (at.row0 + b) * a.to_row + at.head * a.to_head + at.first * 16)[u] =
            make_uint4(~0u, ~0u, ~0u, ~0u);
    return;
  }
  for (uint32_t b = lane; b < a.beams; b += 32)
    if (mv.parent[b] >= 0)
      put_run(a.to[at.array] + (at.row0 + b) * a.to_row + at.head * a.to_head + at.first * 16,
              held + mv.slot_of(mv.parent[b]) * tl.units * 16, mv.limit[b] * 16);
  put_runs_end();
}

// Everything else.  U: the unit that all addresses, strides and widths are multiples
// of.  kFlat: a token's units follow the one's before.
template <typename U, bool kFlat>
__global__ void __launch_bounds__(kThreads) reorder_kernel(const __grid_constant__ ReorderArgs a, const __grid_constant__ Tiles tl) {
  extern __shared__ __align__(16) unsigned char raw[];
  U* held = reinterpret_cast<U*>(raw);
  __shared__ Moves mv;
  const uint32_t t = threadIdx.x;
  const TilePlace at(a, tl);
  find_moves(a, tl, at.row0, at.first, mv);
  const uint32_t many = mv.many;
  if (many == 0) return;
  const auto place = [&](uint64_t u, uint64_t token) -> uint64_t {  // bytes of unit u behind a row's first
    if constexpr (kFlat) return u * sizeof(U);
    const uint64_t n = u / tl.run;
    return n * token + (u - n * tl.run) * sizeof(U);
  };
  const char* from = a.from[at.array] + at.head * a.from_head;
  char* to = a.to[at.array] + at.head * a.to_head;
#pragma unroll 4
  for (uint32_t i = t; i < many * tl.units; i += kThreads) {
    const uint32_t s = i / tl.units, u = i - s * tl.units;
    if (u < mv.have[s])
      held[i] = *reinterpret_cast<const U*>(from + (at.row0 + mv.from[s]) * a.from_row + place(at.first + u, a.from_token));
  }
  __syncthreads();
  for (uint32_t b = 0; b < a.beams; ++b) {
    if (mv.parent[b] < 0) continue;
    const uint32_t s = mv.slot_of(mv.parent[b]), n = mv.limit[b];
    for (uint32_t u = t; u < n; u += kThreads)
      *reinterpret_cast<U*>(to + (at.row0 + b) * a.to_row + place(at.first + u, a.to_token)) = held[s * tl.units + u];
  }
}

template <typename U>
cudaError_t launch_units(const ReorderArgs& a, bool flat, cudaStream_t st) {
  constexpr bool kRuns = sizeof(U) == 16;
  Tiles tl = {};
  tl.run = (uint32_t)(a.width / sizeof(U));
  tl.heads = a.heads;
  const uint64_t row = a.tokens * tl.run, most = 65536 / (a.beams * sizeof(U));  // 64 KB of a tile: three blocks an SM
  uint64_t units = 8192 / sizeof(U);
  if (units > most) units = most;
  if (units > row) units = row;
  tl.units = (uint32_t)units;
  const uint64_t per_row = (row + units - 1) / units, blocks = per_row * tl.heads * a.count * a.groups;
  if (per_row > 0x7FFFFFFFu || blocks > 0x7FFFFFFFu) return cudaErrorInvalidValue;
  tl.per_row = (uint32_t)per_row;
  const uint32_t shared = (uint32_t)(units * a.beams * sizeof(U));
  const auto launch = [&](auto kernel, uint32_t threads) {
    if (shared > 32 * 1024) {
      const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 65536);
      if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((uint32_t)blocks);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = st;
    return cudaLaunchKernelEx(&cfg, kernel, a, tl);
  };
  if (flat && kRuns) return launch(reorder_runs_kernel, 32);
  return flat ? launch(reorder_kernel<U, true>, kThreads) : launch(reorder_kernel<U, false>, kThreads);
}

}  // namespace

uint64_t beam_bytes(uint32_t groups, uint32_t beams, uint64_t vocab, uint32_t keep) {
  uint64_t most = 0;
  for (uint32_t width = 4; width <= 8; width *= 2) {  // elements in 16 bytes
    uint32_t vectors;
    uint64_t bytes;
    chunks_of(groups, beams, vocab, keep, width, nullptr, &vectors, &bytes);
    if (bytes > most) most = bytes;
  }
  return (most + 255) / 256 * 256;
}

cudaError_t launch_beam_step(const BeamArgs& a, void* workspace, cudaStream_t st) {
  return a.dtype == BF_F32    ? launch_step<float>(a, workspace, st)
         : a.dtype == BF_BF16 ? launch_step<__nv_bfloat16>(a, workspace, st)
                              : launch_step<__half>(a, workspace, st);
}

cudaError_t launch_reorder(const ReorderArgs& args, cudaStream_t st) {
  ReorderArgs a = args;
  // Heads that follow one another are one run.
  if (a.heads > 1 && a.from_head == a.width && a.to_head == a.width) {
    a.width *= a.heads;
    a.heads = 1;
  }
  const bool flat = a.tokens < 2 || (a.from_token == a.width && a.to_token == a.width);
  uint64_t bits = a.width;
  if (a.tokens > 1) bits |= a.from_token | a.to_token;
  if (a.heads > 1) bits |= a.from_head | a.to_head;
  if ((uint64_t)a.groups * a.beams > 1) bits |= a.from_row | a.to_row;
  for (uint32_t k = 0; k < a.count; ++k) bits |= (uintptr_t)a.from[k] | (uintptr_t)a.to[k];
  if (bits % 16 == 0) return launch_units<uint4>(a, flat, st);
  if (bits % 4 == 0) return launch_units<uint32_t>(a, flat, st);
  return bits % 2 == 0 ? launch_units<uint16_t>(a, flat, st) : launch_units<uint8_t>(a, flat, st);
}

}  // namespace bfk
