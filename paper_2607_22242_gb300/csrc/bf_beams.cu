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
constexpr uint32_t kList = 1024;  // entries of a block's list

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
// Where the warps' values are alike: each warp finds its ceil(2 keep / warps)-th
// largest, and the one of those that enough warps reach is the bound.  One barrier.
// `warps` holds a word for each warp.
__device__ __forceinline__ uint32_t bound_of(uint32_t mine, uint32_t keep, uint32_t* warps) {
  const uint32_t count = blockDim.x / 32, each = min(32u, (2 * keep + count - 1) / count), lane = threadIdx.x % 32;
  uint32_t most = 0;
  for (uint32_t i = 0; i < each; ++i) {
    most = __reduce_max_sync(~0u, mine);
    if (lane == __ffs(__ballot_sync(~0u, mine == most)) - 1u) mine = 0;
  }
  if (lane == 0) warps[threadIdx.x / 32] = most;
  __syncthreads();
  // Warps whose values are reached by `each` of theirs: the ceil(keep / each) largest are enough.
  const uint32_t need = (keep + each - 1) / each, w = lane < count ? warps[lane] : 0;
  uint32_t above = 0;
  for (uint32_t i = 0; i < count; ++i) {
    const uint32_t o = __shfl_sync(~0u, w, i);
    above += o > w || (o == w && i < lane);
  }
  const uint32_t bound = __reduce_max_sync(~0u, lane < count && above == need - 1 ? w : 0);
  return max(bound, kOrderMinusInf + 1);
}
// Where one warp's may be far above another's (beams of different scores): bisection.
__device__ __forceinline__ uint32_t bound_by_halves(uint32_t mine, uint32_t keep) {
  uint32_t lo = kOrderMinusInf + 1, hi = 0xFFFFFFFFu;
  if ((uint32_t)__syncthreads_count(mine >= lo) <= keep) return lo;
  while (hi - lo > 1) {
    const uint32_t mid = lo + (hi - lo) / 2, n = __syncthreads_count(mine >= mid);
    if (n >= keep) {
      lo = mid;
      if (n <= keep + keep / 4) break;
    } else {
      hi = mid;
    }
  }
  return lo;
}

// Where a list would overflow (many equal values): the exact keep-th largest of
// all (key, tie), by counting.  each(f) calls f(key, tie) for all of a thread's
// candidates.  Candidates of at least `key`, and of a tie below `tie` where they have
// just that key, are the best; there are `keep` of them or, with fewer in all, all.
template <typename Key, typename Each>
__device__ __noinline__ void exact_bound(Each each, Key least, uint32_t keep, uint32_t* sums, Key* key, uint64_t* tie) {
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
  uint64_t below = 0, upto = ~0ull;  // the lowest tie that makes it `keep`
  while (upto - below > 1) {
    const uint64_t mid = below + (upto - below) / 2;
    if (count(lo, mid) >= keep) upto = mid;
    else below = mid;
  }
  *key = lo;
  *tie = upto;
}

// Calls put(rank, entry) for the best `keep` of a list of n.
template <typename Key, typename Put>
__device__ __forceinline__ void rank_list(const Entry<Key>* list, uint32_t n, uint32_t keep, Put put) {
  for (uint32_t i = threadIdx.x; i < n; i += blockDim.x) {
    const Entry<Key> e = list[i];
    uint32_t rank = 0;
    for (uint32_t j = 0; j < n; ++j) {
      const Entry<Key> o = list[j];
      rank += o.key > e.key || (o.key == e.key && o.tie < e.tie);
    }
    if (rank < keep) put(rank, e);
  }
}

// ---- rows -------------------------------------------------------------------

struct Candidate {
  float x;  // -inf: none
  uint32_t token;
};

struct Chunks {
  uint32_t per_row, elements;
  float2* heads;    // [rows][per_row]: maximum, sum of e^((x - maximum) / tau)
  Candidate* best;  // [rows][per_row][keep]
};

constexpr uint32_t kThreads = 256;

__device__ __forceinline__ bool is_alive(const BeamArgs& a, uint64_t row) {
  const float score = __ldg(a.scores + row);
  return !(score == kMinusInf) && !(a.finished && __ldg(a.finished + row));
}

// A chunk of a row: V vectors a thread, cut by the row's elements and not by
// addresses, so that equal rows have equal sums.  kAligned: rows start at 16 bytes.
template <typename E, int V, bool kAligned>
__global__ void __launch_bounds__(kThreads) row_kernel(const __grid_constant__ BeamArgs a, const __grid_constant__ Chunks ch) {
  constexpr uint32_t kW = Vec<E>::kWidth;
  __shared__ Entry<uint32_t> list[kList];
  __shared__ uint32_t count, sums, warp_bound[kThreads / 32];
  __shared__ float warp_max[kThreads / 32], warp_sum[kThreads / 32];
  let_next_start();
  const uint32_t row = blockIdx.x / ch.per_row, chunk = blockIdx.x - row * ch.per_row, t = threadIdx.x;
  if (!is_alive(a, row)) return;
  if (t == 0) count = 0;
  const E* x = static_cast<const E*>(a.x) + (uint64_t)row * a.ldx;
  const uint32_t cut = chunk * ch.elements, first = cut + t * kW;
  const uint32_t none = minus_inf_bits(E());
  uint4 u[V];
  if constexpr (kAligned) {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const uint32_t j = first + (uint32_t)k * kThreads * kW;
      u[k] = make_uint4(none, none, none, none);
      if (j + kW <= a.vocab) u[k] = __ldcs(reinterpret_cast<const uint4*>(x + j));
      else if (j < a.vocab) u[k] = load_ends<E>(x + j, 0, (int32_t)(a.vocab - j), none);
    }
  } else {
    const Extent matrix(static_cast<const E*>(a.x), (uint64_t)a.groups * a.beams, a.ldx, a.vocab);
    Unaligned<E> raw[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const uint32_t j = first + (uint32_t)k * kThreads * kW;
      if (j < a.vocab) raw[k].load(x, a.vocab, (int64_t)j, matrix);
    }
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const uint32_t j = first + (uint32_t)k * kThreads * kW;
      u[k] = make_uint4(none, none, none, none);
      if (j + kW <= a.vocab) u[k] = raw[k].take();
      else if (j < a.vocab) u[k] = load_ends<E>(x + j, 0, (int32_t)(a.vocab - j), none);
    }
  }
  const float tmax = max_of<E, V>(u);
  float m = tmax;
#pragma unroll
  for (int d = 16; d; d /= 2) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
  if (t % 32 == 0) warp_max[t / 32] = m;
  __syncthreads();
#pragma unroll
  for (uint32_t w = 0; w < kThreads / 32; ++w) m = fmaxf(m, warp_max[w]);
  // (x - m) c2 as x c2 - r, r = m c2 rounded, where that is of ordinary size, and what r is off
  // by put back into the sum; else (x - m) c2 (rows of the type's lowest values).
  const bool fits = fabsf(m) * a.c2 < 1024.0f;
  const float usable = m == kMinusInf ? 0.0f : m, r1 = fits ? -m * a.c2 : 0.0f, rest = fits ? fmaf(-m, a.c2, m * a.c2) : 0.0f;
  const float2 base = fits ? make_float2(0.0f, 0.0f) : make_float2(-usable, -usable), r = make_float2(r1, r1), c2 = make_float2(a.c2, a.c2);
  float2 s2 = make_float2(0.0f, 0.0f);
#pragma unroll
  for (int k = 0; k < V; ++k) {
    float2 f[kW / 2];
    unpack<E>(u[k], f);
#pragma unroll
    for (uint32_t i = 0; i < kW / 2; ++i) {
      const float2 e = __ffma2_rn(__fadd2_rn(f[i], base), c2, r);
      s2 = __fadd2_rn(s2, make_float2(exp2_of(e.x), exp2_of(e.y)));
    }
  }
  float s = s2.x + s2.y;
#pragma unroll
  for (int d = 16; d; d /= 2) s += __shfl_xor_sync(~0u, s, d);
  if (t % 32 == 0) warp_sum[t / 32] = fmaf(s, rest * 0.693147180559945309f, s);
  // The candidates: all that reach a bound which `keep` threads' maxima reach.
  const uint32_t bound = bound_of(order_of(tmax), a.keep, warp_bound);
  const float least = from_order(bound);
#pragma unroll
  for (int k = 0; k < V; ++k) {
    if (!(max_of<E, 1>(u + k) >= least)) continue;
    float2 f[kW / 2];
    unpack<E>(u[k], f);
#pragma unroll
    for (uint32_t i = 0; i < kW; ++i) {
      const float v = i % 2 ? f[i / 2].y : f[i / 2].x;
      if (v >= least) {
        const uint32_t at = atomicAdd(&count, 1u);
        if (at < kList) list[at] = {order_of(v), first + (uint32_t)k * kThreads * kW + i};
      }
    }
  }
  __syncthreads();
  uint32_t n = count;
  if (n > kList) {
    // From memory again: registers that a call takes by reference would be in memory for everybody.
    const uint32_t some = min(ch.elements, a.vocab - cut);
    const auto each = [=](auto f) {
      for (uint32_t i = t; i < some; i += kThreads) {
        const float v = to_f32(x[cut + i]);
        if (v >= least) f(order_of(v), (uint64_t)i);
      }
    };
    uint32_t key;
    uint64_t tie;
    exact_bound<uint32_t>(each, bound, a.keep, &sums, &key, &tie);
    __syncthreads();
    if (t == 0) count = 0;
    __syncthreads();
    each([&](uint32_t c, uint64_t at) {
      if (c > key || (c == key && at < tie)) list[atomicAdd(&count, 1u)] = {c, at + cut};
    });
    __syncthreads();
    n = count;
  }
  const uint64_t record = (uint64_t)row * ch.per_row + chunk;
  Candidate* best = ch.best + record * a.keep;
  rank_list(list, n, a.keep, [&](uint32_t rank, const Entry<uint32_t>& e) { best[rank] = {from_order(e.key), (uint32_t)e.tie}; });
  for (uint32_t i = min(n, a.keep) + t; i < a.keep; i += kThreads) best[i] = {kMinusInf, 0};
  if (t == 0) {
    float total = 0.0f;
    for (uint32_t w = 0; w < kThreads / 32; ++w) total += warp_sum[w];
    ch.heads[record] = make_float2(m, total);
  }
}

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

// What a beam's continuations are made from: total = base + (x - most) / tau, rank = total * weight.
struct Beam {
  Two base, weight;  // score - ln sum (a finished beam's score); 1 / max(1, length)^penalty
  float most;        // the row's largest logit
  uint32_t state;
};

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

// A group's beams, its list and (kDirect) its logits, in dynamic shared memory.
__host__ __device__ __forceinline__ uint32_t list_of(uint64_t slots) { return slots < kList ? (uint32_t)slots : kList; }
__host__ __device__ __forceinline__ uint32_t group_bytes(uint32_t beams, uint64_t slots, uint64_t logits) {
  return (uint32_t)((beams * sizeof(Beam) + 15) / 16 * 16 + list_of(slots) * sizeof(Entry<uint64_t>) + logits * 4);
}

template <typename E, bool kDirect>
__global__ void __launch_bounds__(kThreads) group_kernel(const __grid_constant__ BeamArgs a, const __grid_constant__ Chunks ch) {
  extern __shared__ __align__(16) unsigned char raw[];
  __shared__ uint32_t count, sums, odd;
  const uint32_t g = blockIdx.x, t = threadIdx.x, warps = blockDim.x / 32, warp = t / 32, lane = t % 32;
  const uint32_t row_slots = kDirect ? a.vocab : ch.per_row * a.keep, slots = a.beams * row_slots, most_listed = list_of(slots);
  Beam* beam = reinterpret_cast<Beam*>(raw);
  Entry<uint64_t>* list = reinterpret_cast<Entry<uint64_t>*>(raw + (a.beams * sizeof(Beam) + 15) / 16 * 16);
  float* logits = reinterpret_cast<float*>(list + most_listed);
  const uint64_t row0 = (uint64_t)g * a.beams;
  const float inv_tau = 1.0f / a.tau;
  if (t == 0) count = odd = 0;
  // Lanes to a row of logits: as many as a short row has.
  const uint32_t row_lanes = row_slots >= 32 ? 32 : 1u << (31 - __clz(row_slots)), row_warps = warps * (32 / row_lanes);
  const uint32_t my_row = t / row_lanes, my_lane = t % row_lanes;
  if constexpr (kDirect) {
    for (uint32_t b = my_row; b < a.beams; b += row_warps)
      for (uint32_t j = my_lane; j < a.vocab; j += row_lanes)
        logits[b * a.vocab + j] = to_f32(static_cast<const E*>(a.x)[(row0 + b) * a.ldx + j]);
  } else {
    wait_for_previous();
  }
  __syncthreads();
  // The beams' maxima and sums: a warp to a beam, or a thread where rows are short.
  const bool by_thread = kDirect && a.vocab <= 16;
  for (uint32_t b = by_thread ? t : warp; b < a.beams; b += by_thread ? blockDim.x : warps) {
    const float score = __ldg(a.scores + row0 + b);
    const uint32_t state = score == kMinusInf ? kDead : a.finished && __ldg(a.finished + row0 + b) ? kFinished : kAlive;
    float m = kMinusInf, s = 0.0f;
    if (state == kAlive) {
      const uint32_t n = kDirect ? a.vocab : ch.per_row, mine = by_thread ? 0 : lane, step = by_thread ? 1 : 32;
      const float2* heads = ch.heads + (row0 + b) * ch.per_row;
      for (uint32_t i = mine; i < n; i += step) m = fmaxf(m, kDirect ? logits[b * a.vocab + i] : __ldca(heads + i).x);
      if (!by_thread)
#pragma unroll
        for (int d = 16; d; d /= 2) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
      const float base = m == kMinusInf ? 0.0f : m;
      for (uint32_t i = mine; i < n; i += step) {
        if constexpr (kDirect) {
          s += expf((logits[b * a.vocab + i] - base) * inv_tau);
        } else {
          const float2 part = __ldca(heads + i);
          s += part.y == 0.0f ? 0.0f : part.y * expf((part.x - base) * inv_tau);
        }
      }
      if (!by_thread)
#pragma unroll
        for (int d = 16; d; d /= 2) s += __shfl_xor_sync(~0u, s, d);
    }
    if (by_thread || lane == 0) {
      Beam o;
      o.state = state == kAlive && m == kMinusInf && s == s ? (uint32_t)kDead : state;
      o.most = o.state == kAlive ? m : 0.0f;
      o.base = {score, 0.0f};
      if (o.state == kAlive) {
        const Two l = log_of(s);
        const Two d = two_sum(score, -l.hi);
        o.base = quick_two(d.hi, d.lo - l.lo);
      }
      o.weight = {1.0f, 0.0f};
      beam[b] = o;
      if (score != score || score == -kMinusInf || s != s) odd = 1;
    }
  }
  __syncthreads();
  if (a.penalty != 0.0f) {  // a thread to a beam: these are of 64 bits
    for (uint32_t b = t; b < a.beams; b += blockDim.x) {
      const int64_t n = __ldg(a.lengths + row0 + b) + (beam[b].state != kFinished);
      const double w = pow((double)(n < 1 ? 1 : n), -(double)a.penalty);
      const float hi = (float)w;
      beam[b].weight = {hi, (float)(w - (double)hi)};
    }
    __syncthreads();
  }
  // All candidates of a thread: f(beam, token, x), x the logit (0 for a finished beam).
  const auto each = [&](auto f) {
    for (uint32_t b = my_row; b < a.beams; b += row_warps) {
      const uint32_t state = beam[b].state;
      if (state == kAlive) {
#pragma unroll 4
        for (uint32_t j = my_lane; j < row_slots; j += row_lanes) {
          if constexpr (kDirect) {
            const float x = logits[b * a.vocab + j];
            if (x > kMinusInf) f(b, j, x);
          } else {
            const uint2 c = __ldca(reinterpret_cast<const uint2*>(ch.best) + (row0 + b) * row_slots + j);
            if (__uint_as_float(c.x) > kMinusInf) f(b, c.y, __uint_as_float(c.x));
          }
        }
      } else if (state == kFinished && my_lane == 0) {
        f(b, 0u, 0.0f);
      }
    }
  };
  const auto key_of = [&](uint32_t b, float x) {
    const Beam& o = beam[b];
    const Two total = o.state == kFinished ? o.base : total_of(o, x, a.tau, inv_tau);
    return order_of(a.penalty != 0.0f ? times(total, o.weight) : total);
  };
  // Equal in both parts: the lower beam, in it the larger logit, then the lower token (8, 32 and 24 bits).
  const auto tie_of = [](uint32_t b, float x, uint32_t token) { return (uint64_t)b << 56 | (uint64_t)~order_of(x) << 24 | token; };
  uint32_t n = 0;
  if (!odd) {
    uint64_t least = 0;
    if (slots > 2 * a.keep && slots > 128 && a.keep <= blockDim.x) {
      uint32_t most = 0;
      each([&](uint32_t b, uint32_t, float x) { most = max(most, (uint32_t)(key_of(b, x) >> 32)); });
      const uint32_t bound = bound_by_halves(most, a.keep);
      least = bound == kOrderMinusInf + 1 ? 0 : (uint64_t)bound << 32;
    }
    each([&](uint32_t b, uint32_t token, float x) {
      const uint64_t key = key_of(b, x);
      if (key >= least) {
        const uint32_t at = atomicAdd(&count, 1u);
        if (at < most_listed) list[at] = {key, tie_of(b, x, token)};
      }
    });
    __syncthreads();
    n = count;
    if (n > most_listed) {
      const auto each_key = [&](auto f) {
        each([&](uint32_t b, uint32_t token, float x) {
          const uint64_t key = key_of(b, x);
          if (key >= least) f(key, tie_of(b, x, token));
        });
      };
      uint64_t key, tie;
      exact_bound<uint64_t>(each_key, (uint64_t)0, a.keep, &sums, &key, &tie);
      __syncthreads();
      if (t == 0) count = 0;
      __syncthreads();
      each_key([&](uint64_t c, uint64_t at) {
        if (c > key || (c == key && at < tie)) list[atomicAdd(&count, 1u)] = {c, at};
      });
      __syncthreads();
      n = count;
    }
  }
  const uint64_t out = (uint64_t)g * a.keep;
  rank_list(list, n, a.keep, [&](uint32_t rank, const Entry<uint64_t>& e) {
    const uint32_t b = (uint32_t)(e.tie >> 56);
    const Beam& o = beam[b];
    const bool was = o.state == kFinished;
    const int64_t token = was ? a.end_token : (int64_t)(e.tie & 0xFFFFFFu);
    a.out_scores[out + rank] = was ? o.base.hi : total_of(o, from_order(~(uint32_t)(e.tie >> 24)), a.tau, inv_tau).hi;
    a.out_tokens[out + rank] = token;
    a.out_parents[out + rank] = (int64_t)(row0 + b);
    if (a.out_finished) a.out_finished[out + rank] = was || token == a.end_token;
    if (a.out_lengths) a.out_lengths[out + rank] = __ldg(a.lengths + row0 + b) + !was;
  });
  for (uint32_t i = min(n, a.keep) + t; i < a.keep; i += blockDim.x) {
    a.out_scores[out + i] = odd ? __int_as_float(0x7FC00000) : kMinusInf;
    a.out_tokens[out + i] = -1;
    a.out_parents[out + i] = (int64_t)(row0 + i % a.beams);
    if (a.out_finished) a.out_finished[out + i] = 0;
    if (a.out_lengths) a.out_lengths[out + i] = 0;
  }
}

constexpr uint64_t kDirectMost = 4096;  // logits of a group that one block takes as they are

// How rows are cut: 8 vectors a thread (4 where each is put together from two), 2
// where there are too few blocks for two on each of 152 SMs.
Chunks chunks_of(uint32_t groups, uint32_t beams, uint64_t vocab, uint32_t keep, uint32_t width, bool aligned, void* workspace,
                 uint32_t* vectors, uint64_t* bytes) {
  Chunks c = {};
  *bytes = 0;
  if (beams * vocab <= kDirectMost) return c;
  const uint64_t rows = (uint64_t)groups * beams;
  const auto per_row = [&](uint32_t v) { return (vocab + kThreads * v * width - 1) / (kThreads * v * width); };
  *vectors = aligned ? 8 : 4;
  if (rows * per_row(*vectors) < 304) *vectors = 2;
  c.per_row = (uint32_t)per_row(*vectors);
  c.elements = kThreads * *vectors * width;
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
  const Chunks c = chunks_of(a.groups, a.beams, a.vocab, a.keep, Vec<E>::kWidth, aligned, workspace, &vectors, &bytes);
  const bool direct = c.per_row == 0;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute after;
  cfg.gridDim = dim3(a.groups);
  cfg.stream = st;
  cfg.attrs = &after;
  if (direct) {
    const uint32_t n = a.beams * a.vocab;
    uint32_t threads = (n / 2 + 31) / 32 * 32;
    threads = threads < 32 ? 32 : threads > kThreads ? kThreads : threads;
    if (threads < a.keep && n > 128) threads = (a.keep + 31) / 32 * 32;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = group_bytes(a.beams, n, n);
    return cudaLaunchKernelEx(&cfg, group_kernel<E, true>, a, c);
  }
  const uint64_t blocks = (uint64_t)a.groups * a.beams * c.per_row;
  const auto rows = [&](auto kernel) { return launch_plain(kernel, blocks, kThreads, st, a, c); };
  const cudaError_t e = aligned ? (vectors == 8 ? rows(row_kernel<E, 8, true>) : rows(row_kernel<E, 2, true>))
                                : (vectors == 4 ? rows(row_kernel<E, 4, false>) : rows(row_kernel<E, 2, false>));
  if (e != cudaSuccess) return e;
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = group_bytes(a.beams, (uint64_t)a.beams * c.per_row * a.keep, 0);
  after.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  after.val.programmaticStreamSerializationAllowed = 1;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, group_kernel<E, false>, a, c);
}

// ---- states -----------------------------------------------------------------

// Rows' tiles by way of shared memory: a block reads a tile of every row that is
// somebody's parent, once, and then writes the tile of every row, so that rows
// may change places.  U: the unit that all addresses, strides and widths are multiples
// of.  Flat: a token's units follow the one's before.
struct Tiles {
  uint32_t units;          // of a tile and row
  uint32_t run;            // units of a token (and head, where heads are apart)
  uint32_t per_row, heads; // tiles; heads that are apart
};

template <typename U, bool kFlat>
__global__ void __launch_bounds__(kThreads) reorder_kernel(const __grid_constant__ ReorderArgs a, const __grid_constant__ Tiles tl) {
  extern __shared__ __align__(16) unsigned char raw[];
  U* held = reinterpret_cast<U*>(raw);
  __shared__ int32_t parent[BF_MAX_BEAMS];       // of each row; -1: stays
  __shared__ uint32_t limit[BF_MAX_BEAMS];       // units of this tile that a row's parent has
  __shared__ uint32_t needed[BF_MAX_BEAMS / 32];
  __shared__ uint32_t slots[BF_MAX_BEAMS];       // slot -> row
  const uint32_t t = threadIdx.x;
  uint64_t i = blockIdx.x;
  const uint32_t tile = i % tl.per_row;
  i /= tl.per_row;
  const uint32_t head = i % tl.heads;
  i /= tl.heads;
  const uint32_t k = i % a.count;
  const uint64_t row0 = i / a.count * a.beams;
  const uint64_t first = (uint64_t)tile * tl.units;
  if (t < BF_MAX_BEAMS / 32) needed[t] = 0;
  __syncthreads();
  for (uint32_t b = t; b < a.beams; b += kThreads) {
    const int64_t p = __ldg(a.parents + row0 + b) - (int64_t)row0;
    int32_t from = p >= 0 && p < (int64_t)a.beams && !(a.in_place && p == (int64_t)b) ? (int32_t)p : -1;
    uint64_t end = a.tokens * tl.run;
    if (from >= 0 && a.lengths) {
      const int64_t n = __ldg(a.lengths + row0 + from);
      end = n <= 0 ? 0 : min((uint64_t)n, a.tokens) * tl.run;
    }
    const uint32_t mine = end > first ? (uint32_t)min(end - first, (uint64_t)tl.units) : 0;
    if (mine == 0) from = -1;
    parent[b] = from;
    limit[b] = mine;
    if (from >= 0) atomicOr(&needed[from / 32], 1u << from % 32);
  }
  __syncthreads();
  uint32_t many = 0;
  for (uint32_t w = 0; w < (a.beams + 31) / 32; ++w) many += __popc(needed[w]);
  if (many == 0) return;
  const auto slot_of = [&](uint32_t p) {
    uint32_t n = __popc(needed[p / 32] & ((1u << p % 32) - 1));
    for (uint32_t w = 0; w < p / 32; ++w) n += __popc(needed[w]);
    return n;
  };
  for (uint32_t b = t; b < a.beams; b += kThreads) {
    if (needed[b / 32] >> b % 32 & 1) slots[slot_of(b)] = b;
  }
  __syncthreads();
  const auto place = [&](uint64_t u, uint64_t token) -> uint64_t {  // bytes of unit u behind a row's first
    if constexpr (kFlat) return u * sizeof(U);
    const uint64_t n = u / tl.run;
    return n * token + (u - n * tl.run) * sizeof(U);
  };
  for (uint32_t s = 0; s < many; ++s) {
    const uint32_t p = slots[s];
    uint32_t n = tl.units;
    {
      uint64_t end = a.tokens * tl.run;
      if (a.lengths) end = min((uint64_t)__ldg(a.lengths + row0 + p), a.tokens) * tl.run;
      n = (uint32_t)min(end - first, (uint64_t)tl.units);
    }
    const char* from = a.from[k] + (row0 + p) * a.from_row + head * a.from_head;
    for (uint32_t u = t; u < n; u += kThreads)
      held[s * tl.units + u] = *reinterpret_cast<const U*>(from + place(first + u, a.from_token));
  }
  __syncthreads();
  for (uint32_t b = 0; b < a.beams; ++b) {
    if (parent[b] < 0) continue;
    const uint32_t s = slot_of(parent[b]), n = limit[b];
    char* to = a.to[k] + (row0 + b) * a.to_row + head * a.to_head;
    for (uint32_t u = t; u < n; u += kThreads)
      *reinterpret_cast<U*>(to + place(first + u, a.to_token)) = held[s * tl.units + u];
  }
}

template <typename U>
cudaError_t launch_units(const ReorderArgs& a, bool flat, cudaStream_t st) {
  Tiles tl = {};
  tl.run = (uint32_t)(a.width / sizeof(U));
  tl.heads = a.heads;
  const uint32_t most = 65536 / (a.beams * sizeof(U));
  const uint64_t row = a.tokens * tl.run;
  uint64_t units = 8192 / sizeof(U);
  if (units > most) units = most;
  if (units > row) units = row;
  tl.units = (uint32_t)units;
  const uint64_t per_row = (row + units - 1) / units, blocks = per_row * tl.heads * a.count * a.groups;
  if (blocks > 0x7FFFFFFFu) return cudaErrorInvalidValue;
  tl.per_row = (uint32_t)per_row;
  const uint32_t shared = (uint32_t)(units * a.beams * sizeof(U));
  const auto launch = [&](auto kernel) {
    if (shared > 32 * 1024) {
      const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 65536);
      if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((uint32_t)blocks);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = st;
    return cudaLaunchKernelEx(&cfg, kernel, a, tl);
  };
  return flat ? launch(reorder_kernel<U, true>) : launch(reorder_kernel<U, false>);
}

}  // namespace

uint64_t beam_bytes(uint32_t groups, uint32_t beams, uint64_t vocab, uint32_t keep) {
  uint64_t most = 256;
  for (uint32_t i = 0; i < 4; ++i) {  // 4 or 8 elements in 16 bytes, aligned or not
    uint32_t vectors;
    uint64_t bytes;
    chunks_of(groups, beams, vocab, keep, i % 2 ? 4 : 8, i / 2, nullptr, &vectors, &bytes);
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
