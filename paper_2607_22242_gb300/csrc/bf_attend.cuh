// bf_attend.cuh -- what the attention kernels share: how a call's keys are cut
// into pieces, and the record that a piece leaves.
//
// With s_t = scale q . k_t over a piece's keys, in units of log2(e):
//   m = max s_t, l = sum 2^(s_t - m), o = sum 2^(s_t - m) v_t,
// and pieces join by their sums weighted with 2^(m_i - max m): out = o / l, lse =
// ln2 (m + log2 l).  All of it is held in 32 bits.
//
// The prompts' keys.  A segment is a prompt, a key head and a tile of up to `rows`
// query vectors (the prompt's answers times the query heads that share the key
// head); it has ceil(length / keys) tiles of keys.  The tiles of all segments, in
// order, are dealt to `parts` blocks in runs of equal length, so that prompts of
// uneven lengths, one long prompt and many short ones all keep every SM busy to
// the end.  A run may begin and end inside a segment; block c's piece of segment
// s leaves its record in slot c + s, which no two pieces share.  Lengths are in
// device memory: blocks find their runs themselves.
#pragma once

#include "bf_answer.h"
#include "bf_elem.cuh"
#include "bf_launches.cuh"

namespace bfk {

// How a call is cut; chosen on the host from the sizes alone.
struct AttendPlan {
  uint32_t rows, row_tiles;      // query vectors of a prefix segment at most, segments of a prompt and key head
  uint32_t held, suffix_held;    // rows of a record: as many as a segment has, to a multiple of 2
  uint32_t keys;                 // of a tile
  uint32_t parts;                // blocks that share the prefix tiles out
  uint32_t suffix_rows, suffix_row_tiles, suffix_splits;  // the answers' own keys: pieces of an answer and key head
  float *prefix, *suffix;        // records
  uint32_t* gave_up;             // of the tiled kernel's blocks; nullptr: it does not run
  uint64_t* before;              // tiles ahead of each prompt, and all; of more than kFewPrompts
  uint32_t record, suffix_record;  // floats of a record
};

// A record, of an even number of rows (16 bytes are read at a time): the outputs of its rows, four dimensions of all rows after four others (so
// that a thread to a row writes, and neighbouring rows are read, whole lines), then (m, l) of each row.
__host__ __device__ __forceinline__ uint32_t record_place(uint32_t rows, uint32_t row, uint32_t d) { return (d / 4 * rows + row) * 4 + d % 4; }
__host__ __device__ __forceinline__ uint32_t record_sums(uint32_t rows, uint32_t dim) { return (dim + 3) / 4 * 4 * rows; }
__host__ __device__ __forceinline__ uint32_t record_floats(uint32_t rows, uint32_t dim) { return record_sums(rows, dim) + 2 * rows; }

constexpr float kNone = -__builtin_huge_valf();

// Weights that are rounded to 16 bits for the second product are taken times 2^kLift, and the maximum less by as much.
// bf16 has the exponents of 32 bits: a weight is off by 2^-8 of itself at most.  f16 has that (2^-11) from 2^-14 on only, and
// nothing below 2^-25, where 100,000 keys together still weigh 0.3 % of the largest.  Weights are at most
// 2^8 (the maximum lags by up to 8) and f16 ends at 2^16: with 2^7 what is lost is below 2^-32 of the largest each.
template <typename E>
constexpr float kLift = 0.0f;
template <>
constexpr float kLift<__half> = 7.0f;

__device__ __forceinline__ float exp2_of(float t) {
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t));
  return e;
}

// A length as given; 0 where it is outside 0..cap (the answers are NaN: bad_length).
__device__ __forceinline__ uint32_t length_of(const int64_t* lengths, uint64_t cap, uint64_t i) {
  if (!lengths) return (uint32_t)cap;
  const int64_t n = __ldg(lengths + i);
  return n < 0 || (uint64_t)n > cap ? 0u : (uint32_t)n;
}
__device__ __forceinline__ bool bad_length(const int64_t* lengths, uint64_t cap, uint64_t i) {
  if (!lengths) return false;
  const int64_t n = __ldg(lengths + i);
  return n < 0 || (uint64_t)n > cap;
}

__device__ __forceinline__ uint64_t sum_lanes(uint64_t v) {
#pragma unroll
  for (int d = 16; d; d /= 2) v += __shfl_xor_sync(~0u, v, d);
  return v;
}

// Key tiles of a prompt in one segment, of the prompts ahead of it, and of all.  Up to kFewPrompts a warp adds up where it
// needs to know; of more prompts `before` has the sums (every warp adding up all was 6 ms of 65,536 prompts, and minutes of millions).
constexpr uint32_t kFewPrompts = 128;
__device__ __forceinline__ uint32_t tiles_of(const AttendArgs& a, uint32_t keys, uint64_t p) {
  return (length_of(a.prefix_len, a.prefix_cap, p) + keys - 1) / keys;
}
// Tiles ahead of prompt p (of all: p the prompts), of more than kFewPrompts.
__device__ __forceinline__ uint64_t tiles_ahead(const AttendArgs& a, const AttendPlan& plan, uint32_t keys, uint64_t p) {
  return a.prefix_len ? __ldg(plan.before + p) : p * (((uint32_t)a.prefix_cap + keys - 1) / keys);
}
// All tiles; by a whole warp.
__device__ __forceinline__ uint64_t tiles_of_all(const AttendArgs& a, const AttendPlan& plan, uint32_t keys) {
  if (a.prompts > kFewPrompts) return tiles_ahead(a, plan, keys, a.prompts);
  uint64_t n = 0;
  for (uint32_t i = threadIdx.x % 32; i < a.prompts; i += 32) n += tiles_of(a, keys, i);
  return sum_lanes(n);
}

// The blocks that share `total` tiles out: none is without a tile, so that between a
// segment's first and last block each one has a piece of it.
__device__ __forceinline__ uint64_t parts_of(const AttendPlan& plan, uint64_t total) { return min((uint64_t)plan.parts, total); }

// A place in the run of all tiles: prompt, segment in it (key head and row tile), tile in that.
struct Place {
  uint32_t prompt, inner, tile;
};
// The place of tile t (below the total) among more than kFewPrompts; by a whole warp.
__device__ __forceinline__ Place place_far(const AttendArgs& a, const AttendPlan& plan, uint32_t keys, uint32_t inners, uint64_t t) {
  const uint32_t lane = threadIdx.x % 32;
  uint64_t lo = 0, hi = a.prompts;  // the last prompt that no more than t tiles are ahead of lies in [lo, hi)
  while (hi - lo > 1) {
    const uint64_t step = (hi - lo + 31) / 32, p = lo + lane * step;
    const uint32_t not_past = __popc(__ballot_sync(~0u, p < hi && tiles_ahead(a, plan, keys, p) * inners <= t));
    lo += (not_past - 1) * step;  // (lane 0's is not)
    hi = min(hi, lo + step);
  }
  const uint64_t in = t - tiles_ahead(a, plan, keys, lo) * inners;
  const uint32_t mine = tiles_of(a, keys, lo);
  return {(uint32_t)lo, (uint32_t)(in / mine), (uint32_t)(in % mine)};
}
// Out of line, for kernels that a few instructions more to fetch are long for.
static __device__ __noinline__ Place place_far_apart(const AttendArgs& a, const AttendPlan& plan, uint32_t keys, uint32_t inners, uint64_t t) {
  return place_far(a, plan, keys, inners, t);
}
// The same among any.
__device__ __forceinline__ Place place_of(const AttendArgs& a, const AttendPlan& plan, uint32_t keys, uint32_t inners, uint64_t t) {
  const uint32_t lane = threadIdx.x % 32;
  if (a.prompts > kFewPrompts) return place_far_apart(a, plan, keys, inners, t);
  uint64_t before = 0;
  for (uint32_t first = 0; first < a.prompts; first += 32) {
    const uint32_t i = first + lane;
    const uint64_t n = i < a.prompts ? (uint64_t)tiles_of(a, keys, i) * inners : 0;
    uint64_t upto = n;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const uint64_t o = __shfl_up_sync(~0u, upto, d);
      if (lane >= d) upto += o;
    }
    const uint32_t past = __ballot_sync(~0u, before + upto > t);
    if (past) {
      const int owner = __ffs(past) - 1;
      const uint64_t at = __shfl_sync(~0u, before + upto - n, owner), mine = __shfl_sync(~0u, n, owner) / inners;
      return {first + owner, (uint32_t)((t - at) / mine), (uint32_t)((t - at) % mine)};
    }
    before += __shfl_sync(~0u, upto, 31);
  }
  return {a.prompts, 0, 0};
}

// The first prompt from p on that is not empty, of more than kFewPrompts; by a whole warp.  (There is one, unless lengths
// change under the call: then there may be none, and nothing goes on.)
__device__ __forceinline__ uint32_t not_empty_from(const AttendArgs& a, uint32_t p) {
  for (; p < a.prompts; p += 32) {
    const uint32_t i = p + threadIdx.x % 32, some = __ballot_sync(~0u, i < a.prompts && length_of(a.prefix_len, a.prefix_cap, i) != 0);
    if (some) return p + __ffs(some) - 1;
  }
  return a.prompts;
}

// The prompts' keys on the tensor cores (bf_attend_tile.cu): what of a call says that it may take them, and, with
// the addresses and strides, does.
inline bool tile_might_take(const AttendArgs& a) { return a.dtype != BF_F32 && a.dim % 8 == 0 && a.dim <= 128 && a.prefix_cap > 0; }
bool tile_takes(const AttendArgs& a);
constexpr uint32_t kTileKeys = 128, kTileParts = 152;  // a block on each SM
cudaError_t launch_tile(const AttendArgs& a, const AttendPlan& plan, cudaStream_t st);

// The answers' own keys on few queries each, and the joining of all (bf_attend_few.cu).
bool few_takes(const AttendArgs& a);
cudaError_t launch_few_queries(const AttendArgs& a, const AttendPlan& plan, cudaStream_t st);

// The blocks [first, last) that have a piece of a row's prefix segment.
struct Owners {
  uint32_t first, last;
  uint64_t segment;
};
// A prompt's tiles among all, by a whole warp: how many there are, and are before it, in one segment of each prompt.
struct Standing {
  uint64_t total, before;
  uint32_t tiles;
};
__device__ __forceinline__ Standing standing_of(const AttendArgs& a, const AttendPlan& plan, uint32_t prompt) {
  const uint32_t keys = plan.keys;
  if (a.prompts > kFewPrompts) return {tiles_ahead(a, plan, keys, a.prompts), tiles_ahead(a, plan, keys, prompt), tiles_of(a, keys, prompt)};
  uint64_t total = 0, before = 0;
  uint32_t mine = 0;
  if (((a.prefix_cap + keys - 1) / keys) * a.prompts < 1ull << 31) {  // sums of 32 bits, an instruction each
    uint32_t all = 0, ahead = 0;
    for (uint32_t i = threadIdx.x % 32; i < a.prompts; i += 32) {
      const uint32_t n = tiles_of(a, keys, i);
      all += n;
      ahead += i < prompt ? n : 0;
      mine += i == prompt ? n : 0;
    }
    total = __reduce_add_sync(~0u, all);
    before = __reduce_add_sync(~0u, ahead);
  } else {
    for (uint32_t i = threadIdx.x % 32; i < a.prompts; i += 32) {
      const uint32_t n = tiles_of(a, keys, i);
      total += n;
      before += i < prompt ? n : 0;
      mine += i == prompt ? n : 0;
    }
    total = sum_lanes(total);
    before = sum_lanes(before);
  }
  return {total, before, __reduce_add_sync(~0u, mine)};
}
__device__ __forceinline__ Owners owners_of(const AttendArgs& a, const AttendPlan& plan, const Standing& s, uint32_t prompt, uint32_t inner) {
  const uint32_t inners = a.kv_heads * plan.row_tiles;
  const uint64_t total = s.total * inners;
  Owners o = {0, 0, (uint64_t)prompt * inners + inner};
  if (s.tiles) {
    const uint64_t at = s.before * inners + (uint64_t)inner * s.tiles, parts = parts_of(plan, total);
    if (total < 1u << 24 && plan.parts < 256) {
      o.first = ((uint32_t)(at + 1) * (uint32_t)parts - 1) / (uint32_t)total;
      o.last = ((uint32_t)(at + s.tiles) * (uint32_t)parts - 1) / (uint32_t)total + 1;
    } else {
      o.first = (uint32_t)(((at + 1) * parts - 1) / total);
      o.last = (uint32_t)(((at + s.tiles) * parts - 1) / total) + 1;
    }
  }
  return o;
}
// Whether an answer's lengths make it NaN.
__device__ __forceinline__ bool bad_answer(const AttendArgs& a, uint32_t prompt, uint64_t answer) {
  return bad_length(a.prefix_len, a.prefix_cap, prompt) || bad_length(a.suffix_len, a.suffix_cap, answer);
}

}  // namespace bfk
