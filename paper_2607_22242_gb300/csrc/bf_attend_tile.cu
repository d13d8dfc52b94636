// bf_attend_tile.cu -- the prompts' keys on the tensor cores: 128 query vectors
// (the answers of a prompt times the query heads that share a key head) against
// tiles of 128 keys, 16-bit types, up to 128 dimensions.
//
// S = Q K^T and O += P V are tcgen05 products with S, P and O in tensor memory; K
// and V come by TMA.  A block has two streams of tiles: of the same queries, even and
// odd tiles of keys (whose sums it joins at a piece's end), or of 256 queries, each
// half with all tiles.  While one stream's weights are made (a thread to a query, 128
// threads), the other's products run: a prompt's keys are read once at the memory's
// rate.  Queries that no thread has are skipped by whole warps.
//
// The maximum that weights are taken against is raised only where a score is above
// it by more than 8 (in log2): weights are at most 2^8, and O in tensor memory is
// rescaled a few times at the beginning of a piece instead of at every tile.
// Weights are rounded to the keys' type, which is what the products take: by at most 2^-8 of
// themselves (bf16) or 2^-11 (f16, those below 2^-21 of the largest by up to 2^-32 of
// it: kLift), as the output is at the end; their sum is of the unrounded ones, in 32 bits.
//
// 131,072 keys of 8 heads of 128 dimensions: 87 us for up to 32 queries a head (6.2 TB/s)
// and 92 for 128: the memory.  256 queries: 121 us, 1.14 PFLOP/s, the tensor cores busy for
// 45 % of it: each stream's way from scores to weights takes 2,300 cycles of the 5,400 a
// tile, its products, behind the other stream's, the rest.  Handing the weights over in halves,
// one pass over the scores and scalar exponentials were no faster.
#include <cuda.h>

#include "bf_attend.cuh"
#include "bf_blackwell.cuh"

namespace bfk {

namespace {

constexpr uint32_t kKeys = 128, kRows = 128;
constexpr uint32_t kSoft = 256, kThreads = kSoft + 96;  // softmax threads; a warp that copies, a warp of products for each stream
// Tensor memory: S of both streams, O of both; with up to 64 dimensions P of both, which otherwise lies where S was.
constexpr uint32_t kColumns = 512, kOutputs = 256, kWeights = 384;
constexpr uint32_t kMaxStages = 12, kMostShared = 227 * 1024;
constexpr float kRaise = 8.0f;

struct TileArgs {
  TensorMap k, v;
  uint32_t stages, chunks;  // of a ring of K and V tiles; columns of 64 elements
  uint32_t columns;         // dimensions, to a multiple of 16
  uint32_t pair;            // 256 queries a block
  uint32_t apart;           // P has columns of its own
  uint32_t* gave_up;        // one word a block
};

struct Shared {
  uint64_t full[kMaxStages], empty[kMaxStages];
  uint64_t q_full, s_full[2], p_full[2], o_done[2];
  uint32_t tensor, gave_up;
  float2 sums[2][kRows];  // (maximum, sum) of the streams
};

// A block's pieces, in order; the same for all its warps.  Up to 128 prompts, whose
// lengths a warp holds (four to a lane), are found by one read; divisions are of 32 bits where they can
// be (two reads and 64 bits took 3,200 to 4,000 cycles of a block's start).
struct Pieces {
  const AttendArgs& a;
  const AttendPlan& plan;
  uint32_t inners, my_len[4];
  uint64_t left;
  Place at;
  uint32_t len, tiles;  // the piece's prompt, and its tiles
  uint32_t head, first_row;

  __device__ __forceinline__ Pieces(const AttendArgs& args, const AttendPlan& p)
      : a(args), plan(p), inners(args.kv_heads * p.row_tiles), my_len{}, left(0), at{0, 0, 0}, len(0), tiles(0), head(0), first_row(0) {
    const uint32_t lane = threadIdx.x % 32;
    uint64_t t0;
    if (a.prompts <= kFewPrompts) {
      uint32_t n = 0, upto;
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j)
        if (4 * lane + j < a.prompts) my_len[j] = length_of(a.prefix_len, a.prefix_cap, 4 * lane + j);
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) n += tiles_of(my_len[j]);
      upto = n;
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const uint32_t o = __shfl_up_sync(~0u, upto, d);
        if (lane >= d) upto += o;
      }
      const uint64_t total = (uint64_t)__shfl_sync(~0u, upto, 31) * inners;
      if (!share(total, &t0)) return;
      const int owner = __ffs(__ballot_sync(~0u, (uint64_t)upto * inners > t0)) - 1;
      uint64_t before = (uint64_t)__shfl_sync(~0u, upto - n, owner) * inners;
      uint32_t mine = 0;
      at.prompt = 4 * (uint32_t)owner;
      for (;; ++at.prompt) {  // of the lane's four
        mine = tiles_of(len_of(at.prompt));
        if (t0 < before + (uint64_t)mine * inners) break;
        before += (uint64_t)mine * inners;
      }
      const uint64_t in = t0 - before;
      at.inner = in >> 32 ? (uint32_t)(in / mine) : (uint32_t)in / mine;
      at.tile = (uint32_t)(in - (uint64_t)at.inner * mine);
    } else {
      if (!share(tiles_of_all(a, plan, kKeys) * inners, &t0)) return;
      at = place_far(a, plan, kKeys, inners, t0);
    }
    find();
  }
  static __device__ __forceinline__ uint32_t tiles_of(uint32_t len) { return (len + kKeys - 1) / kKeys; }
  __device__ __forceinline__ uint32_t len_of(uint32_t prompt) const {  // by a whole warp
    const uint32_t j = prompt % 4, mine = j == 0 ? my_len[0] : j == 1 ? my_len[1] : j == 2 ? my_len[2] : my_len[3];
    return __shfl_sync(~0u, mine, prompt / 4);
  }
  // This block's run of `total` tiles: its first, and how many; false where it has none.
  __device__ __forceinline__ bool share(uint64_t total, uint64_t* t0) {
    const uint32_t parts = (uint32_t)parts_of(plan, total);
    if (blockIdx.x >= parts) return false;
    uint64_t t1;
    if (total < 1u << 24 && plan.parts <= 256) {
      *t0 = (uint32_t)total * blockIdx.x / parts;
      t1 = (uint32_t)total * (blockIdx.x + 1) / parts;
    } else {
      *t0 = total * blockIdx.x / parts;
      t1 = total * (blockIdx.x + 1) / parts;
    }
    left = t1 - *t0;
    return true;
  }
  __device__ __forceinline__ void find() {
    for (;; ++at.prompt) {
      if (left && a.prompts > kFewPrompts) at.prompt = not_empty_from(a, at.prompt);
      if (at.prompt >= a.prompts) left = 0;
      if (left == 0) return;
      len = a.prompts <= kFewPrompts ? len_of(at.prompt) : length_of(a.prefix_len, a.prefix_cap, at.prompt);
      if (len) break;
    }
    tiles = (uint32_t)min((uint64_t)((len + kKeys - 1) / kKeys - at.tile), left);
    head = plan.row_tiles == 1 ? at.inner : at.inner / plan.row_tiles;
    first_row = (at.inner - head * plan.row_tiles) * plan.rows;
  }
  __device__ __forceinline__ bool more() const { return left != 0; }
  __device__ __forceinline__ void next() {
    left -= tiles;
    at.tile = 0;
    if (++at.inner == inners) {
      at.inner = 0;
      ++at.prompt;
    }
    find();
  }
};

// The rings of K and V tiles: one that both streams use whole (256 queries), or one
// for each stream, in the order K, V, K, V of its tiles.  A barrier tells a phase only
// from the one before it, so whoever waits for a place's filling must have waited for
// every filling of that place before: a stream that passed over the other's tiles in a common ring could be a
// round ahead of a copy that is late, and take what was there before.
struct Ring {
  uint32_t stage, phase, first, end;
  __device__ __forceinline__ Ring(uint32_t s, const TileArgs& t) : stage(s * t.stages), phase(0), first(stage), end(stage + t.stages) {}
  __device__ __forceinline__ void step() {
    if (++stage == end) {
      stage = first;
      phase ^= 1;
    }
  }
};

__device__ void copy_tiles(const TileArgs& t, Shared& sh, unsigned char* ring, Pieces& p) {
  const uint32_t bytes = t.chunks * kKeys * 128, streams = t.pair ? 1 : 2;
  Ring rings[2] = {Ring(0, t), Ring(streams - 1, t)};
  bool ok = true;
  for (; ok && p.more(); p.next())
    for (uint32_t i = 0; ok && i < p.tiles; i += streams)
#pragma unroll 1
      for (uint32_t n = 0; n < 2 * streams; ++n) {  // K of the streams' next tiles, then V
        const uint32_t s = streams == 2 ? n & 1 : 0, tile = i + s;
        const bool value = streams == 2 ? n >= 2 : n == 1;
        if (tile >= p.tiles) continue;
        Ring r = s ? rings[1] : rings[0];
        if (!(ok = barrier_wait(&sh.empty[r.stage], r.phase ^ 1, &sh.gave_up))) break;
        if (threadIdx.x % 32 == 0) {
          barrier_expect(&sh.full[r.stage], bytes);
          unsigned char* to = ring + r.stage * bytes;
          const TensorMap* map = value ? &t.v : &t.k;
          const int32_t key = (int32_t)((p.at.tile + tile) * kKeys);
          copy_box(to, map, 0, (int32_t)p.head, key, (int32_t)p.at.prompt, &sh.full[r.stage]);
          if (t.chunks > 1) copy_box(to + kKeys * 128, map, 64, (int32_t)p.head, key, (int32_t)p.at.prompt, &sh.full[r.stage]);
        }
        __syncwarp();
        r.step();
        if (s) rings[1] = r;
        else rings[0] = r;
      }
  // No copy is in flight when the block ends: those of each place's last round have
  // arrived (a place that was never filled is in its first phase, and has nothing to wait for).
  for (uint32_t s = 0; s < streams; ++s) {
    Ring r = s ? rings[1] : rings[0];
    for (uint32_t i = 0; i < t.stages; ++i, r.step())  // the oldest filling of the ring is the next place's
      for (uint32_t n = 0; n < 1u << 22 && !barrier_try(&sh.full[r.stage], r.phase ^ 1); ++n) {
      }
  }
}

// The products of stream s.
template <bool bf16>
__device__ void multiply_tiles(const TileArgs& t, Shared& sh, uint32_t q_at, unsigned char* ring_base, uint32_t s, Pieces& p) {
  const uint32_t bytes = t.chunks * kKeys * 128, tensor = uniform(sh.tensor), lane = threadIdx.x % 32;
  const uint32_t ring_at = shared_address(ring_base);
  const uint32_t scores = product_of(bf16, kKeys, false), outputs = product_of(bf16, t.columns, true);
  const uint32_t s_at = tensor + s * 128, o_at = tensor + kOutputs + s * (t.apart ? 64 : 128), p_at = t.apart ? tensor + kWeights + s * 64 : s_at;
  const uint64_t q = matrix_at(uniform(q_at + (t.pair ? s * t.chunks * kRows * 128 : 0)), 16);
  uint32_t q_phase = 0, p_phase = 0, o_phase = 0;
  Ring r(t.pair ? 0 : s, t);
  bool ok = true;
  for (; ok && p.more(); p.next()) {
    if (!(ok = barrier_wait(&sh.q_full, q_phase, &sh.gave_up))) break;
    q_phase ^= 1;
    tensor_fence_after();
    const uint32_t first = t.pair ? 0 : s, step = t.pair ? 1 : 2;
    const auto score = [&](bool behind) {
      const uint64_t k = matrix_at(uniform(ring_at + r.stage * bytes), 16);
      if (!barrier_wait(&sh.full[r.stage], r.phase, &sh.gave_up)) return false;
      if (behind && !t.apart) {  // the weights that lie where the scores will have been used
        if (!barrier_wait(&sh.o_done[s], o_phase, &sh.gave_up)) return false;
        o_phase ^= 1;
      }
      tensor_fence_after();
      for (uint32_t c = 0; c < t.columns; c += 64) {
        const uint64_t off = c / 64 * (kKeys * 128) / 16;  // of matrix_at's addresses
        if (t.columns - c >= 64) multiply4(s_at, q + off, k + off, scores, c != 0, 2);
        else
          for (uint32_t d = 0; d < t.columns - c; d += 16) multiply(s_at, q + off + d / 8, k + off + d / 8, scores, (c | d) != 0);
      }
      tensor_commit(&sh.s_full[s]);
      tensor_commit(&sh.empty[r.stage]);
      r.step();
      return true;
    };
    if (first < p.tiles) {
      ok = score(false);
    } else {  // a piece of one tile: nobody goes on before this warp has seen its queries' phase
      if (lane == 0) barrier_arrive(&sh.o_done[s]);
      o_phase ^= 1;
    }
    for (uint32_t tile = first; ok && tile < p.tiles; tile += step) {
      const uint64_t v = matrix_at(uniform(ring_at + r.stage * bytes), kKeys * 128);
      if (!(ok = barrier_wait(&sh.full[r.stage], r.phase, &sh.gave_up))) break;
      const uint32_t valid = min(kKeys, p.len - (p.at.tile + tile) * kKeys), deep = (valid + 15) / 16 * 16;
      if (valid < deep) {  // whatever lies behind the prompt's end is not multiplied, not even by 0 (both streams see to it)
        const uint32_t row = t.chunks * 8;  // pieces of 16 bytes
        for (uint32_t n = lane; n < (deep - valid) * row; n += 32) {
          const uint32_t key = valid + n / row, c = n % row;
          *reinterpret_cast<uint4*>(ring_base + r.stage * bytes + c / 8 * (kKeys * 128) + key * 128 + c % 8 * 16) =
              make_uint4(0, 0, 0, 0);
        }
        fence_to_async();
        __syncwarp();
      }
      if (!(ok = barrier_wait(&sh.p_full[s], p_phase, &sh.gave_up))) break;
      p_phase ^= 1;
      tensor_fence_after();
      const bool more = tile != first;
      if (deep == kKeys) {
        multiply4_held(o_at, p_at, v, outputs, more, 8, 128);
        multiply4_held(o_at, p_at + 32, v + 512, outputs, true, 8, 128);
      } else {
        for (uint32_t n = 0; n < deep; n += 16) multiply_held(o_at, p_at + n / 2, v + n * 8, outputs, n != 0 || more);
      }
      tensor_commit(&sh.o_done[s]);
      tensor_commit(&sh.empty[r.stage]);
      r.step();
      if (tile + step < p.tiles) ok = score(true);
      else o_phase ^= 1;  // the last outputs are the softmax threads' to wait for
    }
  }
  // No product is in flight when the block ends; where a wait gave up, one has milliseconds to end.
  if (!ok)
    for (uint32_t n = 0; n < 1u << 16; ++n) __nanosleep(100);
}

// Where the streams' queries lie: both on the same rows, or, where there are at most
// 64 (32), stream 1's on the rows 64 (32) further on, so that its softmax is on other
// schedulers: two warps of one take 1,050 cycles for 64 exponentials, one 440 to 670.
__device__ __forceinline__ uint32_t apart_by(const TileArgs& t, uint32_t rows) { return t.pair || rows > 64 ? 0 : rows > 32 ? 64 : 32; }

// The prompt's query vectors [first_row, ...) of a key head on their way into shared
// memory, 16 bytes a thread and turn; zeros up to a multiple of 32 vectors and in the columns behind the last dimension.
template <typename E>
__device__ __forceinline__ void request_q(const AttendArgs& a, const AttendPlan& plan, const Pieces& p, const TileArgs& t, unsigned char* to) {
  const uint32_t rows = min(plan.rows, a.per_prompt * a.share - p.first_row), most = (rows + 31) / 32 * 32, by = apart_by(t, rows);
  const uint32_t shift = t.chunks > 1 ? 4 : 3, c = threadIdx.x & ((1u << shift) - 1), step = kSoft >> shift;  // pieces of a row: 8 or 16
  const bool flip = a.scale2 < 0.0f, whole = !flip && ((uintptr_t)a.q.data | (uint64_t)a.q.batch * 2 | (uint64_t)a.q.head * 2) % 16 == 0;
  const E* base = static_cast<const E*>(a.q.data) + (int64_t)((uint64_t)p.at.prompt * a.per_prompt) * a.q.batch +
                  (int64_t)(p.head * a.share) * a.q.head + c * 8;
  const uint32_t step_answer = step / a.share, step_head = step - step_answer * a.share;
  uint32_t row = threadIdx.x >> shift, answer = (p.first_row + row) / a.share, head = p.first_row + row - answer * a.share;
#pragma unroll 2
  for (; row < most; row += step) {
    const bool on = row < rows && c * 8 < a.dim;
    const E* q = on ? base + (int64_t)answer * a.q.batch + (int64_t)head * a.q.head : static_cast<const E*>(a.q.data);
    unsigned char* place = to + (row / kRows * t.chunks + c / 8) * (kRows * 128) + row % kRows * 128 + (c % 8 ^ row % 8) * 16;
    if (whole) {
      copy_piece(shared_address(place), q, on);
      if (by) copy_piece(shared_address(place + by * 128), q, on);
    } else {
      uint32_t u[4];
      const uint16_t* h = reinterpret_cast<const uint16_t*>(q);
#pragma unroll
      for (int k = 0; k < 4; ++k) u[k] = on ? (h[2 * k] | (uint32_t)h[2 * k + 1] << 16) ^ (flip ? 0x80008000u : 0u) : 0u;
      *reinterpret_cast<uint4*>(place) = make_uint4(u[0], u[1], u[2], u[3]);
      if (by) *reinterpret_cast<uint4*>(place + by * 128) = make_uint4(u[0], u[1], u[2], u[3]);
    }
    answer += step_answer;
    head += step_head;
    if (head >= a.share) {
      head -= a.share;
      ++answer;
    }
  }
}

// A barrier of the softmax threads that tells all of them whether any of them says so.
__device__ __forceinline__ bool any_of_streams(bool say) {
  uint32_t any;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.aligned.pred q, 1, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(any)
      : "r"((uint32_t)say)
      : "memory");
  return any;
}

// Columns [c0, c1) of a row, times w, into a record: as they are, or added to what is there.
template <bool kAdd>
__device__ __forceinline__ void put_outputs(float* record, uint32_t rows, uint32_t row, bool on, uint32_t c0, uint32_t c1, uint32_t from, float w) {
#pragma unroll 1
  for (uint32_t c = c0; c < c1; c += 32) {
    uint32_t o[32];
    tensor_load32(from + c, o);
    tensor_wait_load(o);
    if (!on) continue;
#pragma unroll
    for (uint32_t k = 0; k < 32; k += 4) {
      if (c + k >= c1) break;
      const float4 x = make_float4(w * __uint_as_float(o[k]), w * __uint_as_float(o[k + 1]), w * __uint_as_float(o[k + 2]), w * __uint_as_float(o[k + 3]));
      float* to = record + record_place(rows, row, c + k);
      if (kAdd) add4(to, x);
      else *reinterpret_cast<float4*>(to) = x;
    }
  }
}

// 64 scores of a row from column c on; -inf behind the prompt's end.
__device__ __forceinline__ void load_scores(uint32_t at, uint32_t c, uint32_t valid, float (&x)[64]) {
  uint32_t raw[64];
  tensor_load32(at + c, raw);
  tensor_load32(at + c + 32, raw + 32);
  tensor_wait_load(raw);
#pragma unroll
  for (uint32_t k = 0; k < 64; ++k) x[k] = __uint_as_float(raw[k]);
  if (c + 64 > valid) {
#pragma unroll
    for (uint32_t k = 0; k < 64; ++k) x[k] = c + k < valid ? x[k] : kNone;
  }
}

// `p`: the block's first piece, whose queries are on their way.
template <typename E>
__device__ void weigh_tiles(const AttendArgs& a, const AttendPlan& plan, const TileArgs& t, Shared& sh, unsigned char* q_to, Pieces& p) {
  const uint32_t s = threadIdx.x / kRows, row = threadIdx.x % kRows, lane = threadIdx.x % 32;
  const uint32_t mine = sh.tensor + (row / 32 * 32 << 16), s_at = mine + s * 128;
  const uint32_t o_at = mine + kOutputs + s * (t.apart ? 64 : 128), p_at = t.apart ? mine + kWeights + s * 64 : s_at;
  const float scale = fmaxf(fabsf(a.scale2), 1e-37f);  // 0 would make NaN of masked scores
  const uint32_t rows_all = a.per_prompt * a.share;
  uint32_t s_phase = 0, o_phase = 0;
  while (p.more()) {
    copies_wait_all();
    fence_to_async();
    tensor_fence_before();
    barrier_arrive(&sh.q_full);
    const uint32_t rows = min(plan.rows, rows_all - p.first_row);
    const uint32_t my_row = t.pair ? s * kRows + row : row - s * apart_by(t, rows);  // (beyond 2^31 where there is none)
    const bool warp_on = my_row - lane < rows, on = my_row < rows;  // some of the warp's rows are there; this one is
    const uint32_t steps = t.pair ? p.tiles : s < p.tiles ? (p.tiles - s + 1) / 2 : 0;
    float m = kNone, l = 0.0f;
    bool ok = true;
    for (uint32_t i = 0; i < steps; ++i) {
      if (!(ok = barrier_wait(&sh.s_full[s], s_phase, &sh.gave_up))) break;
      s_phase ^= 1;
      if (i) {  // the outputs so far, and the weights' place, are free
        if (!(ok = barrier_wait(&sh.o_done[s], o_phase, &sh.gave_up))) break;
        o_phase ^= 1;
      }
      tensor_fence_after();
      if (warp_on) {
        const uint32_t tile = p.at.tile + (t.pair ? i : 2 * i + s), valid = min(kKeys, p.len - tile * kKeys);
        // Twice through the scores, 64 at a time, for their maximum and for the weights: reading them
        // again costs less than holding 128 (spills) and code of twice the length, which a block runs cold at first.
        float top[4] = {kNone, kNone, kNone, kNone};
#pragma unroll 1
        for (uint32_t c = 0; c < kKeys; c += 64) {
          float x[64];
          load_scores(s_at, c, valid, x);
#pragma unroll
          for (uint32_t k = 0; k < 64; k += 8)
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) top[j] = fmaxf(top[j], fmaxf(x[k + j], x[k + j + 4]));
        }
        const float now = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
        float base = m == kNone ? 0.0f : m;
        const bool raise = (now - base) * scale > kRaise || m == kNone;
        if (i == 0) {
          m = now;
        } else if (__any_sync(~0u, raise)) {
          const float to = raise ? fmaxf(m, now) : m, shrink = m == kNone ? 0.0f : exp2_of((m - to) * scale);
          m = to;
          l *= shrink;
          for (uint32_t c = 0; c < t.columns; c += 8) {
            uint32_t o[8];
            tensor_load8(o_at + c, o);
            tensor_wait_load(o);
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] = __float_as_uint(shrink == 0.0f ? 0.0f : __uint_as_float(o[k]) * shrink);
            tensor_store8(o_at + c, o);
          }
          tensor_wait_store();
        }
        base = m == kNone ? 0.0f : m;
        // Scores so large that what the product with the scale is rounded by would show in the weights, all of them or none
        // (beyond 2^25 it is a factor of 2): the maximum is taken off first.
        float lifted = fmaf(-base, scale, kLift<E>);
        const bool large = __any_sync(~0u, fabsf(lifted) > 0x1p20f);
        if (large) lifted = kLift<E>;
        const float2 scale_2 = make_float2(scale, scale), less = make_float2(lifted, lifted);
        float2 sum[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll 1
        for (uint32_t c = 0; c < kKeys; c += 64) {
          float x[64];
          uint32_t w[32];
          load_scores(s_at, c, valid, x);
          if (large) {
#pragma unroll
            for (uint32_t k = 0; k < 64; ++k) x[k] -= base;
          }
#pragma unroll
          for (uint32_t k = 0; k < 32; ++k) {
            const float2 e = __ffma2_rn(make_float2(x[2 * k], x[2 * k + 1]), scale_2, less);
            const float2 v = make_float2(exp2_of(e.x), exp2_of(e.y));
            sum[k % 2] = __fadd2_rn(sum[k % 2], v);
            w[k] = pack2(v, E());
          }
          tensor_store32(p_at + c / 2, w);
        }
        l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
        tensor_wait_store();
      }
      tensor_fence_before();
      __syncwarp();
      if (lane == 0) barrier_arrive(&sh.p_full[s]);
    }
    // The piece's outputs, when all products are done.  Two streams of the same queries:
    // each puts half of the columns there, weighted, and then adds its part to the other half.
    const bool both = !t.pair && p.tiles > 1;
    float* record = plan.prefix + (uint64_t)(blockIdx.x + (uint64_t)p.at.prompt * p.inners + p.at.inner) * plan.record;
    float2* sums = reinterpret_cast<float2*>(record + record_sums(plan.held, a.dim));
    float2 ml = make_float2(m == kNone ? kNone : fmaf(m, scale, -kLift<E>), l);
    float w = 1.0f;
    if (both) {
      const uint32_t by = apart_by(t, rows);
      sh.sums[s][row] = ml;
      asm volatile("bar.sync 1, 256;" ::: "memory");
      const float2 other = sh.sums[1 - s][(row + (s ? 0u - by : by)) % kRows];
      const float most = fmaxf(ml.x, other.x), base = most == kNone ? 0.0f : most;
      w = exp2_of(ml.x - base);
      if (s == 0) ml = make_float2(most, fmaf(exp2_of(other.x - base), other.y, w * ml.y));
    }
    if (ok) {  // (without tiles, this stream's products' warp says that it has seen the piece)
      ok = barrier_wait(&sh.o_done[s], o_phase, &sh.gave_up);
      o_phase ^= 1;
    }
    tensor_fence_after();
    const uint32_t half = both ? (a.dim / 2 + 7) / 8 * 8 : a.dim;
    if (warp_on && (t.pair || steps)) {
      put_outputs<false>(record, plan.held, my_row, on, s && both ? half : 0, s && both ? a.dim : half, o_at, w);
      if (on && (t.pair || s == 0)) sums[my_row] = ml;
    }
    tensor_fence_before();
    if (any_of_streams(!ok || *static_cast<volatile uint32_t*>(&sh.gave_up))) break;  // all go on, or none
    tensor_fence_after();
    p.next();
    if (p.more()) request_q<E>(a, plan, p, t, q_to);  // neither stream has a product left that reads the queries
    if (both && warp_on) put_outputs<true>(record, plan.held, my_row, on, s ? 0 : half, s ? half : a.dim, o_at, w);
    tensor_fence_before();
  }
  copies_wait_all();
}

template <typename E>
__global__ void __launch_bounds__(kThreads, 1) tile_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ AttendPlan plan,
                                                           const __grid_constant__ TileArgs t) {
  extern __shared__ __align__(1024) unsigned char base[];  // queries, ring, barriers
  unsigned char* ring = base + (t.pair ? 2 : 1) * t.chunks * kRows * 128;
  const uint32_t places = (t.pair ? 1 : 2) * t.stages;
  Shared& sh = *reinterpret_cast<Shared*>(ring + places * t.chunks * kKeys * 128);
  const uint32_t warp = threadIdx.x / 32;
  let_next_start();
  if (shared_address(base) % 1024) {  // the swizzle goes by addresses
    if (threadIdx.x == 0) t.gave_up[blockIdx.x] = 1;
    return;
  }
  Pieces p(a, plan);
  if (threadIdx.x == 0) {
    for (uint32_t i = 0; i < places; ++i) {
      barrier_init(&sh.full[i], 1);
      barrier_init(&sh.empty[i], t.pair ? 2 : 1);
    }
    barrier_init(&sh.q_full, kSoft);
    for (uint32_t i = 0; i < 2; ++i) {
      barrier_init(&sh.s_full[i], 1);
      barrier_init(&sh.p_full[i], kRows / 32);
      barrier_init(&sh.o_done[i], 1);
    }
    sh.gave_up = 0;
    fence_barriers();
  }
  if (warp == 9) tensor_alloc(&sh.tensor, kColumns);
  // The first queries are asked for ahead of the rings' copies: behind them they were 7,000 to 14,000 cycles on their way.
  if (warp < 8 && p.more()) request_q<E>(a, plan, p, t, base);
  if (warp == 8 && threadIdx.x % 32 == 0) {
    prefetch_map(&t.k);
    prefetch_map(&t.v);
  }
  tensor_fence_before();
  __syncthreads();
  tensor_fence_after();
  if (warp < 8) weigh_tiles<E>(a, plan, t, sh, base, p);
  else if (warp == 8) copy_tiles(t, sh, ring, p);
  else multiply_tiles<__is_same(E, __nv_bfloat16)>(t, sh, shared_address(base), ring, warp - 9, p);
  tensor_fence_before();
  __syncthreads();
  tensor_fence_after();
  if (warp == 9) tensor_free(sh.tensor, kColumns);
  if (threadIdx.x == 0) t.gave_up[blockIdx.x] = sh.gave_up;
}

using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                            const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                            CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

Encode encoder() {
  static const Encode found = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult how;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &how) != cudaSuccess) p = nullptr;
    return reinterpret_cast<Encode>(p);
  }();
  return found;
}

bool make_map(TensorMap* map, const Vectors& x, const AttendArgs& a) {
  static_assert(sizeof(TensorMap) == sizeof(CUtensorMap), "a tensor map");
  const Encode encode = encoder();
  if (!encode) return false;
  const auto stride = [&](uint64_t count, int64_t s) { return count > 1 ? (cuuint64_t)s * 2 : (cuuint64_t)(a.dim * 2 + 15) / 16 * 16; };
  const cuuint64_t size[4] = {a.dim, a.kv_heads, a.prefix_cap, a.prompts};
  const cuuint64_t strides[3] = {stride(a.kv_heads, x.head), stride(a.prefix_cap, x.token), stride(a.prompts, x.batch)};
  const cuuint32_t box[4] = {64, 1, kKeys, 1}, step[4] = {1, 1, 1, 1};
  return encode(reinterpret_cast<CUtensorMap*>(map), a.dtype == BF_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                4, const_cast<void*>(x.data), size, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool copyable(const Vectors& x, const AttendArgs& a) {
  const auto fits = [](uint64_t count, int64_t s) { return count < 2 || (s > 0 && s % 8 == 0 && s < (1ll << 38)); };
  return (uintptr_t)x.data % 16 == 0 && fits(a.kv_heads, x.head) && fits(a.prefix_cap, x.token) && fits(a.prompts, x.batch);
}

}  // namespace

bool tile_takes(const AttendArgs& a) {
  return tile_might_take(a) && copyable(a.pk, a) && copyable(a.pv, a);
}

cudaError_t launch_tile(const AttendArgs& a, const AttendPlan& plan, cudaStream_t st) {
  TileArgs t = {};
  t.pair = plan.rows == 2 * kRows;
  t.chunks = (a.dim + 63) / 64;
  t.columns = (a.dim + 15) / 16 * 16;
  t.apart = a.dim <= 64;
  t.gave_up = plan.gave_up;
  const uint32_t tile = t.chunks * kKeys * 128, queries = t.pair ? 2 : 1;
  const uint32_t rings = t.pair ? 1 : 2, fit = (kMostShared - sizeof(Shared)) / tile - queries;
  t.stages = (fit < kMaxStages ? fit : kMaxStages) / rings;
  const uint32_t shared = (queries + rings * t.stages) * tile + sizeof(Shared);
  const auto launch = [&](auto kernel) {
    // One limit for all sizes: another thread's call may come between this and the launch.
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared);
    if (e != cudaSuccess) return e;
    // Behind a call of the runtime, which makes the device's context current: a thread's first call has none, and the
    // driver then refuses to make a map.
    if (!make_map(&t.k, a.pk, a) || !make_map(&t.v, a.pv, a)) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(plan.parts);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = st;
    return cudaLaunchKernelEx(&cfg, kernel, a, plan, t);
  };
  return a.dtype == BF_BF16 ? launch(tile_kernel<__nv_bfloat16>) : launch(tile_kernel<__half>);
}

}  // namespace bfk
