// bf_attend.cu -- attention of one token of many answers to a shared prompt and
// to their own tokens: any type, layout and dimension (general_kernel), and the
// joining of all pieces (join_kernel).
#include "bf_attend.cuh"

namespace bfk {

namespace {

// ---- pieces, for any type and layout ----------------------------------------

// A piece: R query vectors against keys [k0, k1), 64 at a time, on 256 threads.
// Everything is staged in shared memory in 32 bits; a thread makes 4 rows by
// R / 16 (scores) or dim / (1024 / R) (outputs) values, so that a value read from
// shared memory is used four times or more.  16 rows are bound by the keys' way here, and
// have keys and values on it at once; 64 by the sums, and have room for two blocks an SM.
// Two prompts of 1,500 keys, 5 answers, 12 query and 4 key heads of 80 dimensions in 32 bits:
// 16.4 us with the joining, one chain of waiting (a tile of a cold block is 19,000 cycles).
constexpr uint32_t kThreads = 256, kKeys = 64, kMaxDim = 256;

template <uint32_t R>
struct Shape {
  static constexpr uint32_t kRowGroups = R / 4, kCols = kThreads / kRowGroups;  // threads by rows and by columns
  static constexpr uint32_t kScores = kKeys / kCols;                            // scores of a thread and row
  static constexpr uint32_t kOuts = kMaxDim / kCols;                            // outputs, at most
  static constexpr uint32_t kRowThreads = kThreads / R;                         // threads of a row's softmax
  static constexpr bool kBoth = R == 16;                                        // keys and values have places of their own
};

__host__ __device__ constexpr uint32_t pitch_of(uint32_t dim) { return (dim + 3) / 4 * 4 + 4; }
template <uint32_t R>
constexpr uint32_t shared_of(uint32_t dim) {
  return 4 * ((R + (Shape<R>::kBoth ? 2 : 1) * kKeys) * pitch_of(dim) + R * (kKeys + 4) + 3 * R);
}

struct Piece {
  const void *k, *v;
  int64_t k_token, v_token;
  uint32_t k0, k1;
  float* record;
  uint32_t held;  // its rows
};

// Four elements of a row from d on, zeros behind its end; `whole`: addresses allow one read.
template <typename E>
__device__ __forceinline__ float4 four(const E* row, uint32_t d, uint32_t dim, bool whole) {
  if (whole && d + 4 <= dim) {
    if constexpr (sizeof(E) == 4) {
      return __ldg(reinterpret_cast<const float4*>(row + d));
    } else {
      const uint2 u = __ldg(reinterpret_cast<const uint2*>(row + d));
      const float2 lo = unpack2(u.x, E()), hi = unpack2(u.y, E());
      return make_float4(lo.x, lo.y, hi.x, hi.y);
    }
  }
  float v[4];
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) v[i] = d + i < dim ? to_f32(row[d + i]) : 0.0f;
  return make_float4(v[0], v[1], v[2], v[3]);
}
template <typename E>
__device__ __forceinline__ bool whole_quads(const E* from, int64_t step) {
  return ((uintptr_t)from | (uint64_t)(step * (int64_t)sizeof(E))) % (4 * sizeof(E)) == 0;
}

// kKeys rows (zeros behind the first `rows`) of one or two matrices: a warp to a row, eight rows of each on their way.
template <typename E, bool kTwo>
__device__ __forceinline__ void stage(float* to, const E* from, int64_t step, float* to2, const E* from2, int64_t step2, uint32_t pitch,
                                      uint32_t rows, uint32_t dim) {
  constexpr uint32_t kWarps = kThreads / 32, kAhead = kKeys / kWarps;
  const bool whole = whole_quads(from, step), whole2 = kTwo && whole_quads(from2, step2);
  const uint32_t warp = threadIdx.x / 32;
  for (uint32_t d = threadIdx.x % 32 * 4; d < pitch - 4; d += 128) {
    float4 x[kAhead], y[kTwo ? kAhead : 1];
#pragma unroll
    for (uint32_t i = 0; i < kAhead; ++i) {
      const uint32_t r = warp + i * kWarps;
      x[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (kTwo) y[i] = x[i];
      if (r < rows) {
        x[i] = four(from + (int64_t)r * step, d, dim, whole);
        if (kTwo) y[i] = four(from2 + (int64_t)r * step2, d, dim, whole2);
      }
    }
#pragma unroll
    for (uint32_t i = 0; i < kAhead; ++i) {
      const uint32_t r = warp + i * kWarps;
      *reinterpret_cast<float4*>(to + r * pitch + d) = x[i];
      if (kTwo) *reinterpret_cast<float4*>(to2 + r * pitch + d) = y[i];
    }
  }
}

// Rows [0, rows) of Q, scaled, are in qs.
template <typename E, uint32_t R>
__device__ void piece(const Piece& p, uint32_t rows, uint32_t dim, float* sm) {
  using S = Shape<R>;
  const uint32_t pitch = pitch_of(dim), t = threadIdx.x, rg = t / S::kCols, cg = t % S::kCols;
  float *qs = sm, *ks = qs + R * pitch, *vs = S::kBoth ? ks + kKeys * pitch : ks, *ps = vs + kKeys * pitch,
        *ms = ps + R * (kKeys + 4), *ls = ms + R, *as = ls + R;
  float o[4][S::kOuts] = {};
  if (t < R) {
    ms[t] = kNone;
    ls[t] = 0.0f;
  }
  for (uint32_t k = p.k0; k < p.k1; k += kKeys) {
    const uint32_t n = min(kKeys, p.k1 - k);
    const E *key0 = static_cast<const E*>(p.k) + (int64_t)k * p.k_token, *value0 = static_cast<const E*>(p.v) + (int64_t)k * p.v_token;
    stage<E, S::kBoth>(ks, key0, p.k_token, vs, value0, p.v_token, pitch, n, dim);
    __syncthreads();
    float s[4][S::kScores] = {};
    for (uint32_t d = 0; d < pitch - 4; d += 4) {
      float4 q[4], c[S::kScores];
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = *reinterpret_cast<const float4*>(qs + (rg * 4 + i) * pitch + d);
#pragma unroll
      for (uint32_t j = 0; j < S::kScores; ++j) c[j] = *reinterpret_cast<const float4*>(ks + (cg + j * S::kCols) * pitch + d);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (uint32_t j = 0; j < S::kScores; ++j)
          s[i][j] = fmaf(q[i].w, c[j].w, fmaf(q[i].z, c[j].z, fmaf(q[i].y, c[j].y, fmaf(q[i].x, c[j].x, s[i][j]))));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (uint32_t j = 0; j < S::kScores; ++j) {
        const uint32_t at = cg + j * S::kCols;
        ps[(rg * 4 + i) * (kKeys + 4) + at] = at < n ? s[i][j] : kNone;
      }
    __syncthreads();
    if (!S::kBoth) stage<E, false>(vs, value0, p.v_token, vs, value0, p.v_token, pitch, n, dim);
    {
      const uint32_t row = t / S::kRowThreads, mine = t % S::kRowThreads;
      float* x = ps + row * (kKeys + 4);
      float m = kNone;
      for (uint32_t j = mine; j < kKeys; j += S::kRowThreads) m = fmaxf(m, x[j]);
#pragma unroll
      for (uint32_t w = S::kRowThreads / 2; w; w /= 2) m = fmaxf(m, __shfl_xor_sync(~0u, m, w));
      const float old = ms[row], now = fmaxf(old, m), base = now == kNone ? 0.0f : now;
      float l = 0.0f;
      for (uint32_t j = mine; j < kKeys; j += S::kRowThreads) {
        const float e = exp2_of(x[j] - base);
        x[j] = j < n ? e : 0.0f;
        l += j < n ? e : 0.0f;
      }
#pragma unroll
      for (uint32_t w = S::kRowThreads / 2; w; w /= 2) l += __shfl_xor_sync(~0u, l, w);
      if (mine == 0) {
        const float shrink = exp2_of(old - base);
        ms[row] = now;
        as[row] = shrink;
        ls[row] = fmaf(ls[row], shrink, l);
      }
    }
    __syncthreads();
    float shrink[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) shrink[i] = as[rg * 4 + i];
#pragma unroll
    for (uint32_t c = 0; c < S::kOuts; ++c) {
      const uint32_t d = cg + c * S::kCols;
      if (d >= dim) break;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i][c] *= shrink[i];
    }
    // Four keys at a time (weights and values behind the last one are 0): one by one, each
    // waited for its reads, 190 cycles of 16 rows.
    for (uint32_t j = 0; j < n; j += 4) {
      float4 w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const float4*>(ps + (rg * 4 + i) * (kKeys + 4) + j);
#pragma unroll
      for (uint32_t c = 0; c < S::kOuts; ++c) {
        const uint32_t d = cg + c * S::kCols;
        if (c * S::kCols >= dim) break;
        float v[4];
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) v[k] = d < dim ? vs[(j + k) * pitch + d] : 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i][c] = fmaf(w[i].w, v[3], fmaf(w[i].z, v[2], fmaf(w[i].y, v[1], fmaf(w[i].x, v[0], o[i][c]))));
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t row = rg * 4 + i;
    if (row >= rows) break;
    float* to = p.record + record_place(p.held, row, cg);
#pragma unroll
    for (uint32_t c = 0; c < S::kOuts; ++c) {  // kCols dimensions further on: kCols / 4 times four of all rows
      if (cg + c * S::kCols >= dim) break;
      to[c * S::kCols * p.held] = o[i][c];
    }
  }
  if (t < rows) {
    float2* ml = reinterpret_cast<float2*>(p.record + record_sums(p.held, dim));
    ml[t] = make_float2(ms[t], ls[t]);
  }
  __syncthreads();
}

// Query vectors [first, first + rows) of a prompt's (or an answer's) for a key head, scaled; zeros up to `most`.
template <typename E>
__device__ __forceinline__ void stage_q(const AttendArgs& a, float* to, uint64_t answer0, uint32_t head, uint32_t first,
                                        uint32_t rows, uint32_t most) {
  const uint32_t pitch = pitch_of(a.dim);
  const E* q = static_cast<const E*>(a.q.data);
  const bool whole = whole_quads(q, a.q.batch) && whole_quads(q, a.q.head);
#pragma unroll 2
  for (uint32_t r = threadIdx.x / 32; r < most; r += kThreads / 32) {
    const uint32_t at = first + r, answer = at / a.share;
    const E* row = q + (int64_t)(answer0 + answer) * a.q.batch + (int64_t)(head * a.share + at - answer * a.share) * a.q.head;
    for (uint32_t d = threadIdx.x % 32 * 4; d < pitch - 4; d += 128) {
      const float4 v = r < rows ? four(row, d, a.dim, whole) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      *reinterpret_cast<float4*>(to + r * pitch + d) = make_float4(v.x * a.scale2, v.y * a.scale2, v.z * a.scale2, v.w * a.scale2);
    }
  }
  __syncthreads();
}

template <typename E, uint32_t R>
__global__ void __launch_bounds__(kThreads, 2) general_kernel(const __grid_constant__ AttendArgs a,
                                                           const __grid_constant__ AttendPlan plan) {
  extern __shared__ float sm[];
  let_next_start();
  if (blockIdx.x < plan.parts) {
    const uint32_t inners = a.kv_heads * plan.row_tiles, rows_all = a.per_prompt * a.share;
    const uint64_t total = tiles_of_all(a, plan, kKeys) * inners;
    const uint64_t parts = parts_of(plan, total);
    if (blockIdx.x >= parts) return;
    const uint64_t t0 = total * blockIdx.x / parts, t1 = total * (blockIdx.x + 1) / parts;
    Place at = place_of(a, plan, kKeys, inners, t0);
    for (uint64_t left = t1 - t0; left && at.prompt < a.prompts;) {
      const uint32_t len = length_of(a.prefix_len, a.prefix_cap, at.prompt), tiles = (len + kKeys - 1) / kKeys;
      if (tiles == 0) {
        at.prompt = a.prompts > kFewPrompts ? not_empty_from(a, at.prompt + 1) : at.prompt + 1;
        continue;
      }
      const uint32_t n = (uint32_t)min((uint64_t)(tiles - at.tile), left);
      const uint32_t head = at.inner / plan.row_tiles, first = at.inner % plan.row_tiles * R, rows = min(R, rows_all - first);
      stage_q<E>(a, sm, (uint64_t)at.prompt * a.per_prompt, head, first, rows, R);
      const Piece p = {static_cast<const E*>(a.pk.data) + at.prompt * a.pk.batch + head * a.pk.head,
                       static_cast<const E*>(a.pv.data) + at.prompt * a.pv.batch + head * a.pv.head,
                       a.pk.token, a.pv.token, at.tile * kKeys, min(len, (at.tile + n) * kKeys),
                       plan.prefix + (uint64_t)(blockIdx.x + (uint64_t)at.prompt * inners + at.inner) * plan.record, plan.held};
      piece<E, R>(p, rows, a.dim, sm);
      left -= n;
      at.tile = 0;
      if (++at.inner == inners) {
        at.inner = 0;
        ++at.prompt;
      }
    }
  } else {
    uint64_t i = blockIdx.x - plan.parts;
    const uint64_t slot = i;
    const uint32_t split = i % plan.suffix_splits;
    i /= plan.suffix_splits;
    const uint32_t first = i % plan.suffix_row_tiles * R;
    i /= plan.suffix_row_tiles;
    const uint32_t head = i % a.kv_heads;
    const uint64_t answer = i / a.kv_heads;
    const uint32_t len = length_of(a.suffix_len, a.suffix_cap, answer), rows = min(R, a.share - first);
    stage_q<E>(a, sm, answer, head, first, rows, R);
    const Piece p = {static_cast<const E*>(a.sk.data) + answer * a.sk.batch + head * a.sk.head,
                     static_cast<const E*>(a.sv.data) + answer * a.sv.batch + head * a.sv.head, a.sk.token, a.sv.token,
                     (uint32_t)((uint64_t)len * split / plan.suffix_splits),
                     (uint32_t)((uint64_t)len * (split + 1) / plan.suffix_splits), plan.suffix + slot * plan.suffix_record,
                     plan.suffix_held};
    piece<E, R>(p, rows, a.dim, sm);
  }
}

// ---- joining ----------------------------------------------------------------

// A warp per query vector and 32 dimensions, a lane to a dimension: 32 pieces at a time, a
// lane to a piece's maximum and sum, and 16 pieces' outputs on their way.  (A warp to
// all dimensions was 11 us where 120 vectors of 80 dimensions join 23 pieces.)
template <typename E>
__global__ void __launch_bounds__(kThreads) join_kernel(const __grid_constant__ AttendArgs a,
                                                        const __grid_constant__ AttendPlan plan) {
  const uint32_t lane = threadIdx.x % 32, heads = a.kv_heads * a.share, columns = (a.dim + 31) / 32;
  const uint64_t warp = (uint64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32, vec = warp / columns;
  const uint32_t d = (uint32_t)(warp - vec * columns) * 32 + lane;
  if (vec >= (uint64_t)a.prompts * a.per_prompt * heads) return;
  const uint32_t answer = (uint32_t)(vec / heads), h = (uint32_t)vec - answer * heads, head = h / a.share, prompt = answer / a.per_prompt;
  const uint32_t srow = h - head * a.share, row = (answer - prompt * a.per_prompt) * a.share + srow;
  const Owners own = owners_of(a, plan, standing_of(a, plan, prompt), prompt, head * plan.row_tiles + row / plan.rows);
  const uint32_t far = own.last - own.first, splits = a.suffix_cap ? plan.suffix_splits : 0, pieces = far + splits;
  const float* prefix = plan.prefix + (own.first + own.segment) * plan.record;
  const uint64_t sslot = (((uint64_t)answer * a.kv_heads + head) * plan.suffix_row_tiles + srow / plan.suffix_rows) * plan.suffix_splits;
  const float* suffix = plan.suffix + sslot * plan.suffix_record;
  const uint32_t r0 = row % plan.rows, r1 = srow % plan.suffix_rows;
  const auto record = [&](uint32_t i) { return i < far ? prefix + (uint64_t)i * plan.record : suffix + (uint64_t)(i - far) * plan.suffix_record; };
  const bool bad = bad_answer(a, prompt, answer);
  wait_for_previous();
  float m = kNone, l = 0.0f, o = 0.0f;
  bool odd = bad;
  for (uint32_t from = 0; from < pieces; from += 32) {
    const uint32_t i = from + lane, some = min(32u, pieces - from);
    float2 ml = make_float2(kNone, 0.0f);
    if (i < pieces) {
      const uint32_t rows = i < far ? plan.held : plan.suffix_held;
      ml = __ldcg(reinterpret_cast<const float2*>(record(i) + record_sums(rows, a.dim)) + (i < far ? r0 : r1));
      if (plan.gave_up && i < far) odd |= __ldcg(plan.gave_up + own.first + i) != 0;
    }
    odd |= ml.y != ml.y;
    float to = fmaxf(m, ml.x);
#pragma unroll
    for (int apart = 16; apart; apart /= 2) to = fmaxf(to, __shfl_xor_sync(~0u, to, apart));
    const float base = to == kNone ? 0.0f : to, shrink = m == kNone ? 0.0f : exp2_of(m - base);
    m = to;
    const float w = ml.y > 0.0f ? exp2_of(ml.x - base) : 0.0f;  // 0: nothing to attend to in that piece
    float sum = ml.y > 0.0f ? w * ml.y : 0.0f;
#pragma unroll
    for (int apart = 16; apart; apart /= 2) sum += __shfl_xor_sync(~0u, sum, apart);
    l = fmaf(l, shrink, sum);
    o = shrink == 0.0f ? 0.0f : o * shrink;
    constexpr uint32_t kAhead = 16;
    for (uint32_t k = 0; k < some; k += kAhead) {
      float x[kAhead];
#pragma unroll
      for (uint32_t j = 0; j < kAhead; ++j) {
        const uint32_t p = from + k + j;
        x[j] = k + j < some && d < a.dim ? __ldcg(record(p) + (p < far ? record_place(plan.held, r0, d) : record_place(plan.suffix_held, r1, d))) : 0.0f;
      }
#pragma unroll
      for (uint32_t j = 0; j < kAhead; ++j) {
        const float f = __shfl_sync(~0u, w, (k + j) % 32);
        if (k + j < some && f > 0.0f) o = fmaf(f, x[j], o);
      }
    }
  }
  odd = __any_sync(~0u, odd || m == -kNone);  // (a score above 32-bit numbers)
  const float nan = __int_as_float(0x7FC00000), inv = odd ? nan : l > 0.0f ? 1.0f / l : 0.0f;
  E* out = static_cast<E*>(const_cast<void*>(a.out.data)) + (int64_t)answer * a.out.batch + (int64_t)h * a.out.head;
  if (d < a.dim) out[d] = from_f32<E>(o * inv);
  if (a.lse && d == 0) a.lse[vec] = odd ? nan : l > 0.0f ? (m + log2f(l)) * 0.693147180559945309f : kNone;
}

// The tiles ahead of each prompt, and all, where there are many: one block, eight prompts a thread and turn.
constexpr uint32_t kCountThreads = 1024, kCounted = 8;
__global__ void __launch_bounds__(kCountThreads) count_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ AttendPlan plan) {
  __shared__ uint64_t warps[2][32];
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  uint64_t before = 0;
  uint32_t turn = 0;
  for (uint64_t first = 0; first < a.prompts; first += kCountThreads * kCounted, turn ^= 1) {
    const uint64_t p = first + threadIdx.x * kCounted;
    uint32_t n[kCounted];
    uint64_t mine = 0;
#pragma unroll
    for (uint32_t j = 0; j < kCounted; ++j) {
      n[j] = p + j < a.prompts ? tiles_of(a, plan.keys, p + j) : 0;
      mine += n[j];
    }
    uint64_t upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const uint64_t o = __shfl_up_sync(~0u, upto, d);
      if (lane >= d) upto += o;
    }
    if (lane == 31) warps[turn][warp] = upto;  // (those of the turn before may still be read)
    __syncthreads();
    const uint64_t w = warps[turn][lane];
    uint64_t at = before + sum_lanes(lane < warp ? w : 0) + upto - mine;
#pragma unroll
    for (uint32_t j = 0; j < kCounted; ++j) {
      if (p + j < a.prompts) plan.before[p + j] = at;
      at += n[j];
    }
    before += sum_lanes(w);
  }
  if (threadIdx.x == 0) plan.before[a.prompts] = before;
}

// ---- the host's part --------------------------------------------------------

constexpr uint32_t kParts = 304;  // two blocks of each of 152 SMs

// `tile`: the prompts' keys go to the tiled kernel.
AttendPlan plan_of(const AttendArgs& a, bool tile, void* workspace, uint64_t* bytes) {
  AttendPlan p = {};
  const uint64_t rows = (uint64_t)a.per_prompt * a.share;
  p.rows = tile ? (rows <= 128 ? 128 : 256) : rows <= 16 ? 16 : 64;
  p.row_tiles = (uint32_t)((rows + p.rows - 1) / p.rows);
  p.keys = tile ? kTileKeys : kKeys;
  p.parts = tile ? kTileParts : kParts;
  p.suffix_rows = tile ? (a.share <= 16 ? 16 : 64) : p.rows;
  p.suffix_row_tiles = (a.share + p.suffix_rows - 1) / p.suffix_rows;
  const uint64_t pieces = (uint64_t)a.prompts * a.per_prompt * a.kv_heads * p.suffix_row_tiles;
  uint64_t splits = pieces ? kParts / pieces : 1;
  const uint64_t most = (a.suffix_cap + kKeys - 1) / kKeys;  // a tile each: the first of a block takes 12 us, one more 4
  splits = splits < most ? splits : most;
  p.suffix_splits = splits < 1 ? 1 : (uint32_t)splits;
  // Records of the rows there are: with all that a tile has room for, 32,768 answers of 4 query heads a key head took 9.3 GB.
  const auto even = [](uint64_t n) { return (uint32_t)(n + 1) / 2 * 2; };
  p.held = even(rows < p.rows ? rows : p.rows);
  p.suffix_held = even(a.share < p.suffix_rows ? a.share : p.suffix_rows);
  p.record = record_floats(p.held, a.dim);
  p.suffix_record = record_floats(p.suffix_held, a.dim);
  char* at = static_cast<char*>(workspace);
  const auto take = [&](uint64_t n) {
    char* q = at;
    at += (n + 255) / 256 * 256;
    return q;
  };
  p.gave_up = reinterpret_cast<uint32_t*>(take(4 * kTileParts));
  if (!tile) p.gave_up = nullptr;
  p.before = reinterpret_cast<uint64_t*>(take(a.prompts > kFewPrompts ? 8 * ((uint64_t)a.prompts + 1) : 0));
  p.prefix = reinterpret_cast<float*>(take(4 * (p.parts + (uint64_t)a.prompts * a.kv_heads * p.row_tiles) * p.record));
  p.suffix = reinterpret_cast<float*>(take(a.suffix_cap ? 4 * pieces * p.suffix_splits * p.suffix_record : 0));
  *bytes = (uint64_t)(at - static_cast<char*>(workspace));
  return p;
}

template <typename E, uint32_t R>
cudaError_t launch_general(uint64_t blocks, cudaStream_t st, const AttendArgs& a, const AttendPlan& p) {
  if (blocks > 0x7FFFFFFFu) return cudaErrorInvalidValue;
  const uint32_t shared = shared_of<R>(a.dim);
  if (shared > 48 * 1024) {  // one limit for all sizes: another thread's call may come between this and the launch
    const cudaError_t e =
        cudaFuncSetAttribute(general_kernel<E, R>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shared_of<R>(kMaxDim));
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((uint32_t)blocks);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = shared;
  cfg.stream = st;
  return cudaLaunchKernelEx(&cfg, general_kernel<E, R>, a, p);
}

template <typename E>
cudaError_t launch_type(const AttendArgs& a, void* workspace, cudaStream_t st) {
  uint64_t bytes = 0;
  const bool tile = tile_takes(a);
  const AttendPlan p = plan_of(a, tile, workspace, &bytes);
  const uint64_t answers = (uint64_t)a.prompts * a.per_prompt;
  const uint64_t suffix = a.suffix_cap ? answers * a.kv_heads * p.suffix_row_tiles * p.suffix_splits : 0;
  cudaError_t e = cudaSuccess;
  if (a.prompts > kFewPrompts && a.prefix_len) e = launch_plain(count_kernel, 1, kCountThreads, st, a, p);
  if (e != cudaSuccess) return e;
  AttendPlan general = p;
  if (tile) {
    e = launch_tile(a, p, st);
    if (e == cudaSuccess && few_takes(a)) return launch_few_queries(a, p, st);
    general.parts = 0;
  }
  if (e == cudaSuccess && general.parts + suffix)
    e = p.suffix_rows == 16 ? launch_general<E, 16>(general.parts + suffix, st, a, general)
                            : launch_general<E, 64>(general.parts + suffix, st, a, general);
  if (e != cudaSuccess) return e;
  const uint64_t warps = answers * a.kv_heads * a.share * ((a.dim + 31) / 32);
  return launch_after(join_kernel<E>, (warps + kThreads / 32 - 1) / (kThreads / 32), kThreads, st, a, p);
}

}  // namespace

uint64_t attend_bytes(const AttendArgs& a) {
  uint64_t bytes = 0;
  plan_of(a, false, nullptr, &bytes);
  if (tile_might_take(a)) {
    uint64_t more = 0;
    plan_of(a, true, nullptr, &more);
    bytes = more > bytes ? more : bytes;
  }
  return bytes;
}

cudaError_t launch_attend(const AttendArgs& a, void* workspace, cudaStream_t st) {
  return a.dtype == BF_F32    ? launch_type<float>(a, workspace, st)
         : a.dtype == BF_BF16 ? launch_type<__nv_bfloat16>(a, workspace, st)
                              : launch_type<__half>(a, workspace, st);
}

}  // namespace bfk
