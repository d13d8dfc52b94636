// bf_attend_few.cu -- an answer's own keys, and the joining of all that was attended
// to: 16-bit types, up to 128 dimensions.
//
// A unit is an answer and key head (and up to 16 of the query heads that share
// it); in a cluster of blocks where there are few, so that an answer's keys are spread over
// several SMs.  Each warp takes 16 keys at a time through a ring of its own in shared
// memory, two steps ahead by asynchronous copies, so that the keys on their way
// cost no registers (kept there, two blocks an SM had 64 KB on their way and stood
// still for half of the time).  The products are the warps' own (16 x 8 x 16): at 4 to
// 16 queries a key the memory is the bound, and a tile of 128 queries would be empty.
//
// Behind its own keys a block waits for the prompts' pieces and joins all of them.
//
// A unit has four warps, or two where there are more units than four warps' blocks fit
// on the GPU at once, and where there are units enough to give every warp one of its own
// (kAlone), it has that: what a warp does once (finding its pieces, joining) was two thirds of the
// instructions.  A call with 128 keys of prompt, 64 dimensions and 32 / 160 / 600 own keys, in us:
//   units  four warps          two                 one
//     608  14.4 / 15.8 / 26.2  -                   15.7 / 22.4 / 45.6
//     912  17.8 / 21.3 / 37.5  13.7 / 17.2 / 33.2  15.8 / 22.4 / 45.9
//   1,216  19.2 / 24.6 / 43.8  17.9 / 24.4 / 49.1  16.4 / 23.7 / 46.6
//   2,432  28.7 / 38.1 / 73.3  23.3 / 34.2 / 76.1  18.6 / 29.7 / 67.7
//
// 134 MB of 64 answers' own keys take about 28 us behind a long prompt's, 4.8 TB/s.
#include <cooperative_groups.h>
#include <type_traits>

#include "bf_attend.cuh"
#include "bf_blackwell.cuh"

namespace bfk {

namespace {

namespace cg = cooperative_groups;

constexpr uint32_t kRows = 16, kMostBlocks = 8;
constexpr uint64_t kAloneUnits = 1216;  // eight an SM, from which on every warp has one
constexpr float kRaise = 8.0f;

struct FewArgs {
  uint32_t row_tiles, blocks, units;  // of a key head's query heads; of a cluster; answers times key heads times row tiles
};

// d += a b, 16 x 8 x 16.
template <typename E>
__device__ __forceinline__ void product(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (__is_same(E, __nv_bfloat16))
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// 8 bytes to shared memory.
__device__ __forceinline__ void copy_pair(uint32_t to, const void* from) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(__cvta_generic_to_global(from)) : "memory");
}
// Four 8 x 8 matrices of 16 bits; the address is of row lane % 8 of matrix lane / 8.
__device__ __forceinline__ void load_matrices(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void load_turned(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}

// DP: dimensions, to a multiple of 64.
template <uint32_t DP, uint32_t kWarps>
struct Few {
  static constexpr uint32_t kPitch = DP + 4, kStages = 3;
  // A step's 16 keys, or values: rows of 128 bytes in columns of 64 dimensions, 16-byte
  // pieces at their place exclusive-or the row modulo 8.
  static constexpr uint32_t kTile = 16 * DP * 2;
  static constexpr uint64_t kRings = kWarps * kStages * 2 * kTile;  // all that warps on their own need
  static constexpr uint64_t kJoining = kWarps * kRows * kPitch * 4 + kRows * (kMostBlocks * kWarps + kTileParts) * 8;  // 16 rows and all pieces
  // The rings; behind the last key, in their place: the warps' outputs of the rows there are, (m, l) and then the
  // weights of a row's pieces, and as many of the prompt's outputs as fit.
  unsigned char ring[kRings > kJoining ? kRings : kJoining];
  float2 sums[kWarps][kRows];
  float inverse[kRows];
};

template <typename E, uint32_t DP, uint32_t kWarps, bool kAlone>
__global__ void __launch_bounds__(kWarps * 32) few_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ AttendPlan plan,
                                                       const __grid_constant__ FewArgs few) {
  extern __shared__ __align__(128) unsigned char raw[];
  using Shared = Few<DP, kWarps>;
  constexpr uint32_t kThreads = kWarps * 32;
  Shared& sh = *reinterpret_cast<Shared*>(raw);
  constexpr uint32_t kStages = Shared::kStages, kTile = Shared::kTile, kPieces = DP / 8;  // pieces of a key
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, c = lane % 4;
  const uint32_t rank = kAlone ? 0 : blockIdx.x % few.blocks;
  uint32_t unit = kAlone ? blockIdx.x * kWarps + warp : blockIdx.x / few.blocks;
  if (kAlone && unit >= few.units) return;
  const uint32_t first = unit % few.row_tiles * kRows;
  unit /= few.row_tiles;
  const uint32_t head = unit % a.kv_heads, rows = min(kRows, a.share - first);
  const uint32_t answer = unit / a.kv_heads, prompt = answer / a.per_prompt;
  // The queries, as first operands of the scores: dimensions 16 j + 2 c + (0 1 | 8 9) of rows g and g + 8.
  uint32_t q[DP / 16][4];
  {
    const E* base = static_cast<const E*>(a.q.data) + (int64_t)answer * a.q.batch + (int64_t)(head * a.share + first) * a.q.head;
    const auto two = [&](uint32_t row, uint32_t d) {
      return row < rows && d < a.dim ? __ldg(reinterpret_cast<const uint32_t*>(base + (int64_t)row * a.q.head + d)) : 0u;
    };
#pragma unroll
    for (uint32_t j = 0; j < DP / 16; ++j) {
      const uint32_t d = 16 * j + 2 * c;
      q[j][0] = two(g, d), q[j][1] = two(g + 8, d), q[j][2] = two(g, d + 8), q[j][3] = two(g + 8, d + 8);
    }
  }
  const uint32_t len = length_of(a.suffix_len, a.suffix_cap, answer), step = kAlone ? 16 : 16 * kWarps * few.blocks;
  uint32_t at = kAlone ? 0 : 16 * (rank * kWarps + warp);

  // Who has the prompt's pieces (ahead of the copies, behind which its reads would queue); an answer's rows may lie in
  // two tiles of queries.
  const uint32_t row0 = (answer - prompt * a.per_prompt) * a.share + first;
  const uint32_t tile0 = row0 / plan.rows, rows0 = min(rows, (tile0 + 1) * plan.rows - row0);
  const Standing standing = standing_of(a, plan, prompt);
  const Owners own0 = owners_of(a, plan, standing, prompt, head * plan.row_tiles + tile0);
  const Owners own1 = rows0 == rows ? own0 : owners_of(a, plan, standing, prompt, head * plan.row_tiles + tile0 + 1);
  const bool bad = bad_answer(a, prompt, answer);
  // The warp's ring: a lane copies a piece of every (32 / kPieces)-th key.
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(sh.ring + warp * kStages * 2 * kTile);
  const uint32_t my_piece = lane % kPieces, my_key = lane / kPieces;
  const E* k_from = static_cast<const E*>(a.sk.data) + (int64_t)answer * a.sk.batch + (int64_t)head * a.sk.head + my_piece * 8;
  const E* v_from = static_cast<const E*>(a.sv.data) + (int64_t)answer * a.sv.batch + (int64_t)head * a.sv.head + my_piece * 8;
  const auto copy = [&](uint32_t stage, uint32_t from) {
#pragma unroll
    for (uint32_t i = 0; i < 16 * kPieces / 32; ++i) {
      const uint32_t key = my_key + i * (32 / kPieces);
      const bool on = from + key < len && my_piece * 8 < a.dim;
      const uint32_t to = ring + stage * 2 * kTile + my_piece / 8 * 2048 + key * 128 + (my_piece % 8 ^ key % 8) * 16;
      const int64_t token = on ? (int64_t)(from + key) : 0;
      copy_piece(to, on ? k_from + token * a.sk.token : static_cast<const E*>(a.q.data), on);
      copy_piece(to + kTile, on ? v_from + token * a.sv.token : static_cast<const E*>(a.q.data), on);
    }
  };
#pragma unroll
  for (uint32_t s = 0; s < kStages - 1; ++s) {
    if (at + s * step < len) copy(s, at + s * step);
    copies_end();
  }

  // What the prompts' kernel wrote is there from here on (it takes whole SMs: blocks of this one hardly start before it ends).
  wait_for_previous();
  const auto record_of = [&](const Owners& own, uint32_t i) { return plan.prefix + (own.first + i + own.segment) * plan.record; };
  const uint32_t quads = a.dim / 4, sums_at = record_sums(plan.held, a.dim), r0 = row0 - tile0 * plan.rows;
  uint32_t gave = 0;
  if (!kAlone) {
    const uint32_t from = own0.first, to = max(own0.last, own1.last);
    if (from + lane < to) gave = __ldca(plan.gave_up + from + lane);
    for (uint32_t i = from + lane + 32; i < to; i += 32) gave |= __ldca(plan.gave_up + i);
  }
  float o[DP / 8][4] = {};
  float m[2] = {kNone, kNone}, l[2] = {0.0f, 0.0f};  // rows g and g + 8; the maxima less by kLift
  // Rows of the matrices that this lane gives the addresses of: of keys for the scores, of values for the outputs.
  const uint32_t k_row = lane % 8, v_row = lane / 8 % 2 * 8 + lane % 8;
  for (uint32_t stage = 0; at < len; at += step, stage = stage + 1 == kStages ? 0 : stage + 1) {
    copies_wait<kStages - 2>();
    __syncwarp();
    const uint32_t ahead = at + (kStages - 1) * step;
    if (ahead < len) copy(stage == 0 ? kStages - 1 : stage - 1, ahead);  // where the step before this one was
    copies_end();
    const uint32_t keys = ring + stage * 2 * kTile, values = keys + kTile;
    float s[2][4] = {};
#pragma unroll
    for (uint32_t j = 0; j < DP / 32; ++j)
#pragma unroll
      for (uint32_t n = 0; n < 2; ++n) {
        const uint32_t piece = 4 * j + lane / 8, key = 8 * n + k_row;
        uint32_t b[4];
        load_matrices(b, keys + piece / 8 * 2048 + key * 128 + (piece % 8 ^ k_row) * 16);
        product<E>(s[n], q[2 * j], b[0], b[1]);
        product<E>(s[n], q[2 * j + 1], b[2], b[3]);
      }
    // Scores of keys at + 8n + 2c + (0, 1): rows g (elements 0, 1) and g + 8 (2, 3).
    float top[2] = {kNone, kNone};
#pragma unroll
    for (uint32_t n = 0; n < 2; ++n)
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) {
        s[n][i] = at + 8 * n + 2 * c + i % 2 < len ? s[n][i] * a.scale2 : kNone;
        top[i / 2] = fmaxf(top[i / 2], s[n][i]);
      }
    bool raise = false;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      top[r] = fmaxf(top[r], __shfl_xor_sync(~0u, top[r], 1));
      top[r] = fmaxf(top[r], __shfl_xor_sync(~0u, top[r], 2));
      raise |= top[r] - (kRaise + kLift<E>) > m[r] || (m[r] == kNone && top[r] > kNone);
    }
    if (__any_sync(~0u, raise)) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float to = fmaxf(m[r], top[r] - kLift<E>), shrink = m[r] == kNone ? 0.0f : exp2_of(m[r] - to);
        m[r] = to;
        l[r] *= shrink;
#pragma unroll
        for (uint32_t n = 0; n < DP / 8; ++n) {
          o[n][2 * r] = shrink == 0.0f ? 0.0f : o[n][2 * r] * shrink;
          o[n][2 * r + 1] = shrink == 0.0f ? 0.0f : o[n][2 * r + 1] * shrink;
        }
      }
    }
    uint32_t w[4];
#pragma unroll
    for (uint32_t n = 0; n < 2; ++n)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float base = m[r] == kNone ? 0.0f : m[r];
        const float2 e = make_float2(exp2_of(s[n][2 * r] - base), exp2_of(s[n][2 * r + 1] - base));
        l[r] += e.x + e.y;
        w[2 * n + r] = pack2(e, E());
      }
#pragma unroll
    for (uint32_t j = 0; j < DP / 16; ++j) {
      const uint32_t piece = 2 * j + lane / 16;
      uint32_t b[4];
      load_turned(b, values + piece / 8 * 2048 + v_row * 128 + (piece % 8 ^ v_row % 8) * 16);
      product<E>(o[2 * j], w, b[0], b[1]);
      product<E>(o[2 * j + 1], w, b[2], b[3]);
    }
    __syncwarp();
  }
  copies_wait<0>();
  if constexpr (kAlone) {
    const float nan = __int_as_float(0x7FC00000);
    const bool pairs = ((uintptr_t)a.out.data | (uint64_t)a.out.batch * 2 | (uint64_t)a.out.head * 2) % 4 == 0;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      l[r] += __shfl_xor_sync(~0u, l[r], 1);
      l[r] += __shfl_xor_sync(~0u, l[r], 2);
      const uint32_t row = g + 8 * r;
      if (row >= rows) continue;
      const Owners& own = row < rows0 ? own0 : own1;
      const uint32_t pr = row < rows0 ? r0 + row : row - rows0, far = own.last - own.first;
      const float* records = record_of(own, 0);
      bool odd = bad || l[r] != l[r];
      float most = m[r];
#pragma unroll 4
      for (uint32_t i = 0; i < far; ++i) {
        const float2 ml = __ldca(reinterpret_cast<const float2*>(records + (uint64_t)i * plan.record + sums_at) + pr);
        odd |= ml.y != ml.y || __ldca(plan.gave_up + own.first + i) != 0;
        most = fmaxf(most, ml.x);
      }
      odd |= most == -kNone;  // a score above 32-bit numbers
      const float base = most == kNone ? 0.0f : most, mine = l[r] > 0.0f ? exp2_of(m[r] - base) : 0.0f;
      float total = l[r] > 0.0f ? mine * l[r] : 0.0f;
#pragma unroll
      for (uint32_t n = 0; n < DP / 8; ++n) {
        o[n][2 * r] = mine > 0.0f ? o[n][2 * r] * mine : 0.0f;
        o[n][2 * r + 1] = mine > 0.0f ? o[n][2 * r + 1] * mine : 0.0f;
      }
      for (uint32_t i = 0; i < far; ++i) {
        const float* record = records + (uint64_t)i * plan.record;
        const float2 ml = __ldca(reinterpret_cast<const float2*>(record + sums_at) + pr);
        float2 x[DP / 8];
#pragma unroll
        for (uint32_t n = 0; n < DP / 8; ++n)
          if (8 * n < a.dim) x[n] = __ldca(reinterpret_cast<const float2*>(record + record_place(plan.held, pr, 8 * n + 2 * c)));
        if (!(ml.y > 0.0f)) continue;  // nothing to attend to in that piece
        const float w = exp2_of(ml.x - base);
        total = fmaf(w, ml.y, total);
#pragma unroll
        for (uint32_t n = 0; n < DP / 8; ++n)
          if (8 * n < a.dim) {
            o[n][2 * r] = fmaf(w, x[n].x, o[n][2 * r]);
            o[n][2 * r + 1] = fmaf(w, x[n].y, o[n][2 * r + 1]);
          }
      }
      const float inv = odd ? nan : total > 0.0f ? 1.0f / total : 0.0f;
      if (a.lse && c == 0)
        a.lse[(uint64_t)answer * (a.kv_heads * a.share) + head * a.share + first + row] =
            odd ? nan : total > 0.0f ? (most + log2f(total)) * 0.693147180559945309f : kNone;
      E* out = static_cast<E*>(const_cast<void*>(a.out.data)) + (int64_t)answer * a.out.batch +
               (int64_t)(head * a.share + first + row) * a.out.head + 2 * c;
#pragma unroll
      for (uint32_t n = 0; n < DP / 8; ++n)
        if (8 * n < a.dim) {
          const uint32_t u = pack2(make_float2(o[n][2 * r] * inv, o[n][2 * r + 1] * inv), E());
          if (pairs) {
            *reinterpret_cast<uint32_t*>(out + 8 * n) = u;
          } else {
            uint16_t* h = reinterpret_cast<uint16_t*>(out + 8 * n);
            h[0] = (uint16_t)u, h[1] = (uint16_t)(u >> 16);
          }
        }
    }
    return;
  }
  __syncthreads();  // the rings are done with
  const uint32_t near = few.blocks * kWarps, most_pieces = near + max(own0.last - own0.first, own1.last - own1.first);
  float* const outputs = reinterpret_cast<float*>(sh.ring);
  float2* const pieces = reinterpret_cast<float2*>(outputs + kWarps * rows * Shared::kPitch);
  const uint32_t held_at = (kWarps * rows * Shared::kPitch * 4 + rows * most_pieces * 8 + 15) / 16 * 16;
  float4* const held = reinterpret_cast<float4*>(sh.ring + held_at) + threadIdx.x;
  const uint32_t most_held = (uint32_t)((sizeof(sh.ring) - held_at) / (kThreads * 16));
  const auto output_of = [&](Shared* from, uint32_t w, uint32_t row, uint32_t d) {
    return reinterpret_cast<float*>(from->ring) + (w * rows + row) * Shared::kPitch + d;
  };
  // How the joining is shared out: four dimensions of a row to a thread, neighbouring rows to neighbours, over the
  // cluster's blocks; where they have threads enough up to eight lanes of a warp share an item's pieces out.
  const uint32_t items = rows * quads;
  uint32_t parts = 1;
  while (parts < 8 && 2 * parts * items <= few.blocks * kThreads) parts *= 2;
  const uint32_t width = 32 / parts, part = lane / width;
  const auto each_item = [&](auto f) {  // f(item, whether there is one, row, first dimension, its pieces' first, how many), by whole warps
    for (uint32_t n0 = (rank * kWarps + warp) * width; n0 < items; n0 += few.blocks * kWarps * width) {
      const uint32_t n = n0 + lane % width, row = n < items ? n % rows : 0, d = n < items ? n / rows * 4 : 0;
      const Owners& own = row < rows0 ? own0 : own1;
      f(n < items, row, d, record_of(own, 0) + record_place(plan.held, row < rows0 ? r0 + row : row - rows0, d), own.last - own.first);
    }
  };
  // The prompt's records of these rows, all on their way at once while the weights are found: (m, l), and what each
  // thread will add up.  (Read where they are used, eight at a time, they were three rounds of 2,000 cycles.)
  for (uint32_t row = warp; row < rows; row += kWarps) {
    const Owners& own = row < rows0 ? own0 : own1;
    const float* from = record_of(own, 0) + sums_at + 2 * (row < rows0 ? r0 + row : row - rows0);
    for (uint32_t i = lane; i < own.last - own.first; i += 32)
      copy_pair((uint32_t)__cvta_generic_to_shared(pieces + row * most_pieces + near + i), from + (uint64_t)i * plan.record);
  }
  copies_end();
  {
    uint32_t n = 0;
    each_item([&](bool, uint32_t, uint32_t, const float* from, uint32_t far) {
      const uint32_t some = min(far > part ? (far - part + parts - 1) / parts : 0u, most_held - n);
#pragma unroll 4
      for (uint32_t j = 0; j < some; ++j)
        copy_piece((uint32_t)__cvta_generic_to_shared(held + (n + j) * kThreads), from + (uint64_t)(part + j * parts) * plan.record, true);
      n += some;
    });
    copies_end();
  }
  // Element i of o[n] is of row g + i / 2 * 8 and dimension 8 n + 2 c + i % 2.
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    l[r] += __shfl_xor_sync(~0u, l[r], 1);
    l[r] += __shfl_xor_sync(~0u, l[r], 2);
    const uint32_t row = g + 8 * r;
    if (row >= rows) continue;
    if (c == 0) sh.sums[warp][row] = make_float2(m[r], l[r]);
#pragma unroll
    for (uint32_t n = 0; n < DP / 8; ++n)
      *reinterpret_cast<float2*>(output_of(&sh, warp, row, 8 * n + 2 * c)) = make_float2(o[n][2 * r], o[n][2 * r + 1]);
  }
  const bool clustered = few.blocks > 1;
  cg::cluster_group cluster = cg::this_cluster();
  copies_wait<1>();
  if (clustered) cluster.sync();
  else __syncthreads();

  // The weights of a row's pieces: of the warps of all blocks here, and of the prompt's.
  const auto peer = [&](uint32_t b) -> Shared* { return clustered ? cluster.map_shared_rank(&sh, b) : &sh; };
  for (uint32_t row = warp; row < rows; row += kWarps) {
    const uint32_t far = row < rows0 ? own0.last - own0.first : own1.last - own1.first;
    float2* const piece = pieces + row * most_pieces;
    bool odd = bad || gave != 0;
    float most = kNone;
    for (uint32_t i = lane; i < near + far; i += 32) {
      if (i < near) piece[i] = peer(i / kWarps)->sums[i % kWarps][row];
      odd |= piece[i].y != piece[i].y;
      most = fmaxf(most, piece[i].x);
    }
#pragma unroll
    for (int d = 16; d; d /= 2) most = fmaxf(most, __shfl_xor_sync(~0u, most, d));
    odd |= most == -kNone;  // a score above 32-bit numbers
    const float base = most == kNone ? 0.0f : most;
    float total = 0.0f;
    for (uint32_t i = lane; i < near + far; i += 32) {
      const float2 ml = piece[i];
      const float w = ml.y > 0.0f ? exp2_of(ml.x - base) : 0.0f;  // 0: nothing to attend to in that piece
      piece[i].x = w;
      total = fmaf(w, ml.y > 0.0f ? ml.y : 0.0f, total);
    }
#pragma unroll
    for (int d = 16; d; d /= 2) total += __shfl_xor_sync(~0u, total, d);
    odd = __any_sync(~0u, odd);
    const float nan = __int_as_float(0x7FC00000);
    if (lane == 0) {
      sh.inverse[row] = odd ? nan : total > 0.0f ? 1.0f / total : 0.0f;
      if (a.lse && rank == 0)
        a.lse[(uint64_t)answer * (a.kv_heads * a.share) + head * a.share + first + row] =
            odd ? nan : total > 0.0f ? (most + log2f(total)) * 0.693147180559945309f : kNone;
    }
  }
  copies_wait<0>();
  __syncthreads();
  const bool whole = ((uintptr_t)a.out.data | (uint64_t)a.out.batch * 2 | (uint64_t)a.out.head * 2) % 8 == 0;
  uint32_t next = 0;
  each_item([&](bool on, uint32_t row, uint32_t d, const float* from, uint32_t far) {
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const float2* piece = pieces + row * most_pieces;
    const auto add = [&](float w, const float4& x) {
      if (w > 0.0f) sum = make_float4(fmaf(w, x.x, sum.x), fmaf(w, x.y, sum.y), fmaf(w, x.z, sum.z), fmaf(w, x.w, sum.w));
    };
    const uint32_t some = min(far > part ? (far - part + parts - 1) / parts : 0u, most_held - next);
#pragma unroll 4
    for (uint32_t j = 0; j < some; ++j) add(piece[near + part + j * parts].x, held[(next + j) * kThreads]);
    next += some;
#pragma unroll 4
    for (uint32_t i = part + some * parts; i < far; i += parts) add(piece[near + i].x, __ldca(reinterpret_cast<const float4*>(from + (uint64_t)i * plan.record)));
#pragma unroll 4
    for (uint32_t i = part; i < near; i += parts)
      add(piece[i].x, *reinterpret_cast<const float4*>(output_of(peer(i / kWarps), i % kWarps, row, d)));
    for (uint32_t apart = width; apart < 32; apart *= 2) {
      sum.x += __shfl_xor_sync(~0u, sum.x, apart);
      sum.y += __shfl_xor_sync(~0u, sum.y, apart);
      sum.z += __shfl_xor_sync(~0u, sum.z, apart);
      sum.w += __shfl_xor_sync(~0u, sum.w, apart);
    }
    if (on && part == 0) {
      const float inv = sh.inverse[row];
      E* out = static_cast<E*>(const_cast<void*>(a.out.data)) + (int64_t)answer * a.out.batch +
               (int64_t)(head * a.share + first + row) * a.out.head + d;
      const uint2 u = make_uint2(pack2(make_float2(sum.x * inv, sum.y * inv), E()), pack2(make_float2(sum.z * inv, sum.w * inv), E()));
      if (whole) {
        *reinterpret_cast<uint2*>(out) = u;
      } else {
        uint16_t* h = reinterpret_cast<uint16_t*>(out);
        h[0] = (uint16_t)u.x, h[1] = (uint16_t)(u.x >> 16), h[2] = (uint16_t)u.y, h[3] = (uint16_t)(u.y >> 16);
      }
    }
  });
  if (clustered) cluster.sync();  // others may still read this block's outputs
}

}  // namespace

bool few_takes(const AttendArgs& a) {
  const auto fits = [](const Vectors& x) { return ((uintptr_t)x.data | (uint64_t)x.batch * 2 | (uint64_t)x.token * 2 | (uint64_t)x.head * 2) % 16 == 0; };
  if (a.dtype == BF_F32 || a.dim % 8 || a.dim > 128 || !fits({a.q.data, a.q.batch, 0, a.q.head})) return false;
  return a.suffix_cap == 0 || (fits(a.sk) && fits(a.sv));
}

cudaError_t launch_few_queries(const AttendArgs& a, const AttendPlan& plan, cudaStream_t st) {
  FewArgs f = {(a.share + kRows - 1) / kRows, 1, 0};
  const uint64_t units = (uint64_t)a.prompts * a.per_prompt * a.kv_heads * f.row_tiles;
  if (units > 0x7FFFFFFFu) return cudaErrorInvalidValue;
  f.units = (uint32_t)units;
  const bool alone = units >= kAloneUnits, two = !alone && units > (a.dim <= 64 ? 608 : 304);
  while (!alone && f.blocks < kMostBlocks && units * f.blocks * 2 <= 304 && a.suffix_cap > 64ull * f.blocks) f.blocks *= 2;  // two an SM
  const auto launch = [&](auto kernel, uint32_t warps, uint64_t shared) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shared);
    if (e != cudaSuccess) return e;
    return launch_shared(kernel, alone ? (units + warps - 1) / warps : units * f.blocks, warps * 32, f.blocks, true, shared, st, a, plan, f);
  };
  const auto launch_dim = [&](auto type, auto dim) {
    using E = decltype(type);
    constexpr uint32_t DP = decltype(dim)::value;
    return alone ? launch(few_kernel<E, DP, 4, true>, 4, Few<DP, 4>::kRings)
           : two ? launch(few_kernel<E, DP, 2, false>, 2, sizeof(Few<DP, 2>))
                 : launch(few_kernel<E, DP, 4, false>, 4, sizeof(Few<DP, 4>));
  };
  const auto launch_type = [&](auto type) {
    return a.dim <= 64 ? launch_dim(type, std::integral_constant<uint32_t, 64>()) : launch_dim(type, std::integral_constant<uint32_t, 128>());
  };
  return a.dtype == BF_BF16 ? launch_type(__nv_bfloat16()) : launch_type(__half());
}

}  // namespace bfk
