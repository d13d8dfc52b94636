// bf_attend_few.cu -- an answer's own keys, and the joining of all that was attended
// to: 16-bit types, up to 128 dimensions.
//
// A block to an answer and key head (and up to 16 of the query heads that share
// it); in a cluster where there are few, so that an answer's keys are spread over
// several SMs.  The keys are read once and by one block, so they go from memory to
// registers in the shape in which the products take them: which dimension, or which
// key, stands where inside a product does not matter as long as both operands agree, and
// 16 bytes of a key's vector are eight of a thread's elements.  The products are the
// warps' own (16 x 8 x 16): at 4 to 16 queries a key the memory is the bound, and a
// tile of 128 queries would be empty.  A warp takes 16 keys at a time; the next keys are
// on their way while the present ones' weights are made, the next values while the
// scores are.
//
// Behind its own keys a block waits for the prompts' pieces and joins all of them.
#include <cooperative_groups.h>

#include "bf_attend.cuh"

namespace bfk {

namespace {

namespace cg = cooperative_groups;

constexpr uint32_t kThreads = 128, kWarps = kThreads / 32, kRows = 16, kMostBlocks = 8;
constexpr float kRaise = 8.0f;

struct FewArgs {
  uint32_t row_tiles, blocks;  // of a key head's query heads; of a cluster
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

__device__ __forceinline__ uint4 load16(const void* p, bool on) {
  return on ? __ldg(reinterpret_cast<const uint4*>(p)) : make_uint4(0, 0, 0, 0);
}

// DP: dimensions, to a multiple of 64.
template <typename E, uint32_t DP>
struct Few {
  static constexpr uint32_t kPitch = DP + 4;
  float o[kWarps][kRows][kPitch];
  float2 sums[kWarps][kRows];
  float weight[kRows][kMostBlocks * kWarps + kTileParts];  // of the pieces: the cluster's warps', then the prompt's
  float inverse[kRows];
};

template <typename E, uint32_t DP>
__global__ void __launch_bounds__(kThreads) few_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ AttendPlan plan,
                                                       const __grid_constant__ FewArgs few) {
  __shared__ Few<E, DP> sh;
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, c = lane % 4;
  const uint32_t rank = blockIdx.x % few.blocks;
  uint64_t unit = blockIdx.x / few.blocks;
  const uint32_t first = unit % few.row_tiles * kRows;
  unit /= few.row_tiles;
  const uint32_t head = unit % a.kv_heads, rows = min(kRows, a.share - first);
  const uint64_t answer = unit / a.kv_heads;
  const uint32_t prompt = (uint32_t)(answer / a.per_prompt);

  // The queries, as first operands of the scores: dimensions 32 j + 8 c + (0 1 | 2 3 | 4 5 | 6 7) of rows g and g + 8.
  uint32_t q[DP / 32][2][4];
  {
    const E* base = static_cast<const E*>(a.q.data) + (int64_t)answer * a.q.batch + (int64_t)(head * a.share + first) * a.q.head;
#pragma unroll
    for (uint32_t j = 0; j < DP / 32; ++j) {
      const uint32_t d = 32 * j + 8 * c;
      const uint4 lo = load16(base + (int64_t)g * a.q.head + d, g < rows && d < a.dim);
      const uint4 hi = load16(base + (int64_t)(g + 8) * a.q.head + d, g + 8 < rows && d < a.dim);
      q[j][0][0] = lo.x, q[j][0][2] = lo.y, q[j][1][0] = lo.z, q[j][1][2] = lo.w;
      q[j][0][1] = hi.x, q[j][0][3] = hi.y, q[j][1][1] = hi.z, q[j][1][3] = hi.w;
    }
  }
  const uint32_t len = length_of(a.suffix_len, a.suffix_cap, answer);
  const E* keys = static_cast<const E*>(a.sk.data) + (int64_t)answer * a.sk.batch + (int64_t)head * a.sk.head;
  const E* values = static_cast<const E*>(a.sv.data) + (int64_t)answer * a.sv.batch + (int64_t)head * a.sv.head;
  uint4 k[2][DP / 32], v[DP / 64][4];
  const auto load_k = [&](uint32_t at) {  // keys at + g and at + 8 + g
#pragma unroll
    for (uint32_t n = 0; n < 2; ++n)
#pragma unroll
      for (uint32_t j = 0; j < DP / 32; ++j) {
        const uint32_t key = at + 8 * n + g, d = 32 * j + 8 * c;
        k[n][j] = load16(keys + (int64_t)key * a.sk.token + d, key < len && d < a.dim);
      }
  };
  const auto load_v = [&](uint32_t at) {  // keys at + 2c + (0, 1, 8, 9), dimensions 64 h + 8 g + (0 .. 7)
#pragma unroll
    for (uint32_t h = 0; h < DP / 64; ++h)
#pragma unroll
      for (uint32_t n = 0; n < 4; ++n) {
        const uint32_t key = at + 2 * c + n % 2 + n / 2 * 8, d = 64 * h + 8 * g;
        v[h][n] = load16(values + (int64_t)key * a.sv.token + d, key < len && d < a.dim);
      }
  };
  float o[DP / 64][8][4] = {};
  float m[2] = {kNone, kNone}, l[2] = {0.0f, 0.0f};  // rows g and g + 8
  const uint32_t step = 16 * kWarps * few.blocks;
  uint32_t at = 16 * (rank * kWarps + warp);
  if (at < len) {
    load_k(at);
    load_v(at);
  }
  // Who has the prompt's pieces (while the keys are on their way); an answer's rows may lie in two tiles of queries.
  const uint32_t row0 = (uint32_t)(answer - (uint64_t)prompt * a.per_prompt) * a.share + first;
  const uint32_t tile0 = row0 / plan.rows, rows0 = min(rows, (tile0 + 1) * plan.rows - row0);
  const Standing standing = standing_of(a, plan.keys, prompt);
  const Owners own0 = owners_of(a, plan, standing, prompt, head * plan.row_tiles + tile0);
  const Owners own1 = rows0 == rows ? own0 : owners_of(a, plan, standing, prompt, head * plan.row_tiles + tile0 + 1);
  const bool bad = bad_answer(a, prompt, answer);
  for (; at < len; at += step) {
    float s[2][4] = {};
#pragma unroll
    for (uint32_t j = 0; j < DP / 32; ++j)
#pragma unroll
      for (uint32_t n = 0; n < 2; ++n) {
        product<E>(s[n], q[j][0], k[n][j].x, k[n][j].y);
        product<E>(s[n], q[j][1], k[n][j].z, k[n][j].w);
      }
    if (at + step < len) load_k(at + step);
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
      raise |= top[r] - kRaise > m[r] || (m[r] == kNone && top[r] > kNone);
    }
    if (__any_sync(~0u, raise)) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float to = fmaxf(m[r], top[r]), shrink = m[r] == kNone ? 0.0f : exp2_of(m[r] - to);
        m[r] = to;
        l[r] *= shrink;
#pragma unroll
        for (uint32_t h = 0; h < DP / 64; ++h)
#pragma unroll
          for (uint32_t e = 0; e < 8; ++e) {
            o[h][e][2 * r] = shrink == 0.0f ? 0.0f : o[h][e][2 * r] * shrink;
            o[h][e][2 * r + 1] = shrink == 0.0f ? 0.0f : o[h][e][2 * r + 1] * shrink;
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
    for (uint32_t h = 0; h < DP / 64; ++h) {
      const uint32_t* v0 = reinterpret_cast<const uint32_t*>(&v[h][0]);
      const uint32_t* v1 = reinterpret_cast<const uint32_t*>(&v[h][1]);
      const uint32_t* v2 = reinterpret_cast<const uint32_t*>(&v[h][2]);
      const uint32_t* v3 = reinterpret_cast<const uint32_t*>(&v[h][3]);
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e) {
        const uint32_t pick = e % 2 ? 0x7632 : 0x5410;
        product<E>(o[h][e], w, __byte_perm(v0[e / 2], v1[e / 2], pick), __byte_perm(v2[e / 2], v3[e / 2], pick));
      }
    }
    if (at + step < len) load_v(at + step);
  }
  // The warp's outputs: element i of o[h][e] is of row g + i / 2 * 8 and dimension 64 h + (2 c + i % 2) 8 + e.
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    l[r] += __shfl_xor_sync(~0u, l[r], 1);
    l[r] += __shfl_xor_sync(~0u, l[r], 2);
    const uint32_t row = g + 8 * r;
    if (row >= rows) continue;
    if (c == 0) sh.sums[warp][row] = make_float2(m[r], l[r]);
#pragma unroll
    for (uint32_t h = 0; h < DP / 64; ++h)
#pragma unroll
      for (uint32_t i = 0; i < 2; ++i)
#pragma unroll
        for (uint32_t e = 0; e < 8; e += 4)
          *reinterpret_cast<float4*>(&sh.o[warp][row][64 * h + (2 * c + i) * 8 + e]) =
              make_float4(o[h][e][2 * r + i], o[h][e + 1][2 * r + i], o[h][e + 2][2 * r + i], o[h][e + 3][2 * r + i]);
  }
  const bool clustered = few.blocks > 1;
  cg::cluster_group cluster = cg::this_cluster();
  if (clustered) cluster.sync();
  else __syncthreads();
  wait_for_previous();

  // The weights of a row's pieces: of the warps of all blocks here, and of the prompt's.
  const uint32_t near = few.blocks * kWarps;
  const auto peer = [&](uint32_t b) -> Few<E, DP>* { return clustered ? cluster.map_shared_rank(&sh, b) : &sh; };
  const auto record_of = [&](const Owners& own, uint32_t i) { return plan.prefix + (own.first + i + own.segment) * plan.record; };
  for (uint32_t row = warp; row < rows; row += kWarps) {
    const Owners own = row < rows0 ? own0 : own1;
    const uint32_t r = row < rows0 ? row0 - tile0 * plan.rows + row : row - rows0, far = own.last - own.first;
    bool odd = bad;
    float most = kNone;
    for (uint32_t i = lane; i < near + far; i += 32) {
      float2 ml;
      if (i < near) {
        ml = peer(i / kWarps)->sums[i % kWarps][row];
      } else {
        ml = __ldcg(reinterpret_cast<const float2*>(record_of(own, i - near) + record_sums(plan.rows, a.dim)) + r);
        odd |= __ldcg(plan.gave_up + own.first + i - near) != 0;
      }
      odd |= ml.y != ml.y;
      most = fmaxf(most, ml.x);
      sh.weight[row][i] = ml.x;
    }
#pragma unroll
    for (int d = 16; d; d /= 2) most = fmaxf(most, __shfl_xor_sync(~0u, most, d));
    const float base = most == kNone ? 0.0f : most;
    float total = 0.0f;
    for (uint32_t i = lane; i < near + far; i += 32) {
      const float l = i < near ? peer(i / kWarps)->sums[i % kWarps][row].y
                               : __ldcg(reinterpret_cast<const float2*>(record_of(own, i - near) + record_sums(plan.rows, a.dim)) + r).y;
      const float w = l > 0.0f ? exp2_of(sh.weight[row][i] - base) : 0.0f;  // 0: nothing to attend to in that piece
      sh.weight[row][i] = w;
      total = fmaf(w, l > 0.0f ? l : 0.0f, total);
    }
#pragma unroll
    for (int d = 16; d; d /= 2) total += __shfl_xor_sync(~0u, total, d);
    odd = __any_sync(~0u, odd);
    const float nan = __int_as_float(0x7FC00000);
    if (lane == 0) {
      sh.inverse[row] = odd ? nan : total > 0.0f ? 1.0f / total : 0.0f;
      if (a.lse && rank == 0)
        a.lse[answer * ((uint64_t)a.kv_heads * a.share) + head * a.share + first + row] =
            odd ? nan : total > 0.0f ? (most + log2f(total)) * 0.693147180559945309f : kNone;
    }
  }
  __syncthreads();
  // Four dimensions of a row to a thread, neighbouring rows to neighbours; the cluster's blocks share them out.
  const uint32_t quads = a.dim / 4;
  const bool whole = ((uintptr_t)a.out.data | (uint64_t)a.out.batch * 2 | (uint64_t)a.out.head * 2) % 8 == 0;
  for (uint32_t n = rank * kThreads + threadIdx.x; n < rows * quads; n += few.blocks * kThreads) {
    const uint32_t row = n % rows, d = n / rows * 4;
    const Owners& own = row < rows0 ? own0 : own1;
    const uint32_t r = row < rows0 ? row0 - tile0 * plan.rows + row : row - rows0, far = own.last - own.first;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const auto add = [&](float w, const float4& x) {
      if (w > 0.0f) sum = make_float4(fmaf(w, x.x, sum.x), fmaf(w, x.y, sum.y), fmaf(w, x.z, sum.z), fmaf(w, x.w, sum.w));
    };
    const float* from = record_of(own, 0) + record_place(plan.rows, r, d);
    constexpr uint32_t kAhead = 8;
    for (uint32_t i = 0; i < far; i += kAhead) {
      float4 x[kAhead];
#pragma unroll
      for (uint32_t k = 0; k < kAhead; ++k)
        if (i + k < far) x[k] = __ldcg(reinterpret_cast<const float4*>(from + (uint64_t)(i + k) * plan.record));
#pragma unroll
      for (uint32_t k = 0; k < kAhead; ++k)
        if (i + k < far) add(sh.weight[row][near + i + k], x[k]);
    }
    for (uint32_t b = 0; b < few.blocks; ++b) {
      const Few<E, DP>* them = peer(b);
#pragma unroll
      for (uint32_t w = 0; w < kWarps; ++w) add(sh.weight[row][b * kWarps + w], *reinterpret_cast<const float4*>(&them->o[w][row][d]));
    }
    {
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
  }
  if (clustered) cluster.sync();  // others may still read this block's outputs
}

}  // namespace

bool few_takes(const AttendArgs& a) {
  const auto fits = [](const Vectors& x) { return ((uintptr_t)x.data | (uint64_t)x.batch * 2 | (uint64_t)x.token * 2 | (uint64_t)x.head * 2) % 16 == 0; };
  if (a.dtype == BF_F32 || a.dim % 8 || a.dim > 128 || !fits({a.q.data, a.q.batch, 0, a.q.head})) return false;
  return a.suffix_cap == 0 || (fits(a.sk) && fits(a.sv));
}

cudaError_t launch_few_queries(const AttendArgs& a, const AttendPlan& plan, cudaStream_t st) {
  FewArgs f = {(a.share + kRows - 1) / kRows, 1};
  const uint64_t units = (uint64_t)a.prompts * a.per_prompt * a.kv_heads * f.row_tiles;
  while (f.blocks < kMostBlocks && units * f.blocks < 304 && a.suffix_cap > 64ull * f.blocks) f.blocks *= 2;
  const auto launch = [&](auto kernel) { return launch_shaped(kernel, units * f.blocks, kThreads, f.blocks, true, st, a, plan, f); };
  if (a.dtype == BF_BF16) return a.dim <= 64 ? launch(few_kernel<__nv_bfloat16, 64>) : launch(few_kernel<__nv_bfloat16, 128>);
  return a.dim <= 64 ? launch(few_kernel<__half, 64>) : launch(few_kernel<__half, 128>);
}

}  // namespace bfk
