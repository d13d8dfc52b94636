// bf_rows.cu -- passes over rows of logits: token log-probabilities and
// entropies, their gradient, the clipped policy loss and both passes of the
// preference loss (arithmetic in bf_rows.cuh).  Compiled once per element type
// (-DBF_ROWS_TYPE=<bf_dtype>).
#include "bf_rows.cuh"

#ifndef BF_ROWS_TYPE
#error "BF_ROWS_TYPE: the element type, a bf_dtype"
#endif

namespace bfk {

namespace {

#if BF_ROWS_TYPE == 0
using E = float;
#elif BF_ROWS_TYPE == 1
using E = __nv_bfloat16;
#else
using E = __half;
#endif
constexpr uint32_t kW = Vec<E>::kWidth;

// `entropy` of a kernel: whether its scores need the rows' entropies, its
// gradient a slope in them.  The policy loss always reports them.
template <RowOp op, bool entropy>
constexpr bool kMoment = op == RowOp::kPolicy || entropy;

template <RowOp op>
constexpr bool kScores = op == RowOp::kScore || op == RowOp::kPairScore;

// The policy loss from its sums, the k-th in lane k of the calling warp.
__device__ __forceinline__ void put_policy_stats(const RowArgs& a, float total) {
  const float surrogate = __shfl_sync(~0u, total, 0), kl = __shfl_sync(~0u, total, 1), h = __shfl_sync(~0u, total, 2);
  if (threadIdx.x == 0) {
    a.stats[0] = -surrogate + (a.kl_coef != 0.0f ? a.kl_coef * kl : 0.0f) - a.entropy_coef * h;
    a.stats[1] = -surrogate;
  } else if (threadIdx.x < kPolicySums) {
    a.stats[threadIdx.x + 1] = total;
  }
}

// The sums of `parts` parts from `from` on, the k-th in thread k.
__device__ __forceinline__ float sum_parts(const float* from, uint64_t parts, float* buf) {
  float v[kPolicySums] = {};
  const float4* part = reinterpret_cast<const float4*>(from);  // kPolicyPart floats each
  constexpr uint32_t kAhead = 8;  // one block reads them all: at one a time it took a fifth of a short call
  for (uint64_t i = threadIdx.x; i < parts; i += kAhead * blockDim.x) {
    float4 lo[kAhead];
    float hi[kAhead];
#pragma unroll
    for (uint32_t j = 0; j < kAhead; ++j) {
      const uint64_t at = i + j * blockDim.x;
      lo[j] = at < parts ? __ldcg(part + 2 * at) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      hi[j] = at < parts ? __ldcg(from + kPolicyPart * at + 4) : 0.0f;
    }
#pragma unroll
    for (uint32_t j = 0; j < kAhead; ++j) {
      v[0] += lo[j].x;
      v[1] += lo[j].y;
      v[2] += lo[j].z;
      v[3] += lo[j].w;
      v[4] += hi[j];
    }
  }
  return block_sums(v, buf);
}

// The loss from its parts' sums, in an order that does not depend on when blocks ran.
__device__ __forceinline__ void policy_stats(const RowArgs& a, uint64_t parts, float* buf) {
  last_sees();
  const float total = sum_parts(a.partial, parts, buf);
  if (threadIdx.x < 32) put_policy_stats(a, total);
}

// (x - m) (hi + lo) as (x - base) hi - r + (x - base) lo: with base = 0 and r =
// m hi rounded it is two products and sums, the small part last, and what r is
// off by (`rest`) goes into the factors once per row, as 1 + rest ln2.  With m hi
// below 1,024 rest is at most 1.5e-4 (m lo, and half a last place of r), so that is
// below 6e-9 off, always short; 1e-12 where m hi is around 10.  Rows of larger logits
// (or all masked by the type's lowest value, where m hi leaves the 32-bit range) take
// base = m, r = 0.
//
// Without `exact` the small part is left out, for gradients of 16 bits: 1e-6 of
// a probability of e^-14.
template <bool exact>
struct Exponent {
  float2 hi, lo, base, r;
  float rest;

  __device__ __forceinline__ Exponent(float m, Scale c) : hi(make_float2(c.hi, c.hi)), lo(make_float2(c.lo, c.lo)) {
    const bool fits = fabsf(m) * c.hi < 1024.0f;
    base = fits ? make_float2(0.0f, 0.0f) : make_float2(-m, -m);
    r = fits ? make_float2(-m * c.hi, -m * c.hi) : make_float2(0.0f, 0.0f);
    rest = fits ? fmaf(exact ? -m : 0.0f, c.lo, fmaf(-m, c.hi, m * c.hi)) : 0.0f;
  }
  // v 2^rest; 2^rest itself, rounded, would be off the same way in every row with this m.
  __device__ __forceinline__ float put_back(float v) const { return fmaf(v, rest * kLn2, v); }
  __device__ __forceinline__ float2 of(float2 x) const {
    x = __fadd2_rn(x, base);
    const float2 t = __ffma2_rn(x, hi, r);
    return exact ? __ffma2_rn(x, lo, t) : t;
  }
};

// NV vectors in registers: their sums against their own maximum (q only with `moment`).
template <int NV, bool moment>
__device__ __forceinline__ RowSums sums_of(const uint4* u, Scale c) {
  const float m = max_of<E, NV>(u);
  const Exponent<true> ex(usable_max(m), c);
  float2 s = {}, q = {};
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    float2 x[kW / 2];
    unpack<E>(u[k], x);
#pragma unroll
    for (uint32_t i = 0; i < kW / 2; ++i) {
      const float2 t = ex.of(x[i]), e = make_float2(exp2_fast(t.x), exp2_fast(t.y));
      s = __fadd2_rn(s, e);
      if (moment) q = __ffma2_rn(e, make_float2(finite_t(t.x), finite_t(t.y)), q);
    }
  }
  const float s1 = s.x + s.y, q1 = fmaf(ex.rest, s1, q.x + q.y);
  return {m, ex.put_back(s1), ex.put_back(q1), m == kMinusInf ? 0.0f : 1.0f};
}

// The gradient of vectors of logits, from a row's factors (o.d only with `tilt`).
template <bool tilt>
struct Grads {
  Exponent<sizeof(E) == 4> ex;
  float2 b, d;

  __device__ __forceinline__ Grads(const RowOut& o, Scale c) : ex(o.m, c) {
    const float b1 = ex.put_back(fmaf(o.d, ex.rest, o.b)), d1 = ex.put_back(o.d);
    b = make_float2(b1, b1);
    d = make_float2(d1, d1);
  }
  __device__ __forceinline__ uint4 of(const uint4& u) const {
    float2 x[kW / 2];
    unpack<E>(u, x);
#pragma unroll
    for (uint32_t i = 0; i < kW / 2; ++i) {
      const float2 t = ex.of(x[i]), e = make_float2(exp2_fast(t.x), exp2_fast(t.y));
      x[i] = __fmul2_rn(e, tilt ? __ffma2_rn(d, make_float2(finite_t(t.x), finite_t(t.y)), b) : b);
    }
    return pack<E>(x);
  }
};

// The gradient of vector v of row x, to row g.
__device__ __forceinline__ void put(const Window<E>& x, const Window<E>& g, uint32_t v, const uint4& d) {
  if (x.shift == g.shift) g.store(v, d);
  else g.store_cut(v, x.shift, d);
}

// The gradients of N vectors of row x, to row g (zeros with `zero`).
template <int N, bool tilt>
__device__ __forceinline__ void put_many(const Window<E>& x, const Window<E>& g, const uint4 (&u)[N], uint32_t v,
                                         uint32_t step, const Grads<tilt>& grads, bool zero) {
  const uint4 none = make_uint4(0, 0, 0, 0);
  if (x.shift == g.shift && g.template all_whole<N>(v, step)) {
    uint4* p = reinterpret_cast<uint4*>(g.at(v));
    if (zero) {
#pragma unroll
      for (int k = 0; k < N; ++k, p += step) __stcs(p, none);
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k, p += step) __stcs(p, grads.of(u[k]));
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) put(x, g, v + k * step, zero ? none : grads.of(u[k]));
  }
}

// ---- the shortest rows (three modes): a thread for each, N elements at most ----
//
// Bound by waiting, not by its bytes: token and logits, then the sequence, then
// the advantage arrive one after the other.  655,360 rows of 3 (f32): 13.5 us of
// a policy loss of 29 us, the counts before it 10 us.

constexpr uint32_t kGroupThreads = 256;

// The part of the policy loss that a block's rows have.  Said before the
// gradient is stored, so that the fence has only these few values to wait for:
// after the stores, it cost a fifth of the kernel's time.  The last block sums
// up at its end.  Above kMostSaying blocks, each warp leaves its part without
// waiting for others and a kernel behind sums up.
__device__ __forceinline__ bool say_policy_part(const RowArgs& a, const RowOut& o, bool mine, uint32_t lanes, float* buf) {
  float v[kPolicySums];
#pragma unroll
  for (uint32_t k = 0; k < kPolicySums; ++k) v[k] = mine ? o.sums[k] : 0.0f;
  if (a.sums_behind) {
#pragma unroll
    for (uint32_t k = 0; k < kPolicySums; ++k)
      for (uint32_t d = 16; d >= lanes && d; d /= 2) v[k] += __shfl_down_sync(~0u, v[k], d);
    if (threadIdx.x % 32 == 0) {
      float* part = a.partial + ((uint64_t)blockIdx.x * (kGroupThreads / 32) + threadIdx.x / 32) * kPolicyPart;
      *reinterpret_cast<float4*>(part) = make_float4(v[0], v[1], v[2], v[3]);
      part[4] = v[4];
    }
    return false;
  }
  const float sum = block_sums(v, buf, lanes);
  if (threadIdx.x >= 32) return false;
  if (threadIdx.x < kPolicySums) a.partial[(uint64_t)blockIdx.x * kPolicyPart + threadIdx.x] = sum;
  return last_to_say(&a.counts->blocks_done, gridDim.x);
}

template <RowOp op, int N>
__global__ void __launch_bounds__(kGroupThreads) short_kernel(const RowArgs a, uint32_t) {
  const uint64_t row = (uint64_t)blockIdx.x * kGroupThreads + threadIdx.x;
  const bool here = row < a.rows;
  if constexpr (kFollows<op>) let_next_start();
  RowIn in = {};
  float v[N];
  const E* x = static_cast<const E*>(a.x) + row * a.ldx;
#pragma unroll
  for (uint32_t j = 0; j < N; ++j) v[j] = here && j < a.vocab ? to_f32(x[j]) : kMinusInf;
  if (here) in = load_row<E, op>(a, row);
  if constexpr (kFollows<op>) wait_for_previous();
  if (here) load_row_late<op>(a, row, in);
  RowSums r = {v[0], 0.0f, 0.0f, 1.0f};
  if constexpr (op != RowOp::kPairGrad) {
#pragma unroll
    for (int j = 1; j < N; ++j) r.m = fmaxf(r.m, v[j]);
    const float ref = usable_max(r.m);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float t = scale_of(a).of(v[j] - ref), e = exp2_fast(t);
      r.s += e;
      r.q = fmaf(e, finite_t(t), r.q);
    }
  }
  RowOut o = {};
  if (here) o = finish_row<op>(a, row, in, r, true);
  __shared__ float buf[kGroupThreads / 32 * kPolicySums];
  bool last = false;
  if constexpr (op == RowOp::kPolicy) last = say_policy_part(a, o, here, 1, buf);
  if constexpr (!kScores<op>) {
    if (here && a.g) {
      E* g = static_cast<E*>(a.g) + row * a.ldg;
#pragma unroll
      for (uint32_t j = 0; j < N; ++j) {
        if (j >= a.vocab) continue;
        float d = in.on ? logit_grad(o, v[j], scale_of(a)) : 0.0f;
        if (in.on && j == in.y) d += o.hit;
        g[j] = from_f32<E>(d);
      }
    }
  }
  if constexpr (op == RowOp::kPolicy) {
    if (!a.sums_behind && __syncthreads_or(last)) policy_stats(a, gridDim.x, buf);
  }
}

// Behind a grid of many blocks: each of these sums up a stretch of the warps'
// parts into its own, the last one those.  1,000,000 rows of 3 (3,907 blocks) 43
// -> 33 us; 655,360 rows (2,560 blocks) 29 -> 27 us, but the launch makes the
// call 33 us on the host: hence the limit.
constexpr uint32_t kMostSaying = 3072, kSumBlocks = 128;

__global__ void __launch_bounds__(kGroupThreads) policy_sum_kernel(const RowArgs a, uint32_t parts) {
  __shared__ float buf[kGroupThreads / 32 * kPolicySums];
  wait_for_previous();
  const uint32_t each = (parts + kSumBlocks - 1) / kSumBlocks, first = min(parts, blockIdx.x * each);
  const float sum = sum_parts(a.partial + (uint64_t)first * kPolicyPart, min(parts, first + each) - first, buf);
  bool last = false;
  float* mine = a.partial + (uint64_t)parts * kPolicyPart;
  if (threadIdx.x < 32) {
    if (threadIdx.x < kPolicySums) mine[blockIdx.x * kPolicyPart + threadIdx.x] = sum;
    last = last_to_say(&a.counts->blocks_done, kSumBlocks);
  }
  if (__syncthreads_or(last)) {
    last_sees();
    const float total = sum_parts(mine, kSumBlocks, buf);
    if (threadIdx.x < 32) put_policy_stats(a, total);
  }
}

// ---- middling rows: 1 to 32 lanes of a warp per row, NV vectors a lane ----
//
// All of a row is read at once and stays in registers; lanes join by shuffles.
// As few lanes as hold the row: what a row costs besides its logits (its loss,
// two exponentials and a logarithm) is paid once per warp, for 32 / lanes rows.
// 65,536 rows of 2,048 bf16, gradient: 101 us, 5.3 TB/s; 200,000 rows of 512 88 us.

template <RowOp op, bool entropy, int NV>
__global__ void __launch_bounds__(kGroupThreads, op == RowOp::kPolicy ? 3 : 4) warp_kernel(const RowArgs a, uint32_t lanes) {
  const uint64_t row = ((uint64_t)blockIdx.x * kGroupThreads + threadIdx.x) / lanes;
  const uint32_t lane = threadIdx.x % lanes;
  const bool here = row < a.rows;
  if constexpr (kFollows<op>) let_next_start();
  RowIn in = {};
  if (here) in = load_row<E, op>(a, row);
  const Window<E> x(const_cast<E*>(static_cast<const E*>(a.x)) + row * a.ldx, a.vocab);
  uint4 u[NV] = {};
  if (in.on) {
    x.load_many(u, lane, lanes, true);
  }
  if constexpr (kFollows<op>) wait_for_previous();
  if (here) load_row_late<op>(a, row, in);
  RowSums r = {};
  if constexpr (op != RowOp::kPairGrad) r = lanes_join(sums_of<NV, kMoment<op, entropy>>(u, scale_of(a)), scale_of(a), lanes);
  RowOut o = {};
  if (here) o = finish_row<op>(a, row, in, r, lane == 0);
  __shared__ float buf[kGroupThreads / 32 * kPolicySums];
  bool last = false;
  if constexpr (op == RowOp::kPolicy) last = say_policy_part(a, o, here && lane == 0, lanes, buf);
  if constexpr (!kScores<op>) {
    if (here && a.g) {
      const Window<E> g(static_cast<E*>(a.g) + row * a.ldg, a.vocab);
      const Grads<entropy> grads(o, scale_of(a));
      put_many(x, g, u, lane, lanes, grads, !in.on);
      if (in.on && in.known && (in.y + x.shift) / kW % lanes == lane)
        g.row[in.y] = from_f32<E>(logit_grad(o, in.xy, scale_of(a)) + o.hit);
    }
  }
  if constexpr (op == RowOp::kPolicy) {
    if (!a.sums_behind && __syncthreads_or(last)) policy_stats(a, gridDim.x, buf);
  }
}

// ---- long rows: a block, or a cluster of blocks, per row ----

constexpr uint32_t kWideThreads = 512;
constexpr uint32_t kMaxCluster = 8;
constexpr int kWideVectors = 8;  // a thread's vectors of a tile
constexpr uint32_t kChunk = 32 * kWideVectors;  // a warp's

__device__ __forceinline__ void cluster_arrive() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Store to the same shared variable of the cluster's block `rank`.
__device__ __forceinline__ void cluster_store(float* p, uint32_t rank, float v) {
  uint32_t here = (uint32_t)__cvta_generic_to_shared(p), there;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(here), "r"(rank));
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there), "f"(v) : "memory");
}

// `cluster` blocks per row, each with `tiles` tiles of kWideVectors vectors a
// thread; the last tile stays in registers between the row's sums and its
// gradient, the others are read again, from L2 as far as the rows on their way fit
// it: two blocks an SM, so 304 rows, 80 MB of 131,072 bf16 (93 % of the second reads
// hit), but 159 MB of 131,072 f32 (44 %: a policy loss of 1,024 rows reads 799 MB from
// memory for 537 MB of logits) and 319 MB of 262,144 f32 (26 %, 910 MB).
// Bound by memory: 8,192 rows of 131,072 bf16, policy loss
// 0.611 ms, 6.2 of 6.67 TB/s measured; 2,048 rows of 32,768 f32, gradient with
// entropies 87 us, 5.9 TB/s; 4,096 rows of 50,001 f16, scores with entropies 60 us,
// 5.4 TB/s (rows at any alignment).
template <RowOp op, bool entropy>
__global__ void __launch_bounds__(kWideThreads, 2) wide_kernel(const RowArgs a, uint32_t cluster, uint32_t tiles) {
  constexpr int NV = kWideVectors;
  constexpr uint32_t kMost = kWideThreads / 32 * kMaxCluster;
  __shared__ float part[4][kMost];  // sums of the row's warps, all blocks'
  const uint64_t row = blockIdx.x / cluster;
  const uint32_t rank = blockIdx.x % cluster, tid = threadIdx.x, threads = blockDim.x;
  if constexpr (kFollows<op>) let_next_start();
  RowIn in = load_row<E, op>(a, row);
  const Window<E> x(const_cast<E*>(static_cast<const E*>(a.x)) + row * a.ldx, a.vocab);
  // A warp's vectors of a tile are neighbours: a row's last ones and what is
  // beyond it fall to few warps, and the others need no test of single vectors
  // (23,439 rows of 16,736 bf16, gradient: 317 -> 287 us; of 16,741 393 -> 336).
  const uint32_t warps = threads / 32, first = (rank * tiles * warps + tid / 32) * kChunk + tid % 32;
  uint4 u[NV];
  RowSums r = {kMinusInf, 0.0f, 0.0f, 0.0f};
  const bool read = in.on;
  if (read) {
    if (cluster > 1 && op != RowOp::kPairGrad) cluster_arrive();  // seen below: the others run
    for (uint32_t tile = 0; tile < tiles; ++tile) {
      if (op == RowOp::kPairGrad && tile + 1 < tiles) continue;
      const uint32_t v = first + tile * warps * kChunk;
      const bool some = v - tid % 32 < x.vectors;  // the same in all of a warp
      if (some) x.load_many(u, v, 32, op == RowOp::kScore || (op != RowOp::kPairScore && tile + 1 == tiles));
      // Only the first blocks find the kernel ahead still running; what it wrote arrives beside the logits.
      if (kFollows<op> && (tile == 0 || op == RowOp::kPairGrad)) {
        wait_for_previous();
        load_row_late<op>(a, row, in);
      }
      if constexpr (op != RowOp::kPairGrad) {
        if (some) {
          const RowSums now = sums_of<NV, kMoment<op, entropy>>(u, scale_of(a));
          r = tile ? join(r, now, scale_of(a)) : now;
        }
      }
    }
    if constexpr (op != RowOp::kPairGrad) {
      r = lanes_join(r, scale_of(a), 32);
      const uint32_t at = rank * warps + tid / 32;
      if (cluster > 1) {
        cluster_wait();
        if (tid % 32 < cluster) {  // a lane per block of the cluster
          cluster_store(&part[0][at], tid % 32, r.m);
          cluster_store(&part[1][at], tid % 32, r.s);
          cluster_store(&part[2][at], tid % 32, r.q);
          cluster_store(&part[3][at], tid % 32, r.one);
        }
        __syncwarp();
        cluster_arrive();
        cluster_wait();
      } else {
        if (tid % 32 == 0) {
          part[0][at] = r.m;
          part[1][at] = r.s;
          part[2][at] = r.q;
          part[3][at] = r.one;
        }
        __syncthreads();
      }
      r = {kMinusInf, 0.0f, 0.0f, 0.0f};
      for (uint32_t w = tid % 32; w < warps * cluster; w += 32) {
        const RowSums other = {part[0][w], part[1][w], part[2][w], part[3][w]};
        r = w < 32 ? other : join(r, other, scale_of(a));
      }
      r = lanes_join(r, scale_of(a), 32);
    }
  }
  if (kFollows<op> && !read) {
    wait_for_previous();
    load_row_late<op>(a, row, in);
  }
  const RowOut o = finish_row<op>(a, row, in, r, rank == 0 && tid == 0);
  bool last = false;
  if constexpr (op == RowOp::kPolicy) {
    if (rank == 0 && tid < 32) {
      if (tid == 0)
        for (uint32_t k = 0; k < kPolicySums; ++k) a.partial[row * kPolicyPart + k] = o.sums[k];
      last = last_to_say(&a.counts->blocks_done, (uint32_t)a.rows);
    }
  }
  if constexpr (!kScores<op>) {
    if (a.g) {
      const Window<E> g(static_cast<E*>(a.g) + row * a.ldg, a.vocab);
      const Grads<entropy> grads(o, scale_of(a));
      for (uint32_t tile = tiles; tile-- > 0;) {
        const uint32_t v = first + tile * warps * kChunk;
        if (v - tid % 32 >= x.vectors) continue;
        if (in.on && tile + 1 < tiles) x.load_many(u, v, 32, true);
        put_many(x, g, u, v, 32, grads, !in.on);
      }
      if (in.on) {
        const uint32_t at = (in.y + x.shift) / kW, chunk = at / kChunk - rank * tiles * warps;  // the vector with the token
        if (in.known && chunk < tiles * warps && chunk % warps == tid / 32 && at % 32 == tid % 32)
          g.row[in.y] = from_f32<E>(logit_grad(o, in.xy, scale_of(a)) + o.hit);
      }
    }
  }
  if constexpr (op == RowOp::kPolicy) {
    __shared__ float sums[kWideThreads / 32 * kPolicySums];
    if (rank == 0 && __syncthreads_or(last)) policy_stats(a, a.rows, sums);
  }
}

// ---- few rows of short answers: a loss in one launch, by one cluster ----

// Up to 8 blocks hold all rows in registers, as the warp kernel does, from
// their sums to their gradient; each block counts the sequences' scored rows for
// itself, and the blocks meet at cluster barriers instead of kernel ends.  Where
// it fits, it takes one launch instead of two (policy) or four (preference):
// 4 pairs, 130 rows of 1,009 f16, 12.6 us against 14.3 and 26 against 33 us on the
// host; 64 mappings, 1,024 rows of 3, 9.4 us against 8.5 and 24 against 26 us on
// the host.  From 2,000 rows on the blocks' counting loses (4,096 rows of 3 14.4
// against 12.4 us).
constexpr uint32_t kFewThreads = 512, kFewSequences = 1024, kFewRows = 1024;

struct FewShape {
  uint32_t sequences, lanes, cluster;
};

template <bool pairs, bool entropy, int NV>
__global__ void __launch_bounds__(kFewThreads, 1) few_kernel(const RowArgs a, const PairArgs p, const int64_t* offsets,
                                                             const FewShape f) {
  constexpr uint32_t kWarps = kFewThreads / 32;
  __shared__ uint32_t begin[kFewSequences + 1], count[kFewSequences];
  __shared__ uint32_t all, used;
  __shared__ float buf[kWarps * kPolicySums], part[kMaxCluster * kPolicySums];
  const uint32_t rank = blockIdx.x, tid = threadIdx.x, rows = (uint32_t)a.rows;
  const uint32_t row = (rank * kFewThreads + tid) / f.lanes, lane = tid % f.lanes;
  const bool here = row < rows;
  cluster_arrive();
  RowIn in = {};
  if (here) in = load_row<E, pairs ? RowOp::kPairScore : RowOp::kPolicy>(a, row);
  const Window<E> x(const_cast<E*>(static_cast<const E*>(a.x)) + row * a.ldx, a.vocab);
  uint4 u[NV] = {};
  if (in.on) {
    x.load_many(u, lane, f.lanes, true);
  }
  if (tid == 0) all = used = 0;
  for (uint32_t s = tid; s <= f.sequences; s += kFewThreads) {
    begin[s] = clamp_offset(offsets[s], rows);
    if (s < f.sequences) count[s] = 0;
  }
  __syncthreads();
  for (uint32_t first = 0; first < rows; first += kFewThreads) {
    const uint32_t r = first + tid;
    const uint32_t seq = r < rows && a.tokens[r] >= 0 ? sequence_at(begin, f.sequences, r) : kNoSequence;
    const uint32_t same = __match_any_sync(~0u, seq), n = (uint32_t)__popc(same);
    if (seq != kNoSequence && tid % 32 == (uint32_t)__ffs(same) - 1) {
      atomicAdd(&all, n);
      if (atomicAdd(&count[seq], n) == 0) atomicAdd(&used, 1u);
    }
  }
  const uint32_t seq = in.on ? sequence_at(begin, f.sequences, row) : kNoSequence;
  in.on = seq != kNoSequence;
  const RowSums r = lanes_join(sums_of<NV, !pairs || entropy>(u, scale_of(a)), scale_of(a), f.lanes);
  __syncthreads();
  RowOut o = {};
  if constexpr (pairs) {
    if (here) finish_row<RowOp::kScore>(a, row, in, r, lane == 0);
    cluster_wait();
    cluster_arrive();  // the rows' log-probabilities are written
    cluster_wait();
    for (uint32_t pair = rank * kWarps + tid / 32; pair < (uint32_t)p.pairs; pair += f.cluster * kWarps) {
      float sum[2] = {0.0f, 0.0f};
#pragma unroll
      for (uint32_t k = 0; k < 2; ++k) {
        for (uint32_t i = begin[2 * pair + k] + tid % 32; i < begin[2 * pair + k + 1]; i += 32)
          if (a.tokens[i] >= 0) sum[k] += __ldcg(a.logprob + i) - (p.ref_logprob ? p.ref_logprob[i] : 0.0f);
#pragma unroll
        for (int d = 16; d; d /= 2) sum[k] += __shfl_xor_sync(~0u, sum[k], d);
      }
      const uint32_t n[2] = {count[2 * pair], count[2 * pair + 1]};
      if (tid % 32 == 0) finish_pair(p, pair, sum, n);
    }
    cluster_arrive();  // the pairs' slopes are written
    cluster_wait();
    if (rank == 0) preference_stats(p, buf);
    if (here && a.g) {
      if (in.on) in.slope_lp = __ldcg(p.seq_slope + seq);
      o = finish_row<RowOp::kScoreGrad>(a, row, in, r, false);
    }
  } else {
    if (in.on) {
      in.w = a.reduction == BF_MEAN_TOKENS ? 1.0f / (float)all
             : a.reduction == BF_MEAN_SEQUENCES ? 1.0f / ((float)count[seq] * (float)used) : 1.0f;
      if (!a.advantage_per_token) in.adv = a.advantage[seq];
    }
    if (here) o = finish_row<RowOp::kPolicy>(a, row, in, r, lane == 0);
    float v[kPolicySums];
#pragma unroll
    for (uint32_t k = 0; k < kPolicySums; ++k) v[k] = lane == 0 ? o.sums[k] : 0.0f;
    const float sum = block_sums(v, buf, f.lanes);
    cluster_wait();
    if (tid < kPolicySums) cluster_store(&part[rank * kPolicySums + tid], 0, sum);
    cluster_arrive();
  }
  if (here && a.g) {
    const Window<E> g(static_cast<E*>(a.g) + row * a.ldg, a.vocab);
    const Grads<entropy> grads(o, scale_of(a));
    put_many(x, g, u, lane, f.lanes, grads, !in.on);
    if (in.on && in.known && (in.y + x.shift) / kW % f.lanes == lane)
      g.row[in.y] = from_f32<E>(logit_grad(o, in.xy, scale_of(a)) + o.hit);
  }
  if constexpr (!pairs) {
    cluster_wait();  // the blocks' sums are in the first one
    if (rank == 0 && tid < 32) {
      float total = 0.0f;
      if (tid < kPolicySums)
        for (uint32_t b = 0; b < f.cluster; ++b) total += part[b * kPolicySums + tid];
      put_policy_stats(a, total);
    }
  }
}

struct WideShape {
  uint32_t cluster, threads, tiles;
};

uint32_t div_up(uint32_t a, uint32_t b) { return (a + b - 1) / b; }

// A cluster only where there are few rows (131,072 bf16 columns, gradient, 1 / 2 /
// 4 / 8 blocks a row: 20 rows 18.6 / 12.4 / 11.3 / 10.4 us, 80 rows 20.4 / 18.4 /
// 14.8 / 14.4, 300 rows 35.9 / 36.8 / 41.2 / 39.5): its blocks have to start together.
// Scores read their rows once: 128 threads, with many rows beside each other
// (4,096 rows of 50,001 f16: 128 / 256 / 512 threads 62 / 66 / 80 us).  A gradient
// reads its row again from L2, so fewer rows at a time: two tiles a thread, up to 512
// threads (2,048 rows of 32,768 f32: 128 / 256 / 512 threads 112 / 96 / 90 us; 8,192 rows
// of 131,072 bf16 920 / 803 / 738 us).  The rule goes by the operation: a policy loss
// without its gradient keeps the gradient's shape (those rows 427 us, their scores 315 us).
WideShape wide_shape(uint64_t rows, uint32_t vectors, bool scores) {
  WideShape s = {1, 0, 1};
  while (s.cluster < kMaxCluster && rows * s.cluster <= 400 && div_up(vectors, s.cluster) > 256) s.cluster *= 2;
  const uint32_t lanes = div_up(div_up(vectors, s.cluster), kWideVectors);
  const uint32_t most = scores ? 128 : lanes / 2 < 128 ? 128 : lanes / 2 < kWideThreads ? div_up(lanes / 2, 32) * 32 : kWideThreads;
  s.tiles = div_up(lanes, most);
  s.threads = div_up(div_up(lanes, s.tiles), 32) * 32;
  return s;
}

uint32_t pow2_up(uint32_t n) {
  uint32_t p = 1;
  while (p < n) p *= 2;
  return p;
}

// Vectors that a row touches: one more where rows may start inside one.
uint32_t vectors_of(const RowArgs& a) {
  const bool aligned = ((uintptr_t)a.x | (uintptr_t)(a.ldx * sizeof(E))) % 16 == 0;
  return div_up(a.vocab + (aligned ? 0 : kW - 1), kW);
}

template <RowOp op, bool entropy>
cudaError_t launch_op(const RowArgs& a, cudaStream_t st) {
  const auto group = [&](auto kernel, uint32_t lanes) {
    const uint64_t blocks = (a.rows * lanes + kGroupThreads - 1) / kGroupThreads;
    RowArgs b = a;
    b.sums_behind = op == RowOp::kPolicy && blocks > kMostSaying;
    const cudaError_t e = launch_shaped(kernel, blocks, kGroupThreads, 1, kFollows<op>, st, b, lanes);
    if (e != cudaSuccess || !b.sums_behind) return e;
    return launch_after(policy_sum_kernel, kSumBlocks, kGroupThreads, st, b, (uint32_t)blocks * (kGroupThreads / 32));
  };
  const uint32_t vectors = vectors_of(a);
  // Vectors a lane, then lanes: 655,360 rows of 16 bf16 (2 vectors) 45 us with 2,
  // 50 with 4; 400,000 of 64 (8 vectors) 56 us with 2 lanes of 4, 66 with 1 of 8;
  // 200,000 of 512 (64 vectors) 119 us with 8 lanes of 8, 169 with 16 of 4, 283 with
  // 32 of 2; policy losses.  Up to 4 KB a row: 131,072 rows of 1,024 bf16 123 us here,
  // 195 with a block a row; 65,536 of 2,048 105 against 111.  Their bytes alone take 9, 17,
  // 62, 81 and 81 us: the shorter the rows, the more the loss's arithmetic and values of
  // each row weigh.
  if (a.vocab <= 4) return group(short_kernel<op, 4>, 1);
  if (vectors <= 2) return group(warp_kernel<op, entropy, 2>, 1);
  if (vectors <= 8) return group(warp_kernel<op, entropy, 4>, pow2_up(div_up(vectors, 4)));
  if (vectors <= 256) return group(warp_kernel<op, entropy, 8>, pow2_up(div_up(vectors, 8)));
  const WideShape s = wide_shape(a.rows, vectors, kScores<op>);
  return launch_shaped(wide_kernel<op, entropy>, a.rows * s.cluster, s.threads, s.cluster, kFollows<op>, st, a, s.cluster,
                       s.tiles);
}

template <bool pairs, bool entropy>
cudaError_t launch_few(const RowArgs& a, const PairArgs& p, const int64_t* offsets, FewShape f, bool two, cudaStream_t st) {
  const auto kernel = two ? few_kernel<pairs, entropy, 2> : few_kernel<pairs, entropy, 8>;
  return launch_shaped(kernel, f.cluster, kFewThreads, f.cluster, false, st, a, p, offsets, f);
}

}  // namespace

#define BF_ROWS_JOIN2(name, t) name##t
#define BF_ROWS_JOIN(name, t) BF_ROWS_JOIN2(name, t)
#define BF_ROWS_NAME(name) BF_ROWS_JOIN(name, BF_ROWS_TYPE)

cudaError_t BF_ROWS_NAME(launch_few_type)(const RowArgs& a, const PairArgs* p, const int64_t* offsets, uint64_t sequences,
                                          bool* done, cudaStream_t st) {
  const uint32_t vectors = vectors_of(a);
  FewShape f = {};
  *done = false;
  if (vectors > 256 || a.rows > kFewRows || sequences > kFewSequences) return cudaSuccess;
  f.lanes = vectors <= 2 ? 1 : pow2_up(div_up(vectors, 8));
  f.sequences = (uint32_t)sequences;
  const uint32_t blocks = div_up((uint32_t)a.rows * f.lanes, kFewThreads);
  if (blocks > kMaxCluster) return cudaSuccess;
  f.cluster = pow2_up(blocks);
  *done = true;
  const bool two = vectors <= 2;
  if (p) return launch_few<true, false>(a, *p, offsets, f, two, st);
  return a.entropy_coef != 0.0f ? launch_few<false, true>(a, PairArgs{}, offsets, f, two, st)
                                : launch_few<false, false>(a, PairArgs{}, offsets, f, two, st);
}

cudaError_t BF_ROWS_NAME(launch_rows_type)(RowOp op, const RowArgs& a, cudaStream_t st) {
  switch (op) {
    case RowOp::kScore: return a.entropy ? launch_op<RowOp::kScore, true>(a, st) : launch_op<RowOp::kScore, false>(a, st);
    case RowOp::kScoreGrad:
      return a.grad_entropy ? launch_op<RowOp::kScoreGrad, true>(a, st) : launch_op<RowOp::kScoreGrad, false>(a, st);
    case RowOp::kPolicy:
      return a.entropy_coef != 0.0f ? launch_op<RowOp::kPolicy, true>(a, st) : launch_op<RowOp::kPolicy, false>(a, st);
    case RowOp::kPairScore: return launch_op<RowOp::kPairScore, false>(a, st);
    default: return launch_op<RowOp::kPairGrad, false>(a, st);
  }
}

}  // namespace bfk
