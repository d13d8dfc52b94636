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

template <RowOp op>
constexpr bool kScores = op == RowOp::kScore || op == RowOp::kPairScore;

// The policy loss from its parts' sums, in an order that does not depend on when blocks ran.
__device__ __forceinline__ void policy_stats(const RowArgs& a, uint64_t parts, float* buf) {
  float total[kPolicySums];
  for (uint32_t k = 0; k < kPolicySums; ++k) {
    float v = 0.0f;
    for (uint64_t i = threadIdx.x; i < parts; i += blockDim.x) v += __ldcg(a.partial + k * parts + i);
    total[k] = block_sum(v, buf);
  }
  if (threadIdx.x == 0) {
    a.stats[0] = -total[0] + a.kl_coef * total[1] - a.entropy_coef * total[2];
    a.stats[1] = -total[0];
    for (uint32_t k = 1; k < kPolicySums; ++k) a.stats[k + 1] = total[k];
  }
}

// Sums of N values against their own maximum.
template <int N>
__device__ __forceinline__ RowSums sums_of(const float* x, float c2) {
  RowSums r = {x[0], 0.0f, 0.0f};
#pragma unroll
  for (int i = 1; i < N; ++i) r.m = fmaxf(r.m, x[i]);
  const float ref = usable_max(r.m);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float t = (x[i] - ref) * c2, e = exp2_fast(t);
    r.s += e;
    r.q = fmaf(e, finite_t(t), r.q);
  }
  return r;
}

// NV vectors in registers: their sums against their own maximum.
template <int NV>
__device__ __forceinline__ RowSums sums_of(const uint4* u, float c2) {
  RowSums r = {kMinusInf, 0.0f, 0.0f};
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    float x[kW];
    unpack<E>(u[k], x);
#pragma unroll
    for (uint32_t i = 0; i < kW; ++i) r.m = fmaxf(r.m, x[i]);
  }
  const float ref = usable_max(r.m);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    float x[kW];
    unpack<E>(u[k], x);
#pragma unroll
    for (uint32_t i = 0; i < kW; ++i) {
      const float t = (x[i] - ref) * c2, e = exp2_fast(t);
      r.s += e;
      r.q = fmaf(e, finite_t(t), r.q);
    }
  }
  return r;
}

template <int NV>
__device__ __forceinline__ void grad_of(const uint4& u, const RowOut& o, float c2, float* g) {
  float x[kW];
  unpack<E>(u, x);
#pragma unroll
  for (uint32_t i = 0; i < kW; ++i) g[i] = logit_grad(o, x[i], c2);
}

// ---- short rows: 1 to 32 lanes of a warp per row, kShort elements a lane ----

constexpr uint32_t kGroupThreads = 256;
constexpr uint32_t kShort = 4;

// The block's part of the policy loss, once its rows are done.
__device__ __forceinline__ void put_policy_block(const RowArgs& a, const RowOut& o, bool mine) {
  __shared__ float buf[kGroupThreads / 32];
  for (uint32_t k = 0; k < kPolicySums; ++k) {
    const float v = block_sum(mine ? o.sums[k] : 0.0f, buf);
    if (threadIdx.x == 0) a.partial[(uint64_t)k * gridDim.x + blockIdx.x] = v;
  }
  if (last_block(&a.counts->blocks_done, gridDim.x)) policy_stats(a, gridDim.x, buf);
}

template <RowOp op>
__global__ void __launch_bounds__(kGroupThreads) short_kernel(const RowArgs a, uint32_t lanes) {
  const uint64_t row = ((uint64_t)blockIdx.x * kGroupThreads + threadIdx.x) / lanes;
  const uint32_t lane = threadIdx.x % lanes;
  const bool here = row < a.rows;
  RowIn in = {};
  if (here) in = load_row<E, op>(a, row);
  const E* x = static_cast<const E*>(a.x) + row * a.ldx;
  float v[kShort];
#pragma unroll
  for (uint32_t i = 0; i < kShort; ++i) {
    const uint32_t j = lane + i * lanes;
    v[i] = in.on && j < a.vocab ? to_f32(x[j]) : kMinusInf;
  }
  RowSums r = {};
  if constexpr (op != RowOp::kPairGrad) r = lanes_join(sums_of<kShort>(v, a.c2), a.c2, lanes);
  RowOut o = {};
  if (here) o = finish_row<op>(a, row, in, r, lane == 0);
  if constexpr (!kScores<op>) {
    if (here && a.g) {
      E* g = static_cast<E*>(a.g) + row * a.ldg;
#pragma unroll
      for (uint32_t i = 0; i < kShort; ++i) {
        const uint32_t j = lane + i * lanes;
        if (j >= a.vocab) continue;
        float d = in.on ? logit_grad(o, v[i], a.c2) : 0.0f;
        if (in.on && j == in.y) d += o.hit;
        g[j] = from_f32<E>(d);
      }
    }
  }
  if constexpr (op == RowOp::kPolicy) put_policy_block(a, o, here && lane == 0);
}

// ---- middling rows: 8 to 32 lanes of a warp per row, NV vectors a lane ----

template <RowOp op, int NV>
__global__ void __launch_bounds__(kGroupThreads) warp_kernel(const RowArgs a, uint32_t lanes) {
  const uint64_t row = ((uint64_t)blockIdx.x * kGroupThreads + threadIdx.x) / lanes;
  const uint32_t lane = threadIdx.x % lanes;
  const bool here = row < a.rows;
  RowIn in = {};
  if (here) in = load_row<E, op>(a, row);
  const Window<E> x(const_cast<E*>(static_cast<const E*>(a.x)) + row * a.ldx, in.on ? a.vocab : 0);
  uint4 u[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) u[k] = x.load(lane + k * lanes);
  RowSums r = {};
  if constexpr (op != RowOp::kPairGrad) r = lanes_join(sums_of<NV>(u, a.c2), a.c2, lanes);
  RowOut o = {};
  if (here) o = finish_row<op>(a, row, in, r, lane == 0);
  if constexpr (!kScores<op>) {
    if (here && a.g) {
      const Window<E> g(static_cast<E*>(a.g) + row * a.ldg, a.vocab);
      const uint32_t shift = in.on ? x.shift : g.shift;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        float d[kW] = {};
        if (in.on) grad_of<NV>(u[k], o, a.c2, d);
        if (shift == g.shift) g.store(lane + k * lanes, d);
        else g.store_cut(lane + k * lanes, shift, d);
      }
      if (in.on && in.known && (in.y + shift) / kW % lanes == lane)
        g.row[in.y] = from_f32<E>(logit_grad(o, in.xy, a.c2) + o.hit);
    }
  }
  if constexpr (op == RowOp::kPolicy) put_policy_block(a, o, here && lane == 0);
}

// ---- long rows: a block, or a cluster of blocks, per row ----

constexpr uint32_t kWideThreads = 512;
constexpr uint32_t kMaxCluster = 8;

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// Store to the same shared variable of the cluster's block `rank`.
__device__ __forceinline__ void cluster_store(float* p, uint32_t rank, float v) {
  uint32_t here = (uint32_t)__cvta_generic_to_shared(p), there;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(here), "r"(rank));
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there), "f"(v) : "memory");
}

// `cluster` blocks per row, each with `tiles` tiles of NV vectors a thread;
// the last tile stays in registers between the row's sums and its gradient.
template <RowOp op, int NV>
__global__ void __launch_bounds__(kWideThreads, 2) wide_kernel(const RowArgs a, uint32_t cluster, uint32_t tiles) {
  constexpr uint32_t kMost = kWideThreads / 32 * kMaxCluster;
  __shared__ float part[3][kMost];  // sums of the row's warps, all blocks'
  const uint64_t row = blockIdx.x / cluster;
  const uint32_t rank = blockIdx.x % cluster, tid = threadIdx.x, threads = blockDim.x;
  const RowIn in = load_row<E, op>(a, row);
  const Window<E> x(const_cast<E*>(static_cast<const E*>(a.x)) + row * a.ldx, a.vocab);
  const uint32_t first = rank * tiles * NV * threads + tid;
  uint4 u[NV];
  RowOut o = {};
  if (in.on) {
    if (cluster > 1 && op != RowOp::kPairGrad) cluster_arrive();  // seen below: the others run
    RowSums r = {kMinusInf, 0.0f, 0.0f};
    for (uint32_t tile = 0; tile < tiles; ++tile) {
      if (op == RowOp::kPairGrad && tile + 1 < tiles) continue;
#pragma unroll
      for (int k = 0; k < NV; ++k) u[k] = x.load(first + (tile * NV + k) * threads);
      if constexpr (op != RowOp::kPairGrad) {
        const RowSums now = sums_of<NV>(u, a.c2);
        r = tiles > 1 ? join(r, now, a.c2) : now;
      }
    }
    if constexpr (op != RowOp::kPairGrad) {
      r = lanes_join(r, a.c2, 32);
      const uint32_t warps = threads / 32, at = rank * warps + tid / 32;
      if (cluster > 1) {
        cluster_wait();
        if (tid % 32 < cluster) {  // a lane per block of the cluster
          cluster_store(&part[0][at], tid % 32, r.m);
          cluster_store(&part[1][at], tid % 32, r.s);
          cluster_store(&part[2][at], tid % 32, r.q);
        }
        __syncwarp();
        cluster_arrive();
        cluster_wait();
      } else {
        if (tid % 32 == 0) {
          part[0][at] = r.m;
          part[1][at] = r.s;
          part[2][at] = r.q;
        }
        __syncthreads();
      }
      r = {kMinusInf, 0.0f, 0.0f};
      for (uint32_t w = tid % 32; w < warps * cluster; w += 32) {
        const RowSums other = {part[0][w], part[1][w], part[2][w]};
        r = w < 32 ? other : join(r, other, a.c2);
      }
      r = lanes_join(r, a.c2, 32);
    }
    o = finish_row<op>(a, row, in, r, rank == 0 && tid == 0);
  } else {
    o = finish_row<op>(a, row, in, {}, rank == 0 && tid == 0);
  }
  if constexpr (op == RowOp::kPolicy) {
    if (rank == 0 && tid == 0)
      for (uint32_t k = 0; k < kPolicySums; ++k) a.partial[k * a.rows + row] = o.sums[k];
  }
  if constexpr (!kScores<op>) {
    if (a.g) {
      const Window<E> g(static_cast<E*>(a.g) + row * a.ldg, a.vocab);
      if (!in.on) {
        const float zero[kW] = {};
        for (uint32_t k = 0; k < NV * tiles; ++k) g.store(first + k * threads, zero);
      } else {
        for (uint32_t tile = tiles; tile-- > 0;) {
          if (tile + 1 < tiles) {
#pragma unroll
            for (int k = 0; k < NV; ++k) u[k] = x.load(first + (tile * NV + k) * threads);
          }
#pragma unroll
          for (int k = 0; k < NV; ++k) {
            const uint32_t v = first + (tile * NV + k) * threads;
            float d[kW];
            grad_of<NV>(u[k], o, a.c2, d);
            if (x.shift == g.shift) g.store(v, d);
            else g.store_cut(v, x.shift, d);
          }
        }
        const uint32_t at = (in.y + x.shift) / kW - rank * tiles * NV * threads;  // the vector with the token
        if (in.known && at < tiles * NV * threads && at % threads == tid)
          g.row[in.y] = from_f32<E>(logit_grad(o, in.xy, a.c2) + o.hit);
      }
    }
  }
  if constexpr (op == RowOp::kPolicy) {
    __shared__ float sums[kWideThreads / 32];
    if (rank == 0 && last_block(&a.counts->blocks_done, (uint32_t)a.rows)) policy_stats(a, a.rows, sums);
  }
}

struct WideShape {
  uint32_t cluster, threads, vectors, tiles;
};

uint32_t div_up(uint32_t a, uint32_t b) { return (a + b - 1) / b; }

WideShape wide_shape(uint64_t rows, uint32_t vectors) {
  WideShape s = {1, 0, 8, 1};
  while (s.cluster < kMaxCluster && div_up(vectors, s.cluster) > 256 * 8) s.cluster *= 2;
  while (s.cluster < kMaxCluster && rows * s.cluster < 304 && div_up(vectors, s.cluster) > 256) s.cluster *= 2;
  const uint32_t each = div_up(vectors, s.cluster);
  s.vectors = each <= 256 * 2 ? 2 : each <= 256 * 4 ? 4 : 8;
  const uint32_t lanes = div_up(each, s.vectors);
  s.tiles = div_up(lanes, kWideThreads);
  s.threads = div_up(div_up(lanes, s.tiles), 32) * 32;
  return s;
}

template <RowOp op, int NV>
cudaError_t launch_wide(const RowArgs& a, const WideShape& s, cudaStream_t st) {
  if (a.rows > 0x7FFFFFFFu / s.cluster) return cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((uint32_t)a.rows * s.cluster);
  cfg.blockDim = dim3(s.threads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = s.cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = s.cluster > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, wide_kernel<op, NV>, a, s.cluster, s.tiles);
}

template <RowOp op>
cudaError_t launch_op(const RowArgs& a, cudaStream_t st) {
  const auto blocks = [&](uint32_t lanes) { return (uint32_t)((a.rows * lanes + kGroupThreads - 1) / kGroupThreads); };
  if (a.vocab <= 32 * kShort) {
    uint32_t lanes = 1;
    while (lanes * kShort < a.vocab) lanes *= 2;
    short_kernel<op><<<blocks(lanes), kGroupThreads, 0, st>>>(a, lanes);
    return cudaGetLastError();
  }
  const uint32_t vectors = div_up(a.vocab + kW - 1, kW);  // at the worst alignment
  if (vectors <= 128) {
    uint32_t lanes = 8;
    while (lanes < 32 && lanes < vectors) lanes *= 2;
    if (vectors <= lanes) warp_kernel<op, 1><<<blocks(lanes), kGroupThreads, 0, st>>>(a, lanes);
    else if (vectors <= 64) warp_kernel<op, 2><<<blocks(lanes), kGroupThreads, 0, st>>>(a, lanes);
    else warp_kernel<op, 4><<<blocks(lanes), kGroupThreads, 0, st>>>(a, lanes);
    return cudaGetLastError();
  }
  const WideShape s = wide_shape(a.rows, vectors);
  switch (s.vectors) {
    case 2: return launch_wide<op, 2>(a, s, st);
    case 4: return launch_wide<op, 4>(a, s, st);
    default: return launch_wide<op, 8>(a, s, st);
  }
}

}  // namespace

#define BF_ROWS_NAME2(t) launch_rows_type##t
#define BF_ROWS_NAME(t) BF_ROWS_NAME2(t)
cudaError_t BF_ROWS_NAME(BF_ROWS_TYPE)(RowOp op, const RowArgs& a, cudaStream_t st) {
  switch (op) {
    case RowOp::kScore: return launch_op<RowOp::kScore>(a, st);
    case RowOp::kScoreGrad: return launch_op<RowOp::kScoreGrad>(a, st);
    case RowOp::kPolicy: return launch_op<RowOp::kPolicy>(a, st);
    case RowOp::kPairScore: return launch_op<RowOp::kPairScore>(a, st);
    default: return launch_op<RowOp::kPairGrad>(a, st);
  }
}

}  // namespace bfk
