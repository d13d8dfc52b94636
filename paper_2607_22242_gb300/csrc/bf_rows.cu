// bf_rows.cu -- passes over rows of logits: token log-probabilities and
// entropies, their gradient, the clipped policy loss and the preference loss
// (arithmetic in bf_rows.cuh).
#include "bf_rows.cuh"

namespace bfk {

namespace {

constexpr uint32_t kRowThreads = 256;

__device__ __forceinline__ RowSums warp_join(RowSums r, float c2) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const RowSums other = {__shfl_xor_sync(~0u, r.m, o), __shfl_xor_sync(~0u, r.s, o), __shfl_xor_sync(~0u, r.q, o)};
    r = join(r, other, c2);
  }
  return r;
}

// The row's sums from every thread's part, in all threads; buf holds a RowSums per warp.
__device__ __forceinline__ RowSums block_join(RowSums r, float c2, RowSums* buf) {
  r = warp_join(r, c2);
  const uint32_t warps = blockDim.x / 32;
  __syncthreads();
  if (threadIdx.x % 32 == 0) buf[threadIdx.x / 32] = r;
  __syncthreads();
  r = buf[0];
  for (uint32_t w = 1; w < warps; ++w) r = join(r, buf[w], c2);
  return r;
}

// Sum over the block's threads, in thread 0; every thread of the block calls it.
__device__ __forceinline__ float block_sum(float v, float* buf) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  __syncthreads();
  if (threadIdx.x % 32 == 0) buf[threadIdx.x / 32] = v;
  __syncthreads();
  float sum = 0.0f;
  if (threadIdx.x == 0)
    for (uint32_t w = 0; w < blockDim.x / 32; ++w) sum += buf[w];
  return sum;
}

// Whether this block is the last of the grid to get here; what the others wrote before is then visible.
__device__ __forceinline__ bool last_block(RowCounts* counts) {
  __shared__ bool last;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(&counts->blocks_done, 1u) == gridDim.x - 1;
  __syncthreads();
  if (last) __threadfence();
  return last;
}

// The policy loss from its rows' sums, in an order that does not depend on when blocks ran.
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

// One block per row: a pass for the row's sums, a second one for its gradient.
template <typename E, RowOp op>
__global__ void __launch_bounds__(kRowThreads) row_kernel(const RowArgs a) {
  __shared__ RowSums buf[kRowThreads / 32];
  for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const RowIn in = load_row<E, op>(a, row);
    const E* x = static_cast<const E*>(a.x) + row * a.ldx;
    RowSums r = {kMinusInf, 0.0f, 0.0f};
    if (in.on) {
      for (uint32_t j = threadIdx.x; j < a.vocab; j += blockDim.x) {
        const float v = to_f32(x[j]);
        if (v > r.m) {
          const float t = (r.m - v) * a.c2, e = exp2_fast(t);
          r = {v, e * r.s, e * (r.q + finite_t(t) * r.s)};
        }
        const float t = (v - usable_max(r.m)) * a.c2, e = exp2_fast(t);
        r.s += e;
        r.q += e * finite_t(t);
      }
      r = block_join(r, a.c2, buf);
    }
    const RowOut o = finish_row<op>(a, row, in, r, threadIdx.x == 0);
    if constexpr (op == RowOp::kPolicy) {
      if (threadIdx.x == 0)
        for (uint32_t k = 0; k < kPolicySums; ++k) a.partial[k * a.rows + row] = o.sums[k];
    }
    if constexpr (op != RowOp::kScore && op != RowOp::kPairScore) {
      if (a.g) {
        E* g = static_cast<E*>(a.g) + row * a.ldg;
        for (uint32_t j = threadIdx.x; j < a.vocab; j += blockDim.x) {
          float v = 0.0f;
          if (in.on) {
            v = logit_grad(o, to_f32(x[j]), a.c2);
            if (j == in.y) v += o.hit;
          }
          g[j] = from_f32<E>(v);
        }
      }
    }
  }
  if constexpr (op == RowOp::kPolicy) {
    __shared__ float sums[kRowThreads / 32];
    if (last_block(a.counts)) policy_stats(a, a.rows, sums);
  }
}

template <typename E>
cudaError_t launch_typed(RowOp op, const RowArgs& a, cudaStream_t st) {
  const uint32_t grid = (uint32_t)(a.rows < (1u << 30) ? a.rows : (1u << 30));
  switch (op) {
    case RowOp::kScore: row_kernel<E, RowOp::kScore><<<grid, kRowThreads, 0, st>>>(a); break;
    case RowOp::kScoreGrad: row_kernel<E, RowOp::kScoreGrad><<<grid, kRowThreads, 0, st>>>(a); break;
    case RowOp::kPolicy: row_kernel<E, RowOp::kPolicy><<<grid, kRowThreads, 0, st>>>(a); break;
    case RowOp::kPairScore: row_kernel<E, RowOp::kPairScore><<<grid, kRowThreads, 0, st>>>(a); break;
    case RowOp::kPairGrad: row_kernel<E, RowOp::kPairGrad><<<grid, kRowThreads, 0, st>>>(a); break;
  }
  return cudaGetLastError();
}

// The sequence whose rows [offsets[s], offsets[s+1]) contain `row`, or
// kNoSequence.  Offsets that do not ascend make rows miss their sequence; no
// read leaves the array.
__device__ __forceinline__ uint32_t sequence_of(uint64_t row, const int64_t* offsets, uint64_t sequences) {
  uint64_t lo = 0, hi = sequences;  // the last s with offsets[s] <= row lies in [lo, hi)
  while (hi - lo > 1) {
    const uint64_t mid = (lo + hi) / 2;
    if (offsets[mid] <= (int64_t)row) lo = mid;
    else hi = mid;
  }
  return offsets[lo] <= (int64_t)row && (int64_t)row < offsets[lo + 1] ? (uint32_t)lo : kNoSequence;
}

// Counts are sums of whole numbers: their order does not matter.
__global__ void __launch_bounds__(kRowThreads) sequence_kernel(const int64_t* tokens, uint64_t rows,
                                                               const int64_t* offsets, uint64_t sequences,
                                                               uint32_t* row_seq, uint32_t* seq_tokens,
                                                               RowCounts* counts) {
  const uint64_t row = (uint64_t)blockIdx.x * kRowThreads + threadIdx.x;
  uint32_t seq = kNoSequence;
  if (row < rows) {
    if (sequences && tokens[row] >= 0) seq = sequence_of(row, offsets, sequences);
    row_seq[row] = seq;
  }
  const uint32_t same = __match_any_sync(~0u, seq), scored = __ballot_sync(~0u, seq != kNoSequence);
  const uint32_t lane = threadIdx.x % 32;
  if (seq != kNoSequence && lane == (uint32_t)__ffs(same) - 1) {
    if (atomicAdd(&seq_tokens[seq], (uint32_t)__popc(same)) == 0u) atomicAdd(&counts->sequences, 1u);
  }
  if (lane == 0 && scored) atomicAdd(&counts->tokens, (uint32_t)__popc(scored));
}

// One block per pair: the rewards beta * sum (lp - ref) of both answers (or of
// their means), the loss of their gap
//   h = reward_0 - reward_1 - margin,  l = -(1 - eps) ln sigma(h) - eps ln sigma(-h)
// and the slopes of the mean loss in each answer's log-probabilities.
__global__ void __launch_bounds__(kRowThreads) pair_kernel(const PairArgs a) {
  __shared__ float buf[kRowThreads / 32];
  for (uint64_t p = blockIdx.x; p < a.pairs; p += gridDim.x) {
    float sum[2];
    for (uint32_t k = 0; k < 2; ++k) {
      const uint64_t seq = 2 * p + k;
      const int64_t lo = a.offsets[seq], hi = a.offsets[seq + 1];
      const uint64_t begin = lo > 0 ? (uint64_t)lo : 0, end = hi > 0 ? min((uint64_t)hi, a.rows) : 0;
      float v = 0.0f;
      for (uint64_t row = begin + threadIdx.x; row < end; row += kRowThreads)
        if (a.row_seq[row] == (uint32_t)seq) v += a.logprob[row] - (a.ref_logprob ? a.ref_logprob[row] : 0.0f);
      sum[k] = block_sum(v, buf);
    }
    if (threadIdx.x == 0) {
      float share[2], reward[2];
      for (uint32_t k = 0; k < 2; ++k) {
        const uint32_t n = a.seq_tokens[2 * p + k];
        share[k] = a.beta * (a.average && n ? 1.0f / (float)n : 1.0f);
        reward[k] = share[k] * sum[k];
        a.rewards[2 * p + k] = reward[k];
      }
      const float h = reward[0] - reward[1] - a.margin, eps = a.label_smoothing;
      const float tail = log1pf(expf(-fabsf(h)));  // ln(1 + e^-|h|)
      const float loss = (1.0f - eps) * (fmaxf(-h, 0.0f) + tail) + eps * (fmaxf(h, 0.0f) + tail);
      const float slope = (eps / (1.0f + expf(-h)) - (1.0f - eps) / (1.0f + expf(h))) * a.grad_scale / (float)a.pairs;
      a.seq_slope[2 * p] = slope * share[0];
      a.seq_slope[2 * p + 1] = -slope * share[1];
      a.partial[p] = loss;
    }
  }
  if (last_block(a.counts)) {
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (uint64_t p = threadIdx.x; p < a.pairs; p += kRowThreads) {
      const float r0 = __ldcg(a.rewards + 2 * p), r1 = __ldcg(a.rewards + 2 * p + 1);
      v[0] += __ldcg(a.partial + p);
      v[1] += r0 > r1 ? 1.0f : 0.0f;
      v[2] += r0;
      v[3] += r1;
    }
    for (uint32_t k = 0; k < 4; ++k) {
      const float total = block_sum(v[k], buf);
      if (threadIdx.x == 0) a.stats[k] = total / (float)a.pairs;
    }
  }
}

}  // namespace

cudaError_t launch_rows(RowOp op, const RowArgs& a, cudaStream_t st) {
  switch (a.dtype) {
    case BF_BF16: return launch_typed<__nv_bfloat16>(op, a, st);
    case BF_F16: return launch_typed<__half>(op, a, st);
    default: return launch_typed<float>(op, a, st);
  }
}

cudaError_t launch_row_sequences(const int64_t* tokens, uint64_t rows, const int64_t* offsets, uint64_t sequences,
                                 uint32_t* row_seq, uint32_t* seq_tokens, RowCounts* counts, cudaStream_t st) {
  // counts and seq_tokens stand side by side (bf_capi_learn.cu)
  cudaError_t e = cudaMemsetAsync(counts, 0, sizeof(RowCounts) + sizeof(uint32_t) * sequences, st);
  if (e != cudaSuccess) return e;
  sequence_kernel<<<(uint32_t)((rows + kRowThreads - 1) / kRowThreads), kRowThreads, 0, st>>>(
      tokens, rows, offsets, sequences, row_seq, seq_tokens, counts);
  return cudaGetLastError();
}

cudaError_t launch_pairs(const PairArgs& a, cudaStream_t st) {
  const uint32_t grid = (uint32_t)(a.pairs < (1u << 30) ? a.pairs : (1u << 30));
  pair_kernel<<<grid, kRowThreads, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace bfk
