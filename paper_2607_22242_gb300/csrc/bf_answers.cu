// bf_answers.cu -- what the losses need beside rows of logits: which answer
// (sequence) each row belongs to, and the preference loss between its passes.
#include "bf_rows.cuh"

namespace bfk {

namespace {

constexpr uint32_t kRowThreads = 256;

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
  if (last_block(&a.counts->blocks_done, gridDim.x)) {
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
