// bf_answers.cu -- what the losses need beside rows of logits: which answer
// (sequence) each row belongs to, and the preference loss between its passes.
#include "bf_rows.cuh"

namespace bfk {

namespace {

// Offsets that do not ascend make rows miss their sequence; no read leaves the
// array.  Counts are sums of whole numbers: their order does not matter.

// Up to kSmallRows rows of up to kSmallSequences sequences: one block, with the
// offsets and the counts in shared memory, no memory to clear first (1,024 rows
// 3.8 us, 8,000 rows 11 us, beside which the rows' kernel reads its logits).
constexpr uint32_t kSmallRows = 16384, kSmallSequences = 4096, kSmallThreads = 1024;

__global__ void __launch_bounds__(kSmallThreads) small_sequence_kernel(const int64_t* tokens, uint32_t rows,
                                                                       const int64_t* offsets, uint32_t sequences,
                                                                       uint32_t* row_seq, uint32_t* seq_tokens,
                                                                       RowCounts* counts) {
  __shared__ uint32_t begin[kSmallSequences + 1], count[kSmallSequences];
  __shared__ uint32_t all;
  let_next_start();
  if (threadIdx.x == 0) all = 0;
  for (uint32_t s = threadIdx.x; s <= sequences; s += kSmallThreads) {
    begin[s] = clamp_offset(offsets[s], rows);
    if (s < sequences) count[s] = 0;
  }
  __syncthreads();
  for (uint32_t first = 0; first < rows; first += kSmallThreads) {
    const uint32_t row = first + threadIdx.x;
    uint32_t seq = kNoSequence;
    if (row < rows) {
      if (tokens[row] >= 0) seq = sequence_at(begin, sequences, row);
      row_seq[row] = seq;
    }
    const uint32_t same = __match_any_sync(~0u, seq);
    if (seq != kNoSequence && threadIdx.x % 32 == (uint32_t)__ffs(same) - 1) {
      atomicAdd(&count[seq], (uint32_t)__popc(same));
      atomicAdd(&all, (uint32_t)__popc(same));
    }
  }
  __syncthreads();
  uint32_t used = 0;
  for (uint32_t first = 0; first < sequences; first += kSmallThreads) {
    const uint32_t s = first + threadIdx.x, n = s < sequences ? count[s] : 0;
    if (s < sequences) seq_tokens[s] = n;
    used += __syncthreads_count(n != 0);
  }
  if (threadIdx.x == 0) *counts = RowCounts{all, used, 0, 0};
}

// Any number: counts and seq_tokens are zero at the start.  A block's rows are
// neighbours, so their sequences are too: one search for its first row by a
// warp (32 probes at a time), then the offsets from there on in shared memory.
// 655,360 rows of 65,536 sequences 10 us; a search of all offsets for each row 38 us.
constexpr uint32_t kRowThreads = 256, kRowsEach = 4, kBlockRows = kRowThreads * kRowsEach;
constexpr uint32_t kOffsets = kBlockRows;

__global__ void __launch_bounds__(kRowThreads) sequence_kernel(const int64_t* tokens, uint64_t rows,
                                                               const int64_t* offsets, uint64_t sequences,
                                                               uint32_t* row_seq, uint32_t* seq_tokens,
                                                               RowCounts* counts, uint32_t per_sequence) {
  __shared__ uint64_t first_seq;
  __shared__ int64_t begin[kOffsets + 1];
  let_next_start();
  const uint64_t first = (uint64_t)blockIdx.x * kBlockRows;
  const uint32_t lane = threadIdx.x % 32;
  bool on[kRowsEach];
#pragma unroll
  for (uint32_t k = 0; k < kRowsEach; ++k) {
    const uint64_t row = first + k * kRowThreads + threadIdx.x;
    on[k] = row < rows && sequences && tokens[row] >= 0;
  }
  if (threadIdx.x < 32) {
    uint64_t lo = 0, hi = sequences ? sequences : 1;
    while (hi - lo > 1) {
      const uint64_t step = (hi - lo + 31) / 32, at = lo + lane * step;
      const uint32_t before = __ballot_sync(~0u, lane == 0 || (at < hi && offsets[at] <= (int64_t)first));
      lo += (31 - __clz(before)) * step;
      hi = min(hi, lo + step);
    }
    if (lane == 0) first_seq = lo;
  }
  __syncthreads();
  const uint64_t s0 = first_seq;
  const uint32_t held = sequences ? (uint32_t)min((uint64_t)kOffsets, sequences - s0) : 0;
  for (uint32_t i = threadIdx.x; i <= held; i += kRowThreads) begin[i] = offsets[s0 + i];
  __syncthreads();
  uint32_t scored = 0, opened = 0;
#pragma unroll
  for (uint32_t k = 0; k < kRowsEach; ++k) {
    const uint64_t row = first + k * kRowThreads + threadIdx.x;
    uint32_t seq = kNoSequence;
    if (on[k]) {
      const uint32_t i = last_at_or_before(begin, 0u, held + 1, (int64_t)row);
      if (i < held) {
        if (begin[i] <= (int64_t)row) seq = (uint32_t)(s0 + i);
      } else if (s0 + held < sequences) {  // many empty sequences: beyond those held
        const uint64_t s = last_at_or_before(offsets, s0 + held, sequences, (int64_t)row);
        if (offsets[s] <= (int64_t)row && (int64_t)row < offsets[s + 1]) seq = (uint32_t)s;
      }
    }
    if (row < rows) row_seq[row] = seq;
    scored += __popc(__ballot_sync(~0u, seq != kNoSequence));
    if (per_sequence) {
      const uint32_t same = __match_any_sync(~0u, seq);
      const bool opens = seq != kNoSequence && lane == (uint32_t)__ffs(same) - 1 &&
                         atomicAdd(&seq_tokens[seq], (uint32_t)__popc(same)) == 0u;
      opened += __popc(__ballot_sync(~0u, opens));
    }
  }
  __shared__ uint32_t sums[2];
  if (threadIdx.x < 2) sums[threadIdx.x] = 0;
  __syncthreads();
  if (lane == 0) {
    atomicAdd(&sums[0], scored);
    atomicAdd(&sums[1], opened);
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    if (sums[0]) atomicAdd(&counts->tokens, sums[0]);
    if (sums[1]) atomicAdd(&counts->sequences, sums[1]);
  }
}

// `each` threads per answer, a pair's two answers side by side in one block, the
// block's pairs next to one another; kAhead rows a thread are read before they are added.
constexpr uint32_t kPairThreads = 512;        // a block's, for short answers
constexpr uint32_t kLongPairThreads = 1024;   // a pair's, at most

__global__ void __launch_bounds__(kLongPairThreads) pair_kernel(const PairArgs a, uint32_t each) {
  constexpr uint32_t kAhead = 4;
  __shared__ float buf[kLongPairThreads / 32 * 4];
  let_next_start();
  wait_for_previous();
  const uint32_t in_block = blockDim.x / (2 * each), mine = threadIdx.x / (2 * each);
  const uint32_t half = threadIdx.x / each % 2, lane = threadIdx.x % each, warps = each / 32;
  for (uint64_t base = (uint64_t)blockIdx.x * in_block; base < a.pairs; base += (uint64_t)gridDim.x * in_block) {
    const uint64_t p = base + mine, seq = 2 * p + half;
    float v = 0.0f;
    if (p < a.pairs) {
      const int64_t lo = a.offsets[seq], hi = a.offsets[seq + 1];
      const uint64_t begin = lo > 0 ? (uint64_t)lo : 0, end = hi > 0 ? min((uint64_t)hi, a.rows) : 0;
      for (uint64_t first = begin + lane; first < end; first += kAhead * each) {
        uint32_t of[kAhead];
        float lp[kAhead], ref[kAhead];
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k) {
          const uint64_t row = first + k * each;
          of[k] = row < end ? a.row_seq[row] : kNoSequence;
          lp[k] = row < end ? a.logprob[row] : 0.0f;
          ref[k] = row < end && a.ref_logprob ? a.ref_logprob[row] : 0.0f;
        }
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k)
          if (of[k] == (uint32_t)seq) v += lp[k] - ref[k];
      }
    }
#pragma unroll
    for (int o = 16; o; o /= 2) v += __shfl_xor_sync(~0u, v, o);
    __syncthreads();
    if (threadIdx.x % 32 == 0) buf[threadIdx.x / 32] = v;
    __syncthreads();
    // by the first warp, which also says that the block is done
    if (threadIdx.x < in_block && base + threadIdx.x < a.pairs) {
      const uint64_t pair = base + threadIdx.x;
      float sum[2];
      for (uint32_t h = 0; h < 2; ++h) {
        sum[h] = 0.0f;
        for (uint32_t w = 0; w < warps; ++w) sum[h] += buf[(2 * threadIdx.x + h) * warps + w];
      }
      const uint32_t n[2] = {a.average ? a.seq_tokens[2 * pair] : 0, a.average ? a.seq_tokens[2 * pair + 1] : 0};
      finish_pair(a, pair, sum, n);
    }
  }
  bool last = false;
  if (threadIdx.x < 32) last = last_to_say(&a.counts->blocks_done, gridDim.x);
  if (__syncthreads_or(last)) {
    last_sees();
    preference_stats(a, buf);
  }
}

}  // namespace

cudaError_t launch_row_sequences(const int64_t* tokens, uint64_t rows, const int64_t* offsets, uint64_t sequences,
                                 bool per_sequence, uint32_t* row_seq, uint32_t* seq_tokens, RowCounts* counts,
                                 cudaStream_t st) {
  if (rows <= kSmallRows && sequences <= kSmallSequences) {
    small_sequence_kernel<<<1, kSmallThreads, 0, st>>>(tokens, (uint32_t)rows, offsets, (uint32_t)sequences, row_seq,
                                                      seq_tokens, counts);
    return cudaGetLastError();
  }
  // counts and seq_tokens stand side by side (bf_capi_learn.cu)
  cudaError_t e = cudaMemsetAsync(counts, 0, sizeof(RowCounts) + (per_sequence ? sizeof(uint32_t) * sequences : 0), st);
  if (e != cudaSuccess) return e;
  sequence_kernel<<<(uint32_t)((rows + kBlockRows - 1) / kBlockRows), kRowThreads, 0, st>>>(
      tokens, rows, offsets, sequences, row_seq, seq_tokens, counts, per_sequence);
  return cudaGetLastError();
}

cudaError_t launch_pairs(const PairArgs& a, cudaStream_t st) {
  // A warp per answer up to 256 rows a pair on average, more threads for longer ones, half a block's at most.
  // Whole call, here and with a block of 512 threads per pair that read one row at a time: 6 pairs of 46,000 rows of
  // 8 logits in 16 bits 39 and 68 us; 6,661 pairs of 24 rows of 4 logits in 32 bits 28 and 55 us.
  uint32_t each = 32;
  while (2 * each < kLongPairThreads && a.rows / a.pairs > 8ull * each) each *= 2;
  const uint32_t threads = max(kPairThreads, 2 * each), in_block = threads / (2 * each);
  const uint64_t blocks = (a.pairs + in_block - 1) / in_block;
  return launch_after(pair_kernel, blocks < (1u << 30) ? blocks : (1u << 30), threads, st, a, each);
}

}  // namespace bfk
