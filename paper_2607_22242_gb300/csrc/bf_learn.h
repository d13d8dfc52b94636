// bf_learn.h -- internal interface between the C ABI (bf_capi_learn.cu) and
// the kernels that learn from makespans: rows of logits (bf_rows.cu) and the
// token embedding (bf_embed.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/bf.h"

namespace bfk {

// What a pass over rows of logits computes.
enum class RowOp { kScore, kScoreGrad, kPolicy, kPairScore, kPairGrad };

constexpr uint32_t kNoSequence = 0xFFFFFFFFu;
constexpr uint32_t kPolicySums = 5;  // surrogate, KL, entropy, clipped share, ratio: weighted sums over the rows
constexpr uint32_t kPolicyPart = 8;  // floats that a part of them takes
constexpr uint32_t kPolicyMoreParts = 256;

// Counts of a call's scored tokens, in its workspace.
struct RowCounts {
  uint32_t tokens;      // scored tokens of all sequences
  uint32_t sequences;   // sequences with at least one
  uint32_t blocks_done; // the last block to finish sums up
  uint32_t pad;
};

// Arguments of a pass.  x: logits; g: their gradient (may be x itself), nullptr for none.
struct RowArgs {
  const void* x;
  void* g;
  uint64_t ldx, ldg;  // row strides in elements
  uint64_t rows;
  uint32_t vocab;
  uint32_t dtype;     // bf_dtype
  const int64_t* tokens;
  float tau, inv_tau;      // temperature, and its reciprocal
  float c2_hi, c2_lo;      // log2(e) / temperature in two parts, the second above 0
  float* logprob;     // nullptr: not wanted
  float* entropy;     // nullptr: not wanted
  // kScoreGrad
  const float* grad_logprob;
  const float* grad_entropy;  // nullptr: none
  // kPolicy, kPairScore, kPairGrad
  const uint32_t* row_seq;  // sequence of each scored row, kNoSequence otherwise
  const uint32_t* seq_tokens;  // scored tokens of each sequence
  RowCounts* counts;
  const float* old_logprob;
  const float* ref_logprob;  // nullptr: none
  const float* advantage;
  uint32_t advantage_per_token;
  uint32_t reduction;  // bf_reduction
  float ratio_lo, ratio_hi, kl_coef, entropy_coef, grad_scale;
  float* partial;  // kPolicy: kPolicyPart floats (the sums) a part; as many as rows, and kPolicyMoreParts more
  bool sums_behind;  // kPolicy: a kernel behind sums the parts up
  float* stats;
  // kPairScore writes and kPairGrad reads what a row's probabilities are made from; kPairGrad's slope of each sequence
  float2* row_softmax;  // (max, 1 / sum)
  const float* seq_slope;
};

// Arguments of the preference loss between its two passes.
struct PairArgs {
  const int64_t* offsets;
  uint64_t pairs, rows;
  const uint32_t* row_seq;
  const uint32_t* seq_tokens;
  RowCounts* counts;
  const float* logprob;
  const float* ref_logprob;  // nullptr: none
  float beta, label_smoothing, margin, grad_scale;
  uint32_t average;
  float* seq_slope;  // 2 * pairs
  float* rewards;    // 2 * pairs
  float* partial;    // the loss of each pair
  float* stats;
};

// Which sequence each scored row belongs to, and how many there are: fills row_seq, counts and, with `per_sequence`,
// seq_tokens.
cudaError_t launch_row_sequences(const int64_t* tokens, uint64_t rows, const int64_t* offsets, uint64_t sequences,
                                 bool per_sequence, uint32_t* row_seq, uint32_t* seq_tokens, RowCounts* counts,
                                 cudaStream_t st);
// One pass over rows of each element type (bf_rows.cu, compiled once per type).
cudaError_t launch_rows_type0(RowOp op, const RowArgs& a, cudaStream_t st);
cudaError_t launch_rows_type1(RowOp op, const RowArgs& a, cudaStream_t st);
cudaError_t launch_rows_type2(RowOp op, const RowArgs& a, cudaStream_t st);
inline cudaError_t launch_rows(RowOp op, const RowArgs& a, cudaStream_t st) {
  return a.dtype == BF_F32 ? launch_rows_type0(op, a, st)
         : a.dtype == BF_BF16 ? launch_rows_type1(op, a, st) : launch_rows_type2(op, a, st);
}
cudaError_t launch_pairs(const PairArgs& a, cudaStream_t st);

// A whole loss (the preference loss with `p`, else the policy loss) in one
// launch, where its rows are few and short; *done tells whether they were.
cudaError_t launch_few_type0(const RowArgs& a, const PairArgs* p, const int64_t* offsets, uint64_t sequences, bool* done,
                             cudaStream_t st);
cudaError_t launch_few_type1(const RowArgs& a, const PairArgs* p, const int64_t* offsets, uint64_t sequences, bool* done,
                             cudaStream_t st);
cudaError_t launch_few_type2(const RowArgs& a, const PairArgs* p, const int64_t* offsets, uint64_t sequences, bool* done,
                             cudaStream_t st);
inline cudaError_t launch_few(const RowArgs& a, const PairArgs* p, const int64_t* offsets, uint64_t sequences, bool* done,
                              cudaStream_t st) {
  return a.dtype == BF_F32 ? launch_few_type0(a, p, offsets, sequences, done, st)
         : a.dtype == BF_BF16 ? launch_few_type1(a, p, offsets, sequences, done, st)
                              : launch_few_type2(a, p, offsets, sequences, done, st);
}

struct EmbedArgs {
  const void* src;  // embed: the table; gradient: the gradient of the output rows
  void* dst;        // embed: the output rows; gradient: the table's gradient
  uint64_t lds, ldd;
  uint64_t rows;    // tokens
  uint32_t vocab, width;
  uint32_t src_dtype, dst_dtype;
  const int64_t* tokens;
  float scale;
  bool accumulate;
};
cudaError_t launch_embed(const EmbedArgs& a, cudaStream_t st);
// Bytes of workspace of a gradient over `rows` tokens.
uint64_t embed_grad_bytes(uint64_t rows, uint32_t width);
cudaError_t launch_embed_grad(const EmbedArgs& a, void* workspace, cudaStream_t st);

}  // namespace bfk
