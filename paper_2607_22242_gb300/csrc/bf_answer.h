// bf_answer.h -- internal interface between the C ABI (bf_capi_answer.cu) and
// the kernels of a decoding step: attention with a shared prefix
// (bf_attend.cu), the choice of continuations and the reordering of states
// (bf_beams.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/bf.h"

namespace bfk {

// Vectors (sequence, token, head): strides in elements.
struct Vectors {
  const void* data;
  int64_t batch, token, head;
};

struct AttendArgs {
  Vectors q, pk, pv, sk, sv, out;
  float* lse;                         // nullptr: not wanted
  const int64_t *prefix_len, *suffix_len;  // nullptr: the capacity
  uint64_t prefix_cap, suffix_cap;
  uint32_t prompts, per_prompt;       // answers of a prompt
  uint32_t kv_heads, share;           // key heads; query heads of each
  uint32_t dim, dtype;
  float scale2;                       // scale * log2(e)
};

// Bytes of workspace of a call of these sizes (only they are read of `a`).
uint64_t attend_bytes(const AttendArgs& a);
cudaError_t launch_attend(const AttendArgs& a, void* workspace, cudaStream_t st);

struct BeamArgs {
  const void* x;  // logits
  uint64_t ldx;
  uint32_t vocab, dtype;
  uint32_t groups, beams, keep;
  const float* scores;
  const uint8_t* finished;   // nullptr: none
  const int64_t* lengths;    // nullptr: no penalty
  int64_t end_token;
  float penalty, tau, c2;    // c2: log2(e) / tau
  float* out_scores;
  int64_t *out_tokens, *out_parents;
  uint8_t* out_finished;     // nullptr: not wanted
  int64_t* out_lengths;      // nullptr: not wanted
};
uint64_t beam_bytes(uint32_t groups, uint32_t beams, uint64_t vocab, uint32_t keep);
cudaError_t launch_beam_step(const BeamArgs& a, void* workspace, cudaStream_t st);

struct ReorderArgs {
  const char* from[BF_MAX_STATES];
  char* to[BF_MAX_STATES];
  uint64_t from_row, from_token, from_head, to_row, to_token, to_head;  // strides in bytes
  uint64_t tokens, width;
  uint32_t heads, count, groups, beams;
  const int64_t *parents, *lengths;  // lengths: nullptr, all tokens
  bool in_place;
};
cudaError_t launch_reorder(const ReorderArgs& a, cudaStream_t st);

}  // namespace bfk
