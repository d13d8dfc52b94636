// bf_capi_learn.cu -- the C ABI's entry points for learning from makespans:
// argument checks, the layout of the caller's workspace and the launches.
#include <cmath>

#include "bf_capi_internal.h"
#include "bf_learn.h"

namespace bfcapi {

namespace {

using bfk::PairArgs;
using bfk::RowArgs;
using bfk::RowCounts;
using bfk::RowOp;

constexpr uint64_t kMaxRows = 0x7FFFFFFFull;
constexpr uint64_t kMaxCols = 1ull << 30;

uint64_t align256(uint64_t x) { return (x + 255) / 256 * 256; }

uint32_t size_of(uint32_t dtype) { return dtype == BF_F32 ? 4u : 2u; }

bool aligned(const void* p, size_t to) { return (uintptr_t)p % to == 0; }

// A matrix argument; `rows` may be 0 with any data pointer.
int check_matrix(const bf_matrix* m, const char* name, const char* who) {
  if (!m) return fail(BF_EINVAL, "%s: %s is NULL", who, name);
  if (m->dtype > BF_F16) return fail(BF_EINVAL, "%s: %s has the unknown type %u", who, name, m->dtype);
  if (m->rows > kMaxRows) return fail(BF_EINVAL, "%s: %s has more than 2^31 - 1 rows", who, name);
  if (m->cols == 0 || m->cols > kMaxCols) return fail(BF_EINVAL, "%s: %s needs 1 to 2^30 columns", who, name);
  if (m->row_stride < m->cols || m->row_stride > (1ull << 40) / (m->rows ? m->rows : 1))
    return fail(BF_EINVAL, "%s: the row stride of %s is below its columns or beyond 2^40 elements in all", who, name);
  if (m->rows && !m->data) return fail(BF_EINVAL, "%s: %s has no data", who, name);
  if (!aligned(m->data, size_of(m->dtype))) return fail(BF_EINVAL, "%s: %s is not aligned to its type", who, name);
  return BF_OK;
}

// An array argument that calls with `count` elements read or write.
int check_array(const void* p, uint64_t count, size_t size, const char* name, const char* who) {
  if (count && !p) return fail(BF_EINVAL, "%s: %s is NULL", who, name);
  if (!aligned(p, size)) return fail(BF_EINVAL, "%s: %s is not aligned to its type", who, name);
  return BF_OK;
}

uint64_t extent(const bf_matrix* m) { return m->rows ? ((m->rows - 1) * m->row_stride + m->cols) * size_of(m->dtype) : 0; }

bool overlap(const bf_matrix* a, const bf_matrix* b) {
  const uintptr_t x = (uintptr_t)a->data, y = (uintptr_t)b->data;
  return x < y + extent(b) && y < x + extent(a);
}

// A gradient: the logits' shape and type; the logits themselves, or apart from them.
int check_grad(const bf_matrix* logits, const bf_matrix* grad, const char* who) {
  if (check_matrix(grad, "grad", who) != BF_OK) return BF_EINVAL;
  if (grad->rows != logits->rows || grad->cols != logits->cols || grad->dtype != logits->dtype)
    return fail(BF_EINVAL, "%s: grad has another shape or type than logits", who);
  if (grad->data == logits->data && grad->row_stride == logits->row_stride) return BF_OK;
  return overlap(logits, grad) ? fail(BF_EINVAL, "%s: grad overlaps logits without being the same matrix", who) : BF_OK;
}

int check_number(float v, bool ok, const char* name, const char* who) {
  return std::isfinite(v) && ok ? BF_OK : fail(BF_EINVAL, "%s: %s = %g is out of its range", who, name, (double)v);
}

// A temperature whose reciprocals, in two parts, are normal 32-bit numbers.
int check_temperature(float v, const char* who) { return check_number(v, v >= 1e-18f && v <= 1e18f, "temperature", who); }

#define BF_TRY(call)                         \
  do {                                       \
    if ((call) != BF_OK) return BF_EINVAL;   \
  } while (0)

RowArgs row_args(const bf_matrix* logits, const int64_t* tokens, float temperature, const bf_matrix* grad) {
  RowArgs a = {};
  a.x = logits->data;
  a.ldx = logits->row_stride;
  a.rows = logits->rows;
  a.vocab = (uint32_t)logits->cols;
  a.dtype = logits->dtype;
  a.tokens = tokens;
  a.inv_tau = 1.0f / temperature;
  a.tau = temperature;
  const double c2 = 1.44269504088896340736 / (double)temperature;
  a.c2_hi = (float)c2;
  if ((double)a.c2_hi >= c2) a.c2_hi = std::nextafterf(a.c2_hi, 0.0f);
  a.c2_lo = (float)(c2 - (double)a.c2_hi);
  if (grad) {
    a.g = grad->data;
    a.ldg = grad->row_stride;
  }
  return a;
}

// The workspace of the losses; the counts and seq_tokens stand side by side (launch_row_sequences).
struct Layout {
  RowCounts* counts;
  uint32_t *seq_tokens, *row_seq;
  float* partial;
  float* logprob;       // preference: where the caller wants none
  float2* row_softmax;  // preference
  float* seq_slope;     // preference
  uint64_t bytes;

  Layout(void* base, uint64_t rows, uint64_t sequences, bool pairs) {
    char* at = static_cast<char*>(base);
    const auto take = [&](uint64_t n) {
      char* p = at;
      at += align256(n);
      return p;
    };
    char* head = take(sizeof(RowCounts) + 4 * sequences);
    counts = reinterpret_cast<RowCounts*>(head);
    seq_tokens = reinterpret_cast<uint32_t*>(head + sizeof(RowCounts));
    row_seq = reinterpret_cast<uint32_t*>(take(4 * rows));
    partial = reinterpret_cast<float*>(take(4 * (pairs ? sequences / 2 : bfk::kPolicyPart * (rows + bfk::kPolicyMoreParts))));
    logprob = nullptr;
    row_softmax = nullptr;
    seq_slope = nullptr;
    if (pairs) {
      logprob = reinterpret_cast<float*>(take(4 * rows));
      row_softmax = reinterpret_cast<float2*>(take(8 * rows));
      seq_slope = reinterpret_cast<float*>(take(4 * sequences));
    }
    bytes = (uint64_t)(at - static_cast<char*>(base));
  }
};

int check_workspace(const void* workspace, uint64_t have, uint64_t need, const char* who) {
  if (!workspace || !aligned(workspace, 256))
    return fail(BF_EINVAL, "%s: the workspace is NULL or not aligned to 256 bytes", who);
  if (have < need)
    return fail(BF_EINVAL, "%s: the workspace has %llu bytes and %llu are needed", who, (unsigned long long)have,
                (unsigned long long)need);
  return BF_OK;
}

int check_counts(uint64_t rows, uint64_t sequences, uint64_t* bytes, const char* who) {
  if (!bytes) return fail(BF_EINVAL, "%s: bytes is NULL", who);
  if (rows > kMaxRows || sequences > kMaxRows) return fail(BF_EINVAL, "%s: more than 2^31 - 1 rows or sequences", who);
  return BF_OK;
}

}  // namespace

}  // namespace bfcapi

using namespace bfcapi;

extern "C" {

int bf_token_logprobs(const bf_matrix* logits, const int64_t* d_tokens, float temperature, float* d_logprob,
                      float* d_entropy, void* cuda_stream) {
  const char* who = "bf_token_logprobs";
  BF_TRY(check_matrix(logits, "logits", who));
  BF_TRY(check_array(d_tokens, logits->rows, 8, "tokens", who));
  BF_TRY(check_array(d_logprob, logits->rows, 4, "logprob", who));
  BF_TRY(check_array(d_entropy, 0, 4, "entropy", who));
  BF_TRY(check_temperature(temperature, who));
  if (logits->rows == 0) return BF_OK;
  RowArgs a = row_args(logits, d_tokens, temperature, nullptr);
  a.logprob = d_logprob;
  a.entropy = d_entropy;
  const cudaError_t e = bfk::launch_rows(RowOp::kScore, a, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? BF_OK : cuda_fail(e, who);
}

int bf_token_logprobs_grad(const bf_matrix* logits, const int64_t* d_tokens, float temperature,
                           const float* d_grad_logprob, const float* d_grad_entropy, const bf_matrix* grad,
                           void* cuda_stream) {
  const char* who = "bf_token_logprobs_grad";
  BF_TRY(check_matrix(logits, "logits", who));
  BF_TRY(check_grad(logits, grad, who));
  BF_TRY(check_array(d_tokens, logits->rows, 8, "tokens", who));
  BF_TRY(check_array(d_grad_logprob, logits->rows, 4, "grad_logprob", who));
  BF_TRY(check_array(d_grad_entropy, 0, 4, "grad_entropy", who));
  BF_TRY(check_temperature(temperature, who));
  if (logits->rows == 0) return BF_OK;
  RowArgs a = row_args(logits, d_tokens, temperature, grad);
  a.grad_logprob = d_grad_logprob;
  a.grad_entropy = d_grad_entropy;
  const cudaError_t e = bfk::launch_rows(RowOp::kScoreGrad, a, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? BF_OK : cuda_fail(e, who);
}

int bf_policy_loss_workspace(uint64_t rows, uint64_t sequences, uint64_t* bytes) {
  BF_TRY(check_counts(rows, sequences, bytes, "bf_policy_loss_workspace"));
  *bytes = Layout(nullptr, rows, sequences, false).bytes;
  return BF_OK;
}

int bf_policy_loss(const bf_matrix* logits, const bf_policy_args* args, float* d_stats, float* d_logprob,
                   const bf_matrix* grad, void* d_workspace, uint64_t workspace_bytes, void* cuda_stream) {
  const char* who = "bf_policy_loss";
  BF_TRY(check_matrix(logits, "logits", who));
  if (!args) return fail(BF_EINVAL, "%s: args is NULL", who);
  if (grad) BF_TRY(check_grad(logits, grad, who));
  const uint64_t rows = logits->rows, sequences = args->sequences;
  uint64_t need = 0;
  BF_TRY(check_counts(rows, sequences, &need, who));
  BF_TRY(check_array(args->tokens, rows, 8, "tokens", who));
  BF_TRY(check_array(args->offsets, 1, 8, "offsets", who));
  BF_TRY(check_array(args->old_logprob, rows, 4, "old_logprob", who));
  BF_TRY(check_array(args->ref_logprob, 0, 4, "ref_logprob", who));
  BF_TRY(check_array(args->advantage, args->advantage_per_token ? rows : sequences, 4, "advantage", who));
  BF_TRY(check_array(d_stats, 1, 4, "stats", who));
  BF_TRY(check_array(d_logprob, 0, 4, "logprob", who));
  BF_TRY(check_temperature(args->temperature, who));
  BF_TRY(check_number(args->clip_low, args->clip_low >= 0.0f, "clip_low", who));
  BF_TRY(check_number(args->clip_high, args->clip_high >= 0.0f, "clip_high", who));
  BF_TRY(check_number(args->kl_coef, args->kl_coef >= 0.0f, "kl_coef", who));
  BF_TRY(check_number(args->entropy_coef, true, "entropy_coef", who));
  BF_TRY(check_number(args->grad_scale, true, "grad_scale", who));
  if (args->kl_coef > 0.0f && !args->ref_logprob && rows)
    return fail(BF_EINVAL, "%s: a KL term needs ref_logprob", who);
  if (args->reduction > BF_SUM) return fail(BF_EINVAL, "%s: unknown reduction %u", who, args->reduction);
  const Layout ws(d_workspace, rows, sequences, false);
  BF_TRY(check_workspace(d_workspace, workspace_bytes, ws.bytes, who));
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (rows == 0) {
    const cudaError_t e = cudaMemsetAsync(d_stats, 0, sizeof(float) * BF_POLICY_STATS, st);
    return e == cudaSuccess ? BF_OK : cuda_fail(e, who);
  }
  RowArgs a = row_args(logits, args->tokens, args->temperature, grad);
  a.logprob = d_logprob;
  a.row_seq = ws.row_seq;
  a.seq_tokens = ws.seq_tokens;
  a.counts = ws.counts;
  a.old_logprob = args->old_logprob;
  a.ref_logprob = args->ref_logprob;
  a.advantage = args->advantage;
  a.advantage_per_token = args->advantage_per_token;
  a.reduction = args->reduction;
  a.ratio_lo = 1.0f - args->clip_low;
  a.ratio_hi = 1.0f + args->clip_high;
  a.kl_coef = args->kl_coef;
  a.entropy_coef = args->entropy_coef;
  a.grad_scale = args->grad_scale;
  a.partial = ws.partial;
  a.stats = d_stats;
  bool done = false;
  cudaError_t e = bfk::launch_few(a, nullptr, args->offsets, sequences, &done, st);
  if (done || e != cudaSuccess) return e == cudaSuccess ? BF_OK : cuda_fail(e, who);
  e = bfk::launch_row_sequences(args->tokens, rows, args->offsets, sequences,
                                args->reduction == BF_MEAN_SEQUENCES, ws.row_seq, ws.seq_tokens, ws.counts, st);
  if (e == cudaSuccess) e = bfk::launch_rows(RowOp::kPolicy, a, st);
  return e == cudaSuccess ? BF_OK : cuda_fail(e, who);
}

int bf_preference_loss_workspace(uint64_t rows, uint64_t pairs, uint64_t* bytes) {
  if (pairs > kMaxRows / 2) return fail(BF_EINVAL, "bf_preference_loss_workspace: more than 2^30 - 1 pairs");
  BF_TRY(check_counts(rows, 2 * pairs, bytes, "bf_preference_loss_workspace"));
  *bytes = Layout(nullptr, rows, 2 * pairs, true).bytes;
  return BF_OK;
}

int bf_preference_loss(const bf_matrix* logits, const bf_preference_args* args, float* d_stats, float* d_rewards,
                       float* d_logprob, const bf_matrix* grad, void* d_workspace, uint64_t workspace_bytes,
                       void* cuda_stream) {
  const char* who = "bf_preference_loss";
  BF_TRY(check_matrix(logits, "logits", who));
  if (!args) return fail(BF_EINVAL, "%s: args is NULL", who);
  if (grad) BF_TRY(check_grad(logits, grad, who));
  const uint64_t rows = logits->rows, pairs = args->pairs;
  if (pairs > kMaxRows / 2) return fail(BF_EINVAL, "%s: more than 2^30 - 1 pairs", who);
  BF_TRY(check_array(args->tokens, rows, 8, "tokens", who));
  BF_TRY(check_array(args->offsets, 1, 8, "offsets", who));
  BF_TRY(check_array(args->ref_logprob, 0, 4, "ref_logprob", who));
  BF_TRY(check_array(d_stats, 1, 4, "stats", who));
  BF_TRY(check_array(d_rewards, pairs, 4, "rewards", who));
  BF_TRY(check_array(d_logprob, 0, 4, "logprob", who));
  BF_TRY(check_temperature(args->temperature, who));
  BF_TRY(check_number(args->beta, args->beta > 0.0f, "beta", who));
  BF_TRY(check_number(args->label_smoothing, args->label_smoothing >= 0.0f && args->label_smoothing < 1.0f,
                      "label_smoothing", who));
  BF_TRY(check_number(args->margin, true, "margin", who));
  BF_TRY(check_number(args->grad_scale, true, "grad_scale", who));
  const Layout ws(d_workspace, rows, 2 * pairs, true);
  BF_TRY(check_workspace(d_workspace, workspace_bytes, ws.bytes, who));
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  RowArgs a = row_args(logits, args->tokens, args->temperature, grad);
  a.logprob = d_logprob ? d_logprob : ws.logprob;
  PairArgs p = {};
  p.offsets = args->offsets;
  p.pairs = pairs;
  p.rows = rows;
  p.row_seq = ws.row_seq;
  p.seq_tokens = ws.seq_tokens;
  p.counts = ws.counts;
  p.logprob = a.logprob;
  p.ref_logprob = args->ref_logprob;
  p.beta = args->beta;
  p.label_smoothing = args->label_smoothing;
  p.margin = args->margin;
  p.grad_scale = args->grad_scale;
  p.average = args->average;
  p.seq_slope = ws.seq_slope;
  p.rewards = d_rewards;
  p.partial = ws.partial;
  p.stats = d_stats;
  cudaError_t e = cudaSuccess;
  if (rows && pairs) {
    bool done = false;
    e = bfk::launch_few(a, &p, args->offsets, 2 * pairs, &done, st);
    if (done || e != cudaSuccess) return e == cudaSuccess ? BF_OK : cuda_fail(e, who);
  }
  if (rows) {
    a.row_seq = ws.row_seq;
    a.row_softmax = ws.row_softmax;
    e = bfk::launch_row_sequences(args->tokens, rows, args->offsets, 2 * pairs, args->average != 0, ws.row_seq,
                                  ws.seq_tokens, ws.counts, st);
    if (e == cudaSuccess) e = bfk::launch_rows(RowOp::kPairScore, a, st);
  } else {
    e = cudaMemsetAsync(ws.counts, 0, sizeof(RowCounts) + 8 * pairs, st);
  }
  if (e == cudaSuccess && pairs == 0) e = cudaMemsetAsync(d_stats, 0, sizeof(float) * BF_PREFERENCE_STATS, st);
  if (e == cudaSuccess && pairs) e = bfk::launch_pairs(p, st);
  if (e == cudaSuccess && grad && rows) {
    a.logprob = nullptr;
    a.seq_slope = ws.seq_slope;
    e = bfk::launch_rows(RowOp::kPairGrad, a, st);
  }
  return e == cudaSuccess ? BF_OK : cuda_fail(e, who);
}

int bf_embed(const bf_matrix* table, const int64_t* d_tokens, float scale, const bf_matrix* out, void* cuda_stream) {
  const char* who = "bf_embed";
  BF_TRY(check_matrix(table, "table", who));
  BF_TRY(check_matrix(out, "out", who));
  if (out->cols != table->cols || out->dtype != table->dtype)
    return fail(BF_EINVAL, "%s: out has another width or type than table", who);
  if (table->rows == 0) return fail(BF_EINVAL, "%s: table has no rows", who);
  if (overlap(table, out)) return fail(BF_EINVAL, "%s: out overlaps table", who);
  BF_TRY(check_array(d_tokens, out->rows, 8, "tokens", who));
  BF_TRY(check_number(scale, true, "scale", who));
  if (out->rows == 0) return BF_OK;
  const bfk::EmbedArgs a = {table->data, out->data, table->row_stride, out->row_stride, out->rows, (uint32_t)table->rows,
                            (uint32_t)table->cols, table->dtype, out->dtype, d_tokens, scale, false};
  const cudaError_t e = bfk::launch_embed(a, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? BF_OK : cuda_fail(e, who);
}

int bf_embed_grad_workspace(uint64_t rows, uint64_t width, uint64_t* bytes) {
  BF_TRY(check_counts(rows, 0, bytes, "bf_embed_grad_workspace"));
  if (width == 0 || width > kMaxCols) return fail(BF_EINVAL, "bf_embed_grad_workspace: width must be 1 to 2^30");
  *bytes = bfk::embed_grad_bytes(rows, (uint32_t)width);
  return BF_OK;
}

int bf_embed_grad(const bf_matrix* grad_out, const int64_t* d_tokens, float scale, uint32_t accumulate,
                  const bf_matrix* grad_table, void* d_workspace, uint64_t workspace_bytes, void* cuda_stream) {
  const char* who = "bf_embed_grad";
  BF_TRY(check_matrix(grad_out, "grad_out", who));
  BF_TRY(check_matrix(grad_table, "grad_table", who));
  if (grad_out->cols != grad_table->cols) return fail(BF_EINVAL, "%s: grad_table has another width than grad_out", who);
  if (grad_table->rows == 0) return fail(BF_EINVAL, "%s: grad_table has no rows", who);
  if (overlap(grad_out, grad_table)) return fail(BF_EINVAL, "%s: grad_table overlaps grad_out", who);
  BF_TRY(check_array(d_tokens, grad_out->rows, 8, "tokens", who));
  BF_TRY(check_number(scale, true, "scale", who));
  if (grad_out->rows)
    BF_TRY(check_workspace(d_workspace, workspace_bytes,
                           bfk::embed_grad_bytes(grad_out->rows, (uint32_t)grad_out->cols), who));
  const bfk::EmbedArgs a = {grad_out->data, grad_table->data, grad_out->row_stride, grad_table->row_stride,
                            grad_out->rows, (uint32_t)grad_table->rows, (uint32_t)grad_out->cols, grad_out->dtype,
                            grad_table->dtype, d_tokens, scale, accumulate != 0};
  const cudaError_t e = bfk::launch_embed_grad(a, d_workspace, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? BF_OK : cuda_fail(e, who);
}

}  // extern "C"
