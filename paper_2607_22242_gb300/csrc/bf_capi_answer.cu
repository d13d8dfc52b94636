// bf_capi_answer.cu -- the C ABI's entry points of a decoding step: argument
// checks and the launches.
#include "bf_answer.h"
#include "bf_capi_checks.h"

namespace bfcapi {

namespace {

constexpr uint64_t kMaxHeads = 65536, kMaxDim = 1ull << 16, kMaxElements = 1ull << 42;
constexpr uint64_t kMaxVocab = 1ull << 24;  // a group's kept logits are counted in 32 bits

// Elements from a cache's first to behind its last (checked strides).
uint64_t span(const bf_cache* c) {
  if (!c->batch || !c->tokens || !c->heads) return 0;
  return (c->batch - 1) * c->batch_stride + (c->tokens - 1) * c->token_stride + (c->heads - 1) * c->head_stride + c->dim;
}

bool stride_fits(uint64_t count, uint64_t stride) { return count < 2 || stride <= kMaxElements / (count - 1); }

int check_cache(const bf_cache* c, const char* name, const char* who) {
  if (!c) return fail(BF_EINVAL, "%s: %s is NULL", who, name);
  if (c->dtype > BF_F16) return fail(BF_EINVAL, "%s: %s has the unknown type %u", who, name, c->dtype);
  if (c->batch > kMaxRows || c->tokens > kMaxRows || c->heads > kMaxHeads)
    return fail(BF_EINVAL, "%s: %s has more than 2^31 - 1 sequences or tokens, or 65536 heads", who, name);
  if (c->heads == 0) return fail(BF_EINVAL, "%s: %s has no heads", who, name);
  if (c->dim == 0 || c->dim > kMaxDim) return fail(BF_EINVAL, "%s: %s has vectors of 0 or over 65536 dimensions", who, name);
  if (!stride_fits(c->batch, c->batch_stride) || !stride_fits(c->tokens, c->token_stride) ||
      !stride_fits(c->heads, c->head_stride) || span(c) > kMaxElements)
    return fail(BF_EINVAL, "%s: %s spans more than 2^42 elements", who, name);
  if (span(c) && !c->data) return fail(BF_EINVAL, "%s: %s has no data", who, name);
  if (!aligned(c->data, size_of(c->dtype))) return fail(BF_EINVAL, "%s: %s is not aligned to its type", who, name);
  return BF_OK;
}

int check_like(const bf_cache* c, const bf_cache* k, const char* name, const char* other, const char* who) {
  if (c->batch != k->batch || c->tokens != k->tokens || c->heads != k->heads || c->dim != k->dim || c->dtype != k->dtype)
    return fail(BF_EINVAL, "%s: %s has another shape or type than %s", who, name, other);
  return BF_OK;
}

// Bytes of an argument; none where there is no argument.
struct Bytes {
  const void* data;
  uint64_t count;
  const char* name;
};
bool overlap(const Bytes& a, const Bytes& b) {
  const uintptr_t x = (uintptr_t)a.data, y = (uintptr_t)b.data;
  return a.data && b.data && a.count && b.count && x < y + b.count && y < x + a.count;
}
Bytes bytes_of(const bf_cache* c, const char* name) {
  return c ? Bytes{c->data, span(c) * size_of(c->dtype), name} : Bytes{nullptr, 0, name};
}

// Whether two of the vectors of a one-token cache share elements.
bool folded(const bf_cache* c) {
  const uint64_t n[2] = {c->batch, c->heads}, s[2] = {c->batch_stride, c->head_stride};
  for (int inner = 0; inner < 2; ++inner) {
    const int o = 1 - inner;
    const uint64_t run = (n[inner] > 1 ? (n[inner] - 1) * s[inner] : 0) + c->dim;
    if ((n[inner] < 2 || s[inner] >= c->dim) && (n[o] < 2 || s[o] >= run)) return false;
  }
  return true;
}

bfk::Vectors vectors(const bf_cache* c) {
  if (!c) return {nullptr, 0, 0, 0};
  return {c->data, (int64_t)c->batch_stride, (int64_t)c->token_stride, (int64_t)c->head_stride};
}

// The sizes of an attention call, checked against each other.
int attend_sizes(const bf_cache* q, const bf_cache* pk, const bf_cache* sk, bfk::AttendArgs* a, const char* who) {
  BF_TRY(check_cache(q, "q", who));
  BF_TRY(check_cache(pk, "prefix_k", who));
  if (sk) BF_TRY(check_cache(sk, "suffix_k", who));
  if (q->tokens != 1) return fail(BF_EINVAL, "%s: q has %llu tokens per answer instead of 1", who, (unsigned long long)q->tokens);
  if (q->dim > 256) return fail(BF_EINVAL, "%s: vectors of more than 256 dimensions", who);
  if (pk->dim != q->dim || pk->dtype != q->dtype)
    return fail(BF_EINVAL, "%s: prefix_k has other dimensions or another type than q", who);
  if (q->heads % pk->heads) return fail(BF_EINVAL, "%s: the heads of q are no multiple of those of prefix_k", who);
  if (q->batch && (pk->batch == 0 || q->batch % pk->batch))
    return fail(BF_EINVAL, "%s: the answers are no multiple of the prompts", who);
  if (sk) {
    if (sk->batch != q->batch) return fail(BF_EINVAL, "%s: suffix_k has not one sequence per answer", who);
    if (sk->heads != pk->heads || sk->dim != q->dim || sk->dtype != q->dtype)
      return fail(BF_EINVAL, "%s: suffix_k has other heads, dimensions or another type than prefix_k", who);
  }
  if (q->batch * q->heads > kMaxRows) return fail(BF_EINVAL, "%s: more than 2^31 - 1 query vectors", who);
  *a = bfk::AttendArgs{};
  a->prompts = (uint32_t)pk->batch;
  a->per_prompt = q->batch ? (uint32_t)(q->batch / pk->batch) : 0;
  a->kv_heads = (uint32_t)pk->heads;
  a->share = (uint32_t)(q->heads / pk->heads);
  a->dim = (uint32_t)q->dim;
  a->dtype = q->dtype;
  a->prefix_cap = pk->tokens;
  a->suffix_cap = sk ? sk->tokens : 0;
  return BF_OK;
}

// Where row r's bytes end, from its first on.
uint64_t row_extent(const bf_states* s) {
  return (s->tokens - 1) * s->token_stride + (s->heads - 1) * s->head_stride + s->width;
}

int check_states(const bf_states* s, const char* name, const char* who) {
  if (!s) return fail(BF_EINVAL, "%s: %s is NULL", who, name);
  if (s->rows > kMaxRows || s->tokens > kMaxRows || s->heads > kMaxRows || s->width > kMaxRows)
    return fail(BF_EINVAL, "%s: %s has more than 2^31 - 1 rows, tokens, heads or bytes", who, name);
  if (s->heads && s->width > kMaxRows / s->heads) return fail(BF_EINVAL, "%s: %s has tokens of 2^31 bytes or more", who, name);
  if (!stride_fits(s->rows, s->row_stride) || !stride_fits(s->tokens, s->token_stride) || !stride_fits(s->heads, s->head_stride))
    return fail(BF_EINVAL, "%s: %s spans more than 2^42 bytes", who, name);
  return BF_OK;
}

// Whether rows of a layout share bytes with each other, or a row's runs do.
bool folded(const bf_states* s) {
  struct Dim {
    uint64_t n, stride;
  } d[3] = {{s->rows, s->row_stride}, {s->tokens, s->token_stride}, {s->heads, s->head_stride}};
  for (int i = 0; i < 3; ++i)  // smallest stride first, dimensions of one ahead
    for (int j = i + 1; j < 3; ++j)
      if ((d[i].n > 1 ? d[i].stride : 0) > (d[j].n > 1 ? d[j].stride : 0)) {
        const Dim t = d[i];
        d[i] = d[j];
        d[j] = t;
      }
  uint64_t run = s->width;
  for (const Dim& x : d) {
    if (x.n < 2) continue;
    if (x.stride < run) return true;
    run = (x.n - 1) * x.stride + run;
  }
  return false;
}

// From an array's first byte to behind its last.
uint64_t whole_extent(const bf_states* s) { return (s->rows - 1) * s->row_stride + row_extent(s); }

// Whether two arrays share bytes; ones of the same layout may lie between each other's rows.
bool overlap(const void* a, const bf_states* la, const void* b, const bf_states* lb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  const uint64_t ea = whole_extent(la), eb = whole_extent(lb);
  if (x >= y + eb || y >= x + ea) return false;
  const uint64_t r = la->row_stride;
  if (la->rows < 2 || r != lb->row_stride || r == 0 || row_extent(la) > r || row_extent(lb) > r) return true;
  const uint64_t d = y >= x ? (y - x) % r : (r - (x - y) % r) % r;  // b's rows behind a's
  return d < row_extent(la) || r - d < row_extent(lb);
}

}  // namespace

}  // namespace bfcapi

using namespace bfcapi;

extern "C" {

int bf_prefix_attention_workspace(const bf_cache* q, const bf_cache* prefix_k, const bf_cache* suffix_k, uint64_t* bytes) {
  const char* who = "bf_prefix_attention_workspace";
  if (!bytes) return fail(BF_EINVAL, "%s: bytes is NULL", who);
  bfk::AttendArgs a;
  BF_TRY(attend_sizes(q, prefix_k, suffix_k, &a, who));
  *bytes = bfk::attend_bytes(a);
  return BF_OK;
}

int bf_prefix_attention(const bf_cache* q, const bf_cache* prefix_k, const bf_cache* prefix_v, const bf_cache* suffix_k,
                        const bf_cache* suffix_v, const bf_attention_args* args, const bf_cache* out, float* d_lse,
                        void* d_workspace, uint64_t workspace_bytes, void* cuda_stream) {
  const char* who = "bf_prefix_attention";
  bfk::AttendArgs a;
  BF_TRY(attend_sizes(q, prefix_k, suffix_k, &a, who));
  BF_TRY(check_cache(prefix_v, "prefix_v", who));
  BF_TRY(check_like(prefix_v, prefix_k, "prefix_v", "prefix_k", who));
  if ((suffix_k == nullptr) != (suffix_v == nullptr))
    return fail(BF_EINVAL, "%s: only one of suffix_k and suffix_v is NULL", who);
  if (suffix_v) {
    BF_TRY(check_cache(suffix_v, "suffix_v", who));
    BF_TRY(check_like(suffix_v, suffix_k, "suffix_v", "suffix_k", who));
  }
  if (!args) return fail(BF_EINVAL, "%s: args is NULL", who);
  BF_TRY(check_array(args->prefix_lengths, 0, 8, "prefix_lengths", who));
  BF_TRY(check_array(args->suffix_lengths, 0, 8, "suffix_lengths", who));
  BF_TRY(check_number(args->scale, std::fabs(args->scale) <= 1e30f, "scale", who));
  BF_TRY(check_cache(out, "out", who));
  BF_TRY(check_like(out, q, "out", "q", who));
  if (folded(out)) return fail(BF_EINVAL, "%s: vectors of out overlap", who);
  BF_TRY(check_array(d_lse, 0, 4, "lse", who));
  const Bytes outputs[] = {bytes_of(out, "out"), {d_lse, q->batch * q->heads * 4, "lse"}};
  const Bytes inputs[] = {bytes_of(q, "q"),
                          bytes_of(prefix_k, "prefix_k"),
                          bytes_of(prefix_v, "prefix_v"),
                          bytes_of(suffix_k, "suffix_k"),
                          bytes_of(suffix_v, "suffix_v"),
                          {args->prefix_lengths, prefix_k->batch * 8, "prefix_lengths"},
                          {suffix_k ? args->suffix_lengths : nullptr, q->batch * 8, "suffix_lengths"}};
  for (const Bytes& o : outputs)
    for (const Bytes& i : inputs)
      if (overlap(o, i)) return fail(BF_EINVAL, "%s: %s overlaps %s", who, o.name, i.name);
  if (overlap(outputs[0], outputs[1])) return fail(BF_EINVAL, "%s: out overlaps lse", who);
  if (q->batch == 0) return BF_OK;
  const uint64_t need = bfk::attend_bytes(a);
  BF_TRY(check_workspace(d_workspace, workspace_bytes, need, who));
  a.q = vectors(q);
  a.pk = vectors(prefix_k);
  a.pv = vectors(prefix_v);
  a.sk = vectors(suffix_k);
  a.sv = vectors(suffix_v);
  a.out = vectors(out);
  a.lse = d_lse;
  a.prefix_len = args->prefix_lengths;
  a.suffix_len = suffix_k ? args->suffix_lengths : nullptr;
  a.scale2 = (float)((double)args->scale * 1.44269504088896340736);
  const cudaError_t e = bfk::launch_attend(a, d_workspace, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? BF_OK : cuda_fail(e, who);
}

int bf_beam_step_workspace(uint64_t groups, uint32_t beams, uint64_t vocab, uint32_t keep, uint64_t* bytes) {
  const char* who = "bf_beam_step_workspace";
  if (!bytes) return fail(BF_EINVAL, "%s: bytes is NULL", who);
  if (beams == 0 || beams > BF_MAX_BEAMS || keep == 0 || keep > BF_MAX_BEAMS)
    return fail(BF_EINVAL, "%s: beams and keep must be 1 to %d", who, BF_MAX_BEAMS);
  if (groups > kMaxRows / BF_MAX_BEAMS || vocab == 0 || vocab > kMaxVocab)
    return fail(BF_EINVAL, "%s: more than 2^23 - 1 groups, or a vocabulary of 0 or over 2^24", who);
  *bytes = bfk::beam_bytes((uint32_t)groups, beams, vocab, keep);
  return BF_OK;
}

int bf_beam_step(const bf_matrix* logits, const bf_beam_args* args, float* d_scores, int64_t* d_tokens, int64_t* d_parents,
                 uint8_t* d_finished, int64_t* d_lengths, void* d_workspace, uint64_t workspace_bytes, void* cuda_stream) {
  const char* who = "bf_beam_step";
  BF_TRY(check_matrix(logits, "logits", who));
  if (!args) return fail(BF_EINVAL, "%s: args is NULL", who);
  uint64_t need = 0;
  BF_TRY(bf_beam_step_workspace(args->groups, args->beams, logits->cols, args->keep, &need));
  if (logits->rows != args->groups * args->beams) return fail(BF_EINVAL, "%s: logits has not groups * beams rows", who);
  BF_TRY(check_array(args->scores, logits->rows, 4, "scores", who));
  BF_TRY(check_array(args->lengths, 0, 8, "lengths", who));
  if (args->end_token < -1) return fail(BF_EINVAL, "%s: end_token is below -1", who);
  if (args->finished && args->end_token < 0) return fail(BF_EINVAL, "%s: finished beams need an end_token", who);
  BF_TRY(check_number(args->length_penalty, args->length_penalty >= 0.0f && args->length_penalty <= 65536.0f, "length_penalty", who));
  if (args->length_penalty > 0.0f && !args->lengths && logits->rows)
    return fail(BF_EINVAL, "%s: a length penalty needs lengths", who);
  BF_TRY(check_temperature(args->temperature, who));
  const uint64_t places = args->groups * args->keep;
  BF_TRY(check_array(d_scores, places, 4, "out scores", who));
  BF_TRY(check_array(d_tokens, places, 8, "out tokens", who));
  BF_TRY(check_array(d_parents, places, 8, "out parents", who));
  BF_TRY(check_array(d_lengths, 0, 8, "out lengths", who));
  if (d_lengths && !args->lengths && logits->rows) return fail(BF_EINVAL, "%s: out lengths need lengths", who);
  if (args->groups == 0) return BF_OK;
  if (need) BF_TRY(check_workspace(d_workspace, workspace_bytes, need, who));
  // What a group reads again may not be what another one has written.
  const struct {
    const void* data;
    uint64_t bytes;
  } arrays[] = {{d_scores, places * 4}, {d_tokens, places * 8}, {d_parents, places * 8}, {d_finished, places}, {d_lengths, places * 8},
                {args->scores, logits->rows * 4}, {args->finished, logits->rows}, {args->lengths, logits->rows * 8},
                {logits->data, ((logits->rows - 1) * logits->row_stride + logits->cols) * (logits->dtype == BF_F32 ? 4 : 2)}};
  for (uint32_t i = 0; i < 5; ++i)
    for (uint32_t j = i + 1; j < 9; ++j)
      if (arrays[i].data && arrays[j].data && (uintptr_t)arrays[i].data < (uintptr_t)arrays[j].data + arrays[j].bytes &&
          (uintptr_t)arrays[j].data < (uintptr_t)arrays[i].data + arrays[i].bytes)
        return fail(BF_EINVAL, "%s: an output overlaps an input or another output", who);
  bfk::BeamArgs a = {};
  a.x = logits->data;
  a.ldx = logits->row_stride;
  a.vocab = (uint32_t)logits->cols;
  a.dtype = logits->dtype;
  a.groups = (uint32_t)args->groups;
  a.beams = args->beams;
  a.keep = args->keep;
  a.scores = args->scores;
  a.finished = args->finished;
  a.lengths = args->lengths;
  a.end_token = args->end_token;
  a.penalty = args->length_penalty;
  a.tau = args->temperature;
  a.c2 = (float)(1.44269504088896340736 / (double)args->temperature);
  a.out_scores = d_scores;
  a.out_tokens = d_tokens;
  a.out_parents = d_parents;
  a.out_finished = d_finished;
  a.out_lengths = d_lengths;
  const cudaError_t e = bfk::launch_beam_step(a, d_workspace, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? BF_OK : cuda_fail(e, who);
}

int bf_beam_reorder(void* const* from, const bf_states* from_layout, void* const* to, const bf_states* to_layout,
                    uint32_t count, const int64_t* d_parents, uint32_t beams, const int64_t* d_lengths, void* cuda_stream) {
  const char* who = "bf_beam_reorder";
  BF_TRY(check_states(from_layout, "from_layout", who));
  BF_TRY(check_states(to_layout, "to_layout", who));
  const bf_states *f = from_layout, *t = to_layout;
  if (f->rows != t->rows || f->tokens != t->tokens || f->heads != t->heads || f->width != t->width)
    return fail(BF_EINVAL, "%s: to_layout has another shape than from_layout", who);
  if (count > BF_MAX_STATES) return fail(BF_EINVAL, "%s: more than %d arrays", who, BF_MAX_STATES);
  if (beams == 0 || beams > BF_MAX_BEAMS) return fail(BF_EINVAL, "%s: beams must be 1 to %d", who, BF_MAX_BEAMS);
  if (f->rows % beams) return fail(BF_EINVAL, "%s: the rows are no multiple of the beams", who);
  BF_TRY(check_array(d_parents, f->rows, 8, "parents", who));
  BF_TRY(check_array(d_lengths, 0, 8, "lengths", who));
  if (count && (!from || !to)) return fail(BF_EINVAL, "%s: from or to is NULL", who);
  if (count == 0 || f->rows == 0 || f->tokens == 0 || f->heads == 0 || f->width == 0) return BF_OK;
  if (folded(t)) return fail(BF_EINVAL, "%s: rows of to_layout overlap", who);
  const bool same = (f->rows < 2 || f->row_stride == t->row_stride) && (f->tokens < 2 || f->token_stride == t->token_stride) &&
                    (f->heads < 2 || f->head_stride == t->head_stride);
  bfk::ReorderArgs a = {};
  for (uint32_t k = 0; k < count; ++k) {
    if (!from[k] || !to[k]) return fail(BF_EINVAL, "%s: array %u is NULL", who, k);
    a.from[k] = static_cast<const char*>(from[k]);
    a.to[k] = static_cast<char*>(to[k]);
  }
  // What every block reads again may not be what another one has written.
  const Bytes read[] = {{d_parents, f->rows * 8, "parents"}, {d_lengths, f->rows * 8, "lengths"}};
  for (uint32_t k = 0; k < count; ++k)
    for (const Bytes& r : read)
      if (overlap({to[k], whole_extent(t), "to"}, r)) return fail(BF_EINVAL, "%s: array %u of to overlaps %s", who, k, r.name);
  const bool in_place = same && from[0] == to[0];
  for (uint32_t k = 0; k < count; ++k) {
    if (in_place != (same && from[k] == to[k])) return fail(BF_EINVAL, "%s: only some of the arrays are reordered in place", who);
    for (uint32_t j = 0; j < count; ++j) {
      if (j < k && overlap(to[j], t, to[k], t)) return fail(BF_EINVAL, "%s: arrays %u and %u of to overlap", who, j, k);
      if (!in_place && overlap(from[j], f, to[k], t))
        return fail(BF_EINVAL, "%s: array %u of to overlaps array %u of from", who, k, j);
    }
  }
  a.from_row = f->row_stride;
  a.from_token = f->token_stride;
  a.from_head = f->head_stride;
  a.to_row = t->row_stride;
  a.to_token = t->token_stride;
  a.to_head = t->head_stride;
  a.tokens = f->tokens;
  a.width = f->width;
  a.heads = (uint32_t)f->heads;
  a.count = count;
  a.groups = (uint32_t)(f->rows / beams);
  a.beams = beams;
  a.parents = d_parents;
  a.lengths = d_lengths;
  a.in_place = in_place;
  const cudaError_t e = bfk::launch_reorder(a, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? BF_OK : cuda_fail(e, who);
}

}  // extern "C"
