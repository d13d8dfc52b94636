// bf_rows.cuh -- the arithmetic of one row of logits, shared by the kernels in
// bf_rows.cu.
//
// With x the row's logits, y its token and tau the temperature:
//   m = max_j x_j,  t_j = (x_j - m) log2(e) / tau,  e_j = 2^t_j,  s = sum_j e_j,  q = sum_j e_j t_j
//   log-probability  lp = (x_y - m) / tau - ln s
//   entropy          H  = ln s - ln2 q / s
// and for a loss with slopes A = dL/dlp and C = dL/dH of this row,
//   dL/dx_j = e_j (B + D t_j) + [j = y] A / tau
//   B = -(A + C (H - ln s)) / (tau s),  D = -C ln2 / (tau s).
// x - m is taken before the product with log2(e)/tau: a row of the type's
// lowest values would overflow in x log2(e)/tau, and here has m among them.
// log2(e)/tau is held in two parts: its rounding alone shifts every ln s of a
// batch the same way (by up to 6e-8 |t|), and a preference loss adds some
// hundred of them up to a reward.
#pragma once

#include "bf_elem.cuh"
#include "bf_launches.cuh"
#include "bf_learn.h"

namespace bfk {

constexpr float kLn2 = 0.693147180559945309f;
constexpr float kMinusInf = -__builtin_huge_valf();

__device__ __forceinline__ float exp2_fast(float t) {
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t));
  return e;
}

// log2(e) / tau = hi + lo with lo > 0, so that an infinite product has one sign.
struct Scale {
  float hi, lo, inv_tau;
  // A difference of logits as an exponent of 2, and its exponential.
  __device__ __forceinline__ float of(float d) const { return fmaf(d, lo, d * hi); }
  __device__ __forceinline__ float exp_of(float d) const { return expf(d * inv_tau); }
};

// ex2.approx cuts its result off: evenly over an octave its values are 5.0e-8 too
// small on average (measured in 2^20 points of each of 12), except at 0.  The
// probabilities do not mind, their sum being as much too small; ln s does, as
// above, so ln s is put right by the share of s that is short, and sums are joined
// by expf.  With 4.0e-8 log-probabilities of normal logits are off by 5e-9 on
// average at 3 to 10,000 of them, 1.2e-8 at 100,000 (torch's in 32 bits: 3e-9 at 3,
// 1.2e-8 at 1,000, 1.8e-8 at 100,000); with 5.0e-8 by 7e-9 and 2.0e-8.  Logits of
// another distribution, whose exponents fill their octaves otherwise, have another mean.
constexpr float kExp2Short = 4.0e-8f;

// ln v + more = big + low for a v that is 0 (any value then), NaN or normal.  `more` is below half a last place of v and
// of ln v, where it would mostly be rounded away; low is small (|low| < 0.42) and keeps it.  v = 2^k f with f in [3/4,
// 3/2), and Cody and Waite's ln 2 = 355/512 - 2.12e-4, of which k times the first is exact.
struct Log {
  float big, low;
};
__device__ __forceinline__ Log log_of(float v, float more) {
  const int bits = __float_as_int(v), k = (bits - __float_as_int(0.75f)) >> 23;
  const float low = logf(__int_as_float(bits - k * (1 << 23))) + fmaf((float)k, -2.12194440054690583e-4f, more);
  return {(float)k * 0.693359375f, v == v ? low : v};
}
// a - l, rounded once but for what rounds `low`.
__device__ __forceinline__ float less(float a, const Log& l) {
  const float d = a - l.big, part = d - a, left = (a - (d - part)) - (l.big + part);
  return fabsf(d) < -kMinusInf ? d + (left - l.low) : d - l.low;
}

// Maximum, sum and first moment of the exponentials of some of a row's logits,
// and how much of the sum came from exponents of 0.
// m is -inf, the others 0 where there is no logit above -inf.
struct RowSums {
  float m, s, q, one;
};

// t as a factor beside e = 2^t: where e is 0, a finite one (0 * -inf would be NaN).
__device__ __forceinline__ float finite_t(float t) { return fmaxf(t, -160.0f); }

// The max that exponents are taken against: 0 in a row without a logit above -inf.
__device__ __forceinline__ float usable_max(float m) { return m == kMinusInf ? 0.0f : m; }

// r's sums against the maximum m (>= r.m).
__device__ __forceinline__ RowSums against(const RowSums& r, float m, const Scale& c) {
  const float d = r.m - usable_max(m), e = c.exp_of(d);
  return {m, e * r.s, e * (r.q + finite_t(c.of(d)) * r.s), e * r.one};
}

__device__ __forceinline__ RowSums join(const RowSums& a, const RowSums& b, const Scale& c) {
  const float m = fmaxf(a.m, b.m);
  const RowSums x = against(a, m, c), y = against(b, m, c);
  return {m, x.s + y.s, x.q + y.q, x.one + y.one};
}

__device__ __forceinline__ Scale scale_of(const RowArgs& a) { return {a.c2_hi, a.c2_lo, a.inv_tau}; }

// What a row brings besides its logits.
struct RowIn {
  bool on;          // scored
  bool known;       // its token is inside the vocabulary
  uint32_t y;
  float xy;         // its token's logit
  float w;          // kPolicy: its weight in the loss
  float old_lp, ref_lp, adv;
  float slope_lp, slope_h;  // kScoreGrad; slope_lp also kPairGrad
};

// What its gradient is made from, and its terms of the loss.
struct RowOut {
  float m;          // usable max
  float b, d, hit;  // dL/dx_j = e_j (b + d t_j), plus hit at the token
  float sums[kPolicySums];
};

// Whether an op's rows depend on work that its own launch may overlap: what the
// kernels before it in the call write is read after wait_for_previous().
template <RowOp op>
constexpr bool kFollows = op == RowOp::kPolicy || op == RowOp::kPairScore || op == RowOp::kPairGrad;

// The part of a row that the caller's arrays give.
template <typename E, RowOp op>
__device__ __forceinline__ RowIn load_row(const RowArgs& a, uint64_t row) {
  RowIn in = {};
  const int64_t y = a.tokens[row];
  in.on = y >= 0;
  in.known = y < (int64_t)a.vocab;
  in.y = (uint32_t)y;
  if constexpr (op == RowOp::kScoreGrad) {
    in.slope_lp = a.grad_logprob[row];
    if (a.grad_entropy) in.slope_h = a.grad_entropy[row];
  }
  if constexpr (op == RowOp::kPolicy) {
    in.old_lp = a.old_logprob[row];
    if (a.ref_logprob) in.ref_lp = a.ref_logprob[row];
    if (a.advantage_per_token) in.adv = a.advantage[row];
  }
  if (in.on && in.known) in.xy = to_f32(static_cast<const E*>(a.x)[row * a.ldx + in.y]);
  return in;
}

// The part that the call's earlier kernels give; a row of no sequence is not scored.
template <RowOp op>
__device__ __forceinline__ void load_row_late(const RowArgs& a, uint64_t row, RowIn& in) {
  if constexpr (kFollows<op>) {
    const uint32_t seq = a.row_seq[row];
    in.on = seq != kNoSequence;
    if (!in.on) return;
    if constexpr (op == RowOp::kPolicy) {
      in.w = a.reduction == BF_MEAN_TOKENS ? 1.0f / (float)a.counts->tokens
             : a.reduction == BF_MEAN_SEQUENCES ? 1.0f / ((float)a.seq_tokens[seq] * (float)a.counts->sequences) : 1.0f;
      if (!a.advantage_per_token) in.adv = a.advantage[seq];
    }
    if constexpr (op == RowOp::kPairGrad) in.slope_lp = a.seq_slope[seq];
  }
}

// The row's outputs from its sums (written by the caller's leading thread) and
// its gradient's factors.  A token outside the vocabulary makes its row's values
// NaN, whatever its logits; else a row without a logit above -inf has
// log-probability -inf, entropy 0, loss term 0 and gradient 0.
template <RowOp op>
__device__ __forceinline__ RowOut finish_row(const RowArgs& a, uint64_t row, const RowIn& in, const RowSums& r,
                                             bool leader) {
  RowOut o = {};
  if (!in.on) {
    if (leader) {
      if (a.logprob) a.logprob[row] = 0.0f;
      if (a.entropy) a.entropy[row] = 0.0f;
    }
    return o;
  }
  if constexpr (op == RowOp::kPairGrad) {  // from what its scoring pass kept
    const float2 kept = a.row_softmax[row];
    const float slope = in.known ? in.slope_lp * a.inv_tau : __int_as_float(0x7FC00000);
    o.m = kept.x;
    if (kept.y == 0.0f && in.known) return o;  // no logit above -inf: 0 whatever the pair's slope
    o.b = -slope * kept.y;
    o.hit = slope;
    return o;
  }
  const bool none = r.s == 0.0f;
  o.m = usable_max(r.m);
  const float inv_s = none ? 0.0f : 1.0f / r.s;
  const Log log_s = log_of(r.s, kExp2Short * (r.s - r.one) * inv_s);
  const float ln_s = log_s.big + log_s.low;
  float lp = none ? kMinusInf : less((in.xy - o.m) / a.tau, log_s);
  float h = none ? 0.0f : ln_s - kLn2 * r.q * inv_s;
  if (!in.known) lp = h = __int_as_float(0x7FC00000);
  if (leader) {
    if (a.logprob) a.logprob[row] = lp;
    if (a.entropy) a.entropy[row] = h;
  }
  if constexpr (op == RowOp::kPairScore) {
    if (leader) a.row_softmax[row] = make_float2(o.m, inv_s);
  }
  if constexpr (op == RowOp::kScore || op == RowOp::kPairScore) return o;
  if (none && in.known) return o;
  float slope_lp = in.known ? in.slope_lp : lp, slope_h = in.slope_h;
  if constexpr (op == RowOp::kPolicy) {
    const float ratio = expf(lp - in.old_lp);
    const bool clipped = in.adv >= 0.0f ? ratio > a.ratio_hi : ratio < a.ratio_lo;
    const float held = clipped ? (in.adv >= 0.0f ? a.ratio_hi : a.ratio_lo) : ratio;
    float kl = 0.0f;
    slope_lp = clipped ? 0.0f : -in.adv * ratio;
    if (a.ref_logprob) {
      const float u = in.ref_lp - lp, em1 = expm1f(u);
      kl = u == -kMinusInf ? u : em1 - u;
      if (a.kl_coef != 0.0f) slope_lp -= a.kl_coef * em1;  // e^u may be infinite, and 0 of it is nothing
    }
    o.sums[0] = in.w * held * in.adv;
    o.sums[1] = in.w * kl;
    o.sums[2] = in.w * h;
    o.sums[3] = clipped ? in.w : 0.0f;
    o.sums[4] = in.w * ratio;
    slope_lp *= in.w * a.grad_scale;
    slope_h = -a.entropy_coef * in.w * a.grad_scale;
  }
  o.b = -(slope_lp + slope_h * (h - ln_s)) * a.inv_tau * inv_s;
  o.d = -slope_h * kLn2 * a.inv_tau * inv_s;
  o.hit = slope_lp * a.inv_tau;
  return o;
}

// A logit's gradient, without the token's own part.
__device__ __forceinline__ float logit_grad(const RowOut& o, float x, Scale c) {
  const float t = c.of(x - o.m);
  return exp2_fast(t) * fmaf(o.d, finite_t(t), o.b);
}

// The sums of `lanes` neighbouring lanes (a power of two) joined, in all of them.
__device__ __forceinline__ RowSums lanes_join(RowSums r, const Scale& c, uint32_t lanes) {
  float m = r.m;
  for (uint32_t o = lanes / 2; o; o /= 2) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
  r = against(r, m, c);
  for (uint32_t o = lanes / 2; o; o /= 2) {
    r.s += __shfl_xor_sync(~0u, r.s, o);
    r.q += __shfl_xor_sync(~0u, r.q, o);
    r.one += __shfl_xor_sync(~0u, r.one, o);
  }
  return r;
}

// One pair, from both answers' sums of lp - ref and numbers of scored rows: the
// rewards beta * sum (or beta * mean), the loss of their gap
//   h = reward_0 - reward_1 - margin,  l = -(1 - eps) ln sigma(h) - eps ln sigma(-h)
// and the slopes of the mean loss in each answer's log-probabilities.
__device__ __forceinline__ void finish_pair(const PairArgs& a, uint64_t p, const float (&sum)[2], const uint32_t (&n)[2]) {
  float share[2], reward[2];
#pragma unroll
  for (uint32_t k = 0; k < 2; ++k) {
    share[k] = a.beta * (a.average && n[k] ? 1.0f / (float)n[k] : 1.0f);
    reward[k] = share[k] * sum[k];
    a.rewards[2 * p + k] = reward[k];
  }
  const float h = reward[0] - reward[1] - a.margin, eps = a.label_smoothing;
  const float tail = log1pf(expf(-fabsf(h)));  // ln(1 + e^-|h|)
  const float slope = (eps / (1.0f + expf(-h)) - (1.0f - eps) / (1.0f + expf(h))) * a.grad_scale / (float)a.pairs;
  a.seq_slope[2 * p] = slope * share[0];
  a.seq_slope[2 * p + 1] = -slope * share[1];
  const float smooth = eps > 0.0f ? eps * (fmaxf(h, 0.0f) + tail) : 0.0f;  // the gap may be infinite: a banned token
  a.partial[p] = (1.0f - eps) * (fmaxf(-h, 0.0f) + tail) + smooth;
}

// Sums of N values over the block's threads: the k-th in thread k.  Every thread of the block calls it with the same
// `lanes`: only every lanes-th one (a power of two, at most 32) brings values.  buf: N floats per warp, not in use.
template <uint32_t N>
__device__ __forceinline__ float block_sums(float (&v)[N], float* buf, uint32_t lanes = 1) {
#pragma unroll
  for (uint32_t k = 0; k < N; ++k)
    for (uint32_t o = 16; o >= lanes && o; o /= 2) v[k] += __shfl_down_sync(~0u, v[k], o);
  if (threadIdx.x % 32 == 0) {
#pragma unroll
    for (uint32_t k = 0; k < N; ++k) buf[threadIdx.x / 32 * N + k] = v[k];
  }
  __syncthreads();
  float sum = 0.0f;
  if (threadIdx.x < N)
    for (uint32_t w = 0; w < blockDim.x / 32; ++w) sum += buf[w * N + threadIdx.x];
  return sum;
}

// The preference loss from its pairs, once all are visible; every thread of the block calls it.  buf: 4 floats per warp.
__device__ __forceinline__ void preference_stats(const PairArgs& a, float* buf) {
  float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (uint64_t p = threadIdx.x; p < a.pairs; p += blockDim.x) {
    const float r0 = __ldcg(a.rewards + 2 * p), r1 = __ldcg(a.rewards + 2 * p + 1);
    v[0] += __ldcg(a.partial + p);
    v[1] += r0 > r1 ? 1.0f : 0.0f;
    v[2] += r0;
    v[3] += r1;
  }
  const float total = block_sums(v, buf);
  if (threadIdx.x < 4) a.stats[threadIdx.x] = total / (float)a.pairs;
}

// The last s in [0, sequences) with offsets[s] <= row, by halving [lo, hi).
template <typename T, typename I>
__device__ __forceinline__ I last_at_or_before(const T* offsets, I lo, I hi, T row) {
  while (hi - lo > 1) {
    const I mid = (lo + hi) / 2;
    if (offsets[mid] <= row) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Offsets as 32-bit rows, those outside [0, rows] moved to its ends: a row is before the same ones.
__device__ __forceinline__ uint32_t clamp_offset(int64_t o, uint32_t rows) {
  return o < 0 ? 0u : o > (int64_t)rows ? rows : (uint32_t)o;
}

// The sequence of a row, from clamped offsets in shared memory.
__device__ __forceinline__ uint32_t sequence_at(const uint32_t* begin, uint32_t sequences, uint32_t row) {
  if (!sequences) return kNoSequence;
  const uint32_t s = last_at_or_before(begin, 0u, sequences, row);
  return begin[s] <= row && row < begin[s + 1] ? s : kNoSequence;
}

// Whether this block is the last of `blocks` to say so; called by the warp whose
// lanes wrote what the last one reads (last_sees() there).
__device__ __forceinline__ bool last_to_say(uint32_t* done, uint32_t blocks) {
  __syncwarp();
  uint32_t before = 0;
  if (threadIdx.x % 32 == 0) {
    __threadfence();
    before = atomicAdd(done, 1u);
  }
  return __shfl_sync(~0u, before, 0) == blocks - 1;
}
__device__ __forceinline__ void last_sees() { __threadfence(); }

}  // namespace bfk
