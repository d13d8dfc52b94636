"""The operators that learn from makespans against their 64-bit forms (learn_ref.py).

Tolerances.  A log-probability is (x_y - m)/tau - ln s: two roundings of the first term, and ln of a sum whose relative
error is at most 2^-22 (ex2) + 2^-23 |t| of each term (t e^t is below 0.6) + a few 2^-24 of the summation: 1e-5 absolute
and 1e-6 relative hold with room for every size here.  A gradient is a product of such numbers: 5e-5 of the size of its
parts (the ratio e^(lp - old) takes lp's absolute error as a relative one, and the policy's slope is the sum of a ratio's
and a KL term's part, which may cancel), plus one rounding to the output's type.
"""
import ctypes

import numpy as np
import pytest

import learn_ref as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_22242_gb300 import bf  # noqa: E402

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ROUND = {"f32": 2.0 ** -23, "bf16": 2.0 ** -8, "f16": 2.0 ** -10}     # twice half a unit in the last place
LEAST = {"f32": 1e-37, "bf16": 1e-37, "f16": 2.0 ** -24}              # below which a type rounds absolutely
INF = float("inf")


@pytest.fixture(scope="module", autouse=True)
def _built():
    assert torch.cuda.is_available()
    bf.load()


def gpu(a, dtype=torch.float32):
    return torch.as_tensor(np.asarray(a)).to(dtype).cuda()


def host(t):
    return t.double().cpu().numpy()


def make_logits(rng, rows, vocab, dtype, stride=0, shift=0, spread=2.0):
    """A (rows, vocab) view into a larger buffer of NaN, its base moved by `shift` elements, and its values."""
    width = vocab + stride
    buf = torch.full((rows * width + shift + 16,), float("nan"), dtype=TYPES[dtype], device="cuda")
    view = buf[shift:shift + rows * width].view(rows, width)[:, :vocab] if rows else torch.empty(
        0, vocab, dtype=TYPES[dtype], device="cuda")
    view.copy_(torch.from_numpy(rng.normal(0, spread, (rows, vocab))))
    return buf, view, host(view)


def make_tokens(rng, rows, vocab, off=0.15):
    y = rng.integers(0, vocab, rows)
    return np.where(rng.random(rows) < off, -1, y)


def close_scores(got, want):
    got = host(got)
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine])
    assert np.all(np.abs(got[fine] - want[fine]) <= 1e-5 + 1e-6 * np.abs(want[fine]))


def close_grad(got, want, size, dtype, factor=1.0):
    bound = factor * (5e-5 * size + ROUND[dtype] * np.abs(want)) + LEAST[dtype]
    off = np.abs(host(got) - factor * want)
    assert np.all(off <= bound), float((off / bound).max())


# rows x vocab, extra row stride, shift of the base (elements)
SHAPES = [(1, 1, 0, 0), (1, 3, 0, 0), (5, 2, 0, 1), (64, 3, 0, 0), (7, 3, 5, 1), (33, 31, 0, 0), (40, 8, 0, 0),
          (17, 33, 2, 3), (12, 64, 0, 0), (9, 255, 1, 0), (6, 256, 0, 0), (5, 1000, 0, 0), (4, 1009, 0, 7),
          (3, 2048, 8, 0), (3, 2050, 0, 2), (3, 4099, 0, 0), (2, 8191, 3, 1), (2, 16384, 0, 0), (3, 20011, 0, 5),
          (2, 32768, 0, 0), (2, 50001, 0, 0), (1, 131072, 0, 0), (2, 131073, 0, 1), (1, 270001, 0, 0),
          (200, 4096, 0, 0), (330, 1111, 0, 0), (1000, 40, 0, 0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,stride,shift", SHAPES)
def test_scores_and_gradient(rows, vocab, stride, shift, dtype):
    rng = np.random.default_rng([rows, vocab, stride])
    tau = (1.0, 0.7, 1.5)[(rows + vocab) % 3]
    buf, x, xd = make_logits(rng, rows, vocab, dtype, stride, shift)
    y = make_tokens(rng, rows, vocab)
    lp, h = bf.token_logprobs(x, gpu(y, torch.int64), temperature=tau, entropy=True)
    want_lp, want_h = R.scores(xd, y, tau)
    close_scores(lp, want_lp)
    close_scores(h, want_h)
    assert torch.equal(lp, bf.token_logprobs(x, gpu(y, torch.int64), temperature=tau))
    a, c = rng.normal(0, 1, rows).astype(np.float32), rng.normal(0, 0.1, rows).astype(np.float32)
    for entropy in (True, False):
        args = (gpu(y, torch.int64), gpu(a), gpu(c) if entropy else None)
        g = bf.token_logprobs_grad(x, *args, temperature=tau)
        want, size = R.scores_grad(xd, y, a.astype(np.float64), c.astype(np.float64) * entropy, tau)
        close_grad(g, want, size, dtype)
        # into another layout, and in place of the logits; what lies beside the rows stays
        other, out, _ = make_logits(rng, rows, vocab, dtype, stride=1, shift=shift + 1)
        around = torch.isnan(other).sum()
        bf.token_logprobs_grad(x, *args, temperature=tau, out=out)
        assert torch.equal(out, g) and torch.isnan(other).sum() == around
    around = torch.isnan(buf).sum()
    bf.token_logprobs_grad(x, *args, temperature=tau, out=x)
    assert torch.equal(x, g) and torch.isnan(buf).sum() == around


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [3, 40, 700, 3000, 20000])
@pytest.mark.parametrize("level,tau", [(0.0, 1e-3), (0.0, 1e3), (3e4, 1.0), (-3e4, 0.01), (900.0, 0.5), (0.0, 1e-18),
                                       (0.0, 1e18)])
def test_large_logits_and_temperatures(vocab, dtype, level, tau):
    """Logits far from 0 or divided by little: the exponents' differences are exact where their terms are large.  An
    exponent t is off by 2^-23 |t| and a log-probability as much as its own size, 1e-6 of it.  An exponential below 2^-126
    is taken as 0: its part of the gradient, (|a| + 100 |c|) 2^-126 / tau at most, is missing."""
    rng = np.random.default_rng(vocab)
    buf, x, _ = make_logits(rng, 9, vocab, dtype)
    x.add_(level)
    xd = host(x)
    y = make_tokens(rng, 9, vocab)
    tau = float(np.float32(tau))
    lp, h = bf.token_logprobs(x, gpu(y, torch.int64), temperature=tau, entropy=True)
    want_lp, want_h = R.scores(xd, y, tau)
    close_scores(lp, want_lp)
    close_scores(h, want_h)
    a, c = rng.normal(0, 1, 9).astype(np.float32), rng.normal(0, 0.1, 9).astype(np.float32)
    g = bf.token_logprobs_grad(x, gpu(y, torch.int64), gpu(a), gpu(c), temperature=tau)
    want, size = R.scores_grad(xd, y, a.astype(np.float64), c.astype(np.float64), tau)
    big = np.abs(want) > 65504 if dtype == "f16" else np.abs(want) > 3e38  # beyond the type's range: infinite
    got = host(g)
    assert np.all(np.isinf(got[big]) | (np.abs(got[big]) > 6e4))
    flushed = (np.abs(a) + 100 * np.abs(c)).astype(np.float64)[:, None] * 2.0 ** -126 / tau
    bound = 5e-5 * size + ROUND[dtype] * np.abs(want) + LEAST[dtype] + flushed
    fine = ~big & (np.abs(want) + bound < (65504 if dtype == "f16" else 3e38))
    assert np.all(np.abs(got[fine] - want[fine]) <= bound[fine])


@pytest.mark.parametrize("vocab,rows", [(3, 60000), (390, 8000), (6000, 4000), (50001, 1000)])
def test_scores_are_not_off_the_same_way(vocab, rows):
    """A preference loss adds hundreds of log-probabilities up, so what they are all off by counts.  Their errors are
    roundings to 32 bits (below 2^-21 each, of either sign: 4 standard deviations of their mean are allowed), and half a
    unit of the sum of exponentials where its last bit decides: 3e-8."""
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    x = torch.randn(rows, vocab, generator=gen, device="cuda") * 2
    y = torch.randint(vocab, (rows,), generator=gen, device="cuda")
    for tau in (1.0, 0.7):
        want = torch.log_softmax(x.double() / float(np.float32(tau)), 1).gather(1, y[:, None])[:, 0]
        off = (bf.token_logprobs(x, y, temperature=tau).double() - want).mean().item()
        assert abs(off) < 3e-8 + 4 * 2.0 ** -21 / np.sqrt(12 * rows), off


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [5, 40, 1500, 9000, 40000])
def test_masked_logits(dtype, vocab):
    """Banned tokens (-inf or the type's lowest value), rows with nothing left, values in rows that are not scored."""
    rng = np.random.default_rng(vocab)
    _, x, _ = make_logits(rng, 9, vocab, dtype)
    low = torch.finfo(TYPES[dtype]).min
    y = rng.integers(0, vocab, 9)
    x[0] = -INF
    x[1, 1:] = -INF
    y[1] = 0
    x[2, y[2]] = -INF
    x[3] = low
    x[4, rng.random(vocab) < 0.5] = low
    x[5] = float("nan")
    x[6] = INF
    y[5] = y[6] = -1
    x[7, rng.random(vocab) < 0.9] = -INF
    x[7, y[7]] = 3.0
    xd = host(x)
    a, c = rng.normal(0, 1, 9).astype(np.float32), rng.normal(0, 0.1, 9).astype(np.float32)
    for tau in (1.0, 0.5):
        lp, h = bf.token_logprobs(x, gpu(y, torch.int64), temperature=tau, entropy=True)
        want_lp, want_h = R.scores(xd, y, tau)
        got = host(lp)
        big = np.isfinite(want_lp) & (want_lp < -1e30)  # x_y is the lowest value: (x_y - m) / tau may pass 32 bits
        assert np.all((got[big] == -INF) | (np.abs(got[big] / want_lp[big] - 1) < 1e-5))
        close_scores(lp[~torch.from_numpy(big).cuda()], want_lp[~big])
        close_scores(h, want_h)
        g = bf.token_logprobs_grad(x, gpu(y, torch.int64), gpu(a), gpu(c), temperature=tau)
        want, size = R.scores_grad(xd, y, a.astype(np.float64), c.astype(np.float64), tau)
        close_grad(g, want, size, dtype)
        assert not g[0].any() and not g[5].any() and not g[6].any()


def test_values_that_are_no_numbers():
    """A token outside the vocabulary, NaN and +inf make their own row NaN and no other."""
    x = torch.zeros(4, 50, device="cuda")
    y = torch.tensor([50, 1, 2, 3], device="cuda")
    x[1, 7] = float("nan")
    x[2, 7] = INF
    lp, h = bf.token_logprobs(x, y, entropy=True)
    assert torch.isnan(lp).tolist() == [True, True, True, False]
    g = bf.token_logprobs_grad(x, y.clamp(max=49), torch.ones(4, device="cuda"))
    assert torch.isnan(g[1]).any() and torch.isnan(g[2]).any()
    assert not torch.isnan(g[0]).any() and not torch.isnan(g[3]).any()


# ---- policy loss ----

def policy_case(seed, lengths, vocab, dtype, tau=1.0, before=0, after=0, **layout):
    rng = np.random.default_rng(seed)
    offsets = np.concatenate([[0], np.cumsum(lengths)]) + before
    rows = int(offsets[-1]) + after
    buf, x, xd = make_logits(rng, rows, vocab, dtype, **layout)
    y = make_tokens(rng, rows, vocab)
    lp = R.scores(xd, np.maximum(y, 0), tau)[0]
    d = rng.normal(0, 0.25, rows)
    for edge in (np.log(0.8), np.log(1.3)):  # no ratio within 1e-3 of a clip edge: both sides clip alike
        d = np.where(np.abs(d - edge) < 1e-3, d + 4e-3, d)
    old = (lp - d).astype(np.float32)
    ref = (lp + rng.normal(0, 0.4, rows)).astype(np.float32)
    return dict(rng=rng, x=x, xd=xd, y=y, offsets=offsets, old=old, ref=ref, buf=buf, rows=rows,
                adv=rng.normal(0, 1, len(lengths)).astype(np.float32),
                adv_row=rng.normal(0, 1, rows).astype(np.float32))


def run_policy(c, **kw):
    per = kw.get("advantage_per_token", False)
    return bf.policy_loss(c["x"], gpu(c["y"], torch.int64), gpu(c["offsets"], torch.int64), gpu(c["old"]),
                          gpu(c["adv_row" if per else "adv"]), clip_high=0.3, **kw)


LENGTHS = {"ones": [1] * 5, "ragged": [3, 0, 7, 1, 0, 12, 2], "one": [19], "empty": [0, 0], "many": [4] * 50}
POLICY = [("tokens", 0.0, 0.0, 1.0, False), ("sequences", 0.2, 0.05, 0.7, False), ("sum", 0.1, 0.0, 1.3, True),
          ("tokens", 0.3, -0.02, 1.0, True)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("reduction,kl,entropy,tau,per", POLICY)
@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("vocab", [3, 37, 1009, 6000])
def test_policy(vocab, lengths, reduction, kl, entropy, tau, per, dtype):
    c = policy_case([vocab, len(lengths)], LENGTHS[lengths], vocab, dtype, tau, before=2, after=3)
    kw = dict(kl_coef=kl, entropy_coef=entropy, temperature=tau, reduction=reduction, advantage_per_token=per)
    got = run_policy(c, ref_logprob=gpu(c["ref"]) if kl else None, **kw)
    f64 = lambda v: v.astype(np.float64)
    stats, lp, g, size, _ = R.policy(c["xd"], c["y"], c["offsets"], f64(c["old"]), f64(c["adv_row" if per else "adv"]),
                                     f64(c["ref"]) if kl else None, 0.2, 0.3, kl, entropy, tau, reduction, per)
    close_scores(got.logprob, lp)
    total = max(1.0, float(np.abs(f64(c["adv_row"])).sum()) if reduction == "sum" else 4.0)
    assert np.all(np.abs(host(got.stats) - stats) <= 5e-5 * (total + np.abs(stats)))
    close_grad(got.grad, g, size, dtype)
    # the same bits again; without the gradient; scaled; in place
    again = run_policy(c, ref_logprob=gpu(c["ref"]) if kl else None, **kw)
    assert all(torch.equal(u, v) for u, v in zip(got, again))
    only = run_policy(c, ref_logprob=gpu(c["ref"]) if kl else None, grad=False, **kw)
    assert only.grad is None and torch.equal(only.stats, got.stats)
    scaled = run_policy(c, ref_logprob=gpu(c["ref"]) if kl else None, grad_scale=64.0, **kw)
    close_grad(scaled.grad, g, size, dtype, 64.0)
    same = run_policy(c, ref_logprob=gpu(c["ref"]) if kl else None, out=c["x"], **kw)
    assert same.grad is c["x"] and torch.equal(c["x"], got.grad) and torch.equal(same.stats, got.stats)


@pytest.mark.parametrize("vocab,lengths", [(50001, [5, 2]), (131072, [3]), (9, [40] * 200), (700, [33] * 20),
                                           (3, [10] * 20000), (16, [70000])])
def test_policy_sizes(vocab, lengths):
    """Large vocabularies, many rows, one long sequence: against the same formulas in 64 bits on the GPU."""
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    rows = sum(lengths)
    x = torch.randn(rows, vocab, generator=gen, device="cuda") * 2
    y = torch.randint(vocab, (rows,), generator=gen, device="cuda")
    offsets = torch.tensor([0] + np.cumsum(lengths).tolist(), device="cuda")
    z = torch.log_softmax(x.double(), 1)
    lp = z.gather(1, y[:, None])[:, 0]
    d = torch.randn(rows, generator=gen, device="cuda") * 0.05  # inside the clip's range
    old, ref = (lp - d.clamp(-0.15, 0.15)).float(), (lp + d).float()
    adv = torch.randn(len(lengths), generator=gen, device="cuda")
    got = bf.policy_loss(x, y, offsets, old, adv, ref, kl_coef=0.1, reduction="sequences")
    n = torch.tensor(lengths, device="cuda", dtype=torch.float64)
    seq = torch.repeat_interleave(torch.arange(len(lengths), device="cuda"), torch.tensor(lengths, device="cuda"))
    w = 1.0 / (n[seq] * len(lengths))
    r, u = torch.exp(lp - old.double()), ref.double() - lp
    k = torch.expm1(u) - u
    p = z.exp()
    h = -(p * z).sum(1)
    A = adv.double()[seq]
    want = torch.stack([(w * v).sum() for v in (-r * A + 0.1 * k, -r * A, k, h, torch.zeros_like(k), r)])
    assert torch.all((got.stats.double() - want).abs() <= 5e-5 * (4 + want.abs()))
    close_scores(got.logprob, lp.cpu().numpy())
    a, parts = w * (-A * r - 0.1 * torch.expm1(u)), w * ((A * r).abs() + 0.1 * (torch.exp(u) + 1))
    hit = torch.zeros_like(p).scatter_(1, y[:, None], 1.0)
    off = (got.grad.double() - a[:, None] * (hit - p)).abs()
    assert torch.all(off <= 5e-5 * parts[:, None] * (hit + p) + 1e-37)


def test_policy_edges():
    x = torch.randn(4, 6, device="cuda")
    y = torch.tensor([0, 1, 2, 3], device="cuda")
    old, adv = torch.zeros(4, device="cuda"), torch.ones(2, device="cuda")
    # no rows
    r = bf.policy_loss(x[:0], y[:0], torch.tensor([0, 0, 0], device="cuda"), old[:0], adv)
    assert r.stats.tolist() == [0.0] * 6 and r.grad.shape == (0, 6)
    # no sequences, and no scored row: nothing is scored
    for offsets, tokens, a in (([0], y, adv[:0]), ([0, 2, 4], y * 0 - 1, adv)):
        for reduction in bf.REDUCTIONS:
            r = bf.policy_loss(x, tokens, torch.tensor(offsets, device="cuda"), old, a, reduction=reduction)
            assert r.stats.tolist() == [0.0] * 6 and not r.grad.any() and not r.logprob.any()
    # offsets outside the rows, or that do not ascend: rows without a sequence are not scored, nothing faults
    for offsets in ([-7, 2, 900], [3, 1, 0], [-9, -8, -7], [1 << 40, 5, 1 << 41]):
        r = bf.policy_loss(x, y, torch.tensor(offsets, device="cuda"), old, adv)
        assert torch.isfinite(r.stats).all() and torch.isfinite(r.grad).all()
    # a row whose mask leaves nothing counts, with a term and a gradient of 0
    x[1] = -INF
    r = bf.policy_loss(x, y, torch.tensor([0, 2, 4], device="cuda"), old, adv, old, kl_coef=0.1, entropy_coef=0.1)
    assert torch.isfinite(r.stats).all() and torch.isfinite(r.grad).all() and r.logprob[1] == -INF
    assert not r.grad[1].any() and r.grad[0].any()


def test_policy_ratio_beyond_range():
    """A ratio that overflows is clipped for A >= 0 and multiplies nothing for A = 0."""
    x = torch.zeros(2, 4, device="cuda")
    y = torch.tensor([0, 1], device="cuda")
    old = torch.full((2,), -200.0, device="cuda")
    r = bf.policy_loss(x, y, torch.tensor([0, 1, 2], device="cuda"), old, torch.tensor([0.0, 1.0], device="cuda"))
    assert r.stats[1].item() == pytest.approx(-0.6) and not r.grad.any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(1000000, 3), (900, 3), (1000000, 7), (500000, 46), (200000, 455), (40000, 2500)])
def test_log_probabilities_are_not_off_to_one_side(rows, vocab, dtype):
    """A preference loss adds many up: their mean error is far below a rounding."""
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    errors = []
    for _ in range(max(1, 200000 // rows)):
        x = (torch.randn(rows, vocab, generator=gen, device="cuda") * 2).to(TYPES[dtype])
        y = torch.randint(vocab, (rows,), generator=gen, device="cuda")
        x[torch.arange(rows, device="cuda"), y] += (torch.rand(rows, generator=gen, device="cuda") * 4).to(TYPES[dtype])
        want = torch.cat([torch.log_softmax(x[a:a + 50000].double(), 1).gather(1, y[a:a + 50000, None])[:, 0]
                          for a in range(0, rows, 50000)])
        # a pair of half the rows each takes the way of few rows where there are few
        got = bf.preference_loss(x, y, torch.tensor([0, rows // 2, rows], device="cuda"), grad=False).logprob
        errors.append(got.double() - want)
    errors = torch.cat(errors)
    # A value's own roundings, of either sign, are a few 2^-24 of sizes up to 8, so their mean over n rows is within 4
    # standard errors of 0; what is left is held to 1e-8, a fifth of ex2.approx's shortfall of 5e-8.
    assert abs(errors.mean().item()) <= 1e-8 + 4 * errors.std().item() / len(errors) ** 0.5


# ---- preference loss ----

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("eps,margin,average,reference,tau", [(0.0, 0.0, False, True, 1.0), (0.1, 0.5, True, False, 0.7),
                                                              (0.2, -0.3, False, True, 1.2)])
@pytest.mark.parametrize("lengths", [[1, 1], [3, 0, 7, 1, 0, 12], [0, 0], [9, 30], [4] * 40])
@pytest.mark.parametrize("vocab", [3, 37, 1009, 6000])
def test_preference(vocab, lengths, eps, margin, average, reference, tau, dtype):
    c = policy_case([vocab, len(lengths)], lengths, vocab, dtype, tau, before=1, after=2, stride=vocab % 2)
    ref = c["ref"] if reference else None
    kw = dict(beta=0.3, label_smoothing=eps, margin=margin, average=average, temperature=tau)
    call = lambda **more: bf.preference_loss(c["x"], gpu(c["y"], torch.int64), gpu(c["offsets"], torch.int64),
                                             None if ref is None else gpu(ref), **kw, **more)
    got = call()
    stats, rewards, lp, g, size = R.preference(c["xd"], c["y"], c["offsets"],
                                               None if ref is None else ref.astype(np.float64), 0.3, eps, margin,
                                               average, tau)
    close_scores(got.logprob, lp)
    reach = 0.3 * (1e-5 + 1e-6 * np.abs(lp).max(initial=0)) * max(max(lengths), 1) + 1e-6
    assert np.all(np.abs(host(got.rewards) - rewards) <= reach + 1e-6 * np.abs(rewards))
    assert np.all(np.abs(host(got.stats) - stats) <= 2 * reach + 1e-5 * np.abs(stats))
    # a pair's slope moves by at most a quarter of its gap's error, and the sigmoid's own value is never below e^-|gap|
    close_grad(got.grad, g, size * (1 + 4e4 * reach), dtype)
    assert all(torch.equal(u, v) for u, v in zip(got, call()))
    only = call(grad=False)
    assert only.grad is None and torch.equal(only.stats, got.stats)
    close_grad(call(grad_scale=0.5).grad, g, size * (1 + 4e4 * reach), dtype, 0.5)
    call(out=c["x"])
    assert torch.equal(c["x"], got.grad)


@pytest.mark.parametrize("dtype,vocab,lengths,unscored", [
    ("bf16", 16384, [300, 280, 1, 0, 0, 0, 700, 3, 20, 900, 33, 34, 2, 500, 400, 401], 0.2),
    ("f32", 9001, [1500, 1400, 5, 6, 900, 800, 0, 700], 0.0),
    ("f16", 20000, [2000, 1], 0.5), ("bf16", 2500, [40] * 400, 0.3), ("bf16", 131072, [30, 31, 32, 33, 1, 2], 0.1)])
def test_preference_sizes(dtype, vocab, lengths, unscored):
    """Rows enough for several stretches of L2's size, pairs of every length among them, in 64 bits on the GPU."""
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    rows, before, after = sum(lengths), 3, 5
    total = rows + before + after
    x = (torch.randn(total, vocab, generator=gen, device="cuda") * 2).to(TYPES[dtype])
    y = torch.randint(vocab, (total,), generator=gen, device="cuda")
    y[torch.rand(total, generator=gen, device="cuda") < unscored] = -1
    cuts = (np.cumsum([0] + lengths) + before).tolist()
    offsets = torch.tensor(cuts, device="cuda")
    seq = torch.full((total,), -1, device="cuda")
    for k, (a, b) in enumerate(zip(cuts, cuts[1:])):
        seq[a:b] = k
    on = (seq >= 0) & (y >= 0)
    lp = torch.zeros(total, dtype=torch.float64, device="cuda")
    for a in range(0, total, 512):
        z = torch.log_softmax(x[a:a + 512].double(), 1)
        lp[a:a + 512] = z.gather(1, y[a:a + 512].clamp(min=0)[:, None])[:, 0]
    lp = torch.where(on, lp, 0.0)
    ref = (lp + 0.3 * torch.randn(total, generator=gen, device="cuda")).float()
    got = bf.preference_loss(x, y, offsets, ref, beta=0.2, label_smoothing=0.1, margin=0.1)
    close_scores(got.logprob, lp.cpu().numpy())
    reward = torch.zeros(len(lengths), dtype=torch.float64, device="cuda")
    reward.index_add_(0, seq[on], 0.2 * (lp - ref.double())[on])
    # a row's error is a rounding of at most 2^-21 (32-bit values near 16) and as much of the sum it is added to
    reach = 0.2 * 2.0 ** -21 * max(lengths) + 1e-6
    assert torch.all((got.rewards.double() - reward).abs() <= reach)
    h = reward[0::2] - reward[1::2] - 0.1
    pairs = len(lengths) // 2
    up, down = torch.sigmoid(h), torch.sigmoid(-h)
    loss = -(0.9 * torch.nn.functional.logsigmoid(h) + 0.1 * torch.nn.functional.logsigmoid(-h)).mean()
    want = torch.stack([loss, (reward[0::2] > reward[1::2]).double().mean(), reward[0::2].mean(), reward[1::2].mean()])
    assert torch.all((got.stats.double() - want).abs() <= 2 * reach + 1e-5 * want.abs())
    slope = 0.2 * (0.1 * up - 0.9 * down) / pairs
    parts = 0.2 * (0.1 * up + 0.9 * down) / pairs
    both = lambda v, s: torch.stack([v, s * v], 1).reshape(-1)
    a, size = both(slope, -1.0), both(parts, 1.0)
    for r in range(0, total, 512):
        t, q = y[r:r + 512], seq[r:r + 512]
        p = torch.softmax(x[r:r + 512].double(), 1)
        hit = torch.zeros_like(p).scatter_(1, t.clamp(min=0)[:, None], 1.0)
        live = on[r:r + 512, None]
        w = torch.where(live, a[q.clamp(min=0)][:, None] * (hit - p), 0.0)
        far = torch.where(live, size[q.clamp(min=0)][:, None] * (hit + p), 0.0)
        bound = (5e-5 + 2 * reach) * far + ROUND[dtype] * w.abs() + LEAST[dtype]
        assert torch.all((got.grad[r:r + 512].double() - w).abs() <= bound)
    again = bf.preference_loss(x, y, offsets, ref, beta=0.2, label_smoothing=0.1, margin=0.1)
    assert all(torch.equal(u, v) for u, v in zip(got, again))
    only = bf.preference_loss(x, y, offsets, ref, beta=0.2, label_smoothing=0.1, margin=0.1, grad=False)
    assert torch.all((only.rewards.double() - reward).abs() <= reach)
    bf.preference_loss(x, y, offsets, ref, beta=0.2, label_smoothing=0.1, margin=0.1, out=x)
    assert torch.equal(x, got.grad)


def test_preference_offsets_that_do_not_ascend():
    x = torch.randn(40, 6000, device="cuda")
    y = torch.randint(6000, (40,), device="cuda")
    for offsets in ([-7, 20, 900], [30, 10, 0], [1 << 40, 5, 1 << 41], [20, 30, 0, 10, 40], [0, 40, 0, 40, 0]):
        r = bf.preference_loss(x, y, torch.tensor(offsets, device="cuda"))
        assert torch.isfinite(r.stats).all() and torch.isfinite(r.grad).all()
    r = bf.preference_loss(x, y * 0 - 1, torch.tensor([0, 10, 40], device="cuda"))
    assert r.stats[0].item() == pytest.approx(np.log(2)) and not r.grad.any()


def test_preference_edges():
    x = torch.randn(4, 6, device="cuda")
    y = torch.tensor([0, 1, 2, 3], device="cuda")
    r = bf.preference_loss(x, y, torch.tensor([0], device="cuda"))  # no pairs
    assert r.stats.tolist() == [0.0] * 4 and not r.grad.any()
    r = bf.preference_loss(x[:0], y[:0], torch.tensor([0, 0, 0], device="cuda"))  # a pair without rows
    assert r.stats[0].item() == pytest.approx(np.log(2)) and r.rewards.tolist() == [0.0, 0.0]
    r = bf.preference_loss(x, y * 0 - 1, torch.tensor([0, 2, 4], device="cuda"))
    assert r.stats[0].item() == pytest.approx(np.log(2)) and not r.grad.any()
    for offsets in ([-7, 2, 900], [3, 1, 0], [1 << 40, 5, 1 << 41]):
        assert torch.isfinite(bf.preference_loss(x, y, torch.tensor(offsets, device="cuda")).stats).all()
    # a gap of a thousand: the loss is linear and the gradient saturates
    big = torch.tensor([0.0, 0.0, 0.0, 0.0], device="cuda")
    r = bf.preference_loss(x, y, torch.tensor([0, 2, 4], device="cuda"), big, margin=1e4)
    assert r.stats[0].item() == pytest.approx(1e4, rel=1e-3) and torch.isfinite(r.grad).all()


@pytest.mark.parametrize("pairs,longest", [(1003, 25), (1, 256), (5, 300), (9, 700), (3, 1500), (2, 3000), (7, 9000),
                                           (2048, 3)])
@pytest.mark.parametrize("average", [False, True])
def test_pairs_of_any_length(pairs, longest, average):
    """Few threads per answer and many, several pairs together and an odd one behind, in 64 bits on the GPU."""
    gen = torch.Generator(device="cuda").manual_seed(pairs)
    lengths = torch.randint(longest // 2, longest + 1, (2 * pairs,), generator=gen, device="cuda")
    lengths[1::7] = 0
    offsets = torch.nn.functional.pad(lengths.cumsum(0), (1, 0)) + 2
    rows, vocab = int(offsets[-1]) + 3, 5
    x = torch.randn(rows, vocab, generator=gen, device="cuda")
    y = torch.randint(vocab, (rows,), generator=gen, device="cuda")
    y[torch.rand(rows, generator=gen, device="cuda") < 0.2] = -1
    seq = torch.full((rows,), -1, device="cuda")
    seq[2:rows - 3] = torch.arange(2 * pairs, device="cuda").repeat_interleave(lengths)
    on = (seq >= 0) & (y >= 0)
    lp = torch.log_softmax(x.double(), 1).gather(1, y.clamp(min=0)[:, None])[:, 0]
    ref = (lp + 0.3 * torch.randn(rows, generator=gen, device="cuda")).float()
    got = bf.preference_loss(x, y, offsets, ref, beta=0.2, average=average)
    sums = torch.zeros(2 * pairs, dtype=torch.float64, device="cuda")
    sums.index_add_(0, seq[on], (lp - ref.double())[on])
    counted = torch.bincount(seq[on], minlength=2 * pairs)
    reward = 0.2 * sums / (counted.clamp(min=1) if average else 1)
    # a row's error is a rounding of at most 2^-21 (32-bit values near 16) and as much of the sum it is added to
    reach = 0.2 * 2.0 ** -21 * longest + 1e-6
    assert torch.all((got.rewards.double() - reward).abs() <= reach)
    loss = torch.nn.functional.softplus(reward[1::2] - reward[0::2])
    assert abs(got.stats[0].item() - loss.mean().item()) <= 2 * reach + 1e-6 * loss.mean().item()
    mean = torch.stack([(reward[0::2] > reward[1::2]).double().mean(), reward[0::2].mean(), reward[1::2].mean()])
    close = (reward[0::2] - reward[1::2]).abs() <= 2 * reach  # either answer of such a pair may come out ahead
    slack = torch.tensor([close.double().mean().item(), reach, reach], dtype=torch.float64, device="cuda") + 1e-6
    assert torch.all((got.stats[1:].double() - mean).abs() <= slack + 1e-6 * mean.abs())
    again = bf.preference_loss(x, y, offsets, ref, beta=0.2, average=average)
    assert all(torch.equal(u, v) for u, v in zip(got, again))


def test_long_sequences_of_pairs():
    gen = torch.Generator(device="cuda").manual_seed(5)
    rows, vocab = 60000, 5
    x = torch.randn(rows, vocab, generator=gen, device="cuda")
    y = torch.randint(vocab, (rows,), generator=gen, device="cuda")
    offsets = torch.tensor([0, 25000, rows], device="cuda")
    r = bf.preference_loss(x, y, offsets, average=True, beta=2.0)
    lp = torch.log_softmax(x.double(), 1).gather(1, y[:, None])[:, 0]
    want = 2.0 * torch.stack([lp[:25000].mean(), lp[25000:].mean()])
    assert torch.all((r.rewards.double() - want).abs() < 1e-5)


# ---- embedding ----

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,width,stride", [(1, 1, 1, 0), (5, 3, 7, 0), (33, 10, 64, 0), (100, 7, 130, 3),
                                                     (64, 500, 256, 0), (1000, 20, 33, 0), (3000, 2, 16, 0),
                                                     (2100, 70000, 12, 0), (40, 300, 2048, 8), (4500, 4099, 40, 1),
                                                     (70, 9, 2047, 0), (300, 50, 513, 0), (90, 11, 66, 6), (50, 7, 15, 2)])
def test_embed(rows, vocab, width, stride, dtype):
    rng = np.random.default_rng([rows, vocab, width])
    _, table, td = make_logits(rng, vocab, width, dtype, stride, stride % 2)
    tokens = make_tokens(rng, rows, vocab)
    out = bf.embed(table, gpu(tokens, torch.int64), scale=1.7)
    want = R.embed(td, tokens, float(np.float32(1.7)))
    assert np.all(np.abs(host(out) - want) <= (ROUND[dtype] + 2.0 ** -23) * np.abs(want) + LEAST[dtype])
    _, dout, dd = make_logits(rng, rows, width, dtype, stride, stride % 2)
    g, size = R.embed_grad(dd, tokens, vocab, float(np.float32(0.3)))
    # a sum of n terms in 32 bits: at most n 2^-24 of the sum of magnitudes
    bound = max(rows, 4) * 2.0 ** -24 * size + LEAST[dtype]
    got = bf.embed_grad(dout, gpu(tokens, torch.int64), vocab, scale=0.3)
    assert np.all(np.abs(host(got) - g) <= bound + ROUND[dtype] * np.abs(g))
    assert torch.equal(got, bf.embed_grad(dout, gpu(tokens, torch.int64), vocab, scale=0.3))
    # in 32 bits, added to what is there, rows apart
    wide = torch.full((vocab, width + 5), 2.0, device="cuda")
    bf.embed_grad(dout, gpu(tokens, torch.int64), vocab, scale=0.3, out=wide[:, :width], accumulate=True)
    assert np.all(np.abs(host(wide[:, :width]) - (2.0 + g)) <= bound + 2.0 ** -22 * (2.0 + np.abs(g)))
    assert torch.all(wide[:, width:] == 2.0)
    into = torch.full((vocab, width + 5), 2.0, device="cuda", dtype=TYPES["bf16"])
    bf.embed_grad(dout, gpu(tokens, torch.int64), vocab, scale=0.3, out=into[:, :width])
    assert np.all(np.abs(host(into[:, :width]) - g) <= bound + ROUND["bf16"] * np.abs(g))
    assert torch.all(into[:, width:] == 2.0)


@pytest.mark.parametrize("tokens", ["one", "sorted", "reversed", "two", "none"])
@pytest.mark.parametrize("rows", [31, 32, 33, 1024, 1025, 70000])
def test_embed_grad_runs(rows, tokens):
    """Runs of equal tokens that end at, before and behind the ends of tiles."""
    t = torch.arange(rows, device="cuda")
    ids = {"one": t * 0 + 2, "sorted": t // 7, "reversed": (rows - 1 - t) // 64, "two": (t % 2) * 4, "none": t * 0 - 1}[tokens]
    vocab, width = max(5, rows // 7 + 2), 24
    dout = torch.randint(-8, 9, (rows, width), device="cuda").float()  # whole numbers: sums are exact
    got = bf.embed_grad(dout, ids, vocab)
    on = ids >= 0
    want = torch.zeros(vocab, width, dtype=torch.float64, device="cuda").index_add_(0, ids[on], dout[on].double())
    assert torch.equal(got.double(), want)


def test_embed_edges():
    table = torch.randn(4, 8, device="cuda")
    assert bf.embed(table, torch.empty(0, dtype=torch.int64, device="cuda")).shape == (0, 8)
    out = bf.embed(table, torch.tensor([4, -1, 3, 1 << 40], device="cuda"))
    assert torch.isnan(out[0]).all() and not out[1].any() and torch.equal(out[2], table[3]) and torch.isnan(out[3]).all()
    none = bf.embed_grad(torch.empty(0, 8, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda"), 3)
    assert not none.any() and none.shape == (3, 8)
    dout = torch.ones(4, 8, device="cuda")
    g = bf.embed_grad(dout, torch.tensor([9, -1, 2, 1 << 40], device="cuda"), 3)  # outside the table: left out
    assert torch.equal(g, torch.tensor([[0.0], [0.0], [1.0]], device="cuda").expand(3, 8))
    bf.embed_grad(dout, torch.tensor([9, -1, 2, 2], device="cuda"), 3, out=g, accumulate=True)
    assert torch.equal(g, torch.tensor([[0.0], [0.0], [3.0]], device="cuda").expand(3, 8))


# ---- all of them ----

def test_offsets_past_32_bits():
    """More than 2^32 logits: the last rows are read and written where they are."""
    rows, vocab = 66000, 65600
    x = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    y = torch.zeros(rows, dtype=torch.int64, device="cuda")
    last = torch.randn(3, vocab, device="cuda").to(torch.bfloat16)
    x[-3:] = last
    y[-3:] = torch.tensor([1, 2, vocab - 1])
    lp = bf.token_logprobs(x, y)
    want = torch.log_softmax(last.double(), 1).gather(1, y[-3:, None])[:, 0]
    assert torch.all((lp[-3:].double() - want).abs() < 2e-5)
    assert torch.all((lp[:-3] + float(np.log(vocab))).abs() < 2e-5)
    weight = torch.zeros(rows, device="cuda")
    weight[-3:] = 1.0
    bf.token_logprobs_grad(x, y, weight, out=x)
    p = torch.softmax(last.double(), 1)
    hit = torch.zeros_like(p).scatter_(1, y[-3:, None], 1.0)
    assert torch.all((x[-3:].double() - (hit - p)).abs() <= 5e-5 * (hit + p) + 2.0 ** -8 * (hit - p).abs())
    assert not x[:-3].any()


def test_other_stream_and_capture():
    """Work goes to the given stream, and a captured call replays on new inputs."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(300, 999, generator=gen, device="cuda")
    y = torch.randint(999, (300,), generator=gen, device="cuda")
    offsets, adv = torch.tensor([0, 100, 300], device="cuda"), torch.tensor([1.0, -1.0], device="cuda")
    old = torch.full((300,), -6.0, device="cuda")
    table = torch.randn(999, 64, device="cuda")
    want = (bf.token_logprobs(x, y), *bf.policy_loss(x, y, offsets, old, adv), bf.embed(table, y),
            *bf.preference_loss(x, y, offsets, old), bf.embed_grad(x, y, 999))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    late = torch.zeros_like(x)
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        late.copy_(x)
    for stream in (side, side.cuda_stream):
        got = (bf.token_logprobs(late, y, stream=stream), *bf.policy_loss(late, y, offsets, old, adv, stream=stream),
               bf.embed(table, y, stream=stream), *bf.preference_loss(late, y, offsets, old, stream=stream),
               bf.embed_grad(late, y, 999, stream=stream))
        side.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(got, want))
    late.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = (bf.token_logprobs(late, y), *bf.policy_loss(late, y, offsets, old, adv), bf.embed(table, y),
               *bf.preference_loss(late, y, offsets, old), bf.embed_grad(late, y, 999))
    for _ in range(2):
        late.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(got, want))


def test_binding_refuses():
    x, y = torch.zeros(4, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    offsets, f = torch.tensor([0, 2, 4], device="cuda"), torch.zeros(4, device="cuda")
    bad = [lambda: bf.token_logprobs(x.double(), y), lambda: bf.token_logprobs(x.cpu(), y),
           lambda: bf.token_logprobs(x[0], y), lambda: bf.token_logprobs(x.t(), y.new_zeros(8)),
           lambda: bf.token_logprobs(x, y[:3]), lambda: bf.token_logprobs(x, y.int()),
           lambda: bf.token_logprobs(x, y.cpu()), lambda: bf.token_logprobs_grad(x, y, f.double()),
           lambda: bf.policy_loss(x, y, offsets, f, f[:3]), lambda: bf.policy_loss(x, y, offsets, f, f[:2], f[:2]),
           lambda: bf.policy_loss(x, y, offsets, f, f[:2], reduction="mean"),
           lambda: bf.policy_loss(x, y, offsets[:0], f, f[:2]),
           lambda: bf.preference_loss(x, y, offsets[:2]), lambda: bf.embed(x, y, out=x.new_zeros(3, 8)),
           lambda: bf.embed_grad(x, y, 3, accumulate=True), lambda: bf.embed_grad(x, y, 3, out=x.new_zeros(2, 8))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    refused = [lambda: bf.token_logprobs(x, y, temperature=0.0), lambda: bf.token_logprobs(x.expand(4, 8)[:, :0], y),
               lambda: bf.token_logprobs(x[:1].expand(4, 8), y),
               lambda: bf.token_logprobs_grad(x[:, :4], y, f, out=x[:, 2:6]),
               lambda: bf.token_logprobs_grad(x, y, f, out=x.new_zeros(4, 7)),
               lambda: bf.token_logprobs_grad(x, y, f, out=x.new_zeros(4, 8, dtype=torch.float16)),
               lambda: bf.policy_loss(x, y, offsets, f, f[:2], kl_coef=0.1),
               lambda: bf.policy_loss(x, y, offsets, f, f[:2], clip_low=-0.1),
               lambda: bf.policy_loss(x, y, offsets, f, f[:2], entropy_coef=float("nan")),
               lambda: bf.preference_loss(x, y, offsets, beta=0.0),
               lambda: bf.preference_loss(x, y, offsets, label_smoothing=1.0),
               lambda: bf.embed(x, y, scale=float("inf")), lambda: bf.embed(x, y, out=x),
               lambda: bf.embed(x, y, out=x.new_zeros(4, 9)), lambda: bf.embed_grad(x, y, 4, out=x),
               lambda: bf.embed_grad(x, y, 0)]
    for call in refused:
        with pytest.raises(bf.BfError) as e:
            call()
        assert e.value.code == bf.BF_EINVAL
    torch.cuda.synchronize()


def test_workspace_is_checked():
    lib = bf.load()
    x, y = torch.zeros(4, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    need = ctypes.c_uint64(0)
    assert lib.bf_embed_grad_workspace(4, 8, ctypes.byref(need)) == bf.BF_OK and need.value > 0
    work = torch.empty(need.value + 512, dtype=torch.uint8, device="cuda")
    out = torch.zeros(4, 8, device="cuda")
    call = lambda ptr, size: lib.bf_embed_grad(bf._matrix(x, "x"), y.data_ptr(), 1.0, 0, bf._matrix(out, "out"), ptr, size, 0)
    assert call(work.data_ptr(), need.value) == bf.BF_OK
    assert call(work.data_ptr(), need.value - 1) == bf.BF_EINVAL
    assert call(work.data_ptr() + 8, need.value) == bf.BF_EINVAL
    assert call(None, need.value) == bf.BF_EINVAL
    torch.cuda.synchronize()
