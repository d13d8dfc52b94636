"""Corners of the operators that learn from makespans: tokens outside the vocabulary, infinite terms beside coefficients
of 0, rows whose mask leaves nothing, sums of many blocks, and what autograd is told."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_22242_gb300 import bf  # noqa: E402

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ROUND = {"f32": 2.0 ** -23, "bf16": 2.0 ** -8, "f16": 2.0 ** -10}     # twice half a unit in the last place
INF = float("inf")

# Rows x vocabulary: a thread, some lanes and a block or cluster per row; the losses of the first three run in one launch.
SHAPES = [(8, 3), (8, 50), (8, 700), (1100, 3), (1100, 50), (1100, 700), (8, 6000), (500, 6000), (4, 131073)]


@pytest.fixture(scope="module", autouse=True)
def _built():
    assert torch.cuda.is_available()
    bf.load()


def draw(rows, vocab, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows + vocab)
    x = (torch.randn(rows, vocab, generator=gen, device="cuda") * 2).to(TYPES[dtype])
    return gen, x, torch.randint(vocab, (rows,), generator=gen, device="cuda")


def cuts(rows, parts):
    return torch.tensor([rows * k // parts for k in range(parts + 1)], device="cuda")


# ---- a token outside the vocabulary makes its row's values NaN, and no other's ----

def with_unknown(y, vocab):
    """The tokens with the first and last outside the vocabulary, the last by its high bits alone."""
    y = y.clone()
    y[0], y[-1] = vocab, (1 << 32) + 1
    return y, y >= vocab


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_unknown_token_in_scores(rows, vocab, dtype):
    gen, x, y = draw(rows, vocab, dtype)
    y, out = with_unknown(y, vocab)
    x[0] = -INF  # a mask that leaves nothing does not hide it
    lp, h = bf.token_logprobs(x, y, entropy=True)
    assert torch.equal(torch.isnan(lp), out) and torch.equal(torch.isnan(h), out)
    a, c = torch.randn(rows, generator=gen, device="cuda"), torch.randn(rows, generator=gen, device="cuda")
    known = torch.where(out, -1, y)
    for slopes in ((a, c), (a, None), (torch.zeros_like(a), c), (torch.zeros_like(a), None)):
        g = bf.token_logprobs_grad(x, y, *slopes)
        assert torch.isnan(g[out]).all()
        assert torch.equal(g[~out], bf.token_logprobs_grad(x, known, *slopes)[~out])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_unknown_token_in_losses(rows, vocab, dtype):
    gen, x, y = draw(rows, vocab, dtype)
    y, out = with_unknown(y, vocab)
    x[0] = -INF
    old, adv = torch.full((rows,), -2.0, device="cuda"), torch.tensor([1.0, -1.0], device="cuda")
    for entropy_coef in (0.0, 0.01):
        got = bf.policy_loss(x, y, cuts(rows, 2), old, adv, entropy_coef=entropy_coef)
        known = bf.policy_loss(x, y.clamp(max=vocab - 1), cuts(rows, 2), old, adv, entropy_coef=entropy_coef)
        assert torch.isnan(got.stats[0]) and torch.equal(torch.isnan(got.logprob), out)
        assert torch.isnan(got.grad[out]).all() and torch.equal(got.grad[~out], known.grad[~out])
    # the first of two pairs has it: its gap has no value
    y[-1] = 0
    out[-1] = False
    got = bf.preference_loss(x, y, cuts(rows, 4))
    known = bf.preference_loss(x, torch.where(out, -1, y), cuts(rows, 4))
    assert torch.equal(torch.isnan(got.logprob), out) and torch.isnan(got.rewards).tolist() == [True, False, False, False]
    assert torch.isnan(got.grad[0]).all()
    assert torch.equal(got.grad[rows // 2:], known.grad[rows // 2:]) and torch.isfinite(known.grad).all()


# ---- infinite terms beside coefficients of 0 ----

def with_far_reference(rows, vocab, dtype):
    """Rows of which the second's ratio to the reference overflows and the third's token is banned though drawn."""
    gen, x, y = draw(rows, vocab, dtype)
    y[2] = 1
    x[2, 1] = -INF
    lp = bf.token_logprobs(x, y)
    assert lp[2] == -INF
    ref = torch.where(torch.isinf(lp), -3.0, lp + 0.1)
    ref[1] += 100.0
    old = torch.where(torch.isinf(lp), -3.0, lp - 0.05)
    return x, y, old, ref, torch.randn(2, generator=gen, device="cuda")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_reference_that_is_only_watched(rows, vocab, dtype):
    """kl_coef = 0: the KL is reported, and neither the loss nor the gradient has anything of it."""
    x, y, old, ref, adv = with_far_reference(rows, vocab, dtype)
    for entropy_coef in (0.0, 0.02):
        kw = dict(entropy_coef=entropy_coef)
        got = bf.policy_loss(x, y, cuts(rows, 2), old, adv, ref, **kw)
        want = bf.policy_loss(x, y, cuts(rows, 2), old, adv, **kw)
        others = [0, 1, 3, 4, 5]
        assert torch.equal(got.stats[others], want.stats[others]) and torch.isfinite(want.stats).all()
        assert torch.equal(got.grad, want.grad) and torch.isfinite(want.grad).all()


@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_kl_of_a_banned_token_is_infinite(rows, vocab):
    """e^u - u - 1 with u = ref - lp = inf, alone and in the loss."""
    x, y, old, ref, adv = with_far_reference(rows, vocab, "f32")
    ref[1] -= 100.0
    for kl_coef in (0.0, 0.1):
        got = bf.policy_loss(x, y, cuts(rows, 2), old, adv, ref, kl_coef=kl_coef)
        assert got.stats[2] == INF and (got.stats[0] == INF) == (kl_coef > 0.0)
        assert torch.isfinite(got.grad[[0, 1, 3]]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [s for s in SHAPES if s[0] >= 8])
def test_pair_with_a_banned_token(rows, vocab, dtype):
    """A gap of +inf costs nothing without smoothing, one of -inf everything; slopes are finite either way."""
    _, x, y = draw(rows, vocab, dtype)
    offsets = cuts(rows, 4)
    for answer, loss, smoothed in ((1, 0.0, INF), (0, INF, INF)):
        z, t = x.clone(), y.clamp(min=1)
        at = rows * answer // 4
        t[at] = 0
        z[at, 0] = -INF
        got = bf.preference_loss(z, t, offsets)
        assert got.rewards[answer] == -INF and torch.isfinite(got.grad).all()
        if loss == 0.0:  # the mean has the other pair's loss alone: some roundings of it, 2^-24 each
            gap = (got.rewards[2] - got.rewards[3]).double()
            assert got.stats[0].item() == pytest.approx(0.5 * torch.nn.functional.softplus(-gap).item(), rel=2.0 ** -19)
            assert not got.grad[:rows // 2].any()
        else:
            assert got.stats[0] == INF and got.grad[:rows // 2].any()
        got = bf.preference_loss(z, t, offsets, label_smoothing=0.1)
        assert got.stats[0] == smoothed and torch.isfinite(got.grad).all()


# ---- rows whose mask leaves nothing ----

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [s for s in SHAPES if s[0] >= 8])
def test_pair_with_masked_rows_in_both_answers(rows, vocab, dtype):
    """The pair's gap has no value, but a row with no logit above -inf has a gradient of 0 all the same."""
    _, x, y = draw(rows, vocab, dtype)
    masked = [0, rows // 4]
    x[masked] = -INF
    got = bf.preference_loss(x, y, cuts(rows, 4))
    assert got.rewards[:2].tolist() == [-INF, -INF] and not got.grad[masked].any()
    y[masked] = -1
    want = bf.preference_loss(x, y, cuts(rows, 4))
    assert torch.equal(got.grad[rows // 2:], want.grad[rows // 2:]) and torch.isfinite(want.grad).all()


# ---- autograd ----

def test_autograd_sees_what_is_written():
    """A tensor that autograd keeps and a call writes over is refused in the backward pass, as after torch's own in-place
    operations, instead of giving a wrong gradient."""
    y, f = torch.tensor([0, 1, 2, 3], device="cuda"), torch.zeros(4, device="cuda")
    offsets, table = torch.tensor([0, 2, 4], device="cuda"), torch.randn(4, 8, device="cuda")
    calls = [lambda t: bf.token_logprobs_grad(t, y, f + 1, out=t),
             lambda t: bf.policy_loss(t, y, offsets, f, f[:2] + 1, out=t),
             lambda t: bf.preference_loss(t, y, offsets, out=t),
             lambda t: bf.embed(table, y, out=t),
             lambda t: bf.embed_grad(table, y, 4, out=t),
             lambda t: bf.embed_grad(table, y, 4, out=t, accumulate=True)]
    for call in calls:
        for over in (lambda t: t, lambda t: t.detach()):
            leaf = torch.randn(4, 8, device="cuda", requires_grad=True)
            kept = leaf.exp()  # its backward pass multiplies by what exp gave
            call(over(kept))
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                kept.sum().backward()
    # what is not written over stays usable, and tensors without a version are written as before
    leaf = torch.randn(4, 8, device="cuda", requires_grad=True)
    kept = leaf.exp()
    bf.policy_loss(kept, y, offsets, f, f[:2] + 1)
    kept.sum().backward()
    assert torch.equal(leaf.grad, kept.detach())
    with torch.inference_mode():
        t = torch.randn(4, 8, device="cuda")
        want = bf.token_logprobs_grad(t, y, f + 1)
        assert torch.equal(bf.token_logprobs_grad(t, y, f + 1, out=t), want)


# ---- sums of many blocks ----

@pytest.mark.parametrize("rows,vocab,dtype,reduction", [(1000003, 3, "f32", "tokens"), (1000003, 7, "bf16", "sequences"),
                                                        (200001, 512, "bf16", "sum"), (820001, 4, "f16", "sum")])
def test_policy_of_many_blocks(rows, vocab, dtype, reduction):
    """More blocks than sum up in one launch.  A term is made of a log-probability given to 32 bits: its ratio is off by
    2^-22 of itself (a difference's rounding and expf's), its KL term by as much of e^u + |u| + 1, and is weighed and added
    in fewer than 40 roundings of 2^-24: 3e-6 of the sum of magnitudes, far below what one warp's part weighs (4 rows:
    2e-5).  An entropy is within 1e-5."""
    gen, x, y = draw(rows, vocab, dtype)
    y[torch.rand(rows, generator=gen, device="cuda") < 0.1] = -1
    sequences = rows // 13
    offsets = torch.sort(torch.randint(rows + 1, (sequences + 1,), generator=gen, device="cuda")).values
    seq = torch.searchsorted(offsets, torch.arange(rows, device="cuda"), right=True) - 1
    on = (y >= 0) & (seq >= 0) & (seq < sequences)
    at = seq.clamp(0, sequences - 1)
    parts = [torch.log_softmax(x[a:a + 50000].double(), 1) for a in range(0, rows, 50000)]
    lp = torch.cat([z.gather(1, y[50000 * k:50000 * k + 50000].clamp(min=0)[:, None])[:, 0] for k, z in enumerate(parts)])
    h = torch.cat([-(z.exp() * z).sum(1) for z in parts])
    del parts
    d = 0.25 * torch.randn(rows, generator=gen, device="cuda").double()
    for edge in (0.8, 1.2):  # no ratio within 1e-3 of a clip edge
        d = torch.where((d.exp() - edge).abs() < 1e-3, d + 4e-3, d)
    old, ref = (lp - d).float(), (lp + 0.4 * torch.randn(rows, generator=gen, device="cuda")).float()
    adv = torch.randn(sequences, generator=gen, device="cuda")
    kw = dict(kl_coef=0.05, entropy_coef=0.01, reduction=reduction)
    got = bf.policy_loss(x, y, offsets, old, adv, ref, **kw)
    assert torch.all((got.logprob.double() - torch.where(on, lp, 0.0)).abs() <= 1e-5 + 1e-6 * lp.abs())
    lp = got.logprob.double()
    n = torch.bincount(at[on], minlength=sequences).double()
    w = {"tokens": 1.0 / n.sum(), "sequences": 1.0 / (n[at].clamp(min=1) * (n > 0).sum()), "sum": 1.0}[reduction]
    w = torch.where(on, w, 0.0)
    A, r = adv.double()[at], torch.exp(torch.where(on, lp - old.double(), 0.0))
    low, high = 1.0 - float(torch.tensor(0.2)), 1.0 + float(torch.tensor(0.2))
    stopped = ((A >= 0) & (r > high)) | ((A < 0) & (r < low))
    held = torch.where(stopped, torch.where(A >= 0, high, low), r)
    u = torch.where(on, ref.double() - lp, 0.0)
    k = torch.expm1(u) - u
    terms = {1: -held * A, 2: k, 4: stopped.double(), 5: r}
    size = {1: (held * A).abs(), 2: u.exp() + u.abs() + 1, 4: stopped.double(), 5: r}
    for i, v in terms.items():
        assert abs(got.stats[i].item() - (w * v).sum().item()) <= 3e-6 * (w * size[i]).sum().item(), i
    assert abs(got.stats[3].item() - (w * h).sum().item()) <= 1e-5 * w.sum().item() + 3e-6 * (w * h).sum().item()
    s = got.stats.double()
    made = s[1] + 0.05 * s[2] - 0.01 * s[3]
    assert abs(s[0] - made) <= 2.0 ** -21 * (s[1].abs() + 0.05 * s[2] + 0.01 * s[3])
    a = w * (torch.where(stopped, 0.0, -A * r) - 0.05 * torch.expm1(u))
    part = w * (torch.where(stopped, 0.0, (A * r).abs()) + 0.05 * (u.exp() + 1))
    for f in range(0, rows, 50000):
        z, t = torch.log_softmax(x[f:f + 50000].double(), 1), slice(f, f + 50000)
        p = z.exp()
        hit = torch.zeros_like(p).scatter_(1, y[t].clamp(min=0)[:, None], 1.0)
        tilt = p * (z + h[t][:, None])
        want = a[t][:, None] * (hit - p) + 0.01 * w[t][:, None] * tilt
        far = part[t][:, None] * (hit + p) + 0.01 * w[t][:, None] * (tilt.abs() + p)
        least = 2.0 ** -24 if dtype == "f16" else 1e-37
        assert torch.all((got.grad[t].double() - want).abs() <= 5e-5 * far + ROUND[dtype] * want.abs() + least)
    # the same bits again; without the gradient; in place
    again = bf.policy_loss(x, y, offsets, old, adv, ref, **kw)
    assert all(torch.equal(i, j) for i, j in zip(got, again))
    assert torch.equal(bf.policy_loss(x, y, offsets, old, adv, ref, grad=False, **kw).stats, got.stats)
    same = bf.policy_loss(x, y, offsets, old, adv, ref, out=x, **kw)
    assert torch.equal(x, got.grad) and torch.equal(same.stats, got.stats)


@pytest.mark.parametrize("reduction", bf.REDUCTIONS)
@pytest.mark.parametrize("answers,longest,empty", [(40, 900, 3000), (200, 12, 5000), (2000, 40, 30), (3, 40000, 1025)])
def test_many_empty_sequences(answers, longest, empty, reduction):
    """Thousands of empty sequences between others change nothing for those: more than a block's rows have offsets."""
    gen = torch.Generator(device="cuda").manual_seed(answers)
    lengths = torch.randint(1, longest + 1, (answers,), generator=gen, device="cuda")
    wide = torch.zeros(answers, empty + 1, dtype=torch.int64, device="cuda")
    wide[:, empty // 2] = lengths
    close = torch.nn.functional.pad(lengths.cumsum(0), (1, 0)) + 1
    far = torch.nn.functional.pad(wide.flatten().cumsum(0), (1, 0)) + 1
    rows = int(close[-1]) + 2
    x = torch.randn(rows, 5, generator=gen, device="cuda")
    y = torch.randint(-1, 5, (rows,), generator=gen, device="cuda")
    old = torch.full((rows,), -1.6, device="cuda")
    adv = torch.randn(answers, generator=gen, device="cuda")
    spread = torch.zeros_like(wide, dtype=torch.float32)
    spread[:, empty // 2] = adv
    got = bf.policy_loss(x, y, far, old, spread.flatten(), reduction=reduction)
    want = bf.policy_loss(x, y, close, old, adv, reduction=reduction)
    on = (y >= 0) & (torch.arange(rows, device="cuda") >= 1) & (torch.arange(rows, device="cuda") < rows - 2)
    assert torch.equal(want.logprob != 0, on)
    assert torch.equal(got.logprob, want.logprob) and torch.equal(got.grad, want.grad)
    # 32-bit sums of weighed terms whose blocks may differ: under 40 roundings of 2^-24 on either side
    size = torch.tensor([max(1.0, adv.abs().max().item()) * 8] * 6, device="cuda") * (on.sum() if reduction == "sum" else 1)
    assert torch.all((got.stats - want.stats).abs() <= 80 * 2.0 ** -24 * size)


def test_many_empty_pairs():
    """Pairs without rows between others: rewards by the rows that are there, a loss of ln 2 for the empty ones."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    pairs, empty = 30, 1500
    lengths = torch.randint(300, 900, (pairs, 2), generator=gen, device="cuda")
    wide = torch.zeros(pairs, empty + 1, 2, dtype=torch.int64, device="cuda")
    wide[:, empty // 3] = lengths
    offsets = torch.nn.functional.pad(wide.flatten().cumsum(0), (1, 0))
    rows = int(offsets[-1])
    x = torch.randn(rows, 5, generator=gen, device="cuda")
    y = torch.randint(-1, 5, (rows,), generator=gen, device="cuda")
    got = bf.preference_loss(x, y, offsets, average=True, beta=1.0)
    seq = torch.arange(2 * pairs, device="cuda").repeat_interleave(lengths.flatten())
    on = y >= 0
    sums = torch.zeros(2 * pairs, dtype=torch.float64, device="cuda").index_add_(0, seq[on], got.logprob.double()[on])
    want = sums / torch.bincount(seq[on], minlength=2 * pairs)
    rewards = got.rewards.view(pairs, empty + 1, 2)
    # at most 900 terms of one sign by 32 threads, then over those, divided and multiplied: under 40 roundings of 2^-24
    assert torch.all((rewards[:, empty // 3].flatten().double() / want - 1).abs() <= 40 * 2.0 ** -24)
    rest = torch.cat([rewards[:, :empty // 3], rewards[:, empty // 3 + 1:]], 1)
    assert not rest.any()
    gap = want.view(pairs, 2)
    loss = (torch.nn.functional.softplus(gap[:, 1] - gap[:, 0]).sum() + pairs * empty * 0.6931471805599453) / (pairs * (empty + 1))
    assert got.stats[0].item() == pytest.approx(loss.item(), rel=1.5e-5)  # 90 terms a thread, then over 512: 110 roundings and the gaps' own
