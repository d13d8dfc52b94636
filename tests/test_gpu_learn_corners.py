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
