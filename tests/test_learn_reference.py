"""The plain 64-bit forms the GPU tests compare with: their gradients against central differences of their losses."""
import numpy as np
import pytest

import learn_ref as R

OFFSETS = [0, 3, 3, 8, 9]


def _case(seed=0, rows=9, vocab=7):
    rng = np.random.default_rng(seed)
    x = rng.normal(0, 2, (rows, vocab))
    tokens = rng.integers(0, vocab, rows)
    tokens[4] = -1
    return rng, x, tokens


def _differences(f, x, g, h=1e-6):
    rng = np.random.default_rng(1)
    for _ in range(5):
        v = rng.normal(0, 1, x.shape)
        got = (f(x + h * v) - f(x - h * v)) / (2 * h)
        assert abs(got - (g * v).sum()) < 1e-7 * (1 + np.abs(g).sum())


@pytest.mark.parametrize("tau", [1.0, 0.7])
def test_scores(tau):
    rng, x, tokens = _case()
    a, c = rng.normal(0, 1, 9), rng.normal(0, 1, 9)
    def f(z):
        lp, h = R.scores(z, tokens, tau)
        return (a * lp + c * h).sum()
    on = tokens >= 0
    _differences(f, x, R.scores_grad(x, tokens, a * on, c * on, tau)[0])


@pytest.mark.parametrize("reduction", ["tokens", "sequences", "sum"])
@pytest.mark.parametrize("kl,entropy,tau", [(0.0, 0.0, 1.0), (0.3, 0.05, 1.3)])
def test_policy(reduction, kl, entropy, tau):
    rng, x, tokens = _case()
    lp, _ = R.scores(x, tokens, tau)
    old, ref, adv = lp - rng.normal(0, 0.3, 9), lp + rng.normal(0, 0.3, 9), rng.normal(0, 1, 4)
    kw = dict(ref=ref, kl_coef=kl, entropy_coef=entropy, tau=tau, reduction=reduction)
    stats, _, g, _, margin = R.policy(x, tokens, OFFSETS, old, adv, **kw)
    assert margin.min() > 1e-4  # away from the clip's edges, where the loss has a kink
    assert 0 < stats[4]         # some rows are clipped
    _differences(lambda z: R.policy(z, tokens, OFFSETS, old, adv, **kw)[0][0], x, g)


@pytest.mark.parametrize("average", [False, True])
@pytest.mark.parametrize("eps,margin", [(0.0, 0.0), (0.1, 0.5)])
def test_preference(average, eps, margin):
    rng, x, tokens = _case()
    ref = rng.normal(-2, 0.5, 9)
    kw = dict(ref=ref, beta=0.7, eps=eps, margin=margin, average=average)
    _differences(lambda z: R.preference(z, tokens, OFFSETS, **kw)[0][0], x, R.preference(x, tokens, OFFSETS, **kw)[3])


def test_embed_grad():
    rng = np.random.default_rng(0)
    tokens, dout = np.array([2, 0, 2, -1, 4]), rng.normal(0, 1, (5, 3))
    table = rng.normal(0, 1, (5, 3))
    _differences(lambda w: (R.embed(w, tokens, 0.5) * dout).sum(), table, R.embed_grad(dout, tokens, 5, 0.5)[0])
