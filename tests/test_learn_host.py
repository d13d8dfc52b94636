"""Refusals of the learning entry points that need no GPU: every check comes before any CUDA call."""
import ctypes

import pytest

from paper_2607_22242_gb300 import _build, bf

SOME = 1 << 20  # an aligned address that no refused call reads


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return bf.load()


def mat(rows=4, cols=8, stride=8, dtype=0, data=SOME):
    return bf.Matrix(data, rows, cols, stride, dtype, 0)


BAD_LOGITS = [mat(dtype=3), mat(cols=0, stride=0), mat(stride=7), mat(data=None), mat(data=SOME + 2),
              mat(data=SOME + 1, dtype=1), mat(rows=1 << 31), mat(cols=(1 << 30) + 1, stride=(1 << 30) + 1),
              mat(stride=1 << 39)]


@pytest.mark.parametrize("i", range(len(BAD_LOGITS)))
def test_bad_logits(lib, i):
    x = BAD_LOGITS[i]
    assert lib.bf_token_logprobs(x, SOME, 1.0, SOME, None, None) == bf.BF_EINVAL
    assert bf.last_error().startswith("bf_token_logprobs: ")
    assert lib.bf_token_logprobs_grad(x, SOME, 1.0, SOME, None, x, None) == bf.BF_EINVAL
    assert lib.bf_policy_loss(x, policy(), SOME, None, None, SOME, 1 << 30, None) == bf.BF_EINVAL
    assert lib.bf_preference_loss(x, preference(), SOME, SOME, None, None, SOME, 1 << 30, None) == bf.BF_EINVAL
    assert lib.bf_embed(x, SOME, 1.0, mat(data=1 << 24), None) == bf.BF_EINVAL
    assert lib.bf_embed_grad(x, SOME, 1.0, 0, mat(data=1 << 24), SOME, 1 << 30, None) == bf.BF_EINVAL


def policy(**kw):
    a = dict(tokens=SOME, offsets=SOME, old_logprob=SOME, ref_logprob=None, advantage=SOME, sequences=2,
             advantage_per_token=0, reduction=0, clip_low=0.2, clip_high=0.2, kl_coef=0.0, entropy_coef=0.0,
             temperature=1.0, grad_scale=1.0)
    a.update(kw)
    return bf.PolicyArgs(**a)


def preference(**kw):
    a = dict(tokens=SOME, offsets=SOME, ref_logprob=None, pairs=1, average=0, beta=0.1, label_smoothing=0.0, margin=0.0,
             temperature=1.0, grad_scale=1.0)
    a.update(kw)
    return bf.PreferenceArgs(**a)


NAN, INF = float("nan"), float("inf")
BAD_POLICY = [dict(tokens=None), dict(offsets=None), dict(old_logprob=None), dict(advantage=None), dict(tokens=SOME + 4),
              dict(offsets=SOME + 4), dict(old_logprob=SOME + 2), dict(ref_logprob=SOME + 1), dict(advantage=SOME + 1),
              dict(sequences=1 << 31), dict(reduction=3), dict(clip_low=-0.1), dict(clip_high=NAN), dict(kl_coef=-1.0),
              dict(kl_coef=0.1), dict(entropy_coef=INF), dict(temperature=0.0), dict(temperature=-1.0),
              dict(temperature=INF), dict(temperature=1e-19), dict(temperature=1e19), dict(grad_scale=NAN)]


@pytest.mark.parametrize("kw", BAD_POLICY, ids=str)
def test_bad_policy(lib, kw):
    assert lib.bf_policy_loss(mat(), policy(**kw), SOME, None, None, SOME, 1 << 30, None) == bf.BF_EINVAL
    assert bf.last_error().startswith("bf_policy_loss: ")


BAD_PREFERENCE = [dict(tokens=None), dict(offsets=None), dict(tokens=SOME + 4), dict(offsets=SOME + 1),
                  dict(ref_logprob=SOME + 1), dict(pairs=1 << 30), dict(beta=0.0), dict(beta=NAN),
                  dict(label_smoothing=-0.1), dict(label_smoothing=1.0), dict(margin=INF), dict(temperature=0.0),
                  dict(grad_scale=INF)]


@pytest.mark.parametrize("kw", BAD_PREFERENCE, ids=str)
def test_bad_preference(lib, kw):
    assert lib.bf_preference_loss(mat(), preference(**kw), SOME, SOME, None, None, SOME, 1 << 30, None) == bf.BF_EINVAL
    assert bf.last_error().startswith("bf_preference_loss: ")


def test_bad_buffers(lib):
    x, far = mat(), mat(data=1 << 24)
    assert lib.bf_token_logprobs(None, SOME, 1.0, SOME, None, None) == bf.BF_EINVAL
    assert lib.bf_token_logprobs(x, None, 1.0, SOME, None, None) == bf.BF_EINVAL
    assert lib.bf_token_logprobs(x, SOME, 1.0, None, None, None) == bf.BF_EINVAL
    assert lib.bf_token_logprobs(x, SOME, 1.0, SOME, SOME + 2, None) == bf.BF_EINVAL
    for grad in (None, mat(rows=3, data=1 << 24), mat(cols=7, data=1 << 24), mat(dtype=1, data=1 << 24),
                 mat(data=SOME + 4), mat(stride=9)):
        assert lib.bf_token_logprobs_grad(x, SOME, 1.0, SOME, None, grad, None) == bf.BF_EINVAL
    assert lib.bf_policy_loss(x, None, SOME, None, None, SOME, 1 << 30, None) == bf.BF_EINVAL
    assert lib.bf_policy_loss(x, policy(), None, None, None, SOME, 1 << 30, None) == bf.BF_EINVAL
    assert lib.bf_policy_loss(x, policy(), SOME, None, None, None, 1 << 30, None) == bf.BF_EINVAL
    assert lib.bf_policy_loss(x, policy(), SOME, None, None, SOME + 128, 1 << 30, None) == bf.BF_EINVAL
    assert lib.bf_policy_loss(x, policy(), SOME, None, None, SOME, 64, None) == bf.BF_EINVAL
    assert lib.bf_preference_loss(x, preference(), SOME, None, None, None, SOME, 1 << 30, None) == bf.BF_EINVAL
    assert lib.bf_preference_loss(x, preference(), SOME, SOME, None, None, SOME, 64, None) == bf.BF_EINVAL
    assert lib.bf_embed(x, SOME, 1.0, mat(cols=9, stride=9, data=1 << 24), None) == bf.BF_EINVAL
    assert lib.bf_embed(x, SOME, 1.0, mat(dtype=1, data=1 << 24), None) == bf.BF_EINVAL
    assert lib.bf_embed(x, SOME, 1.0, mat(data=SOME + 64), None) == bf.BF_EINVAL
    assert lib.bf_embed(mat(rows=0), SOME, 1.0, far, None) == bf.BF_EINVAL
    assert lib.bf_embed(x, SOME, NAN, far, None) == bf.BF_EINVAL
    assert lib.bf_embed_grad(x, SOME, 1.0, 0, mat(cols=9, stride=9, data=1 << 24), SOME, 1 << 30, None) == bf.BF_EINVAL
    assert lib.bf_embed_grad(x, SOME, 1.0, 0, mat(data=SOME + 64), SOME, 1 << 30, None) == bf.BF_EINVAL
    assert lib.bf_embed_grad(x, SOME, 1.0, 0, mat(rows=0, data=1 << 24), SOME, 1 << 30, None) == bf.BF_EINVAL
    assert lib.bf_embed_grad(x, SOME, 1.0, 0, far, SOME, 8, None) == bf.BF_EINVAL


@pytest.mark.parametrize("temperature", [0.0, -1.0, 1e-40, 1e-19, 1e19, INF, NAN])
def test_bad_temperature(lib, temperature):
    assert lib.bf_token_logprobs(mat(), SOME, temperature, SOME, None, None) == bf.BF_EINVAL
    assert lib.bf_token_logprobs_grad(mat(), SOME, temperature, SOME, None, mat(), None) == bf.BF_EINVAL
    assert lib.bf_preference_loss(mat(), preference(temperature=temperature), SOME, SOME, None, None, SOME, 1 << 30,
                                  None) == bf.BF_EINVAL


def test_no_rows_is_a_call_without_work(lib):
    empty = mat(rows=0, data=None)
    assert lib.bf_token_logprobs(empty, None, 1.0, None, None, None) == bf.BF_OK
    assert lib.bf_token_logprobs_grad(empty, None, 1.0, None, None, empty, None) == bf.BF_OK
    assert lib.bf_embed(mat(data=1 << 24), None, 1.0, empty, None) == bf.BF_OK


def test_workspaces(lib):
    n = ctypes.c_uint64(0)
    for query in (lib.bf_policy_loss_workspace, lib.bf_preference_loss_workspace, lib.bf_embed_grad_workspace):
        sizes = []
        for rows, groups in ((0, 1), (1, 1), (1000, 1), (1000, 100), (1 << 20, 1 << 10)):
            assert query(rows, groups, ctypes.byref(n)) == bf.BF_OK
            assert n.value % 256 == 0
            sizes.append(n.value)
        assert sizes == sorted(sizes)
        assert query(1 << 31, 1, ctypes.byref(n)) == bf.BF_EINVAL
        assert query(1, 1, None) == bf.BF_EINVAL
    assert lib.bf_policy_loss_workspace(1, 1 << 31, ctypes.byref(n)) == bf.BF_EINVAL
    assert lib.bf_preference_loss_workspace(1, 1 << 30, ctypes.byref(n)) == bf.BF_EINVAL
    assert lib.bf_embed_grad_workspace(1, 0, ctypes.byref(n)) == bf.BF_EINVAL
