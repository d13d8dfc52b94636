"""Refusals of the entry points of a decoding step that need no GPU: every check comes before any CUDA call."""
import ctypes

import pytest

from paper_2607_22242_gb300 import _build, bf

SOME, FAR = 1 << 20, 1 << 30  # aligned addresses that no refused call reads
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return bf.load()


def cache(batch=4, tokens=1, heads=4, dim=64, dtype=1, data=SOME, **strides):
    s = dict(batch_stride=tokens * heads * dim, token_stride=heads * dim, head_stride=dim)
    s.update(strides)
    return bf.Cache(data, batch, tokens, heads, dim, s["batch_stride"], s["token_stride"], s["head_stride"], dtype, 0)


def at(c):
    return None if c is None else ctypes.addressof(c)


def workspace(lib, q, pk, sk, n):
    return lib.bf_prefix_attention_workspace(at(q), at(pk), at(sk), n)


def attend(lib, q=None, pk=None, pv=None, sk=None, sv=None, out=None, lse=None, work=SOME, have=1 << 40, **kw):
    a = dict(prefix_lengths=None, suffix_lengths=None, scale=0.125)
    a.update(kw)
    q, pk = q or cache(), pk or cache(2, 10, 2)
    pv = pv or cache(pk.batch, pk.tokens, pk.heads, pk.dim, pk.dtype)
    out = out or cache(q.batch, 1, q.heads, q.dim, q.dtype, data=FAR)
    args = bf.AttentionArgs(a["prefix_lengths"], a["suffix_lengths"], a["scale"], 0)
    return lib.bf_prefix_attention(*[at(c) for c in (q, pk, pv, sk, sv, args, out)], lse, work, have, None)


BAD_ATTENTION = [
    dict(q=cache(dtype=3)), dict(q=cache(data=None)), dict(q=cache(data=SOME + 1)), dict(q=cache(tokens=2)), dict(q=cache(heads=0)),
    dict(q=cache(heads=3)), dict(q=cache(dim=0)), dict(q=cache(dim=257), pk=cache(2, 10, 2, 257)), dict(q=cache(5)),
    dict(q=cache(dtype=0)), dict(q=cache(dim=32)), dict(q=cache(1 << 31)), dict(q=cache(batch_stride=1 << 42)),
    dict(q=cache(heads=65537)), dict(pk=cache(0, 10, 2)), dict(pk=cache(2, 1 << 31, 2)), dict(pk=cache(2, 10, 2, data=None)),
    dict(pk=cache(2, 10, 2, token_stride=1 << 41)), dict(pv=cache(2, 9, 2)), dict(pv=cache(2, 10, 2, dtype=2)),
    dict(pv=cache(2, 10, 2, data=SOME + 1)), dict(sk=cache(4, 5, 2)), dict(sv=cache(4, 5, 2)),
    dict(sk=cache(3, 5, 2), sv=cache(3, 5, 2)), dict(sk=cache(4, 5, 1), sv=cache(4, 5, 1)), dict(sk=cache(4, 5, 2), sv=cache(4, 6, 2)),
    dict(out=cache()), dict(out=cache(data=SOME + 128)), dict(out=cache(3, data=FAR)), dict(out=cache(dtype=2, data=FAR)),
    dict(out=cache(data=FAR, batch_stride=0)), dict(out=cache(data=FAR, head_stride=32)), dict(out=cache(data=FAR, batch_stride=200)),
    dict(lse=SOME + 2), dict(scale=NAN), dict(scale=INF), dict(scale=-1e31), dict(prefix_lengths=SOME + 4), dict(suffix_lengths=SOME + 4),
    dict(work=None), dict(work=SOME + 8), dict(have=64),
]


@pytest.mark.parametrize("i", range(len(BAD_ATTENTION)))
def test_bad_attention(lib, i):
    assert attend(lib, **BAD_ATTENTION[i]) == bf.BF_EINVAL
    assert bf.last_error().startswith("bf_prefix_attention: ")


def test_attention_null(lib):
    c, far = cache(), cache(data=FAR)
    args = bf.AttentionArgs(None, None, 0.1, 0)
    for call in ((None, c, c, None, None, args, far), (c, None, c, None, None, args, far), (c, c, None, None, None, args, far),
                 (c, c, c, None, None, None, far), (c, c, c, None, None, args, None)):
        assert lib.bf_prefix_attention(*[at(v) for v in call], None, SOME, 1 << 40, None) == bf.BF_EINVAL


def test_attention_without_answers(lib):
    empty = cache(0, data=None)
    assert attend(lib, q=empty, out=empty, work=None, have=0) == bf.BF_OK


def test_attention_workspace(lib):
    n = ctypes.c_uint64(0)
    sizes = []
    for answers, tokens in ((2, 1), (4, 100), (64, 100), (256, 1000)):
        assert workspace(lib, cache(answers), cache(2, tokens, 2), cache(answers, tokens, 2), ctypes.byref(n)) == bf.BF_OK
        sizes.append(n.value)
        assert n.value % 256 == 0 and n.value > 0
    assert sizes == sorted(sizes)
    assert workspace(lib, cache(), cache(2, 10, 2), None, ctypes.byref(n)) == bf.BF_OK
    assert workspace(lib, cache(), cache(2, 10, 2), None, None) == bf.BF_EINVAL
    assert workspace(lib, cache(3), cache(2, 10, 2), None, ctypes.byref(n)) == bf.BF_EINVAL


def mat(rows=8, cols=50, stride=50, dtype=1, data=SOME):
    return bf.Matrix(data, rows, cols, stride, dtype, 0)


def beams(**kw):
    a = dict(scores=SOME, finished=None, lengths=None, groups=2, beams=4, keep=4, end_token=-1, length_penalty=0.0, temperature=1.0)
    a.update(kw)
    return bf.BeamArgs(**a)


def step(lib, x=None, args=None, scores=SOME, tokens=SOME, parents=SOME, finished=None, lengths=None, work=SOME, have=1 << 30):
    x, args = x or mat(), args or beams()
    return lib.bf_beam_step(at(x), at(args), scores, tokens, parents, finished, lengths, work, have, None)


BAD_BEAMS = [
    dict(x=mat(dtype=3)), dict(x=mat(data=None)), dict(x=mat(rows=7)), dict(x=mat(stride=49)), dict(x=mat(cols=0)),
    dict(x=mat(cols=(1 << 24) + 1, stride=(1 << 24) + 1)), dict(args=beams(scores=None)), dict(args=beams(scores=SOME + 2)),
    dict(args=beams(beams=0)), dict(args=beams(beams=257)), dict(args=beams(keep=0)), dict(args=beams(keep=257)),
    dict(args=beams(groups=3)), dict(args=beams(groups=1 << 40)), dict(args=beams(end_token=-2)), dict(args=beams(finished=SOME)),
    dict(args=beams(length_penalty=0.5)), dict(args=beams(length_penalty=-0.5, lengths=SOME)),
    dict(args=beams(length_penalty=NAN, lengths=SOME)), dict(args=beams(lengths=SOME + 4)), dict(args=beams(temperature=0.0)),
    dict(args=beams(temperature=1e19)), dict(scores=None), dict(scores=SOME + 1), dict(tokens=None), dict(tokens=SOME + 4),
    dict(parents=None), dict(parents=SOME + 4), dict(lengths=SOME), dict(lengths=SOME + 4, args=beams(lengths=SOME)),
    dict(x=mat(cols=5000, stride=5000), work=None), dict(x=mat(cols=5000, stride=5000), work=SOME + 4),
    dict(x=mat(cols=5000, stride=5000), have=64),
]


@pytest.mark.parametrize("i", range(len(BAD_BEAMS)))
def test_bad_beams(lib, i):
    assert step(lib, **BAD_BEAMS[i]) == bf.BF_EINVAL
    assert bf.last_error().startswith("bf_beam_step")


@pytest.mark.parametrize("a,b", [(a, b) for a in range(5) for b in range(a + 1, 9)])
def test_beams_overlap(lib, a, b):
    """An output in the last bytes of an input or of another output."""
    where = [SOME + (i << 20) for i in range(9)]  # scores, tokens, parents, finished, lengths; scores, finished, lengths, logits
    length = [32, 64, 64, 8, 64, 32, 8, 64, 7 * 100 + 100][b]
    where[a] = where[b] + length - 8
    args = beams(scores=where[5], finished=where[6], lengths=where[7], end_token=1)
    assert step(lib, mat(data=where[8]), args, *where[:5]) == bf.BF_EINVAL
    assert "overlaps" in bf.last_error()


def test_beams_null_and_none(lib):
    x, args = mat(), beams()
    assert lib.bf_beam_step(None, at(args), SOME, SOME, SOME, None, None, SOME, 1 << 30, None) == bf.BF_EINVAL
    assert lib.bf_beam_step(at(x), None, SOME, SOME, SOME, None, None, SOME, 1 << 30, None) == bf.BF_EINVAL
    assert step(lib, x=mat(rows=0, data=None), args=beams(groups=0, scores=None), scores=None, tokens=None, parents=None, work=None, have=0) == bf.BF_OK


def test_beams_workspace(lib):
    n = ctypes.c_uint64(0)
    sizes = []
    for groups, vocab, keep in ((1, 3, 1), (1, 5000, 4), (8, 5000, 4), (8, 131072, 4), (64, 131072, 256)):
        assert lib.bf_beam_step_workspace(groups, 4, vocab, keep, ctypes.byref(n)) == bf.BF_OK
        sizes.append(n.value)
        assert n.value % 256 == 0
    assert sizes == sorted(sizes)
    for bad in ((1, 0, 10, 1), (1, 257, 10, 1), (1, 4, 10, 0), (1, 4, 10, 257), (1 << 23, 4, 10, 1), (1, 4, 0, 1), (1, 4, (1 << 24) + 1, 1)):
        assert lib.bf_beam_step_workspace(*bad, ctypes.byref(n)) == bf.BF_EINVAL
    assert lib.bf_beam_step_workspace(1, 4, 10, 1, None) == bf.BF_EINVAL


def layout(rows=8, tokens=10, heads=1, width=64, **strides):
    s = dict(row_stride=tokens * heads * width, token_stride=heads * width, head_stride=width)
    s.update(strides)
    return bf.States(rows, tokens, heads, width, s["row_stride"], s["token_stride"], s["head_stride"])


def reorder(lib, a=None, b=None, frm=(SOME,), to=(FAR,), parents=SOME, beams=4, lengths=None, count=None):
    table = lambda v: None if v is None else (ctypes.c_void_p * max(1, len(v)))(*v)
    return lib.bf_beam_reorder(table(frm), a or layout(), table(to), b or a or layout(), len(frm) if count is None else count, parents,
                               beams, lengths, None)


BAD_REORDER = [
    dict(b=layout(rows=4)), dict(b=layout(tokens=9)), dict(b=layout(heads=2, width=32)), dict(beams=0), dict(beams=3), dict(beams=257),
    dict(parents=None), dict(parents=SOME + 4), dict(lengths=SOME + 4), dict(frm=(None,)), dict(to=(None,)), dict(frm=None, count=1),
    dict(to=None, count=1), dict(count=129), dict(a=layout(rows=1 << 31)), dict(a=layout(tokens=1 << 31)), dict(a=layout(width=1 << 31)),
    dict(a=layout(row_stride=1 << 42)), dict(a=layout(heads=1 << 16, width=1 << 16)), dict(b=layout(row_stride=639)),
    dict(b=layout(token_stride=63)), dict(b=layout(row_stride=0)), dict(frm=(SOME, SOME), to=(FAR, FAR)),
    dict(frm=(SOME, SOME), to=(FAR, FAR + 5119)), dict(to=(SOME + 64,)), dict(frm=(SOME, FAR), to=(SOME, FAR + (1 << 20))),
    dict(frm=(SOME, FAR), to=(FAR, SOME)), dict(b=layout(row_stride=1280), to=(SOME,)),
]


@pytest.mark.parametrize("i", range(len(BAD_REORDER)))
def test_bad_reorder(lib, i):
    assert reorder(lib, **BAD_REORDER[i]) == bf.BF_EINVAL
    assert bf.last_error().startswith("bf_beam_reorder: ")


def test_reorder_of_nothing(lib):
    assert reorder(lib, frm=(), to=()) == bf.BF_OK
    for empty in (layout(rows=0), layout(tokens=0), layout(heads=0), layout(width=0)):
        assert reorder(lib, a=empty, b=empty, frm=(SOME,), to=(SOME,)) == bf.BF_OK
