"""The operators of a decoding step on the GPU against plain 64-bit forms.

Tolerances.  Attention: a score's 32-bit sum of `dim` products is off by (dim + 4) 2^-24 of the sum of their magnitudes,
scaled; its exponential by 2^-22 more, and by half a last place of exponents of up to 2^7 (2^-17 of the weight at most
for |s - max| < 128, below which weights do not count); the sums of n weights by (n + 16) 2^-24.  Weights rounded to a 16-bit type are off by
half a step (fp16: or 2^-25 of the largest, below 2^-14), and the output, rounded once, by half a step.
Beams: the exponentials are off by 2^-22, their sums over a thread's 64, 13 joins and the chunks by 2^-24 each, the
exponents by 2^-23 of themselves, which weigh in by at most their mean under softmax, log2 of the vocabulary; scores are rounded once.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import answer_ref as ref  # noqa: E402
from paper_2607_22242_gb300 import bf  # noqa: E402

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -9, "f16": 2.0 ** -12}  # half a step, relative to the power of two below
INF, NAN = float("inf"), float("nan")


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.fail("no CUDA device: GPU tests need one")
    bf.load()


def np64(t):
    return t.detach().double().cpu().numpy()


def half(t):
    """Half a step of type t, relative to the value."""
    return torch.finfo(TYPES[t]).eps / 2


# ---- attention ------------------------------------------------------------------------------------------------------

def attention_inputs(prompts, each, heads, kv_heads, dim, prefix, suffix, dtype, seed=0, spread=1.5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *n: torch.randn(*n, generator=gen, device="cuda").to(TYPES[dtype])
    n = prompts * each
    own = (None, None) if suffix is None else (rand(n, suffix, kv_heads, dim), rand(n, suffix, kv_heads, dim))
    return (spread * rand(n, heads, dim), rand(prompts, prefix, kv_heads, dim), rand(prompts, prefix, kv_heads, dim), *own)


def check_attention(x, dtype, prefix_lengths=None, suffix_lengths=None, scale=None, got=None):
    q, pk, pv, sk, sv = x
    prompts, answers = pk.shape[0], q.shape[0]
    pl = [pk.shape[1]] * prompts if prefix_lengths is None else prefix_lengths
    sl = [0 if sk is None else sk.shape[1]] * answers if suffix_lengths is None else suffix_lengths
    length = lambda v: None if v is None else torch.tensor(v, dtype=torch.int64, device="cuda")
    scale = q.shape[2] ** -0.5 if scale is None else scale
    if got is None:
        got = bf.prefix_attention(*x, prefix_lengths=length(prefix_lengths),
                                  suffix_lengths=length(suffix_lengths) if sk is not None else None, scale=scale, lse=True)
    out, lse = (np64(t) for t in got)
    a = [None if t is None else np64(t) for t in x]
    want, want_lse, size, most = ref.attention(*a, pl, sl, scale)
    n = np.array([pl[i // (answers // prompts)] + sl[i] for i in range(answers)])[:, None]
    weight = 2 * (q.shape[2] + 4) * 2.0 ** -24 * abs(scale) * most + 2.0 ** -22 + 2.0 ** -17
    total = weight + (n + 16) * 2.0 ** -24
    tiny = 0.0
    if dtype != "f32":
        weight = weight + half(dtype)
        if dtype == "f16":
            tiny = n[:, :, None] * 2.0 ** -25 * max([np.abs(t[np.isfinite(t)]).max(initial=0) for t in (a[2], *a[4:]) if t is not None])
    bound = (weight + total)[:, :, None] * size + tiny + half(dtype) * np.abs(want) * (1 + 2.0 ** -8) + (2.0 ** -25 if dtype == "f16" else 0)
    assert np.array_equal(np.isnan(out), np.isnan(want))
    worst = np.nanmax(np.abs(out - want) / np.maximum(bound, 1e-300), initial=0.0)
    assert worst <= 1.0
    none = np.isneginf(want_lse)
    assert np.array_equal(none, np.isneginf(lse)) and not out[none].any()
    with np.errstate(invalid="ignore"):
        off = np.where(none, 0.0, np.abs(lse - want_lse))
    worst = (off / (total + 2.0 ** -23 * (np.abs(np.where(none, 0, want_lse)) + most * abs(scale)))).max(initial=0.0)
    assert worst <= 1.0


SHAPES = [  # prompts, answers of each, heads, key heads, dim, prefix, suffix
    (1, 1, 1, 1, 64, 1, 1), (1, 1, 8, 2, 64, 600, 32), (1, 4, 8, 2, 128, 129, 1), (2, 5, 12, 4, 80, 333, 21),
    (3, 7, 7, 1, 40, 257, 130), (1, 33, 8, 2, 128, 515, 9), (1, 70, 4, 1, 64, 300, 33), (2, 3, 32, 8, 128, 1025, 65),
    (1, 2, 20, 1, 96, 64, 64), (5, 1, 4, 4, 8, 63, 17), (2, 2, 2, 1, 256, 90, 20), (1, 3, 3, 3, 1, 40, 5),
    (2, 3, 4, 2, 33, 70, 11), (1, 16, 4, 1, 200, 140, 70), (1, 130, 2, 1, 128, 200, 3),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_attention(shape, dtype):
    check_attention(attention_inputs(*shape, dtype, seed=sum(shape)), dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,each", [(64, 2), (128, 20), (40, 33), (50, 3)])
def test_attention_lengths(dtype, dim, each):
    """Prompts and answers of every length around a tile's end, some of none at all, in one batch."""
    prefix = [0, 1, 63, 64, 65, 127, 128, 129, 300, 0, 256]
    x = attention_inputs(len(prefix), each, 4, 2, dim, 300, 140, dtype, seed=dim)
    suffix = [(0, 1, 2, 31, 63, 64, 65, 100, 140)[i % 9] for i in range(len(prefix) * each)]
    check_attention(x, dtype, prefix, suffix)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("each,share", [(2, 2), (40, 4), (5, 30)])
def test_attention_many_tiles(dtype, dim, each, share):
    """Many tiles of keys and several pieces to each block, of uneven prompts."""
    rng = np.random.default_rng(dim + each)
    prompts, kv_heads = 20, 8
    x = attention_inputs(prompts, each, kv_heads * share, kv_heads, dim, 2500, None, dtype, seed=each)
    lengths = rng.integers(0, 2501, prompts)
    lengths[:3] = 2500, 0, 1
    on = torch.tensor(lengths, device="cuda")
    out, lse = bf.prefix_attention(*x[:3], prefix_lengths=on, lse=True)
    q, k, v = (t.double() for t in x[:3])
    s = torch.einsum("pagsd,ptgd->pagst", q.view(prompts, each, kv_heads, share, dim), k) * dim ** -0.5
    s = s.masked_fill((torch.arange(2500, device="cuda") >= on[:, None])[:, None, None, None], -INF)
    top = s.max(-1, keepdim=True).values.clamp(min=-1e300)
    w = torch.exp(s - top)
    total = w.sum(-1, keepdim=True)
    want = torch.einsum("pagst,ptgd->pagsd", w, v) / total.clamp(min=1e-300)
    size = torch.einsum("pagst,ptgd->pagsd", w, v.abs()) / total.clamp(min=1e-300)
    out, lse = out.double().view(want.shape), lse.double().view(total.shape)
    # As check_attention, with the bounds of 2,500 keys and of the largest score and value.
    most = torch.einsum("pagsd,ptgd->pagst", q.view(prompts, each, kv_heads, share, dim).abs(), k.abs()).max().item() * dim ** -0.5
    weight = 2 * (dim + 4) * 2.0 ** -24 * most + 2.0 ** -22 + 2.0 ** -17
    sums = weight + 2516 * 2.0 ** -24
    tiny = 2500 * 2.0 ** -25 * v.abs().max() + 2.0 ** -25 if dtype == "f16" else 0.0
    bound = (weight + half(dtype) + sums) * size + tiny + half(dtype) * (1 + 2.0 ** -8) * want.abs()
    assert ((out - want).abs() <= bound).all()
    none = total == 0
    assert not out[none.expand_as(out)].any() and torch.isneginf(lse[none]).all()
    assert ((lse - top - torch.log(total))[~none].abs() <= sums + 2.0 ** -23 * (most + 20)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("prompts,each", [(33, 3), (128, 9), (130, 17), (200, 1)])
def test_attention_many_prompts(dtype, dim, prompts, each):
    """More prompts than a warp has lanes, most of one tile or none, some of a few."""
    x = attention_inputs(prompts, each, 8, 2, dim, 400, 20, dtype, seed=prompts)
    prefix = [(0, 1, 128, 17, 0, 129, 400, 64, 127)[i % 9] for i in range(prompts)]
    prefix[prompts // 2:prompts // 2 + 5] = [0] * 5
    prefix[-1] = 300
    check_attention(x, dtype, prefix, [(20, 0, 7, 16)[i % 4] for i in range(prompts * each)])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 72, 128])
@pytest.mark.parametrize("each,share", [(1, 16), (2, 40), (9, 4)])
def test_attention_many_pieces(dtype, dim, each, share):
    """One prompt's keys in pieces of all blocks, more of them than an answer's joining holds at once."""
    x = attention_inputs(1, each, share, 1, dim, 19700, 90, dtype, seed=each)
    check_attention(x, dtype, [19650], [90 - i for i in range(each)])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("prompts,kv_heads", [(1, 1), (2, 2), (4, 2), (9, 2)])
def test_attention_shared_widely(dtype, dim, prompts, kv_heads):
    """An answer's 20 query heads of a key head in two parts, some of which lie in two tiles of a prompt's queries."""
    x = attention_inputs(prompts, 40, 20 * kv_heads, kv_heads, dim, 700, 100, dtype, seed=prompts)
    check_attention(x, dtype, [700 - 150 * (i % 5) for i in range(prompts)], [(100, 0, 1, 33, 64)[i % 5] for i in range(40 * prompts)])


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_nothing(dtype):
    x = attention_inputs(2, 3, 4, 2, 64, 10, 4, dtype)
    check_attention(x, dtype, [0, 10], [0, 1, 0, 0, 4, 0])
    q = x[0]
    out, lse = bf.prefix_attention(q, x[1][:, :0], x[2][:, :0], lse=True)
    assert not out.any() and torch.isneginf(lse).all()
    out, lse = bf.prefix_attention(q, x[1][:, :0], x[2][:, :0], x[3], x[4], lse=True)
    check_attention((q, x[1], x[2], x[3], x[4]), dtype, [0, 0], None, got=(out, lse))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 72, 30])
def test_attention_without_suffix(dtype, dim):
    check_attention(attention_inputs(2, 9, 8, 4, dim, 190, None, dtype), dtype, [190, 77])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 72, 30])
def test_attention_behind_lengths(dtype, dim):
    """NaN and infinities behind every length change nothing."""
    x = attention_inputs(3, 4, 4, 2, dim, 200, 70, dtype, seed=3)
    pl, sl = [130, 0, 199], [70, 0, 1, 33, 64, 65, 2, 3, 69, 5, 6, 7]
    for t, lengths, bad in ((x[1], pl, NAN), (x[2], pl, INF), (x[3], sl, -INF), (x[4], sl, NAN)):
        for i, n in enumerate(lengths):
            t[i, n:] = bad
    check_attention(x, dtype, pl, sl)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 30])
def test_attention_bad_lengths(dtype, dim):
    """A length outside its cache makes its answers NaN and no others."""
    x = attention_inputs(3, 2, 4, 2, dim, 100, 20, dtype)
    to = lambda v: torch.tensor(v, device="cuda")
    good, good_lse = bf.prefix_attention(*x, prefix_lengths=to([100, 0, 50]), suffix_lengths=to([20, 1, 2, 3, 4, 5]), lse=True)
    out, lse = bf.prefix_attention(*x, prefix_lengths=to([100, 101, 50]), suffix_lengths=to([20, -1, 2, 3, 1 << 40, 5]), lse=True)
    bad = torch.tensor([0, 1, 1, 1, 1, 0], dtype=torch.bool)
    assert torch.isnan(out[bad]).all() and torch.isnan(lse[bad]).all()
    assert torch.equal(out[~bad], good[~bad]) and torch.equal(lse[~bad], good_lse[~bad])


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_layouts(dtype):
    """Heads ahead of tokens, strided queries and outputs, broadcast keys, offsets that break 16-byte alignment."""
    for dim in (64, 128):
        base = attention_inputs(2, 6, 8, 2, dim, 150, 40, dtype, seed=7)
        pl, sl = [150, 90], [40, 0, 1, 2, 39, 17, 33, 34, 35, 36, 37, 38]
        ahead = tuple(base[:1]) + tuple(t.transpose(1, 2).contiguous().transpose(1, 2) for t in base[1:])
        check_attention(ahead, dtype, pl, sl)

        def shifted(t, by):
            buf = torch.zeros(t.numel() + t.shape[0] * 24 + 64, dtype=t.dtype, device="cuda")
            inner = t[0].numel() + 24
            s = buf.as_strided(t.shape, (inner, *t.stride()[1:]), by)
            s.copy_(t)
            return s
        check_attention(tuple(shifted(t, 8) for t in base), dtype, pl, sl)
        check_attention(tuple(shifted(t, 1 + i) for i, t in enumerate(base)), dtype, pl, sl)
        one = attention_inputs(1, 6, 8, 1, dim, 150, 40, dtype, seed=8)
        wide = (one[0], *(t.expand(t.shape[0], t.shape[1], 4, dim) for t in one[1:]))
        check_attention(wide, dtype)
        many = (base[0], base[1][:1].expand(2, -1, -1, -1), base[2][:1].expand(2, -1, -1, -1), base[3], base[4])
        check_attention(many, dtype, pl, sl)
        out = torch.full((12, 11, dim + 16), 5.0, dtype=TYPES[dtype], device="cuda")
        got = bf.prefix_attention(*base, lse=True, out=out[:, 1:9, 8:8 + dim])
        check_attention(base, dtype, got=got)
        out[:, 1:9, 8:8 + dim] = 5.0
        assert (out == 5.0).all()
        out = torch.empty(8, 12, dim + 1, dtype=TYPES[dtype], device="cuda").transpose(0, 1)[:, :, 1:]
        check_attention(base, dtype, got=bf.prefix_attention(*base, lse=True, out=out))


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_extremes(dtype):
    """Large scores, a scale below 0, keys that grow from tile to tile, one key that takes all, keys of the lowest value."""
    x = attention_inputs(1, 9, 4, 2, 64, 700, 50, dtype, seed=5)
    check_attention(x, dtype, scale=3.0)
    check_attention(x, dtype, scale=-0.2)
    check_attention(x, dtype, scale=0.0)
    grow = torch.linspace(0.01, 4.0, 700, device="cuda").to(TYPES[dtype])[None, :, None, None]
    check_attention((x[0], x[1] * grow, *x[2:]), dtype)
    check_attention((x[0], x[1] * grow.flip(1), *x[2:]), dtype)
    y = [t.clone() for t in x]
    y[1][0, 333] = y[0][0, 0] * 8  # a score far above the others' for some heads, far below for others
    check_attention(tuple(y), dtype)
    low = torch.finfo(TYPES[dtype]).min
    y = [t.clone() for t in x]
    y[0].abs_()
    y[1][:, ::2] = low if dtype == "f16" else -1e30  # scores of about -1e6 and -1e31: no weight
    y[3][:, :7] = low if dtype == "f16" else -1e30
    q = [t for t in y]
    out = bf.prefix_attention(*q)
    keep_p, keep_s = torch.arange(1, 700, 2, device="cuda"), torch.arange(7, 50, device="cuda")
    want = bf.prefix_attention(q[0], q[1][:, keep_p], q[2][:, keep_p], q[3][:, keep_s], q[4][:, keep_s])
    assert torch.allclose(out.float(), want.float(), rtol=4 * half(dtype), atol=8 * half(dtype))


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_not_finite(dtype):
    """NaN in a query or a used key makes that row NaN; keys of -inf scores leave a row without weights empty."""
    x = attention_inputs(1, 3, 2, 1, 64, 80, 5, dtype, seed=6)
    clean = bf.prefix_attention(*x)
    y = [t.clone() for t in x]
    y[0][1, 1, 5] = NAN
    out, lse = bf.prefix_attention(*y, lse=True)
    assert torch.isnan(out[1, 1]).all() and torch.isnan(lse[1, 1])
    keep = torch.ones(3, 2, dtype=torch.bool)
    keep[1, 1] = False
    assert torch.equal(out[keep], clean[keep])
    y = [t.clone() for t in x]
    y[1][0, 40, 0, 3] = NAN
    assert torch.isnan(bf.prefix_attention(*y)).all()
    y = [t.clone() for t in x]
    y[3][2, 4, 0, 3] = NAN
    out = bf.prefix_attention(*y)
    assert torch.isnan(out[2]).all() and torch.equal(out[:2], clean[:2])
    y = [t.clone() for t in x]
    y[0].fill_(1.0)
    y[1].fill_(-INF)
    y[3].fill_(-INF)
    out, lse = bf.prefix_attention(*y, lse=True)
    assert not out.any() and torch.isneginf(lse).all()
    y[3][1, 2].fill_(0.5)
    out, lse = bf.prefix_attention(*y, lse=True)
    assert torch.allclose(out[1].float(), y[4][1, 2].float().expand(2, -1), rtol=half(dtype)) and torch.isneginf(lse[0]).all()


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("f16", 64), ("f32", 80)])
def test_attention_long(dtype, dim):
    """A prompt of many tiles for one answer and for many, and the joining of two halves by their sums."""
    x = attention_inputs(1, 3, 4, 2, dim, 20011, 300, dtype, seed=9)
    check_attention(x, dtype)
    a, la = bf.prefix_attention(x[0], x[1][:, :9000], x[2][:, :9000], lse=True)
    b, lb = bf.prefix_attention(x[0], x[1][:, 9000:], x[2][:, 9000:], x[3], x[4], lse=True)
    m = torch.maximum(la, lb)
    wa, wb = torch.exp(la - m)[..., None], torch.exp(lb - m)[..., None]
    joined = (a.float() * wa + b.float() * wb) / (wa + wb)
    whole = bf.prefix_attention(*x)
    assert torch.allclose(joined, whole.float(), rtol=0, atol=8 * half(dtype))


def test_attention_same_bits_and_graph():
    """The same call gives the same bits, also captured and replayed over new inputs, and on another stream."""
    x = attention_inputs(2, 16, 8, 2, 128, 900, 60, "bf16", seed=10)
    pl, sl = torch.tensor([900, 333], device="cuda"), torch.arange(32, device="cuda")
    kw = dict(prefix_lengths=pl, suffix_lengths=sl, lse=True)
    first, lse = bf.prefix_attention(*x, **kw)
    for _ in range(20):
        again, lse2 = bf.prefix_attention(*x, **kw)
        assert torch.equal(first, again) and torch.equal(lse, lse2)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        other, _ = bf.prefix_attention(*x, **kw)
    third, _ = bf.prefix_attention(*x, **kw, stream=side)
    side.synchronize()
    assert torch.equal(first, other) and torch.equal(first, third)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held, _ = bf.prefix_attention(*x, **kw)
    for seed in (11, 12):
        y = attention_inputs(2, 16, 8, 2, 128, 900, 60, "bf16", seed=seed)
        for a, b in zip(x, y):
            a.copy_(b)
        pl.copy_(torch.tensor([seed, 900 - seed], device="cuda"))
        sl.copy_(sl.flip(0))
        graph.replay()
        want, _ = bf.prefix_attention(*x, **kw)
        assert torch.equal(held, want)


def test_attention_refusals():
    x = attention_inputs(2, 2, 4, 2, 64, 10, 4, "bf16")
    q, pk, pv, sk, sv = x
    call = bf.prefix_attention
    with pytest.raises(ValueError):
        call(q[0], pk, pv)
    with pytest.raises(ValueError):
        call(q, pk[0], pv)
    with pytest.raises(ValueError):
        call(q.double(), pk, pv)
    with pytest.raises(ValueError):
        call(q.transpose(1, 2), pk, pv)
    with pytest.raises(ValueError):
        call(q, pk, pv, prefix_lengths=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        call(q, pk, pv, suffix_lengths=torch.zeros(4, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        call(q.cpu(), pk, pv)
    for bad in ((q, pk.float(), pv.float()), (q, pk, pv[:, :9]), (q[:3], pk, pv), (q[:, :3], pk, pv), (q, pk, pv, sk[:3], sv[:3]),
                (q, pk, pv, sk), (q, pk, pv, sk[:, :, :1], sv[:, :, :1])):
        with pytest.raises(bf.BfError) as e:
            call(*bad)
        assert e.value.code == bf.BF_EINVAL
    for out in (q, torch.empty_like(q[:, :2]), torch.empty_like(q).float(), torch.empty(1, 4, 64, dtype=q.dtype, device="cuda").expand(4, 4, 64)):
        with pytest.raises(bf.BfError):
            call(q, pk, pv, out=out)
    with pytest.raises(bf.BfError):
        call(q, pk, pv, scale=NAN)
    empty = call(q[:0], pk, pv)
    assert empty.shape == (0, 4, 64)


# ---- beams ----------------------------------------------------------------------------------------------------------

def check_beams(logits, scores, beams, keep=None, finished=None, lengths=None, end_token=-1, penalty=0.0, tau=1.0, got=None):
    keep = beams if keep is None else keep
    to = lambda v, t: None if v is None else torch.tensor(v, dtype=t, device="cuda")
    if got is None:
        got = bf.beam_step(logits, torch.tensor(scores, device="cuda"), beams, keep=keep, finished=to(finished, torch.bool),
                           lengths=to(lengths, torch.int64), length_penalty=penalty, end_token=end_token, temperature=tau)
    x = np64(logits)
    vocab = x.shape[1]
    tau32 = float(np.float32(tau))
    want = ref.beam_step(x, np.float32(scores), beams, keep, finished, lengths, end_token, float(np.float32(penalty)), tau32)
    best, tokens, parents, ended = (t.cpu().numpy() for t in got[:4])
    n_got = None if got.lengths is None else got.lengths.cpu().numpy()
    off = 2.0 ** -22 + (64 + 13 + vocab / 4096) * 2.0 ** -24 + max(1.0, np.log2(vocab)) * 2.0 ** -23
    for g, rows in enumerate(want):
        place = {(r[3], r[2]): i for i, r in enumerate(rows)}
        seen = set()
        for j in range(keep):
            here = (int(parents[g, j]), int(tokens[g, j]))
            if j >= len(rows):
                assert best[g, j] == -np.inf and here == (g * beams + j % beams, -1) and not ended[g, j]
                assert n_got is None or n_got[g, j] == 0
                continue
            assert here in place and here not in seen, (g, j, here)
            seen.add(here)
            rank, total, _, _, end, n = rows[place[here]]
            slack = off / max(1, n if penalty else 1) ** penalty + 1e-12
            assert rank >= rows[j][0] - 2 * slack, (g, j, here, rank, rows[j])
            alone = all(abs(rows[i][0] - rows[j][0]) > 2 * slack or rows[i][0] == rows[j][0] for i in (j - 1, j + 1) if 0 <= i < len(rows))
            if alone:
                assert here == (rows[j][3], rows[j][2]), (g, j, here, rows[max(0, j - 1):j + 2])
            assert abs(best[g, j] - total) <= off + 2.0 ** -24 * abs(total)
            assert bool(ended[g, j]) == end and (n_got is None or n_got[g, j] == n)
    return got


def beam_inputs(groups, beams, vocab, dtype, seed=0, banned=0.0):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(groups * beams, vocab)) * 2.0
    if banned:
        x[rng.random(x.shape) < banned] = -np.inf
    scores = np.float32(-rng.random(groups * beams) * 6)
    return torch.tensor(x, dtype=torch.float32, device="cuda").to(TYPES[dtype]), scores.tolist(), rng


BEAMS = [  # groups, beams, vocabulary, keep
    (1, 1, 1, 1), (3, 4, 3, 4), (50, 16, 3, 16), (2, 3, 7, 6), (5, 8, 100, 8), (1, 4, 4096, 4), (2, 2, 2049, 5),
    (1, 4, 5003, 8), (3, 5, 16384, 10), (2, 3, 16385, 1), (2, 1, 33001, 256), (1, 2, 70001, 200), (1, 64, 300, 64),
    (2, 256, 20, 256), (1, 256, 40, 100), (90, 4, 9001, 4), (1, 33, 129, 66), (2, 40, 70000, 33), (1, 130, 40003, 256),
    (40, 9, 17000, 9), (1, 1, 1 << 20, 3), (6, 8, 30000, 128), (2, 8, 16384, 256), (3, 5, 600, 20), (3, 9, 1100, 30), (5, 3, 1500, 24),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", BEAMS, ids=str)
def test_beams(shape, dtype):
    groups, beams, vocab, keep = shape
    x, scores, _ = beam_inputs(groups, beams, vocab, dtype, seed=sum(shape))
    check_beams(x, scores, beams, keep)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(6, 8, 3, 8), (4, 8, 600, 16), (3, 6, 9001, 12)], ids=str)
def test_beams_options(shape, dtype):
    """Finished and dead beams, a length penalty, a temperature, banned tokens."""
    groups, beams, vocab, keep = shape
    x, scores, rng = beam_inputs(groups, beams, vocab, dtype, seed=sum(shape), banned=0.4)
    rows = groups * beams
    finished = (rng.random(rows) < 0.4).tolist()
    lengths = rng.integers(0, 30, rows).tolist()
    for i in range(0, rows, 5):
        scores[i] = -INF
    for i in np.nonzero(finished)[0]:
        x[int(i)] = NAN  # not used
    check_beams(x, scores, beams, keep, finished, lengths, end_token=1, penalty=0.8, tau=0.6)
    check_beams(x, scores, beams, keep, finished, None, end_token=vocab + 5, tau=1.7)
    check_beams(x, scores, beams, keep, finished, lengths, end_token=0)
    check_beams(x, scores, beams, keep, [True] * rows, lengths, end_token=0, penalty=1.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,beams,keep", [
    (1025, 4, 90), (1100, 6, 64), (2049, 4, 16), (4097, 5, 100), (8193, 4, 1), (16385, 3, 40), (33000, 2, 200), (50001, 2, 32)])
@pytest.mark.parametrize("pad", [0, 1, 2, 3, 5])
def test_beams_cuts(vocab, beams, keep, pad, dtype):
    """Rows a little longer than a tile or a chunk, at every alignment, groups few and many: rows cut in all ways."""
    for groups in (1, 40 if vocab < 9000 else 3):
        x, scores, _ = beam_inputs(groups, beams, vocab, dtype, seed=vocab + pad)
        wide = torch.full((groups * beams, vocab + pad), 60000.0, dtype=x.dtype, device="cuda")
        wide[:, pad // 2:pad // 2 + vocab] = x
        check_beams(wide[:, pad // 2:pad // 2 + vocab], scores, beams, keep)


def test_beams_long_rows():
    """A row of many more chunks than a thread of a group's block has."""
    for vocab in (4900000, 4900001):
        x, scores, _ = beam_inputs(1, 1, vocab, "bf16", seed=5)
        check_beams(x, scores, 1, 8)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [5, 1000, 20000, 50001, 300000])
def test_beams_ties(vocab, dtype):
    """Equal logits everywhere, equal rows at every alignment, a few values only: ties go to the lower beam and token."""
    same = torch.zeros(6, vocab, dtype=TYPES[dtype], device="cuda")
    got = check_beams(same, [-1.0] * 6, 3, 9)
    first = [[g * 3 + j // vocab for j in range(9)] for g in range(2)]
    assert got.parents.tolist() == first and got.tokens.tolist() == [[j % vocab for j in range(9)]] * 2
    rng = np.random.default_rng(vocab)
    row = torch.tensor(rng.normal(size=vocab), dtype=torch.float32, device="cuda").to(TYPES[dtype])
    got = bf.beam_step(row.expand(8, vocab).contiguous(), torch.full((8,), -2.0, device="cuda"), 8, keep=16)
    order = torch.sort(row.float(), descending=True, stable=True).indices[:2].tolist()
    assert got.parents[0].tolist() == [i % 8 for i in range(16)]
    assert got.tokens[0].tolist() == [order[0]] * 8 + [order[1]] * 8
    few = torch.tensor(rng.integers(0, 3, (4, vocab)), dtype=torch.float32, device="cuda").to(TYPES[dtype])
    check_beams(few, [-1.0, -1.5, -1.0, -1.0], 2, 40 if vocab > 5 else 10)
    many = torch.zeros(120, vocab, dtype=TYPES[dtype], device="cuda")  # more lists than are noted
    got = bf.beam_step(many, torch.zeros(120, device="cuda"), 120, keep=256)
    assert got.parents[0].tolist() == [j // vocab for j in range(256)] and got.tokens[0].tolist() == [j % vocab for j in range(256)]
    signed = torch.zeros(2, vocab, dtype=TYPES[dtype], device="cuda")
    signed[:, 1::2] = -0.0
    got = bf.beam_step(signed, torch.zeros(2, device="cuda"), 2, keep=4)
    assert got.tokens.tolist() == [[0, 1, 2, 3]] and got.parents.tolist() == [[0] * 4]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [40, 9001])
def test_beams_empty(vocab, dtype):
    """Rows without a token left, groups without a beam alive, fewer continuations than places."""
    x, scores, _ = beam_inputs(3, 4, vocab, dtype, seed=1)
    x[0:3] = -INF
    x[3] = -INF
    x[3, 7], x[3, 20] = 1.0, 2.0
    scores[4:8] = [-INF] * 4
    got = check_beams(x, scores, 4, 8)
    assert got.tokens[0].tolist() == [20, 7] + [-1] * 6 and got.tokens[1].tolist() == [-1] * 8
    x[3] = -INF
    check_beams(x, scores, 4, 8)
    low = torch.finfo(TYPES[dtype]).min
    x[8:] = low
    x[9, 5] = 0.0
    check_beams(x, scores, 4, 3)


@pytest.mark.parametrize("vocab", [40, 9001])
def test_beams_not_finite(vocab):
    """NaN or +inf among a live beam's logits or scores makes its group NaN, and no other."""
    x, scores, _ = beam_inputs(4, 2, vocab, "bf16", seed=2)
    good = bf.beam_step(x, torch.tensor(scores, device="cuda"), 2)
    bad = x.clone()
    bad[1, 3], bad[4, vocab - 1] = NAN, INF
    s = torch.tensor(scores, device="cuda")
    s[6] = NAN
    got = bf.beam_step(bad, s, 2)
    assert torch.isnan(got.scores[[0, 2, 3]]).all() and (got.tokens[[0, 2, 3]] == -1).all()
    assert got.parents.tolist()[0] == [0, 1] and torch.equal(got.scores[1], good.scores[1]) and torch.equal(got.tokens[1], good.tokens[1])
    s = torch.tensor(scores, device="cuda")
    s[1] = -INF
    alive = bf.beam_step(bad[:2], s[:2], 2)
    assert (alive.parents == 0).all() and torch.isfinite(alive.scores).all()


def test_beams_strides_and_repeats():
    x, scores, _ = beam_inputs(2, 4, 9001, "f16", seed=3)
    wide = torch.full((8, 9100), 60000.0, dtype=torch.float16, device="cuda")
    for shift in (0, 1, 5, 64):
        view = wide[:, shift:shift + 9001]
        view.copy_(x)
        first = check_beams(view, scores, 4)
        for _ in range(10):
            again = bf.beam_step(view, torch.tensor(scores, device="cuda"), 4)
            assert all(torch.equal(a, b) for a, b in zip(first[:4], again[:4]))
        wide.fill_(60000.0)
    s = torch.tensor(scores, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = bf.beam_step(x, s, 4)
    for seed in (4, 5):
        y, new, _ = beam_inputs(2, 4, 9001, "f16", seed=seed)
        x.copy_(y)
        s.copy_(torch.tensor(new))
        graph.replay()
        check_beams(x, new, 4, got=held)


@pytest.mark.parametrize("tau", [1e-18, 1e-3, 1e4, 1e18])
def test_beams_temperatures(tau):
    """Temperatures at the ends of their range: the order within a beam is the logits'."""
    for vocab in (50, 9001):
        x, _, _ = beam_inputs(1, 1, vocab, "f32", seed=6)
        got = bf.beam_step(x, torch.zeros(1, device="cuda"), 1, keep=5, temperature=tau)
        assert got.tokens[0, 0].item() == x[0].argmax().item() and torch.isfinite(got.scores[0, 0])
        if tau <= 1e4:
            assert got.tokens[0].tolist() == torch.topk(x[0], 5).indices.tolist()


def test_beams_refusals():
    x, scores, _ = beam_inputs(2, 4, 50, "f32")
    s = torch.tensor(scores, device="cuda")
    for kw in (dict(beams=3), dict(beams=0), dict(beams=257)):
        with pytest.raises(ValueError):
            bf.beam_step(x, s, **kw)
    for kw in (dict(scores=s[:7]), dict(scores=s.double()), dict(finished=torch.zeros(8, device="cuda")),
               dict(lengths=torch.zeros(8, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            bf.beam_step(x, kw.pop("scores", s), 4, **kw)
    on = torch.zeros(8, dtype=torch.bool, device="cuda")
    for kw in (dict(keep=0), dict(keep=257), dict(finished=on), dict(length_penalty=1.0), dict(length_penalty=-1.0),
               dict(temperature=0.0), dict(temperature=NAN), dict(end_token=-2)):
        with pytest.raises(bf.BfError) as e:
            bf.beam_step(x, s, 4, **kw)
        assert e.value.code == bf.BF_EINVAL
    none = bf.beam_step(x[:0], s[:0], 4)
    assert none.tokens.shape == (0, 4)


# ---- states ---------------------------------------------------------------------------------------------------------

def random_states(shape, dtype, count, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randint(-100, 100, shape, generator=gen, device="cuda").to(dtype) for _ in range(count)]


STATES = [  # groups, beams, tokens, the rest
    (1, 1, 1, ()), (2, 4, 7, ()), (1, 8, 512, (2, 64)), (3, 5, 33, (3, 5)), (2, 16, 100, (64,)), (1, 256, 9, (4,)),
    (40, 3, 70, (1, 40)), (1, 2, 3000, (8, 128)), (2, 33, 50, (2, 9)),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.int64, torch.uint8], ids=str)
@pytest.mark.parametrize("shape", STATES, ids=str)
@pytest.mark.parametrize("in_place", [True, False])
def test_reorder(shape, dtype, in_place):
    groups, beams, tokens, rest = shape
    rows = groups * beams
    rng = np.random.default_rng(sum(shape[:3]))
    states = random_states((rows, tokens, *rest), dtype, 3)
    keep = [t.clone() for t in states]
    for kind in range(4):
        local = rng.integers(0, beams, (groups, beams)) if kind < 2 else np.tile(np.roll(np.arange(beams), 1), (groups, 1)) if kind == 2 \
            else np.tile(np.arange(beams)[::-1], (groups, 1))
        parents = (local + beams * np.arange(groups)[:, None]).reshape(-1)
        lengths = rng.integers(0, tokens + 1, rows) if kind % 2 else None
        if lengths is not None:
            lengths[0] = tokens
        y = torch.tensor(parents, device="cuda")
        n = None if lengths is None else torch.tensor(lengths, device="cuda")
        before = [t.clone() for t in states]
        out = None if in_place else random_states((rows, tokens, *rest), dtype, 3, seed=kind + 1)
        held = None if in_place else [t.clone() for t in out]
        got = bf.beam_reorder(states, y, beams, lengths=n, out=out)
        host = lambda t: t.view(torch.int16).cpu().numpy() if t.dtype == torch.bfloat16 else t.cpu().numpy()
        for k in range(3):
            want = ref.reorder(host(before[k]), parents, beams, lengths, None if in_place else host(held[k]))
            assert np.array_equal(host(got[k]), want)
            if not in_place:
                assert torch.equal(states[k], before[k])
    assert len(keep) == 3


def test_reorder_layouts():
    """Heads ahead of tokens, keys and values between each other, padded tokens, unaligned views, one tensor."""
    rng = np.random.default_rng(0)
    parents = rng.integers(0, 6, 12) + np.repeat([0, 6], 6)
    lengths = rng.integers(0, 41, 12)
    y, n = torch.tensor(parents, device="cuda"), torch.tensor(lengths, device="cuda")
    both = random_states((12, 2, 40, 4, 24), torch.float16, 1)[0]
    ahead = random_states((12, 4, 40, 24), torch.float16, 1)[0].transpose(1, 2)
    padded = random_states((12, 45, 4, 31), torch.float16, 1)[0]
    odd = random_states((12, 40 * 4 * 24 + 3), torch.float16, 1)[0]
    later = random_states((40, 12, 4, 24), torch.float16, 1)[0].transpose(0, 1)
    views = [[both[:, 0], both[:, 1]], [ahead], [padded[:, 2:42, 1:4, 3:28]], [odd[:, 1:1 + 3840].view(12, 40, 96)], [later]]
    for given in views:
        before = [t.cpu().numpy().copy() for t in given]
        bf.beam_reorder(given if len(given) > 1 else given[0], y, 6, lengths=n)
        for t, b in zip(given, before):
            assert np.array_equal(t.cpu().numpy(), ref.reorder(b, parents, 6, lengths))
    fresh = torch.zeros(12, 40, 4, 24, dtype=torch.float16, device="cuda")
    got = bf.beam_reorder(ahead, y, 6, lengths=n, out=fresh)
    assert got is fresh and np.array_equal(fresh.cpu().numpy(), ref.reorder(ahead.cpu().numpy(), parents, 6, lengths, np.zeros_like(fresh.cpu().numpy())))


def test_reorder_rows_that_stay():
    """Parents outside their group and negative lengths leave a row as it was; lengths beyond the end count as the end."""
    x = random_states((8, 20, 3), torch.float32, 1)[0]
    before = x.cpu().numpy().copy()
    parents, lengths = [1, 4, -1, 0, 7, 1 << 40, 5, 6], [20, 99, 3, 3, 3, -4, 20, 20]
    bf.beam_reorder(x, torch.tensor(parents, device="cuda"), 4, lengths=torch.tensor(lengths, device="cuda"))
    want = before.copy()
    want[0] = before[1]
    want[3] = before[0]
    want[4] = before[7]
    want[7] = before[6]
    assert np.array_equal(x.cpu().numpy(), want)


def test_reorder_refusals():
    x = random_states((8, 20, 3), torch.float32, 2)
    y = torch.zeros(8, dtype=torch.int64, device="cuda")
    for bad in (lambda: bf.beam_reorder(x[0][:, 0, 0], y, 4), lambda: bf.beam_reorder([x[0], x[1][:, :19]], y, 4),
                lambda: bf.beam_reorder(x[0], y[:7], 4), lambda: bf.beam_reorder(x[0], y.int(), 4),
                lambda: bf.beam_reorder(x, y, 4, out=[x[1]]), lambda: bf.beam_reorder(x[0].cpu(), y, 4),
                lambda: bf.beam_reorder(x[0], y, 4, out=x[1].double()), lambda: bf.beam_reorder(x[0], y, 4, out=x[1][:, :19])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: bf.beam_reorder(x[0], y, 3), lambda: bf.beam_reorder(x[0], y, 0), lambda: bf.beam_reorder([x[0], x[0]], y, 4),
                lambda: bf.beam_reorder(x, y, 4, out=[x[1], x[0]]), lambda: bf.beam_reorder(x[0][:, :19], y, 4, out=x[0][:, 1:]),
                lambda: bf.beam_reorder(x[0][:1].expand(8, 20, 3), y, 4)):
        with pytest.raises(bf.BfError):
            bad()
    assert bf.beam_reorder([], y, 4) == []


# ---- together -------------------------------------------------------------------------------------------------------

def test_decoding_step_by_step():
    """A small model answers two prompts with beams: embedding, attention over shared prompt and own caches, the choice of
    continuations and the reordering of caches, against the same search over whole answers in 64 bits."""
    vocab, width, heads, kv_heads, dim, beams, steps, prompt = 29, 32, 4, 2, 16, 4, 6, 37
    gen = torch.Generator().manual_seed(3)
    draw = lambda *n: (torch.randn(*n, generator=gen) / n[0] ** 0.5).cuda()
    table, wq, wk, wv = draw(vocab, width) * 5, draw(width, heads * dim) * 2, draw(width, kv_heads * dim), draw(width, kv_heads * dim)
    wo, head = draw(heads * dim, width), draw(width, vocab) * 3
    groups = 2
    rows = groups * beams
    card = torch.randint(vocab, (groups, prompt), generator=gen).cuda()
    lengths = torch.tensor([prompt, 20], device="cuda")
    x = bf.embed(table, card.reshape(-1)).view(groups, prompt, width)
    pk, pv = (x @ wk).view(groups, prompt, kv_heads, dim), (x @ wv).view(groups, prompt, kv_heads, dim)
    caches = [torch.zeros(rows, steps, kv_heads, dim, device="cuda") for _ in range(2)]
    history = torch.full((rows, steps + 1), -1, dtype=torch.int64, device="cuda")
    history[:, 0] = 1
    scores = torch.tensor([0.0] + [-INF] * (beams - 1), device="cuda").repeat(groups)
    finished = torch.zeros(rows, dtype=torch.bool, device="cuda")
    for t in range(steps):
        x = bf.embed(table, history[:, t].contiguous())
        caches[0][:, t], caches[1][:, t] = (x @ wk).view(rows, kv_heads, dim), (x @ wv).view(rows, kv_heads, dim)
        out = bf.prefix_attention((x @ wq).view(rows, heads, dim), pk, pv, *caches, prefix_lengths=lengths,
                                  suffix_lengths=torch.full((rows,), t + 1, device="cuda"))
        logits = (x + out.view(rows, -1) @ wo) @ head
        step = bf.beam_step(logits, scores, beams, finished=finished, end_token=0)
        parents = step.parents.view(-1)
        bf.beam_reorder(caches, parents, beams, lengths=torch.full((rows,), t + 1, device="cuda"))
        bf.beam_reorder(history, parents, beams)
        history[:, t + 1] = step.tokens.view(-1)
        scores, finished = step.scores.view(-1), step.finished.view(-1)

    d = lambda v: v.double().cpu().numpy()
    E, Q, K, V, O, H = (d(v) for v in (table, wq, wk, wv, wo, head))

    def next_logprobs(g, tokens):
        n = int(lengths[g])
        xs = np.concatenate([E[card[g, :n].cpu().numpy()], E[tokens]])
        q = (xs[-1] @ Q).reshape(heads, dim)
        k, v = (xs @ K).reshape(-1, kv_heads, dim), (xs @ V).reshape(-1, kv_heads, dim)
        out = []
        for h in range(heads):
            s = k[:, h // 2] @ q[h] / dim ** 0.5
            w = np.exp(s - s.max())
            out.append((w @ v[:, h // 2]) / w.sum())
        z = (xs[-1] + np.concatenate(out) @ O) @ H
        return z - z.max() - np.log(np.exp(z - z.max()).sum())

    for g in range(groups):
        found = [([1], 0.0, False)]
        for _ in range(steps):
            new = []
            for tokens, score, end in found:
                new += [(tokens + [0], score, True)] if end else [(tokens + [v], score + lp, v == 0) for v, lp in enumerate(next_logprobs(g, tokens))]
            found = sorted(new, key=lambda c: -c[1])[:beams]
        mine = slice(g * beams, (g + 1) * beams)
        assert [c[0] for c in found] == history[mine].tolist()
        assert np.allclose([c[1] for c in found], d(scores[mine]), rtol=0, atol=1e-4)
        assert [c[2] for c in found] == finished[mine].tolist()


def test_calls_of_several_threads():
    """Calls of four threads, each on a stream of its own, on the same inputs."""
    import threading
    x = attention_inputs(2, 8, 8, 2, 64, 700, 50, "bf16", seed=21)
    logits, scores, _ = beam_inputs(4, 4, 9001, "bf16", seed=21)
    s = torch.tensor(scores, device="cuda")
    state = random_states((16, 40, 2, 8), torch.float32, 1)[0]
    want = bf.prefix_attention(*x)
    step = bf.beam_step(logits, s, 4)
    moved = bf.beam_reorder(state.clone(), step.parents, 4)
    torch.cuda.synchronize()
    wrong = []

    def work():
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(30):
                a, b = bf.prefix_attention(*x), bf.beam_step(logits, s, 4)
                c = bf.beam_reorder(state, b.parents, 4, out=torch.empty_like(state))
                stream.synchronize()
                if not (torch.equal(a, want) and torch.equal(b.tokens, step.tokens) and torch.equal(b.scores, step.scores)
                        and torch.equal(c, moved)):
                    wrong.append(1)

    threads = [threading.Thread(target=work) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_captured_together():
    """A step captured as a whole, replayed over other inputs, beside another graph of the same calls."""
    def inputs(seed):
        x = attention_inputs(2, 4, 4, 2, 64, 300, 20, "f16", seed=seed)
        logits, scores, _ = beam_inputs(2, 4, 5003, "f16", seed=seed)
        return [*x, logits, torch.tensor(scores, device="cuda"), random_states((8, 20, 2, 8), torch.float16, 1, seed=seed)[0]]

    def step(x):
        out = bf.prefix_attention(*x[:5])
        best = bf.beam_step(x[5], x[6], 4)
        return out, best.scores, best.tokens, bf.beam_reorder(x[7], best.parents, 4, out=torch.empty_like(x[7])), \
            bf.beam_reorder(x[7], best.parents, 4)

    sets, graphs = [inputs(1), inputs(2)], []
    for x in sets:
        step([t.clone() for t in x])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            held = step(x)
        graphs.append((g, held))
    for seed in (3, 4):
        for k, x in enumerate(sets):
            fresh = inputs(10 * seed + k)
            for a, b in zip(x, fresh):
                a.copy_(b)
        for g, _ in graphs:
            g.replay()
        for k, (_, held) in enumerate(graphs):
            want = step(inputs(10 * seed + k))
            assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_far_offsets():
    """Sequences, rows and states more than 2^32 elements behind each other."""
    far = (1 << 32) + 64
    buf = torch.empty(far + (1 << 22), dtype=torch.bfloat16, device="cuda")
    near = attention_inputs(2, 3, 4, 2, 64, 300, 20, "bf16", seed=30)
    shape, strides = near[1].shape, (far, *near[1].stride()[1:])
    for which in (1, 2):  # keys, then values, of the second prompt far away
        view = buf.as_strided(shape, strides)
        view.copy_(near[which])
        x = [*near]
        x[which] = view
        assert torch.equal(bf.prefix_attention(*x), bf.prefix_attention(*near))
    own = buf.as_strided((2, *near[3].shape[1:]), (far, *near[3].stride()[1:]))
    own.copy_(near[3][:2])
    q = near[0][:2]
    assert torch.equal(bf.prefix_attention(q, near[1], near[2], own, near[4][:2]),
                       bf.prefix_attention(q, near[1], near[2], near[3][:2], near[4][:2]))
    for vocab in (50, 9001):
        x, scores, _ = beam_inputs(1, 2, vocab, "bf16", seed=31)
        view = buf.as_strided(x.shape, (far, 1))
        view.copy_(x)
        check_beams(view, scores, 2, 5)
    rows = buf.as_strided((2, 30, 2, 32), (far, 64, 32, 1))
    rows.copy_(near[3][:1, :1, :1, :1].expand(2, 30, 2, 32))
    rows[1] += 1
    want = rows.flip(0).clone()
    bf.beam_reorder(rows, torch.tensor([1, 0], device="cuda"), 2)
    assert torch.equal(rows, want)
