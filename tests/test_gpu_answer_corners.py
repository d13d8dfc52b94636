"""Corners of the operators of a decoding step on the GPU."""
import ctypes
import math
import threading

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_22242_gb300 import bf  # noqa: E402
from test_gpu_answer import attention_inputs, beam_inputs, check_beams, half  # noqa: E402

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
INF = float("inf")


@pytest.fixture(scope="module", autouse=True)
def _built():
    assert torch.cuda.is_available()
    bf.load()


# ---- weights far below the largest ----

def check_one_above_many(dtype, tokens, prompts, each, own):
    """Two keys 25.04 above all others (in log2), which together weigh up to 0.4 % of them and have eight times their value.
    Rounded to f16 where the largest is 1, the others' weights would be 0: below half of f16's lowest number, 2^-24."""
    above = torch.tensor(17.359375).to(TYPES[dtype]).item()  # (17.375 in bf16)
    value, first = 8.0, (0, 128)  # a key in each of a prompt's two streams of tiles
    q = torch.zeros(prompts * each, 1, 8, dtype=TYPES[dtype], device="cuda")
    q[..., 0] = 1.0
    k = torch.zeros(prompts * each if own else prompts, tokens, 1, 8, dtype=TYPES[dtype], device="cuda")
    v = torch.full_like(k, value)
    for t in first:
        k[:, t, :, 0], v[:, t] = above, 1.0
    if own:  # behind a prompt that is empty
        args, lengths = (q, k[:prompts, :1], v[:prompts, :1], k, v), torch.zeros(prompts, dtype=torch.int64, device="cuda")
    else:
        args, lengths = (q, k, v), None
    out, lse = bf.prefix_attention(*args, prefix_lengths=lengths, scale=1.0, lse=True)
    w = math.exp(-above)
    total = len(first) + (tokens - len(first)) * w
    want = (len(first) + (tokens - len(first)) * w * value) / total
    # As in test_gpu_answer.py (one product a score, exact); the others' weights are off by half a step, or by half of
    # f16's lowest step, 2^-25 where the largest is 2^7 or more.
    weight = 2.0 ** -22 + 2.0 ** -17 + (tokens + 16) * 2.0 ** -24
    rounded = 0.0 if dtype == "f32" else half(dtype) * (want - 1) * 2
    tiny = tokens * 2.0 ** -32 * value if dtype == "f16" else 0.0
    bound = weight * want + rounded + tiny + half(dtype) * want
    assert dtype != "f16" or want - 1 > bound
    assert (out.double() - want).abs().max().item() <= bound
    assert (lse.double() - above - math.log(total)).abs().max().item() <= weight + 2.0 ** -23 * 40


@pytest.mark.parametrize("dtype,prompts,each", [("bf16", 152, 1), ("f16", 152, 1), ("bf16", 152, 200), ("f16", 152, 200), ("f32", 19, 30)])
def test_prompt_of_one_above_many(dtype, prompts, each):
    """152 prompts, so that every block has a whole prompt as one piece; a tile of queries for one stream and for both."""
    check_one_above_many(dtype, 131072, prompts, each, False)


@pytest.mark.parametrize("dtype,answers", [("bf16", 1216), ("f16", 1216), ("bf16", 400), ("f16", 400), ("f16", 700), ("f32", 40)])
def test_answers_of_one_above_many(dtype, answers):
    """The answers' own keys, by a warp each, by two and by four."""
    check_one_above_many(dtype, 131072, 1, answers, True)

# ---- scores of any size ----

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [1e6, -1e6, 1e8, 1e12, 1e20, 1e30, -1e30])
@pytest.mark.parametrize("dim,each", [(64, 3), (128, 40), (128, 100), (64, 70), (40, 9)])
def test_attention_of_large_scores(dim, each, scale, dtype):
    """Scores far beyond what exponentials tell apart: the key of the largest has all the weight, wherever it lies."""
    x = attention_inputs(2, each, 4, 2, dim, 700, 50, dtype, seed=each, spread=1.0)
    q, pk, pv, sk, sv = (t.double() for t in x)
    k, v = (torch.cat([p.repeat_interleave(each, 0), s], 1) for p, s in ((pk, sk), (pv, sv)))
    s = torch.einsum("agsd,atgd->agst", q.view(-1, 2, 2, dim), k) * float(np.float32(scale))
    top, at = s.topk(2, -1)
    size = torch.einsum("agsd,atgd->agst", q.view(-1, 2, 2, dim).abs(), k.abs()).max().item() * abs(scale)
    # A score is off by (dim + 4) 2^-24 of the sum of its products' magnitudes, scaled and rounded; two that are closer than
    # twice that and what a weight of 2^-40 takes are not looked at.
    off = (dim + 6) * 2.0 ** -24 * size
    sure = top[..., 0] - top[..., 1] > 2 * off + 28
    assert sure.double().mean() > 0.9
    want = torch.gather(v.transpose(1, 2), 2, at[..., :1].expand(-1, -1, -1, dim))
    out, lse = bf.prefix_attention(*x, scale=scale, lse=True)
    got = out.double().view(want.shape)
    near = (got - want).abs() <= half(dtype) * want.abs() + 700 * 2.0 ** -40 * 8 + (2.0 ** -25 if dtype == "f16" else 0) + 2.0 ** -22 * want.abs()
    assert near[sure].all()
    assert ((lse.double().view(top[..., 0].shape) - top[..., 0]).abs() <= 2 * off + 8).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("own", [False, True])
def test_attention_of_scores_beyond_32_bits(own, dtype):
    """A score of +inf makes its answer NaN, one of -inf has no weight."""
    x = attention_inputs(1, 3, 4, 2, 64, 300, 50, dtype, seed=1)
    q, pk, pv, sk, sv = (t.clone() for t in x)
    q.fill_(3e4)
    pk.fill_(-3e4 if own else 3e4)
    sk.fill_(3e4 if own else -3e4)
    out, lse = bf.prefix_attention(q, pk, pv, sk, sv, scale=1e30, lse=True)
    assert torch.isnan(out).all() and torch.isnan(lse).all()


# ---- calls from threads of their own ----

def plain_call(x):
    """A call of the C entry point again and again with what it was given once: (call, its output)."""
    lib, code = bf.load(), bf._dtype_code(x[0].dtype)
    caches = [bf.Cache(t.data_ptr(), t.shape[0], 1 if t.dim() == 3 else t.shape[1], t.shape[-2], t.shape[-1], t.stride(0),
                       0 if t.dim() == 3 else t.stride(1), t.stride(-2), code, 0) for t in x]
    out, need = torch.empty_like(x[0]), ctypes.c_uint64(0)
    caches.append(bf.Cache(out.data_ptr(), *[getattr(caches[0], f) for f in ("batch", "tokens", "heads", "dim")],
                           out.stride(0), 0, out.stride(1), code, 0))
    at = [ctypes.addressof(c) for c in caches]
    args = bf.AttentionArgs(None, None, x[0].shape[2] ** -0.5, 0)
    assert lib.bf_prefix_attention_workspace(at[0], at[1], at[3], ctypes.byref(need)) == bf.BF_OK
    work, stream = torch.empty(need.value, dtype=torch.uint8, device="cuda"), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    held = (caches, args, work, stream, *x)
    where, given = ctypes.addressof(args), (work.data_ptr(), need.value, stream.cuda_stream)
    return lambda: lib.bf_prefix_attention(*at[:5], where, at[5], None, *given) if held else None, out


@pytest.mark.parametrize("dtype,dim,each", [("bf16", 64, 2), ("f16", 128, 70), ("f32", 64, 2), ("bf16", 30, 2)])
def test_first_call_of_a_thread(dtype, dim, each):
    """A call from a thread that has made no other call of CUDA: the device's context is not current there."""
    x = attention_inputs(1, each, 4, 2, dim, 300, 20, dtype, seed=dim)
    want = bf.prefix_attention(*x)
    call, out = plain_call(x)
    torch.cuda.synchronize()
    status = []
    thread = threading.Thread(target=lambda: status.append(call()))
    thread.start()
    thread.join()
    torch.cuda.synchronize()
    assert status == [bf.BF_OK], bf.last_error()
    assert torch.equal(out, want)


def test_threads_of_different_shapes():
    """Calls whose kernels are the same and whose shared memory is not, each from a thread of its own: all are valid."""
    sets = [attention_inputs(1, 2, 4, 2, 64, 300, 20, "bf16", seed=1), attention_inputs(1, 70, 8, 2, 128, 300, 20, "bf16", seed=2),
            attention_inputs(1, 2, 4, 2, 40, 90, 20, "f32", seed=3), attention_inputs(1, 2, 4, 2, 256, 90, 20, "f32", seed=4),
            attention_inputs(1, 9, 4, 1, 30, 90, 20, "bf16", seed=5), attention_inputs(1, 9, 4, 1, 250, 90, 20, "bf16", seed=6)]
    want = [bf.prefix_attention(*x) for x in sets]
    calls = [plain_call(x) for x in sets]
    torch.cuda.synchronize()
    refused = [0] * len(sets)

    def work(i):
        torch.cuda.synchronize()
        for _ in range(10000):
            refused[i] += calls[i][0]() != bf.BF_OK

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(sets))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert refused == [0] * len(sets)
    assert all(torch.equal(out, w) for (_, out), w in zip(calls, want))


# ---- rows whose logits are not alike all along ----

def uneven(kind, x):
    """Logits of (rows x vocab) with ranges of tokens that are banned, or in an order."""
    vocab = x.shape[1]
    if kind == "first":
        x[:, :min(20000, vocab // 3)] = -INF
    elif kind == "halves":  # of every 4,096, and so of whatever a block takes
        on = torch.arange(vocab, device="cuda") // max(1, vocab // 8) % 2 == 0
        x.masked_fill_(on, -INF)
    elif kind == "few":  # a few tokens are left at the beginning
        keep = x[:, 5:60:11].clone()
        x[:, :vocab // 2] = -INF
        x[:, 5:60:11] = keep
    elif kind == "ascending":
        x.copy_(x.sort(1).values)
    elif kind == "lower":
        x[:, :vocab // 2] -= 50
    return x


KINDS = ["first", "halves", "few", "ascending", "lower"]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("vocab,keep", [(9001, 16), (70001, 200), (131072, 32)])
def test_beams_of_uneven_rows(vocab, keep, kind, dtype):
    """Rows cut into one tile a block, and (310 of 131,072) two, of which the first and the last group are checked."""
    x, scores, _ = beam_inputs(31, 10, vocab, dtype, seed=vocab)
    x, s = uneven(kind, x), torch.tensor(scores, device="cuda")
    for groups in (31, 1):
        got = bf.beam_step(x[:10 * groups], s[:10 * groups], 10, keep=keep)
        for g in (0, 30)[:groups]:
            rows = slice(10 * g, 10 * g + 10)
            mine = [None if t is None else t[g:g + 1] for t in got]
            mine[2] = mine[2] - 10 * g
            check_beams(x[rows], scores[rows], 10, keep, got=bf.BeamStep(*mine))


def time_of(call):
    for _ in range(3):
        call()
    best = INF
    for _ in range(5):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        for _ in range(5):
            call()
        b.record()
        b.synchronize()
        best = min(best, a.elapsed_time(b))
    return best


@pytest.mark.parametrize("kind", KINDS)
def test_beams_of_uneven_rows_take_no_longer(kind):
    """Not many times as long as rows that are alike all along (ascending ones have the largest beside each other,
    many of them equal in 16 bits, and are read twice)."""
    x = torch.randn(512, 131072, device="cuda").bfloat16()
    scores = -torch.rand(512, device="cuda")
    alike = time_of(lambda: bf.beam_step(x, scores, 8, keep=16))
    x = uneven(kind, x)
    took = time_of(lambda: bf.beam_step(x, scores, 8, keep=16))
    assert took <= 4 * alike


# ---- thousands of prompts ----

def prompts_of(count, dim, tokens, own, dtype, lengths=None):
    gen = torch.Generator(device="cuda").manual_seed(count)
    rand = lambda *n: torch.randn(*n, generator=gen, device="cuda").to(TYPES[dtype])
    x = (rand(count, 2, dim), rand(count, tokens, 1, dim), rand(count, tokens, 1, dim), rand(count, own, 1, dim), rand(count, own, 1, dim))
    return x, torch.randint(0, tokens + 1, (count,), generator=gen, device="cuda") if lengths is None else lengths


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("count,dim", [(129, 64), (9000, 64), (20000, 40), (9000, 30)])
@pytest.mark.parametrize("kind", ["any", "runs", "none", "last", "full"])
def test_attention_of_thousands_of_prompts(count, dim, kind, dtype):
    """Prompts of any length; thousands that are empty behind each other; none that is not; the last alone; all full."""
    x, n = prompts_of(count, dim, 200, 5, dtype)
    if kind == "runs":
        n[count // 9:count // 2] = 0
        n[-count // 4:] = 0
    elif kind in ("none", "last"):
        n.zero_()
        n[-1] = 131 if kind == "last" else 0
    given = None if kind == "full" else n
    out, lse = bf.prefix_attention(*x, prefix_lengths=given, lse=True)
    q, pk, pv, sk, sv = (t.double() for t in x)
    k, v = torch.cat([pk, sk], 1)[:, :, 0], torch.cat([pv, sv], 1)[:, :, 0]
    s = torch.einsum("phd,ptd->pht", q, k) * dim ** -0.5
    if given is not None:
        at = torch.arange(205, device="cuda")
        s = s.masked_fill(((at >= n[:, None]) & (at < 200))[:, None], -INF)
    w = torch.softmax(s, -1)
    want, size = torch.einsum("pht,ptd->phd", w, v), torch.einsum("pht,ptd->phd", w, v.abs())
    # As test_gpu_answer.py, with the largest score's products and 205 keys.
    most = torch.einsum("phd,ptd->pht", q.abs(), k.abs()).max().item() * dim ** -0.5
    weight = 2 * (dim + 4) * 2.0 ** -24 * most + 2.0 ** -22 + 2.0 ** -17
    total = weight + 221 * 2.0 ** -24
    rounded = 0.0 if dtype == "f32" else half(dtype)
    bound = (weight + rounded + total) * size + (205 * 2.0 ** -32 * 6 + 2.0 ** -25 if dtype == "f16" else 0.0) + half(dtype) * (1 + 2.0 ** -8) * want.abs()
    assert ((out.double() - want).abs() <= bound).all()
    assert ((lse.double() - torch.logsumexp(s, -1)).abs() <= total + 2.0 ** -23 * (most + 20)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lengths", [False, True])
def test_attention_time_is_of_the_prompts(lengths, dtype):
    """Eight times the prompts take not much more than eight times as long (20 to 30 where every unit adds up all lengths)."""
    took = []
    for count in (8192, 65536):
        x, n = prompts_of(count, 64, 64, 16, dtype)
        took.append(time_of(lambda: bf.prefix_attention(*x, prefix_lengths=n if lengths else None)))
    assert took[1] <= 16 * took[0], took


# ---- length penalties ----

@pytest.mark.parametrize("penalty", [1.0, 1.8, 2.5, 13.0, 30.0, 200.0, 5000.0, 65536.0])
@pytest.mark.parametrize("vocab,beams,keep", [(3, 4, 6), (3, 16, 16), (100, 16, 40), (9001, 6, 12)])
def test_beams_of_large_penalties(vocab, beams, keep, penalty):
    """total / n^penalty where n^penalty is beyond 32-bit numbers, for totals of both signs."""
    groups = 8
    x, _, rng = beam_inputs(groups, beams, vocab, "f32", seed=vocab + beams)
    scores = np.float32(rng.uniform(-12, 12, groups * beams))
    lengths = rng.choice([0, 1, 2, 3, 40, 41, 999, 10 ** 6, 10 ** 12], (groups, beams))
    lengths[1] = 39  # all alike
    lengths[2] = 39 + np.arange(beams) % 2
    lengths = lengths.reshape(-1)
    finished = rng.random(groups * beams) < 0.3
    got = bf.beam_step(x, torch.tensor(scores, device="cuda"), beams, keep=keep, finished=torch.tensor(finished, device="cuda"),
                       lengths=torch.tensor(lengths, device="cuda"), length_penalty=penalty, end_token=1)
    z = torch.log_softmax(x.double(), 1).cpu().numpy()
    off = 2.0 ** -22 + (64 + 13 + vocab / 4096) * 2.0 ** -24 + max(1.0, np.log2(vocab)) * 2.0 ** -23  # of a total, as check_beams
    for g in range(groups):
        found = []  # (sign, what orders the ranks of that sign, beam, token, total, length)
        for b in range(g * beams, (g + 1) * beams):
            n = int(lengths[b]) + (not finished[b])
            for v, t in [(1, float(scores[b]))] if finished[b] else list(enumerate(scores[b] + z[b])):
                sign = 1 if t > 0 else -1
                found.append((sign, sign * (math.log(abs(t)) - penalty * math.log(max(1, n))), b, int(v), t, n))
        found.sort(key=lambda c: (-c[0], -c[1], c[2], c[3]))
        place = {c[2:4]: c for c in found}
        seen = set()
        for j in range(min(keep, len(found))):
            here = (int(got.parents[g, j]), int(got.tokens[g, j]))
            assert here in place and here not in seen
            seen.add(here)
            c, best = place[here], found[j]
            near = 4 * off / min(abs(c[4]), abs(best[4])) + 1e-8 * (1 + penalty * 2.0 ** -10)
            assert (c[0] == best[0] and abs(c[1] - best[1]) <= near) or abs(c[4]) < 4 * off or abs(best[4]) < 4 * off, (g, j, c, best)
            assert abs(float(got.scores[g, j]) - c[4]) <= off + 2.0 ** -24 * abs(c[4])
            assert int(got.lengths[g, j]) == c[5]


def test_beams_of_a_penalty_over_equal_totals():
    """Beams that differ by their lengths alone: the longer is better where totals are negative, whatever the penalty."""
    for vocab in (1, 4099):
        x = torch.zeros(8, vocab, device="cuda")
        for penalty in (0.5, 20.0, 28.0, 40.0, 1000.0, 65536.0):
            lengths = torch.tensor([9, 40, 3, 41, 7, 1 << 40, 0, 100], device="cuda")
            got = bf.beam_step(x[:, :1] if vocab == 1 else x, torch.full((8,), -2.0, device="cuda"), 8, keep=8, lengths=lengths,
                               length_penalty=penalty)
            if vocab == 1:
                assert got.parents[0].tolist() == [5, 7, 3, 1, 0, 4, 2, 6]
            else:
                assert got.parents[0].tolist() == [5] * 8 and got.tokens[0].tolist() == list(range(8))
