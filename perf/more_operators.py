"""Operators for answering: what is timed, and their plain forms.

A scheduling model answers a workflow's prompt with many candidate mappings: beams, or samples that are graded against each
other.  These operators are a decoding step of such a model: attention of every answer's last token to the prompt that the
answers share and to the answer itself, the choice of the best continuations over beams and vocabulary, and the reordering
of the beams' states.  A case names the operator (``op``), its sizes and options; ``own`` chooses between the package's
kernels and the plain form in elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def _attend(name, prompts, answers, heads, kv_heads, dim, prefix, suffix, dtype, lse=False, fill=1.0):
    """`answers` per prompt; `prefix` and `suffix`: the caches' tokens, filled to the share `fill` on average."""
    return dict(name=name, op="attend", prompts=prompts, answers=answers, heads=heads, kv_heads=kv_heads, dim=dim,
                prefix=prefix, suffix=suffix, dtype=dtype, lse=lse, fill=fill)


def _step(name, groups, beams, vocab, dtype, keep, finished=0.0, penalty=0.0, temperature=1.0, banned=0.0):
    return dict(name=name, op="step", groups=groups, beams=beams, vocab=vocab, dtype=dtype, keep=keep, finished=finished,
                penalty=penalty, temperature=temperature, banned=banned)


def _reorder(name, groups, beams, tensors, tokens, heads, dim, dtype, fill=1.0):
    return dict(name=name, op="reorder", groups=groups, beams=beams, tensors=tensors, tokens=tokens, heads=heads, dim=dim,
                dtype=dtype, fill=fill)


def listed():
    return [
        # Four candidate mappings of one small workflow under a small model: latency counts.
        _attend("attend 4 mappings", 1, 4, 8, 2, 64, 600, 32, "bf16"),
        # Sixteen sampled answers to one workflow's cards and instructions.
        _attend("attend 16 answers", 1, 16, 32, 8, 128, 8191, 256, "bf16"),
        # A batch of workflows of uneven sizes, sixteen samples of each.
        _attend("attend a batch", 64, 16, 16, 4, 64, 2048, 160, "f16", fill=0.75),
        # Sixty-four answers to a prompt with a long log of past runs.
        _attend("attend a long prompt", 1, 64, 32, 8, 128, 131072, 512, "bf16", fill=0.9),
        # A model kept in 32 bits, an odd head size, the sums returned for a caller's own joining.
        _attend("attend in 32 bits", 2, 5, 12, 4, 80, 1500, 100, "f32", lse=True, fill=0.8),
        # One step of a small beam over a large vocabulary: latency counts.
        _step("step of 4 beams", 1, 4, 131072, "bf16", 4),
        # Beams over modes, three tokens: 4096 workflows, 16 partial mappings each.
        _step("step of mappings", 4096, 16, 3, "f32", 16),
        # Text answers to a batch of workflows, twice as many continuations kept as there are beams.
        _step("step of text beams", 64, 8, 131072, "bf16", 16, finished=0.2),
        # Wide beams ranked by mean log-probabilities, tokens banned by the grammar; rows start at any alignment.
        _step("step ranked by length", 16, 32, 50001, "f16", 32, finished=0.3, penalty=0.7, temperature=0.8, banned=0.1),
        # The caches of one small layer behind a step of four beams.
        _reorder("reorder 4 beams", 1, 4, 2, 512, 2, 64, "bf16", fill=0.8),
        # Four layers' caches of a batch of beams of uneven lengths.
        _reorder("reorder a batch", 64, 8, 8, 512, 8, 128, "bf16", fill=0.6),
    ]


def _log_size(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return min(hi, max(lo, n))


def draw(rng):
    op = rng.choice(["attend", "attend", "step", "step", "reorder"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    if op == "attend":
        dim = rng.choice([64, 128, 64, 128, 80, 96, 40])
        kv_heads, shared = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 7, 8])
        prompts, answers = _log_size(rng, 1, 64), _log_size(rng, 1, 64)
        suffix = _log_size(rng, 1, max(2, min(512, (1 << 26) // (dim * kv_heads * prompts * answers))))
        most = (1 << 26) // (dim * kv_heads * prompts)
        rows = prompts * answers * kv_heads * shared
        most = min(most, (1 << (28 if dtype != "f32" else 25)) // rows, 131072)
        return dict(op=op, prompts=prompts, answers=answers, heads=kv_heads * shared, kv_heads=kv_heads, dim=dim,
                    prefix=_log_size(rng, 1, max(2, most)), suffix=suffix, dtype=dtype, lse=rng.random() < 0.3,
                    fill=rng.choice([1.0, 0.75, 0.6]))
    if op == "step":
        vocab, beams = _log_size(rng, 3, 131072), _log_size(rng, 1, 64)
        groups = _log_size(rng, 1, max(1, min(4096, (1 << 25) // (vocab * beams))))
        keep = rng.choice([beams, beams, min(2 * beams, beams * vocab), 1])
        return dict(op=op, groups=groups, beams=beams, vocab=vocab, dtype=dtype, keep=keep, finished=rng.choice([0.0, 0.3]),
                    penalty=rng.choice([0.0, 1.0, 0.6]), temperature=rng.choice([1.0, 0.7, 1.3]), banned=rng.choice([0.0, 0.2]))
    groups, beams = _log_size(rng, 1, 64), _log_size(rng, 1, 32)
    heads, dim, tensors = rng.choice([1, 2, 5, 8]), rng.choice([40, 64, 128]), rng.choice([1, 2, 4, 8])
    most = (1 << 30) // (groups * beams * heads * dim * tensors)
    return dict(op=op, groups=groups, beams=beams, tensors=tensors, tokens=_log_size(rng, 1, max(2, min(2048, most))),
                heads=heads, dim=dim, dtype=dtype, fill=rng.choice([1.0, 0.8, 0.55]))


# ---- inputs ---------------------------------------------------------------------------------------------------------

END = 2          # the token that ends an answer
APART = 1e-5     # continuations of different beams whose ranks are closer than this are moved apart
CHUNK = 1 << 24  # logits handled at a time in 64 bits


def _lengths(count, capacity, fill, rng):
    """`count` lengths of up to `capacity`, the first one full: spread about `fill` of it."""
    n = np.rint(capacity * rng.uniform(2 * fill - 1, 1.0, count)).astype(np.int64)
    n[0] = capacity
    return n


def _gen(case, seed):
    rng = np.random.default_rng([int(seed), len(case["op"])] + [v for k, v in sorted(case.items()) if type(v) is int])
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(rng.integers(1 << 40)))
    return rng, gen


def _make_attend(case, seed):
    rng, gen = _gen(case, seed)
    dtype, d, hk = TYPES[case["dtype"]], case["dim"], case["kv_heads"]
    randn = lambda *n: torch.randn(*n, generator=gen, device="cuda", dtype=dtype)
    prompts, rows = case["prompts"], case["prompts"] * case["answers"]
    s = dict(q=randn(rows, case["heads"], d).mul_(1.5),  # some keys stand out, as they do in a trained model
             prefix_k=randn(prompts, case["prefix"], hk, d), prefix_v=randn(prompts, case["prefix"], hk, d),
             suffix_k=randn(rows, case["suffix"], hk, d), suffix_v=randn(rows, case["suffix"], hk, d))
    s["prefix_lengths"] = torch.from_numpy(_lengths(prompts, case["prefix"], case["fill"], rng)).cuda()
    s["suffix_lengths"] = torch.from_numpy(_lengths(rows, case["suffix"], 0.5 + 0.5 * case["fill"], rng)).cuda()
    return s


def _best_of_rows(logits, tau, live, most):
    """The best `most` logits of each row, their tokens and the rows' ln sum e^z, in 64 bits."""
    rows, vocab = logits.shape
    top = min(most, vocab)
    z = torch.full((rows, top), -math.inf, dtype=torch.float64, device="cuda")
    at = torch.zeros(rows, top, dtype=torch.int64, device="cuda")
    norm = torch.zeros(rows, dtype=torch.float64, device="cuda")
    step = max(1, CHUNK // vocab)
    for a in range(0, rows, step):
        x = logits[a:a + step].double() / tau
        norm[a:a + step] = torch.logsumexp(x, 1)
        z[a:a + step], at[a:a + step] = torch.topk(x, top, dim=1)
    z -= torch.where(live, norm, 0.0)[:, None]
    return torch.where(live[:, None], z, -math.inf), at, norm


def _make_step(case, seed):
    rng, gen = _gen(case, seed)
    groups, beams, vocab, tau = case["groups"], case["beams"], case["vocab"], case["temperature"]
    rows = groups * beams
    logits = torch.empty(rows, vocab, dtype=TYPES[case["dtype"]], device="cuda")
    rand = lambda *n: torch.rand(*n, generator=gen, device="cuda")
    for a in range(0, rows, max(1, CHUNK // vocab)):
        b = min(rows, a + max(1, CHUNK // vocab))
        z = torch.randn(b - a, vocab, generator=gen, device="cuda") * 2.0
        likely = torch.randint(vocab, (b - a, 8), generator=gen, device="cuda")  # a few tokens stand out
        z.scatter_add_(1, likely, rand(b - a, 8) * (0.8 * math.log(vocab)))
        if case["banned"]:  # tokens that the answer's grammar (or the budget) forbids at this place
            allowed = torch.gather(z, 1, likely)
            z = torch.where(rand(b - a, vocab) < case["banned"], torch.full_like(z, -math.inf), z)
            z.scatter_(1, likely, allowed)
        logits[a:b] = z.to(logits.dtype)
    finished = rand(rows) < case["finished"]
    lengths = torch.randint(5, 40, (groups, 1), generator=gen, device="cuda").expand(groups, beams)
    lengths = torch.where(finished.view(groups, beams), (lengths * rand(groups, beams)).long() + 1, lengths).reshape(-1)
    weight = lengths.double() + torch.where(finished, 0.0, 1.0)
    weight = weight ** -case["penalty"]
    z, _, _ = _best_of_rows(logits, tau, ~finished, case["keep"] + 1)
    z = torch.where(finished[:, None], torch.full_like(z, -math.inf), z)
    z[:, 0] = torch.where(finished, 0.0, z[:, 0])
    beam = torch.arange(beams, device="cuda").repeat_interleave(z.shape[1])
    scores = torch.empty(rows, device="cuda")
    redo = torch.ones(groups, dtype=torch.bool, device="cuda")
    for _ in range(60):  # scores whose best continuations lie too close for 32 bits are drawn again
        new = -(0.6 + 0.4 * rand(groups, beams)) * (3.0 + 0.2 * beams)
        scores = torch.where(redo[:, None], new, scores.view(groups, beams)).reshape(-1)
        rank = ((scores.double()[:, None] + z) * weight[:, None]).view(groups, -1)
        best, which = torch.topk(rank, min(case["keep"] + 1, rank.shape[1]), dim=1)
        near = (best[:, :-1] - best[:, 1:] < APART) & (beam[which[:, :-1]] != beam[which[:, 1:]]) & torch.isfinite(best[:, 1:])
        redo = near.any(1)
        if not bool(redo.any()):
            break
    s = dict(logits=logits, scores=scores)
    if case["finished"]:
        s["finished"] = finished
    if case["penalty"]:
        s["lengths"] = lengths
    return s


def _make_reorder(case, seed):
    rng, gen = _gen(case, seed)
    groups, beams = case["groups"], case["beams"]
    rows = groups * beams
    shape = (rows, case["tokens"], case["heads"], case["dim"])
    states = [torch.randn(*shape, generator=gen, device="cuda", dtype=TYPES[case["dtype"]]) for _ in range(case["tensors"])]
    # Continuations mostly come from the better beams.
    parents = np.floor(beams * rng.random((groups, beams)) ** 1.7).astype(np.int64) + beams * np.arange(groups)[:, None]
    lengths = _lengths(rows, case["tokens"], case["fill"], rng)
    return dict(states=states, out=[torch.zeros_like(x) for x in states], parents=torch.from_numpy(parents.reshape(-1)).cuda(),
                lengths=torch.from_numpy(lengths).cuda())


MAKE = {"attend": _make_attend, "step": _make_step, "reorder": _make_reorder}


def prepare(case, seed):
    return dict(case=dict(case), **MAKE[case["op"]](case, seed))


# ---- one pass -------------------------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    return (_run_own if own else PLAIN[case["op"]])(case, state)


def _run_own(case, s):
    from paper_2607_22242_gb300 import bf
    if case["op"] == "attend":
        return bf.prefix_attention(s["q"], s["prefix_k"], s["prefix_v"], s["suffix_k"], s["suffix_v"],
                                   prefix_lengths=s["prefix_lengths"], suffix_lengths=s["suffix_lengths"], lse=case["lse"])
    if case["op"] == "step":
        r = bf.beam_step(s["logits"], s["scores"], case["beams"], keep=case["keep"], finished=s.get("finished"),
                         lengths=s.get("lengths"), length_penalty=case["penalty"], end_token=END,
                         temperature=case["temperature"])
        return r.scores, r.tokens, r.parents, r.finished
    return bf.beam_reorder(s["states"], s["parents"], case["beams"], lengths=s["lengths"], out=s["out"])


def _attend_plain(case, s):
    prompts, w, d, hk = case["prompts"], case["answers"], case["dim"], case["kv_heads"]
    share, scale = case["heads"] // hk, 1.0 / math.sqrt(case["dim"])
    q = s["q"].float() * scale
    shared = q.view(prompts, w, hk, share, d).permute(0, 2, 1, 3, 4).reshape(prompts, hk, w * share, d)
    a = torch.matmul(shared, s["prefix_k"].permute(0, 2, 3, 1).float())
    off = torch.arange(case["prefix"], device="cuda") >= s["prefix_lengths"][:, None]
    a = a.masked_fill_(off[:, None, None], -math.inf)
    b = torch.matmul(q.view(prompts * w, hk, share, d), s["suffix_k"].permute(0, 2, 3, 1).float())
    off = torch.arange(case["suffix"], device="cuda") >= s["suffix_lengths"][:, None]
    b = b.masked_fill_(off[:, None, None], -math.inf)
    a = a.view(prompts, hk, w, share, -1).transpose(1, 2)
    b = b.view(prompts, w, hk, share, -1)
    top = torch.maximum(a.max(-1, keepdim=True).values, b.max(-1, keepdim=True).values)
    ea, eb = torch.exp(a - top), torch.exp(b - top)
    total = ea.sum(-1, keepdim=True) + eb.sum(-1, keepdim=True)
    va = torch.matmul(ea.transpose(1, 2).reshape(prompts, hk, w * share, -1), s["prefix_v"].transpose(1, 2).float())
    vb = torch.matmul(eb.reshape(prompts * w, hk, share, -1), s["suffix_v"].transpose(1, 2).float())
    out = va.view(prompts, hk, w, share, d).transpose(1, 2) + vb.view(prompts, w, hk, share, d)
    out = (out / total).reshape(prompts * w, case["heads"], d).to(s["q"].dtype)
    return (out, (top + torch.log(total)).reshape(prompts * w, case["heads"])) if case["lse"] else out


def _step_plain(case, s):
    # In 64 bits: which continuations are the best must not depend on roundings.
    groups, beams, vocab = case["groups"], case["beams"], case["vocab"]
    z = s["logits"].double() / case["temperature"]
    z = z - z.max(1, keepdim=True).values
    z = z - torch.log(torch.exp(z).sum(1, keepdim=True))
    total = s["scores"].double()[:, None] + z
    finished = s.get("finished")
    if finished is not None:
        total = total.masked_fill_(finished[:, None], -math.inf)
        total[:, END] = torch.where(finished, s["scores"].double(), total[:, END])
    rank = total
    if case["penalty"]:
        length = s["lengths"].double() + (1.0 if finished is None else torch.where(finished, 0.0, 1.0).double())
        rank = total / length.clamp(min=1)[:, None] ** case["penalty"]
    at = torch.sort(rank.view(groups, -1), dim=1, descending=True, stable=True).indices[:, :case["keep"]]
    best = torch.gather(total.view(groups, -1), 1, at)
    some = best > -math.inf
    place = torch.arange(case["keep"], device="cuda") % beams
    first = beams * torch.arange(groups, device="cuda")[:, None]
    tokens = torch.where(some, at % vocab, -1)
    parents = first + torch.where(some, at // vocab, place)
    ended = some & (tokens == END)
    if finished is not None:
        ended = ended | (some & finished[parents])
    return best.float(), tokens, parents, ended


def _reorder_plain(case, s):
    on = torch.arange(case["tokens"], device="cuda") < s["lengths"][s["parents"]][:, None]
    for src, dst in zip(s["states"], s["out"]):
        dst.copy_(torch.where(on[:, :, None, None], src[s["parents"]], dst))
    return s["out"]


PLAIN = {"attend": _attend_plain, "step": _step_plain, "reorder": _reorder_plain}


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    size = BYTES[case["dtype"]]
    if case["op"] == "attend":
        rows, d = case["prompts"] * case["answers"], case["dim"]
        prefix, suffix = case["prompts"] * case["prefix"] * case["fill"], rows * case["suffix"] * (0.5 + 0.5 * case["fill"])
        moved = 2 * (prefix + suffix) * case["kv_heads"] * d + 2 * rows * case["heads"] * d
        return {"bytes": moved * size + (4 * rows * case["heads"] if case["lse"] else 0),
                "flops": 4.0 * d * case["heads"] * (case["answers"] * prefix + suffix)}
    if case["op"] == "step":
        rows = case["groups"] * case["beams"]
        read = rows * (1 - case["finished"]) * case["vocab"]
        return {"bytes": read * size + 4 * rows + 21 * case["groups"] * case["keep"], "flops": 4.0 * read}
    rows, b = case["groups"] * case["beams"], case["beams"]
    # Beams that are a parent: those that none of the draws fall on are not read.
    chance = [((i + 1) / b) ** (1 / 1.7) - (i / b) ** (1 / 1.7) for i in range(b)]
    distinct = case["groups"] * sum(1 - (1 - c) ** b for c in chance)
    return {"bytes": case["tensors"] * (rows + distinct) * case["tokens"] * case["fill"] * case["heads"] * case["dim"] * size,
            "flops": 0}


# ---- the operators' definitions in 64 bits --------------------------------------------------------------------------

def exact(case, seed):
    s = MAKE[case["op"]](case, seed)
    f64 = torch.float64
    if case["op"] == "attend":
        w, hk = case["answers"], case["kv_heads"]
        share = case["heads"] // hk
        q = s["q"].to(f64)
        out, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=f64, device="cuda")
        prefix, suffix = s["prefix_lengths"].tolist(), s["suffix_lengths"].tolist()
        for p in range(case["prompts"]):
            mine = slice(p * w, (p + 1) * w)
            longest = max(suffix[mine])
            past = torch.tensor(suffix[mine], device="cuda")[:, None] <= torch.arange(longest, device="cuda")
            for h in range(hk):
                rows = q[mine, h * share:(h + 1) * share] / case["dim"] ** 0.5
                k, v = s["prefix_k"][p, :prefix[p], h].to(f64), s["prefix_v"][p, :prefix[p], h].to(f64)
                sk, sv = s["suffix_k"][mine, :longest, h].to(f64), s["suffix_v"][mine, :longest, h].to(f64)
                far = torch.einsum("wsd,td->wst", rows, k)
                near = torch.einsum("wsd,wtd->wst", rows, sk).masked_fill(past[:, None], -math.inf)
                both = torch.cat([far, near], 2)
                weight = torch.softmax(both, 2)
                lse[mine, h * share:(h + 1) * share] = torch.logsumexp(both, 2)
                out[mine, h * share:(h + 1) * share] = (torch.einsum("wst,td->wsd", weight[..., :prefix[p]], v)
                                                        + torch.einsum("wst,wtd->wsd", weight[..., prefix[p]:], sv))
        return (out, lse) if case["lse"] else out
    if case["op"] == "step":
        beams, keep, rows = case["beams"], case["keep"], case["groups"] * case["beams"]
        finished = s.get("finished", torch.zeros(rows, dtype=torch.bool, device="cuda"))
        z, _, _ = _best_of_rows(s["logits"], case["temperature"], ~finished, keep)
        length = s["lengths"] if case["penalty"] else torch.ones(rows, dtype=torch.int64, device="cuda")
        z, ended = z.cpu().numpy(), finished.cpu().numpy()
        score, length = s["scores"].double().cpu().numpy(), length.cpu().numpy()
        best = np.full((case["groups"], keep), -np.inf)
        for g in range(case["groups"]):
            totals, ranks = [], []
            for b in range(g * beams, (g + 1) * beams):
                t = np.array([score[b]]) if ended[b] else score[b] + z[b]
                totals.append(t)
                ranks.append(t / max(1.0, float(length[b] + (not ended[b]))) ** case["penalty"])
            totals, ranks = np.concatenate(totals), np.concatenate(ranks)
            order = np.argsort(-ranks, kind="stable")[:keep]
            best[g, :len(order)] = totals[order]
        return torch.from_numpy(best).cuda(), None, None, None
    lengths, parents = s["lengths"].tolist(), s["parents"].tolist()
    for src, dst in zip(s["states"], s["out"]):
        for i, p in enumerate(parents):
            dst[i, :lengths[p]] = src[p, :lengths[p]]
    return s["out"]
