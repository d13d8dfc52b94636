"""Operators for learning from makespans: what is timed, and their plain forms.

The search and the evaluations of this package grade the mappings that a scheduling model answers with.  These operators
turn such grades into gradients: log-probabilities of answered tokens, a clipped policy loss with a KL term, a preference
loss over pairs of answers, and the token embedding at the model's other end.  A case names the operator (``op``), its
sizes and options; ``own`` chooses between the package's kernels and the plain form in elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
LARGEST = 1 << 30  # logits of the largest case


def _logprobs(name, rows, vocab, dtype, grad, entropy, scored=1.0, temperature=1.0):
    return dict(name=name, op="logprobs", rows=rows, vocab=vocab, dtype=dtype, grad=grad, entropy=entropy, scored=scored,
                temperature=temperature)


def _policy(name, sequences, rows, vocab, dtype, reduction, scored, kl, entropy, temperature=1.0, banned=0.0):
    return dict(name=name, op="policy", sequences=sequences, rows=rows, vocab=vocab, dtype=dtype, reduction=reduction,
                scored=scored, kl=kl, entropy=entropy, temperature=temperature, banned=banned)


def _preference(name, pairs, rows, vocab, dtype, scored, reference, average, smoothing=0.0, margin=0.0):
    return dict(name=name, op="preference", pairs=pairs, rows=rows, vocab=vocab, dtype=dtype, scored=scored,
                reference=reference, average=average, smoothing=smoothing, margin=margin)


def _embed(name, rows, vocab, width, dtype, grad, skew, padding=0.0, scale=1.0):
    return dict(name=name, op="embed", rows=rows, vocab=vocab, width=width, dtype=dtype, grad=grad, skew=skew,
                padding=padding, scale=scale)


def listed():
    return [
        # One token of a scheduler that answers with text, scored as it is drawn.
        _logprobs("score one token", 1, 131072, "bf16", False, False),
        # The answers of a reference model, with their entropies; an odd vocabulary, so rows start at any alignment.
        _logprobs("score answers", 4096, 50001, "f16", False, True, scored=0.8, temperature=0.7),
        # A caller's own loss on log-probabilities and entropies: their gradient, in 32 bits.
        _logprobs("gradient of scores", 2048, 32768, "f32", True, True, scored=0.9),
        # A mapping policy, three modes a tool: 64 sampled mappings of a workflow of 16 tools.
        _policy("policy 64 mappings", 64, 1024, 3, "f32", "sequences", 1.0, 0.04, 0.01),
        # The same over the standard batch: 4096 workflows of 10 tools, 16 mappings each.
        _policy("policy batch of mappings", 65536, 655360, 3, "f32", "tokens", 1.0, 0.0, 0.01, banned=0.1),
        # A scheduler that answers with text: a step over 64 answers of about 128 tokens, prompts not scored.
        _policy("policy text answers", 64, 8192, 131072, "bf16", "tokens", 0.75, 0.04, 0.0),
        # A few short answers in pairs over a small vocabulary.
        _preference("preference 4 pairs", 4, 130, 1009, "f16", 0.9, True, False),
        # Pairs of answers over a middling vocabulary, rewards by the mean log-probability without a reference model.
        _preference("preference no reference", 16, 8000, 32000, "bf16", 0.8, False, True, margin=0.5),
        # A step of text answers in pairs over a large vocabulary.
        _preference("preference text answers", 16, 6144, 131072, "bf16", 0.75, True, False, smoothing=0.1),
        # The prompts of a step: rows of a large table.
        _embed("embed prompts", 16384, 131072, 2048, "bf16", False, 1.0, scale=math.sqrt(2048)),
        # Tool cards in 500 field tokens, each repeated very often.
        _embed("gradient of tool cards", 81920, 500, 256, "f32", True, 0.0, padding=0.1),
        # The gradient of a large table by the tokens of text: a few very frequent ones, many that do not occur.
        _embed("gradient of a large table", 16384, 131072, 2048, "bf16", True, 1.0, scale=math.sqrt(2048)),
    ]


def _log_size(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    n = min(hi, max(lo, n))
    return n + 1 if n == 3072 else n


def draw(rng):
    op = rng.choice(["logprobs", "policy", "preference", "embed"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if op == "embed":
        vocab, width = _log_size(rng, 3, 131072), _log_size(rng, 16, 4096)
        rows = _log_size(rng, 1, max(1, min(131072, (1 << 26) // width)))
        vocab = min(vocab, (1 << 28) // width)
        return dict(op=op, rows=rows, vocab=vocab, width=width, dtype=dtype, grad=rng.random() < 0.7,
                    skew=rng.choice([0.0, 0.5, 1.0]), padding=rng.choice([0.0, 0.1]), scale=rng.choice([1.0, 0.5, math.sqrt(width)]))
    vocab = _log_size(rng, 3, 131072)
    most = max(2, min(1 << 20, (LARGEST // 2) // (vocab * (2 if dtype == "f32" else 1))))
    rows = _log_size(rng, 1 if op == "logprobs" else 2, most)
    scored = rng.choice([1.0, 0.9, 0.6])
    temperature = rng.choice([1.0, 0.7, 1.3])
    if op == "logprobs":
        return dict(op=op, rows=rows, vocab=vocab, dtype=dtype, grad=rng.random() < 0.5, entropy=rng.random() < 0.5,
                    scored=scored, temperature=temperature)
    groups = _log_size(rng, 1, max(1, rows // 4))
    if op == "policy":
        return dict(op=op, sequences=groups, rows=rows, vocab=vocab, dtype=dtype, reduction=rng.choice(["tokens", "sequences", "sum"]),
                    scored=scored, kl=rng.choice([0.0, 0.04, 0.2]), entropy=rng.choice([0.0, 0.01]), temperature=temperature,
                    banned=rng.choice([0.0, 0.2]))
    return dict(op=op, pairs=max(1, groups // 2), rows=rows, vocab=vocab, dtype=dtype, scored=scored, reference=rng.random() < 0.7,
                average=rng.random() < 0.4, smoothing=rng.choice([0.0, 0.1]), margin=rng.choice([0.0, 0.5]))


# ---- inputs ---------------------------------------------------------------------------------------------------------

CLIP_LOW, CLIP_HIGH, BETA = 0.2, 0.28, 0.1
CHUNK = 1 << 26  # logits handled at a time where inputs are made and in the 64-bit form


def _chunks(rows, vocab, most=CHUNK):
    step = max(1, most // vocab)
    return [(a, min(rows, a + step)) for a in range(0, rows, step)]


def _offsets(rows, sequences, rng):
    """Boundaries of `sequences` answers of uneven lengths (some may be empty) that share out the rows."""
    share = rng.gamma(4.0, 1.0, sequences)
    cuts = np.rint(np.cumsum(share) / share.sum() * rows).astype(np.int64)
    return np.concatenate([[0], cuts[:-1], [rows]])


def _seed(case, seed):
    return [int(seed), case["rows"], case["vocab"]]


def _make(case, seed):
    """The tensors that a case's operator takes, from the seed alone, and nothing that goes by `own`."""
    gen = torch.Generator(device="cuda")
    rng = np.random.default_rng(_seed(case, seed))
    gen.manual_seed(int(rng.integers(1 << 40)))
    rows, vocab, dtype = case["rows"], case["vocab"], TYPES[case["dtype"]]
    rand = lambda *n: torch.rand(*n, generator=gen, device="cuda")
    randn = lambda *n, dtype=torch.float32: torch.randn(*n, generator=gen, device="cuda", dtype=dtype)
    if case["op"] == "embed":
        if case["skew"]:  # frequent tokens first, as in a vocabulary sorted by frequency
            u = rand(rows)
            tokens = torch.exp(u ** (1.0 / (0.5 + case["skew"])) * math.log(vocab)).to(torch.int64).sub_(1).clamp_(0, vocab - 1)
        else:
            tokens = torch.randint(vocab, (rows,), generator=gen, device="cuda")
        tokens = torch.where(rand(rows) < case["padding"], torch.full_like(tokens, -1), tokens)
        if case["grad"]:
            return dict(tokens=tokens, grad_out=randn(rows, case["width"], dtype=dtype))
        return dict(tokens=tokens, table=randn(vocab, case["width"], dtype=dtype).mul_(0.02))
    logits = torch.empty(rows, vocab, dtype=dtype, device="cuda")
    tokens = torch.randint(vocab, (rows,), generator=gen, device="cuda")
    tau = case.get("temperature", 1.0)
    logprob = torch.empty(rows, device="cuda")
    lift = rand(rows) * (2.0 + 0.8 * math.log(vocab))  # an answered token is mostly a likely one
    banned = case.get("banned", 0.0)
    for a, b in _chunks(rows, vocab):
        z = randn(b - a, vocab) * 2.0
        at = torch.arange(b - a, device="cuda")
        if banned:  # tokens that the answer's grammar (or the budget) forbids at this place
            z = torch.where(rand(b - a, vocab) < banned, torch.full_like(z, -math.inf), z)
        z[at, tokens[a:b]] = 2.0 * randn(b - a) + lift[a:b]
        logits[a:b] = z.to(dtype)
        z = logits[a:b].float() / tau
        logprob[a:b] = z[at, tokens[a:b]] - torch.logsumexp(z, 1)
    s = dict(logits=logits)
    if case["op"] == "logprobs":
        s["tokens"] = torch.where(rand(rows) >= case["scored"], torch.full_like(tokens, -1), tokens)
        if case["grad"]:
            s["grad_logprob"] = randn(rows)
            if case["entropy"]:
                s["grad_entropy"] = 0.01 * randn(rows)
        return s
    sequences = case["sequences"] if case["op"] == "policy" else 2 * case["pairs"]
    cuts = _offsets(rows, sequences, rng)
    offsets = torch.from_numpy(cuts).cuda()
    length = offsets[1:] - offsets[:-1]
    row = torch.arange(rows, device="cuda")
    seq = torch.repeat_interleave(torch.arange(sequences, device="cuda"), length, output_size=rows)
    place = (row - offsets[seq]).float() / length[seq].float()
    s.update(offsets=offsets, tokens=torch.where(place < 1.0 - case["scored"], torch.full_like(tokens, -1), tokens))
    drift = lambda size: size * randn(rows)
    if case["op"] == "policy":
        d = drift(0.15)
        # A ratio within 1e-4 of a clip edge would be clipped in one precision and not in another: such ones are moved.
        for edge in (math.log(1.0 - CLIP_LOW), math.log(1.0 + CLIP_HIGH)):
            d = torch.where((d - edge).abs() < 1e-4, d + 1e-3, d)
        s["old_logprob"] = logprob - d
        s["advantage"] = randn(sequences)
        if case["kl"]:
            s["ref_logprob"] = logprob + drift(0.3)
    elif case["reference"]:
        s["ref_logprob"] = logprob + drift(0.3)
    return s


def prepare(case, seed):
    return dict(case=dict(case), **_make(case, seed))


# ---- one pass -------------------------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    return (_run_own if own else _run_plain)(case, state)


def _run_own(case, s):
    from paper_2607_22242_gb300 import bf
    if case["op"] == "embed":
        if case["grad"]:
            return bf.embed_grad(s["grad_out"], s["tokens"], case["vocab"], scale=case["scale"])
        return bf.embed(s["table"], s["tokens"], scale=case["scale"])
    if case["op"] == "logprobs":
        if case["grad"]:
            return bf.token_logprobs_grad(s["logits"], s["tokens"], s["grad_logprob"], s.get("grad_entropy"),
                                          temperature=case["temperature"])
        return bf.token_logprobs(s["logits"], s["tokens"], temperature=case["temperature"], entropy=case["entropy"])
    if case["op"] == "policy":
        r = bf.policy_loss(s["logits"], s["tokens"], s["offsets"], s["old_logprob"], s["advantage"], s.get("ref_logprob"),
                           clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=case["kl"], entropy_coef=case["entropy"],
                           temperature=case["temperature"], reduction=case["reduction"])
        return r.stats, r.logprob, r.grad
    r = bf.preference_loss(s["logits"], s["tokens"], s["offsets"], s.get("ref_logprob"), beta=BETA, margin=case["margin"],
                           label_smoothing=case["smoothing"], average=case["average"])
    return r.stats, r.rewards, r.logprob, r.grad


def _row_index(tokens):
    return torch.arange(tokens.numel(), device=tokens.device), tokens.clamp(min=0)


def _softmax(logits, tau):
    """(x - max) / tau, its exponentials and their sums, in 32 bits."""
    x = logits.float()
    d = (x - x.max(1, keepdim=True).values) / tau
    e = torch.exp(d)
    return d, e, e.sum(1)


def _entropy(d, e, s):
    return torch.log(s) - torch.where(e > 0, e * d, torch.zeros_like(e)).sum(1) / s


def _logit_grad(d, e, s, tokens, tau, a, c=None, h=None):
    """Gradient of sum_t a_t logprob_t + c_t entropy_t in the logits, in 32 bits."""
    at, y = _row_index(tokens)
    p = e / s[:, None]
    g = -a[:, None] * p
    if c is not None:
        g = g - c[:, None] * torch.where(p > 0, p * (d - torch.log(s)[:, None] + h[:, None]), torch.zeros_like(p))
    g[at, y] += a
    return torch.where((tokens >= 0)[:, None], g / tau, torch.zeros_like(g))


def _sequence_of(offsets, rows):
    return torch.bucketize(torch.arange(rows, device=offsets.device), offsets[1:], right=True)


def _sum_by(values, seq, count):
    return torch.zeros(count, dtype=values.dtype, device=values.device).index_add_(0, seq, values)


def _run_plain(case, s):
    tokens = s["tokens"]
    if case["op"] == "embed":
        on = tokens >= 0
        if case["grad"]:
            g = torch.where(on[:, None], s["grad_out"].float() * case["scale"], 0.0)
            out = torch.zeros(case["vocab"], case["width"], device="cuda").index_add_(0, tokens.clamp(min=0), g)
            return out.to(s["grad_out"].dtype)
        return torch.where(on[:, None], s["table"][tokens.clamp(min=0)].float() * case["scale"], 0.0).to(s["table"].dtype)
    logits, tau = s["logits"], case.get("temperature", 1.0)
    at, y = _row_index(tokens)
    on = tokens >= 0
    d, e, total = _softmax(logits, tau)
    lp = torch.where(on, d[at, y] - torch.log(total), 0.0)
    if case["op"] == "logprobs":
        if not case["grad"]:
            return (lp, torch.where(on, _entropy(d, e, total), 0.0)) if case["entropy"] else lp
        h = _entropy(d, e, total) if case["entropy"] else None
        return _logit_grad(d, e, total, tokens, tau, s["grad_logprob"], s.get("grad_entropy"), h).to(logits.dtype)
    offsets = s["offsets"]
    count = offsets.numel() - 1
    seq = _sequence_of(offsets, tokens.numel())
    n = _sum_by(on.float(), seq, count)
    if case["op"] == "policy":
        if case["reduction"] == "tokens":
            w = on.float() / n.sum().clamp(min=1)
        elif case["reduction"] == "sequences":
            w = on.float() / (n[seq].clamp(min=1) * (n > 0).sum().clamp(min=1))
        else:
            w = on.float()
        adv = s["advantage"][seq]
        ratio = torch.exp(torch.where(on, lp - s["old_logprob"], 0.0))
        held = torch.where(adv >= 0, ratio.clamp(max=1 + CLIP_HIGH), ratio.clamp(min=1 - CLIP_LOW))
        clipped = held != ratio
        kl = torch.zeros_like(lp)
        slope = torch.where(clipped, 0.0, -adv * ratio)
        if case["kl"]:
            u = torch.where(on, s["ref_logprob"] - lp, 0.0)
            kl = torch.exp(u) - u - 1
            slope = slope + case["kl"] * (1 - torch.exp(u))
        h = _entropy(d, e, total)
        term = -held * adv + case["kl"] * kl - case["entropy"] * h
        mean = lambda v: (w * v).sum()
        stats = torch.stack([mean(term), mean(-held * adv), mean(kl), mean(h), mean(clipped.float()), mean(ratio)])
        c = -case["entropy"] * w if case["entropy"] else None
        return stats, lp, _logit_grad(d, e, total, tokens, tau, w * slope, c, h).to(logits.dtype)
    pairs = case["pairs"]
    ref = s["ref_logprob"] if case["reference"] else torch.zeros_like(lp)
    share = 1.0 / n.clamp(min=1) if case["average"] else torch.ones_like(n)
    rewards = BETA * _sum_by(torch.where(on, lp - ref, 0.0), seq, count) * share
    gap = rewards[0::2] - rewards[1::2] - case["margin"]
    log_sigmoid = lambda v: torch.minimum(v, torch.zeros_like(v)) - torch.log1p(torch.exp(-v.abs()))
    eps = case["smoothing"]
    loss = -(1 - eps) * log_sigmoid(gap) - eps * log_sigmoid(-gap)
    slope = (eps / (1 + torch.exp(-gap)) - (1 - eps) / (1 + torch.exp(gap))) * BETA / pairs
    stats = torch.stack([loss.mean(), (rewards[0::2] > rewards[1::2]).float().mean(), rewards[0::2].mean(), rewards[1::2].mean()])
    a = torch.stack([slope, -slope], 1).reshape(-1) * share
    return stats, rewards, lp, _logit_grad(d, e, total, tokens, tau, a[seq]).to(logits.dtype)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    rows, vocab, size = case["rows"], case["vocab"], BYTES[case["dtype"]]
    if case["op"] == "embed":
        moved = rows * case["width"]
        if case["grad"]:
            return {"bytes": moved * size + vocab * case["width"] * size + 8 * rows, "flops": moved}
        read = min(rows, vocab) * case["width"]  # the distinct rows of a table, at most
        return {"bytes": (read + moved) * size + 8 * rows, "flops": moved}
    scored = case["scored"] * rows
    read = scored * vocab * size + 8 * rows
    if case["op"] == "logprobs" and not case["grad"]:
        return {"bytes": read + 4 * rows * (2 if case["entropy"] else 1), "flops": scored * vocab * 5}
    return {"bytes": read + rows * vocab * size + 16 * rows, "flops": scored * vocab * 10}


# ---- the operators' definitions in 64 bits --------------------------------------------------------------------------

def exact(case, seed):
    s = _make(case, seed)
    tokens = s["tokens"]
    f64 = torch.float64
    if case["op"] == "embed":
        keep = torch.nonzero(tokens >= 0)[:, 0]
        if not case["grad"]:
            out = torch.zeros(case["rows"], case["width"], dtype=f64, device="cuda")
            out[keep] = s["table"][tokens[keep]].to(f64) * case["scale"]
            return out
        out = torch.zeros(case["vocab"], case["width"], dtype=f64, device="cuda")
        order = keep[torch.argsort(tokens[keep], stable=True)]
        which, many = torch.unique_consecutive(tokens[order], return_counts=True)
        if order.numel():
            sums = torch.segment_reduce(s["grad_out"][order].to(f64), "sum", lengths=many, axis=0)
            out[which] = sums * case["scale"]
        return out
    rows, vocab, tau = case["rows"], case["vocab"], case.get("temperature", 1.0)
    lp = torch.zeros(rows, dtype=f64, device="cuda")
    ent = torch.zeros(rows, dtype=f64, device="cuda")
    for a, b in _chunks(rows, vocab, 1 << 24):
        z = torch.log_softmax(s["logits"][a:b].to(f64) / tau, 1)
        t = tokens[a:b]
        lp[a:b] = torch.where(t >= 0, z.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)
        ent[a:b] = torch.where(t >= 0, torch.special.entr(z.exp()).sum(1), 0.0)

    def gradient(on_logprob, on_entropy):
        g = torch.empty(rows, vocab, dtype=f64, device="cuda")
        for a, b in _chunks(rows, vocab, 1 << 24):
            z = torch.log_softmax(s["logits"][a:b].to(f64) / tau, 1)
            p, t = z.exp(), tokens[a:b]
            hit = torch.zeros_like(p).scatter_(1, t.clamp(min=0)[:, None], 1.0)
            part = on_logprob[a:b, None] * (hit - p)
            if on_entropy is not None:
                part += on_entropy[a:b, None] * (torch.special.entr(p) - p * ent[a:b, None])
            g[a:b] = torch.where(t[:, None] >= 0, part / tau, 0.0)
        return g

    if case["op"] == "logprobs":
        if case["grad"]:
            return gradient(s["grad_logprob"].to(f64), s["grad_entropy"].to(f64) if case["entropy"] else None)
        return (lp, ent) if case["entropy"] else lp
    cuts = s["offsets"].cpu().numpy()
    on = (tokens >= 0).cpu().numpy()
    host = lambda v: v.to(f64).cpu().numpy()
    l = host(lp)
    seq = np.repeat(np.arange(len(cuts) - 1), np.diff(cuts))
    n = np.bincount(seq[on], minlength=len(cuts) - 1)
    to_gpu = lambda v: torch.from_numpy(np.ascontiguousarray(v)).cuda()
    if case["op"] == "policy":
        if case["reduction"] == "tokens":
            w = on / max(1, n.sum())
        elif case["reduction"] == "sequences":
            w = on / np.maximum(1, n[seq]) / max(1, np.count_nonzero(n))
        else:
            w = on.astype(np.float64)
        adv, h = host(s["advantage"])[seq], host(ent)
        r = np.exp(np.where(on, l - host(s["old_logprob"]), 0.0))
        low, high = 1 - CLIP_LOW, 1 + CLIP_HIGH
        gain = np.minimum(r * adv, np.clip(r, low, high) * adv)
        stopped = ((adv >= 0) & (r > high)) | ((adv < 0) & (r < low))
        u = np.where(on, host(s["ref_logprob"]) - l, 0.0) if case["kl"] else np.zeros(rows)
        kl = np.expm1(u) - u
        loss = -gain + case["kl"] * kl - case["entropy"] * h
        stats = np.array([np.sum(w * v) for v in (loss, -gain, kl, h, stopped, r)])
        slope = np.where(stopped, 0.0, -adv * r) - case["kl"] * np.expm1(u)
        return to_gpu(stats), lp, gradient(to_gpu(w * slope), to_gpu(-case["entropy"] * w) if case["entropy"] else None)
    ref = host(s["ref_logprob"]) if case["reference"] else np.zeros(rows)
    reward = BETA * np.bincount(seq[on], weights=(l - ref)[on], minlength=len(cuts) - 1)
    share = 1.0 / np.maximum(1, n) if case["average"] else np.ones(len(n))
    reward = reward * share
    gap = reward[0::2] - reward[1::2] - case["margin"]
    eps, pairs = case["smoothing"], case["pairs"]
    loss = (1 - eps) * np.logaddexp(0, -gap) + eps * np.logaddexp(0, gap)
    sig = np.exp(-np.logaddexp(0, -gap))
    slope = (eps * sig - (1 - eps) * (1 - sig)) * BETA / pairs
    a = np.stack([slope, -slope], 1).reshape(-1) * share
    stats = np.array([loss.mean(), np.mean(reward[0::2] > reward[1::2]), reward[0::2].mean(), reward[1::2].mean()])
    return to_gpu(stats), to_gpu(reward), lp, gradient(to_gpu(a[seq]), None)
