"""Plain 64-bit forms of the operators that learn from makespans, row by row from their definitions (numpy)."""
import numpy as np


def softmax(x, tau):
    """ln p and p of one row of logits (64-bit); None where no logit is above -inf."""
    m = x.max()
    if m == -np.inf:
        return None
    d = (x - m) / tau
    e = np.exp(d)
    return d - np.log(e.sum()), e / e.sum()


def entropy_of(lp, p):
    on = p > 0
    return float(-(p[on] * lp[on]).sum())


def scores(x, tokens, tau=1.0):
    """(log-probabilities, entropies) of rows."""
    out = np.zeros((2, len(tokens)))
    for t, y in enumerate(tokens):
        if y < 0:
            continue
        s = softmax(x[t], tau)
        out[:, t] = (-np.inf, 0.0) if s is None else (s[0][y], entropy_of(*s))
    return out[0], out[1]


def scores_grad(x, tokens, a, c, tau=1.0):
    """Gradient of sum a_t lp_t + c_t H_t, and how large its parts are (for error bounds)."""
    g, size = np.zeros(x.shape), np.zeros(x.shape)
    for t, y in enumerate(tokens):
        s = softmax(x[t], tau) if y >= 0 else None
        if s is None:
            continue
        lp, p = s
        h = entropy_of(lp, p)
        tilt = np.where(p > 0, np.where(p > 0, lp, 0.0) + h, 0.0)
        hit = np.zeros(x.shape[1])
        hit[y] = 1.0
        g[t] = (a[t] * (hit - p) - c[t] * p * tilt) / tau
        size[t] = (abs(a[t]) * (hit + p) + abs(c[t]) * p * (np.abs(tilt) + 1.0)) / tau
    return g, size


def sequence_of(offsets, rows):
    seq = np.full(rows, -1)
    for s in range(len(offsets) - 1):
        seq[offsets[s]:offsets[s + 1]] = s
    return seq


def policy(x, tokens, offsets, old, adv, ref=None, lo=0.2, hi=0.2, kl_coef=0.0, entropy_coef=0.0, tau=1.0,
           reduction="tokens", per_token=False):
    """(stats, log-probabilities of the scored rows, gradient, its parts' size, rows' clip margins)."""
    rows = len(tokens)
    seq = sequence_of(offsets, rows)
    on = (np.asarray(tokens) >= 0) & (seq >= 0)
    n = np.bincount(seq[on], minlength=len(offsets) - 1)
    lp, h = scores(x, np.where(on, tokens, -1), tau)
    stats, a, c, margin = np.zeros(6), np.zeros(rows), np.zeros(rows), np.full(rows, np.inf)
    parts = np.zeros(rows)  # magnitudes of the slope's two terms: they may cancel
    for t in np.nonzero(on)[0]:
        w = {"tokens": 1 / on.sum(), "sequences": 1 / (n[seq[t]] * np.count_nonzero(n)), "sum": 1.0}[reduction]
        if lp[t] == -np.inf and h[t] == 0.0 and x[t].max() == -np.inf:
            continue
        A = adv[t if per_token else seq[t]]
        r = np.exp(lp[t] - old[t])
        gain = min(r * A, np.clip(r, 1 - lo, 1 + hi) * A)
        stopped = (A >= 0 and r > 1 + hi) or (A < 0 and r < 1 - lo)
        u = 0.0 if ref is None else ref[t] - lp[t]
        kl = np.expm1(u) - u
        stats += w * np.array([-gain + kl_coef * kl - entropy_coef * h[t], -gain, kl, h[t], float(stopped), r])
        a[t] = w * ((0.0 if stopped else -A * r) - kl_coef * np.expm1(u))
        parts[t] = w * ((0.0 if stopped else abs(A) * r) + kl_coef * (np.exp(u) + 1))
        c[t] = -w * entropy_coef
        margin[t] = min(abs(r - (1 + hi)), abs(r - (1 - lo)))
    g, _ = scores_grad(x, np.where(on, tokens, -1), a, c, tau)
    _, size = scores_grad(x, np.where(on, tokens, -1), parts, c, tau)
    return stats, lp, g, size, margin


def preference(x, tokens, offsets, ref=None, beta=0.1, eps=0.0, margin=0.0, average=False, tau=1.0):
    """(stats, rewards, log-probabilities, gradient, its parts' size)."""
    rows, pairs = len(tokens), len(offsets) // 2
    seq = sequence_of(offsets, rows)
    on = (np.asarray(tokens) >= 0) & (seq >= 0)
    lp, _ = scores(x, np.where(on, tokens, -1), tau)
    reward, share = np.zeros(2 * pairs), np.zeros(2 * pairs)
    for s in range(2 * pairs):
        mine = np.nonzero(on & (seq == s))[0]
        share[s] = beta / (max(1, len(mine)) if average else 1)
        reward[s] = share[s] * sum(lp[t] - (0.0 if ref is None else ref[t]) for t in mine)
    a, parts = np.zeros(rows), np.zeros(rows)
    loss = 0.0
    for p in range(pairs):
        h = reward[2 * p] - reward[2 * p + 1] - margin
        loss += ((1 - eps) * np.logaddexp(0, -h) + eps * np.logaddexp(0, h)) / pairs
        slope = (eps * np.exp(-np.logaddexp(0, -h)) - (1 - eps) * np.exp(-np.logaddexp(0, h))) / pairs
        part = (eps * np.exp(-np.logaddexp(0, -h)) + (1 - eps) * np.exp(-np.logaddexp(0, h))) / pairs
        for k, sign in ((0, 1), (1, -1)):
            a[seq == 2 * p + k] = sign * slope * share[2 * p + k]
            parts[seq == 2 * p + k] = part * share[2 * p + k]
    g, _ = scores_grad(x, np.where(on, tokens, -1), a, np.zeros(rows), tau)
    _, size = scores_grad(x, np.where(on, tokens, -1), parts, np.zeros(rows), tau)
    r0, r1 = reward[0::2], reward[1::2]
    stats = np.array([loss, np.mean(r0 > r1), r0.mean(), r1.mean()]) if pairs else np.zeros(4)
    return stats, reward, lp, g, size


def embed(table, tokens, scale):
    out = np.zeros((len(tokens), table.shape[1]))
    for t, v in enumerate(tokens):
        if v >= 0:
            out[t] = scale * table[v]
    return out


def embed_grad(grad_out, tokens, vocab, scale):
    """(sums by token, sums of magnitudes by token)."""
    g, size = np.zeros((vocab, grad_out.shape[1])), np.zeros((vocab, grad_out.shape[1]))
    for t, v in enumerate(tokens):
        if 0 <= v < vocab:
            g[v] += scale * grad_out[t]
            size[v] += abs(scale) * np.abs(grad_out[t])
    return g, size
