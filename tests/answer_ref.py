"""Plain 64-bit forms of the operators of a decoding step, from their definitions (numpy)."""
import numpy as np


def attention(q, prefix_k, prefix_v, suffix_k, suffix_v, prefix_lengths, suffix_lengths, scale):
    """(out, ln of the sums, weighted means of |v|, the largest sum |q||k| of a score's products): 64-bit arrays
    (answers x heads x ...); suffix_k and suffix_v may be None."""
    answers, heads, dim = q.shape
    prompts, _, kv_heads, _ = prefix_k.shape
    share, each = heads // kv_heads, answers // prompts
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    lse, most = np.full((answers, heads), -np.inf), np.zeros((answers, heads))
    for a in range(answers):
        p = a // each
        for h in range(heads):
            g = h // share
            k, v = prefix_k[p, :prefix_lengths[p], g], prefix_v[p, :prefix_lengths[p], g]
            if suffix_k is not None:
                k = np.concatenate([k, suffix_k[a, :suffix_lengths[a], g]])
                v = np.concatenate([v, suffix_v[a, :suffix_lengths[a], g]])
            if len(k) == 0:
                continue
            s = scale * (k @ q[a, h])
            m = s.max()
            if m == -np.inf:
                continue
            w = np.exp(s - m)
            on = w > 0
            out[a, h] = (w[on, None] * v[on]).sum(0) / w.sum()
            size[a, h] = (w[on, None] * np.abs(v[on])).sum(0) / w.sum()
            lse[a, h] = m + np.log(w.sum())
            most[a, h] = (np.abs(k) @ np.abs(q[a, h])).max()
    return out, lse, size, most


def continuations(logits, score, finished, length, end_token, penalty, tau):
    """All continuations of one beam: (totals, ranks, tokens, length of a continuation)."""
    if finished:
        total, tokens, n = np.array([score]), np.array([end_token]), length
    else:
        on = logits > -np.inf
        if score == -np.inf or not on.any():
            return np.zeros(0), np.zeros(0), np.zeros(0, np.int64), length + 1
        z = logits / tau
        m = z.max()
        tokens = np.nonzero(on)[0]
        total, n = score + (z[on] - m - np.log(np.exp(z[on] - m).sum())), length + 1
    if score == -np.inf:
        return np.zeros(0), np.zeros(0), np.zeros(0, np.int64), n
    return total, total / max(1, n) ** penalty, tokens, n


def beam_step(logits, scores, beams, keep, finished=None, lengths=None, end_token=-1, penalty=0.0, tau=1.0):
    """For each group, its best continuations in the order of rank (20 more than are kept, at least): a list of (rank,
    total, token, parent, ended, length)."""
    groups = []
    for first in range(0, len(scores), beams):
        rows = []
        for b in range(first, first + beams):
            done = finished is not None and bool(finished[b])
            n0 = 0 if lengths is None else int(lengths[b])
            total, rank, tokens, n = continuations(logits[b], float(scores[b]), done, n0, end_token, penalty, tau)
            best = np.argsort(-rank, kind="stable")[:keep + 20]
            rows += [(-rank[i], b, int(tokens[i]), total[i], done or int(tokens[i]) == end_token, n) for i in best]
        rows.sort(key=lambda x: x[:3])
        groups.append([(-r, t, v, b, e, n) for r, b, v, t, e, n in rows])
    return groups


def reorder(state, parents, beams, lengths=None, out=None):
    """state's rows by their parents (numpy, any type), over what `out` (state itself if None) holds."""
    to = (state if out is None else out).copy()
    for i, p in enumerate(parents):
        if p // beams != i // beams or p < 0:
            continue
        n = state.shape[1] if lengths is None else min(int(lengths[p]), state.shape[1])
        if n > 0:
            to[i, :n] = state[p, :n]
    return to
