"""A small mapping policy fitted to makespans: the learning entry points of :mod:`bf`, put together.

Each tool card (its latencies, load-in, footprint, place in the DAG) becomes a few field tokens; their embeddings
(:func:`bf.embed`) are summed, mixed over the DAG and turned into logits over the three modes.  Mappings are sampled,
:func:`bf.eval_indices` gives their makespans, and either

* ``policy``: the clipped policy loss (:func:`bf.policy_loss`) with each mapping's makespan measured against the other
  samples of its workflow, held near the starting policy by a KL term, or
* ``preference``: the preference loss (:func:`bf.preference_loss`) over pairs of a workflow's samples, the faster first,

gives the gradient in the logits; torch carries it through the two layers between, :func:`bf.embed_grad` into the table.

    python -m paper_2607_22242_gb300.learn_mapping [policy|preference] [steps]
"""
from __future__ import annotations

import math
import sys
from typing import List, Sequence

from . import bf, scenarios
from .scenarios import Scenario

LEVELS = 24      # values of a field: 2 a factor of 2, of what varies over a factor of 4,000
FIELDS = 7       # cpu, gpu, transfer, load-in, footprint over budget, predecessors, successors
MODES = 3


def card_tokens(scn: Scenario) -> List[List[int]]:
    """FIELDS tokens for each tool: field f's value v is token f * LEVELS + v."""
    step = lambda x, unit: min(LEVELS - 1, max(0, int(round(2 * math.log2(max(x, 1) / unit)))))
    rows = []
    for v in range(scn.n):
        values = (step(scn.cpu_us[v], 4096), step(scn.gpu_us[v], 4096), step(scn.xfer_us[v], 1024),
                  step(scn.load_us[v], 4096), min(LEVELS - 1, scn.vram_mib[v] * LEVELS // max(1, scn.vram_budget_mib)),
                  min(LEVELS - 1, bin(scn.pred_mask[v]).count("1")),
                  min(LEVELS - 1, sum(p >> v & 1 for p in scn.pred_mask[:scn.n])))
        rows.append([f * LEVELS + x for f, x in enumerate(values)])
    return rows


class Policy:
    """Logits over the modes of every tool of every workflow, and Adam over its weights."""

    def __init__(self, scns: Sequence[Scenario], width: int = 64, seed: int = 0, rate: float = 0.01):
        import torch
        self.scns = list(scns)
        gen = torch.Generator().manual_seed(seed)
        self.tokens = torch.tensor([t for s in scns for row in card_tokens(s) for t in row], device="cuda")
        n = sum(s.n for s in scns)
        # Each tool also sees the mean of its workflow and the sum of its predecessors.
        mix, first = torch.zeros(2, n, n), 0
        for s in scns:
            mix[0, first:first + s.n, first:first + s.n] = 1.0 / s.n
            for v in range(s.n):
                for u in range(v):
                    mix[1, first + v, first + u] = float(s.pred_mask[v] >> u & 1)
            first += s.n
        self.mix = mix.cuda()
        draw = lambda *shape: (torch.randn(*shape, generator=gen) / math.sqrt(shape[0])).cuda()
        self.table = (0.3 * torch.randn(FIELDS * LEVELS, width, generator=gen)).cuda()
        self.weights = [draw(3 * width, width).requires_grad_(), draw(width, MODES).requires_grad_()]
        self.rate, self.steps = rate, 0
        self.moments = [(torch.zeros_like(w), torch.zeros_like(w)) for w in (self.table, *self.weights)]

    def logits(self):
        """(logits, the embedding rows they came from), both with a gradient to take."""
        import torch
        rows = bf.embed(self.table, self.tokens).requires_grad_()
        x = rows.view(-1, FIELDS, rows.shape[1]).sum(1)
        x = torch.cat([x, self.mix[0] @ x, self.mix[1] @ x], 1)
        return torch.relu(x @ self.weights[0]) @ self.weights[1], rows

    def step(self, logits, rows, grad):
        """One step of Adam along the loss whose gradient in the logits is `grad`."""
        import torch
        grads = torch.autograd.grad(logits, [rows, *self.weights], grad)
        grads = [bf.embed_grad(grads[0], self.tokens, self.table.shape[0]), *grads[1:]]
        self.steps += 1
        with torch.no_grad():
            for w, g, (m, v) in zip((self.table, *self.weights), grads, self.moments):
                m.lerp_(g, 0.1)
                v.lerp_(g * g, 0.01)
                w -= self.rate * (m / (1 - 0.9 ** self.steps)) / ((v / (1 - 0.99 ** self.steps)).sqrt() + 1e-8)


def _makespans(handles, scns, modes):
    """Makespans of sampled mappings: modes is (samples, tools of all workflows); (samples, workflows), infinite where
    a mapping exceeds the budget."""
    import torch
    out, first = [], 0
    for h, s in zip(handles, scns):
        power = torch.tensor([3 ** i for i in range(s.n)], device="cuda")
        ms, fe = bf.eval_indices(h, (modes[:, first:first + s.n] * power).sum(1))
        out.append(torch.where(fe == 1, ms.double(), math.inf))
        first += s.n
    return torch.stack(out, 1)


def train(scns: Sequence[Scenario], method: str = "policy", steps: int = 60, samples: int = 32, seed: int = 0,
          progress=None) -> List[float]:
    """Fit a policy; the mean over the workflows of (makespan of the policy's likeliest mapping / optimum), before the
    first step and after every one (a mapping beyond the budget counts as the all-cpu one)."""
    import torch
    if samples < 2:
        raise ValueError("samples must be at least 2: a workflow's samples are measured against each other")
    torch.manual_seed(seed)
    policy = Policy(scns, seed=seed)
    best = torch.tensor([r.makespan_us for r in bf.search_batch(list(scns))], device="cuda", dtype=torch.float64)
    sizes = [s.n for s in scns]
    tools = sum(sizes)
    handles = [bf.create_scenario(s) for s in scns]
    try:
        cpu = _makespans(handles, scns, torch.zeros(1, tools, dtype=torch.int64, device="cuda"))[0]
        # Rows of a step: sample by sample, workflow by workflow, tool by tool; one answer is one workflow's mapping.
        lengths = torch.tensor(sizes * samples)
        offsets = torch.cat([torch.zeros(1, dtype=torch.int64), lengths.cumsum(0)]).cuda()
        history = []

        def gap(logits):
            ms = _makespans(handles, scns, logits.argmax(1)[None])[0]
            history.append((torch.where(torch.isinf(ms), cpu, ms) / best).mean().item())
            if progress:
                progress(len(history) - 1, history[-1])

        start = policy.logits()[0].detach()
        for _ in range(steps):
            logits, rows = policy.logits()
            now = logits.detach()
            gap(now)
            modes = torch.multinomial(torch.softmax(now, 1), samples, replacement=True).t().contiguous()
            ms = _makespans(handles, scns, modes)
            cost = torch.log(torch.where(torch.isinf(ms), 2 * cpu, ms) / best)  # (samples, workflows)
            wide = logits.repeat(samples, 1)
            flat = modes.reshape(-1)
            ref = bf.token_logprobs(start.repeat(samples, 1), flat)
            if method == "policy":
                advantage = (cost.mean(0) - cost) / (cost.std(0) + 1e-3)
                old = bf.token_logprobs(wide.detach(), flat)
                loss = bf.policy_loss(wide.detach(), flat, offsets, old, advantage.float().reshape(-1), ref,
                                      kl_coef=0.01, entropy_coef=0.01, reduction="sequences")
                policy.step(wide, rows, loss.grad)
            elif method == "preference":
                # Samples s and s + samples / 2 of a workflow are a pair, the faster one first.
                half = samples // 2
                swap = (cost[half:2 * half] < cost[:half]).repeat_interleave(torch.tensor(sizes, device="cuda"), dim=1)
                grid = torch.arange(2 * half * tools, device="cuda").view(2, half, tools)
                pair = torch.stack([torch.where(swap, grid[1], grid[0]), torch.where(swap, grid[0], grid[1])])
                order = torch.cat([pair[k, s, a:a + n] for s in range(half)
                                   for a, n in zip([sum(sizes[:i]) for i in range(len(sizes))], sizes)
                                   for k in (0, 1)])
                cuts = torch.tensor([n for _ in range(half) for n in sizes for _ in (0, 1)]).cumsum(0)
                cuts = torch.cat([torch.zeros(1, dtype=torch.int64), cuts]).cuda()
                chosen = wide[order]
                loss = bf.preference_loss(chosen.detach(), flat[order], cuts, ref[order], beta=0.3)
                policy.step(chosen, rows, loss.grad)
            else:
                raise ValueError("method must be policy or preference")
        gap(policy.logits()[0].detach())
        return history
    finally:
        for h in handles:
            h.close()


if __name__ == "__main__":
    how = sys.argv[1] if len(sys.argv) > 1 else "policy"
    count = int(sys.argv[2]) if len(sys.argv) > 2 else 60
    found = train(scenarios.config4(16), how, count,
                  progress=lambda k, g: print(f"step {k:3d}: makespan / optimum {g:.3f}") if k % 10 == 0 else None)
    print(f"{how}: {found[0]:.3f} -> {found[-1]:.3f} of the optimum in {count} steps")
