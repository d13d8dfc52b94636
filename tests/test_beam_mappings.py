"""The example's beam of mappings: exact for a policy whose tools are independent, and the fastest of it."""
import itertools
import math

import pytest

from paper_2607_22242_gb300 import learn_mapping, scenarios

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _small():
    full = scenarios.config4(3)
    cut = lambda s, m: scenarios.Scenario(m, [p & ((1 << m) - 1) for p in s.pred_mask[:m]], s.cpu_us[:m], s.gpu_us[:m],
                                          s.xfer_us[:m], s.load_us[:m], s.vram_mib[:m], s.vram_budget_mib, s.slowdown_q10)
    return [cut(full[0], 4), cut(full[1], 2), cut(full[2], 4)]


@pytest.mark.parametrize("beams", [1, 5, 16, 40])
def test_likeliest_mappings(beams):
    scns = _small()
    logits = torch.randn(10, 3, generator=torch.Generator().manual_seed(beams)).cuda()
    lp = torch.log_softmax(logits.double(), 1).cpu()
    first = 0
    for s, (modes, scores) in zip(scns, learn_mapping.beam_mappings(logits, scns, beams)):
        every = [(sum(lp[first + t, a].item() for t, a in enumerate(m)), m) for m in itertools.product(range(3), repeat=s.n)]
        every.sort(key=lambda c: -c[0])
        for j in range(beams):
            if j < len(every):
                assert tuple(modes[j].tolist()) == every[j][1]
                assert abs(scores[j].item() - every[j][0]) < 1e-5
            else:
                assert scores[j].item() == -math.inf and (modes[j] == -1).all()
        first += s.n


def test_fastest_of_beam():
    from paper_2607_22242_gb300 import bf
    scns = scenarios.config4(5)
    logits = torch.randn(sum(s.n for s in scns), 3, generator=torch.Generator().manual_seed(0)).cuda()
    optima = [r.makespan_us for r in bf.search_batch(scns)]
    one, many, all_ = (learn_mapping.best_of_beam(logits, scns, b) for b in (1, 16, 243))
    assert all(o <= c <= b for o, b, c in zip(optima, many, all_))
    small = _small()[:1]
    assert learn_mapping.best_of_beam(logits[:4], small, 81) == [bf.search_best(small[0]).makespan_us]
    assert len(one) == 5
