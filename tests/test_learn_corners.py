"""Corners of the learning entry points that need no GPU."""
import ctypes

import pytest

from paper_2607_22242_gb300 import _build, bf, learn_mapping, scenarios


@pytest.mark.parametrize("pairs", [(1 << 30) + 1, 1 << 62, 1 << 63, (1 << 63) + 1, (1 << 64) - 1])
def test_preference_workspace_refuses_pairs_past_the_limit(pairs):
    """Twice the pairs may wrap to few; the loss refuses such a number too."""
    _build.build()
    n = ctypes.c_uint64(7)
    assert bf.load().bf_preference_loss_workspace(1, pairs, ctypes.byref(n)) == bf.BF_EINVAL
    assert n.value == 7


@pytest.mark.parametrize("method", ["policy", "preference"])
@pytest.mark.parametrize("samples", [1, 0, -2])
def test_training_needs_samples_to_compare(method, samples):
    """One sample of a workflow has no spread and no pair: refused before any work, not trained on as NaN."""
    with pytest.raises(ValueError, match="samples"):
        learn_mapping.train(scenarios.config4(1), method, steps=1, samples=samples)
