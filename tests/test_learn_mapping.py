"""The example that fits a mapping policy to makespans."""
import pytest

from paper_2607_22242_gb300 import learn_mapping, scenarios


def test_card_tokens():
    """One token a field, within the field's range."""
    for scn in scenarios.config4(16) + [scenarios.config(i) for i in range(4)]:
        for row in learn_mapping.card_tokens(scn):
            assert len(row) == learn_mapping.FIELDS
            assert all(f * learn_mapping.LEVELS <= t < (f + 1) * learn_mapping.LEVELS for f, t in enumerate(row))


@pytest.mark.gpu
@pytest.mark.parametrize("method", ["policy", "preference"])
def test_training_brings_makespans_down(method):
    """16 workflows of 10 tools: the policy's mappings get closer to the brute-force optimum, and never below it."""
    pytest.importorskip("torch")
    gaps = learn_mapping.train(scenarios.config4(16), method, steps=60)
    assert len(gaps) == 61 and min(gaps) >= 1.0
    assert gaps[-1] - 1.0 < 0.6 * (gaps[0] - 1.0)
