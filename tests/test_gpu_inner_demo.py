"""Inner and outer steps together: a small IsoLoCo run learns its text."""
import pytest

pytestmark = pytest.mark.gpu


def test_a_small_run_learns():
    from paper_2607_03011_gb300 import inner_demo
    losses = inner_demo.run(workers=3, rounds=3, inner_steps=10, tokens=1024, vocab=300, width=64, ff=136, report=lambda s: None)
    assert len(losses) == 4
    # learning the successors takes most of the first loss; a run that only forgets its random start
    # ends at the uniform loss, ln 300 = 5.7
    assert losses[-1] < min(losses[0], 5.7) - 0.5, losses
