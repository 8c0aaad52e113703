"""The decoder-layer example: it learns, and a query asked alone hears what it hears among others."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("rig", ["tiny", "nuscenes"])
def test_example(rig):
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import map_queries
    losses, apart = map_queries.run(rig, steps=8)
    assert losses[-1] < 0.9 * losses[0]
    # bf16 answers of order 1 to 4, each rounded a few times: units of 2^-7 in the last place
    assert apart <= 0.125
