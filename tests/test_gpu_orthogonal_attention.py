"""The example that uses the norm with rotation, the orthogonalised directions and the
Slow Momentum steps together learns its task."""
import math
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_workers_learn_to_repeat_a_token():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import orthogonal_attention as E
    finally:
        sys.path.pop(0)
    losses = E.train(outer=20)
    assert all(math.isfinite(v) for v in losses)
    # a guess among VOCAB tokens costs log(VOCAB) = 4.16
    assert sum(losses[:6]) / 6 > 0.8 * math.log(E.VOCAB)
    assert sum(losses[-6:]) / 6 < 0.5 * math.log(E.VOCAB)
