"""More arguments that the heads' C entry points refuse, without a GPU."""
import pytest

import paper_1910_00643_amd as P
from paper_1910_00643_amd import binding as B

from test_heads_host import _backward, _config, _forward, _heads


@pytest.mark.parametrize("weight", ["q_weight", "k_weight"])
def test_weights_without_the_norm(weight):
    """They were ignored without a word."""
    assert _forward(_config(norm=0, **{weight: 0x700000})) == B.SLOWMO_ERR_ARG
    assert "weights" in P.slowmo_last_error(None)
    assert _backward(_config(norm=0, **{weight: 0x700000}), dwq=None) == B.SLOWMO_ERR_ARG
    assert "weights" in P.slowmo_last_error(None)


def test_arrays_that_reach_past_64_bits():
    """Their extents wrapped, so that overlaps were judged by other addresses."""
    far = 1 << 40
    assert _forward(_config(), slots=0x1000, rows=far, k_out=_heads(0x400000, token=far)) == B.SLOWMO_ERR_ARG
    assert "2^50" in P.slowmo_last_error(None)
    assert _forward(_config(), tokens=1 << 31, q=_heads(0x100000, token=1 << 20)) == B.SLOWMO_ERR_ARG
    assert "2^50" in P.slowmo_last_error(None)
