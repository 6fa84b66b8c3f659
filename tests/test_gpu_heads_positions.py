"""Shapes and strides of the positions that the head norms take."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_heads import DEV, _P, _inputs  # noqa: E402


def test_expanded_positions():
    """Text in a model of three axes: one row of positions for all, read at stride 0."""
    q, k, table, positions, pair_axis, wq, wk = _inputs(5, 37, 3, 2, 64, 64, torch.float32, 3)
    op = _P().HeadNormRotary(64, table, dtype="f32", pair_axis=pair_axis)
    same = positions[1].expand(3, 37)
    g = torch.ones_like(q), torch.ones_like(k)
    got = op.forward(q, k, same, wq, wk) + op.backward(*g, q, k, same, wq, wk)
    want = op.forward(q, k, same.contiguous(), wq, wk) + op.backward(*g, q, k, same.contiguous(), wq, wk)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
