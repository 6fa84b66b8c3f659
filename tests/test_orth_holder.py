"""Orthogonalizer's check of tensors, without a GPU."""
import pytest

torch = pytest.importorskip("torch")

from paper_1910_00643_amd import operators as O  # noqa: E402

from test_heads_holder import Stand  # noqa: E402


def _holder():
    o = object.__new__(O.Orthogonalizer)
    o.shapes, o.ld, o.n_matrices, o.device, o.handle = [(4, 6)], [6], 1, torch.device("cuda:0"), None
    return o


def test_tensors_of_another_gpu_are_refused():
    good, bad = Stand(4096, 4, 6), Stand(4096, 4, 6)
    good.element_size = bad.element_size = lambda: 4
    bad.device = torch.device("cuda:1")
    assert list(_holder().pointer_array([good], torch.float32)) == [4096]
    with pytest.raises(ValueError, match="cuda:1"):
        _holder().pointer_array([bad], torch.float32)
    with pytest.raises(ValueError):
        _holder().pointer_array([good], torch.bfloat16)
