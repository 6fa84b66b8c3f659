"""HeadNormRotary's checks and the structures it hands to the library, without a GPU: stand-ins have
what the holder asks of a tensor."""
import threading

import pytest

torch = pytest.importorskip("torch")

from paper_1910_00643_amd import operators as O  # noqa: E402


class Stand:
    """A contiguous tensor of this shape at this address, as far as the holder looks."""
    is_cuda, device = True, torch.device("cuda:0")

    def __init__(self, at, *shape, dtype=torch.float32):
        self.at, self.shape, self.dtype = at, torch.Size(shape), dtype

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def data_ptr(self):
        return self.at

    def is_contiguous(self):
        return True

    def stride(self):
        st = [1]
        for n in reversed(self.shape[1:]):
            st.insert(0, st[0] * n)
        return tuple(st)


def _op():
    op = O.HeadNormRotary(16, None, dtype="f32", norm=False)
    op.pairs = 8                            # as with a table
    return op


@pytest.mark.parametrize("shape", [(2, 1, 12), (1, 2, 12), (1, 1, 12), (2, 6), (11,), ()], ids=str)
def test_positions_of_other_shapes_are_refused(shape):
    with pytest.raises(AssertionError):
        _op()._config(Stand(64, *shape, dtype=torch.int64), 12, None, None)


@pytest.mark.parametrize("shape,axes,stride", [((12,), 1, 0), ((1, 12), 1, 0), ((3, 12), 3, 12)], ids=str)
def test_positions_of_one_axis_and_of_several(shape, axes, stride):
    cfg = _op()._config(Stand(64, *shape, dtype=torch.int64), 12, None, None)
    assert (cfg.n_axes, cfg.position_stride, cfg.positions) == (axes, stride, 64)
