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


def test_two_threads_on_one_handle(monkeypatch):
    """The library lets another thread run while it is called: each call keeps its own addresses."""
    seen, inside, done = {}, threading.Event(), threading.Event()

    class Library:
        def slowmo_head_norm_rotary(self, cfg, tokens, q, k, q_out, k_out, slots, rows, stream):
            if threading.current_thread().name == "first":
                inside.set()
                assert done.wait(20)
            seen[threading.current_thread().name] = (cfg.positions, tokens, *[r._obj.data for r in (q, k, q_out, k_out)])
            return 0

    monkeypatch.setattr(O, "lib", Library)
    monkeypatch.setattr(O, "_raw_stream", lambda device: 0)
    op = _op()

    def call(base, tokens):
        q, k, yq, yk = (Stand(base + 4096 * i, tokens, 2, 16) for i in range(4))
        op.forward(q, k, Stand(base + 64, tokens, dtype=torch.int64), q_out=yq, k_out=yk)

    first = threading.Thread(target=call, args=(1 << 20, 5), name="first")
    first.start()
    assert inside.wait(20)
    second = threading.Thread(target=call, args=(2 << 20, 7), name="second")
    second.start()
    second.join(20)
    done.set()
    first.join(20)
    for name, base, tokens in (("first", 1 << 20, 5), ("second", 2 << 20, 7)):
        assert seen[name] == (base + 64, tokens, *[base + 4096 * i for i in range(4)])


@pytest.mark.parametrize("axis", [256, 4, -1, -256])
def test_axes_that_are_none_are_refused(axis):
    """256 went into 8 bits as axis 0."""
    table = Stand(1 << 12, 5, 2, 2)
    O.HeadNormRotary(16, table, pair_axis=[0, 3])
    with pytest.raises(AssertionError):
        O.HeadNormRotary(16, table, pair_axis=[0, axis])
