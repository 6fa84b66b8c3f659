"""Attention's and PagedAttention's checks and the structures they hand to the library, without a GPU: stand-ins have
what the holders ask of a tensor."""
import threading

import pytest

torch = pytest.importorskip("torch")

from paper_1910_00643_amd import attention as A  # noqa: E402

ON = torch.device("cuda:0")


class Stand:
    """A tensor of this shape at this address, as far as the holders look."""
    is_cuda = True

    def __init__(self, at, *shape, dtype=torch.float32, device=ON, strides=None):
        self.at, self.shape, self.dtype, self.device, self.strides = at, torch.Size(shape), dtype, device, strides

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def data_ptr(self):
        return self.at

    def is_contiguous(self):
        return self.strides is None

    def stride(self, i=None):
        st = [1]
        for n in reversed(self.shape[1:]):
            st.insert(0, st[0] * n)
        st = tuple(st) if self.strides is None else self.strides
        return st if i is None else st[i]

    def fill_(self, value):
        return self


I64, I32 = torch.int64, torch.int32


class Library:
    """Keeps what it is called with."""

    def __init__(self):
        self.seen, self.inside, self.done = {}, threading.Event(), threading.Event()

    def _note(self, *values):
        name = threading.current_thread().name
        if name == "first":
            self.inside.set()
            assert self.done.wait(20)
        self.seen[name] = values

    def slowmo_attention(self, cfg, batch, at, k_at, tokens, keys, q, k, v, out, lse, stream):
        self._note(batch, at, k_at, tokens, keys, *[r._obj.data for r in (q, k, v, out)], cfg.clear_rest)

    def slowmo_cache_append(self, cfg, pages, tokens, k, v, kc, vc, q, q_out, stream):
        p = pages._obj
        self._note(p.batch, p.columns, p.stride, p.pages, p.lengths, p.offsets, tokens,
                   *[None if r is None else r._obj.data for r in (k, v, kc, vc, q, q_out)])

    def slowmo_paged_attention_bytes(self, *args):
        return 0

    def slowmo_paged_attention(self, cfg, pages, tokens, q, kc, vc, out, lse, space, nbytes, stream):
        self._note(pages._obj.pages, tokens, q._obj.data, kc._obj.data, vc._obj.page_stride, out._obj.data, cfg.causal)


@pytest.fixture
def library(monkeypatch):
    L = Library()
    monkeypatch.setattr(A, "lib", lambda: L)
    monkeypatch.setattr(A, "_raw_stream", lambda device: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch, "empty", lambda shape, **kw: Stand(1 << 40, *shape, dtype=kw["dtype"]))
    return L


def _call(op, base, tokens=5, heads=4, keys=5, **kw):
    t = dict(q=Stand(base, tokens, heads, 16), k=Stand(base + 4096, keys, 2, 16), v=Stand(base + 8192, keys, 2, 16),
             offsets=Stand(base + 64, 3, dtype=I64), k_offsets=None, out=Stand(base + 12288, tokens, heads, 16))
    t.update(kw)
    return op.forward(**t)


def test_what_a_call_hands_over(library):
    _call(A.Attention(16, dtype="f32"), 1 << 20, k_offsets=Stand(72, 3, dtype=I64), keys=7)
    b = 1 << 20
    assert library.seen["MainThread"] == (2, b + 64, 72, 5, 7, b, b + 4096, b + 8192, b + 12288, 0)


@pytest.mark.parametrize("kw", [
    dict(q=Stand(64, 5, 4, 32)), dict(q=Stand(64, 5, 64)), dict(q=Stand(64, 5, 4, 16, dtype=torch.bfloat16)),
    dict(k=Stand(64, 5, 2, 16, device=torch.device("cuda:1"))), dict(v=Stand(64, 6, 2, 16)), dict(out=Stand(64, 5, 2, 16)),
    dict(q=Stand(64, 5, 4, 16, strides=(64, 1, 4))), dict(offsets=Stand(64, 3, dtype=I32)), dict(offsets=Stand(64, 0, dtype=I64)),
    dict(offsets=Stand(64, 3, 1, dtype=I64)), dict(offsets=Stand(64, 3, dtype=I64, strides=(2,))),
    dict(offsets=Stand(64, 3, dtype=I64, device=torch.device("cuda:1"))), dict(k_offsets=Stand(64, 4, dtype=I64)),
], ids=lambda kw: str(list(kw)))
def test_other_tensors_are_refused(library, kw):
    with pytest.raises(ValueError):
        _call(A.Attention(16, dtype="f32"), 1 << 20, **kw)
    assert not library.seen


def _append(op, base, tokens=3, **kw):
    t = dict(k=Stand(base, tokens, 2, 16), v=Stand(base + 4096, tokens, 1, 16), k_cache=Stand(base + 8192, 9, 4, 2, 16),
             v_cache=Stand(base + 16384, 9, 4, 1, 16), pages=Stand(base + 32, 2, 6, dtype=I32),
             lengths=Stand(base + 40, 2, dtype=I64), offsets=Stand(base + 48, 3, dtype=I64), q=Stand(base + 20480, tokens, 4, 16),
             q_out=Stand(base + 24576, tokens, 4, 16))
    t.update(kw)
    return op.append(**t)


def test_what_an_append_hands_over(library):
    b = 1 << 20
    _append(A.PagedAttention(16, dtype="f32"), b)
    assert library.seen["MainThread"] == (2, 6, 6, b + 32, b + 40, b + 48, 3, b, b + 4096, b + 8192, b + 16384, b + 20480, b + 24576)
    _append(A.PagedAttention(16, dtype="f32"), b, q=None, q_out=None)
    assert library.seen["MainThread"][-2:] == (None, None)


@pytest.mark.parametrize("kw", [
    dict(pages=Stand(64, 2, 6, dtype=I64)), dict(pages=Stand(64, 12, dtype=I32)), dict(pages=Stand(64, 2, 6, dtype=I32, strides=(1, 2))),
    dict(lengths=Stand(64, 3, dtype=I64)), dict(lengths=Stand(64, 2, dtype=I32)), dict(offsets=Stand(64, 2, dtype=I64)),
    dict(k_cache=Stand(64, 9, 4, 2, 8)), dict(k_cache=Stand(64, 36, 2, 16)), dict(v_cache=Stand(64, 9, 4, 1, 16, dtype=torch.bfloat16)),
    dict(v=Stand(64, 4, 1, 16)), dict(q=Stand(64, 4, 4, 16), q_out=Stand(128, 4, 4, 16)), dict(q=None), dict(q_out=Stand(64, 3, 2, 16)),
    dict(k_cache=Stand(64, 9, 4, 2, 16, strides=(128, 32, 1, 2))),
], ids=lambda kw: str(list(kw)))
def test_other_places_are_refused(library, kw):
    with pytest.raises(ValueError):
        _append(A.PagedAttention(16, dtype="f32"), 1 << 20, **kw)
    assert not library.seen


def test_tables_that_are_none_are_refused():
    for bad in (Stand(64, 5, 2, 8, dtype=torch.float64), Stand(64, 5, 3, 8), Stand(64, 5, 16), Stand(64, 5, 2, 8, strides=(32, 16, 2))):
        with pytest.raises(ValueError):
            A.PagedAttention(16, bad, dtype="f32")


@pytest.mark.parametrize("kw", [dict(window=0), dict(window=-3), dict(sinks=-1), dict(window=5, sinks=-1)], ids=str)
def test_windows_that_are_none_are_refused(kw):
    for kind in (A.Attention, A.PagedAttention):
        with pytest.raises(ValueError):
            kind(16, **kw)


def test_tensors_that_are_not_on_a_gpu_are_refused():
    x = torch.zeros(3, 1, 16)
    with pytest.raises(ValueError):
        A.Attention(16, dtype="f32").forward(x, x, x, torch.tensor([0, 3]))


def test_two_threads_on_one_handle(library):
    """The library lets another thread run while it is called: each call keeps its own addresses."""
    op, paged = A.Attention(16, dtype="f32"), A.PagedAttention(16, dtype="f32")
    first = threading.Thread(target=_call, args=(op, 1 << 20), name="first")
    first.start()
    assert library.inside.wait(20)
    second = threading.Thread(target=_call, args=(op, 2 << 20), kwargs=dict(tokens=7), name="second")
    second.start()
    second.join(20)
    library.done.set()
    first.join(20)
    for name, b, tokens in (("first", 1 << 20, 5), ("second", 2 << 20, 7)):
        assert library.seen[name] == (2, b + 64, None, tokens, 5, b, b + 4096, b + 8192, b + 12288, 0)
    assert paged._cfg.causal == 1


@pytest.mark.parametrize("many", [1 << 62, (1 << 63) - 1, 1 << 63, (1 << 64) + 1, 10 ** 30])
def test_windows_and_sinks_past_64_bits_are_past_every_length(many):
    for op in (A.Attention(64, window=many, sinks=many), A.PagedAttention(64, window=many, sinks=many)):
        for cfg in (op._cleared, op._kept if isinstance(op, A.Attention) else op._cfg):
            assert cfg.window >= 1 << 30 and cfg.sinks >= 1 << 30
