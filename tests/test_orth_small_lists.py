"""Small matrices beside tiny ones of any length go by one workgroup each: the workspace holds no X for
the launches of products.  Without a GPU, but for the values."""
import ctypes as C

import pytest

from paper_1910_00643_amd import binding as B
from paper_1910_00643_amd import operators as O

LONG = [[(64, 64), (3, 300)], [(1, 1000), (64, 64)], [(40, 64), (17, 604), (60, 33), (900, 2)]]


def _bytes(sizes, out):
    cfg = O.slowmo_orth_config(in_dtype=B.SLOWMO_F32, out_dtype=out, steps=5, scale=0, eps=1e-7)
    rows, cols = ((C.c_int64 * len(sizes))(*v) for v in zip(*sizes))
    return O.lib().slowmo_orth_bytes(cfg, len(sizes), rows, cols, None)


@pytest.mark.parametrize("out", [B.SLOWMO_F32, B.SLOWMO_BF16])
@pytest.mark.parametrize("sizes", LONG, ids=str)
def test_a_long_tiny_matrix_leaves_small_ones_small(sizes, out):
    one = _bytes([(64, 64)], out)
    assert one <= _bytes(sizes, out) < one + 2048
    assert _bytes([(64, 64), (33, 300)], out) > 100000     # a longer one that is not tiny does not


@pytest.mark.gpu
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", LONG, ids=str)
def test_their_values(sizes, out):
    torch = pytest.importorskip("torch")
    from test_gpu_orth import DEV, _P, _exact, _matrix, _near
    x = [_matrix(*s, 3 + i) for i, s in enumerate(sizes)]
    got = [torch.full(s, float("nan"), device=DEV, dtype=torch.float32 if out == "f32" else torch.bfloat16) for s in sizes]
    _P().Orthogonalizer(sizes, dtype="f32", out_dtype=out).orthogonalize(x, got)
    for v, w in zip(x, got):
        _near(w, _exact(v), out)
