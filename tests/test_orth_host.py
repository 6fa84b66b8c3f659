"""The orthogonalising call's C entry points without a GPU: bad arguments are
refused before the device is touched."""
import ctypes as C

import pytest

import paper_1910_00643_amd as P
from paper_1910_00643_amd import binding as B
from paper_1910_00643_amd import operators as O


def _i64(*v):
    return (C.c_int64 * len(v))(*v)


def _config(**kw):
    base = dict(in_dtype=B.SLOWMO_BF16, out_dtype=B.SLOWMO_BF16, steps=5, scale=0, eps=1e-7)
    base.update(kw)
    return O.slowmo_orth_config(**base)


def _bytes(cfg, rows=(64, 300), cols=(132, 70), ld=None, n=None):
    return O.lib().slowmo_orth_bytes(cfg, len(rows) if n is None else n, _i64(*rows), _i64(*cols),
                                     _i64(*ld) if ld else None)


def test_bytes_grow_with_the_list_and_with_paired_halves():
    one, two = _bytes(_config(), (64,), (132,)), _bytes(_config())
    assert 0 < one < two < _bytes(_config(out_dtype=B.SLOWMO_F32))
    assert _bytes(_config(), (0,), (5,)) > 0
    assert C.sizeof(O.slowmo_orth_config) == 32


@pytest.mark.parametrize("kw", [dict(in_dtype=2), dict(out_dtype=-1), dict(steps=0), dict(steps=17),
                                dict(scale=3), dict(eps=-1.0), dict(eps=float("nan"))])
def test_bad_configurations(kw):
    assert _bytes(_config(**kw)) == 0 and P.slowmo_last_error(None)


def test_bad_lists():
    assert _bytes(_config(), (-1,), (4,)) == 0
    assert _bytes(_config(), (65537,), (4,)) == 0
    assert _bytes(_config(), (4,), (8,), (7,)) == 0
    assert _bytes(_config(), n=0) == 0
    assert O.lib().slowmo_orth_bytes(None, 1, _i64(1), _i64(1), None) == 0
    assert O.lib().slowmo_orth_bytes(_config(), 1, None, _i64(1), None) == 0
    bad = (C.c_float * 15)(*([1.0] * 14 + [float("inf")]))
    assert _bytes(_config(coefficients=bad)) == 0


def test_create_refuses_before_the_device_is_used():
    cfg, rows, cols = _config(), _i64(64), _i64(32)
    need = O.lib().slowmo_orth_bytes(cfg, 1, rows, cols, None)
    h = C.c_void_p()

    def create(space, nbytes, out=h):
        return O.lib().slowmo_orth_create(C.byref(out) if out is not None else None, cfg, 1, rows, cols, None,
                                          space, nbytes, None)

    assert create(None, need) == B.SLOWMO_ERR_ARG
    assert create(0x1010, need) == B.SLOWMO_ERR_ALIGN
    assert create(0x10000, need - 1) == B.SLOWMO_ERR_NOMEM
    assert create(0x10000, need, None) == B.SLOWMO_ERR_ARG
    assert not h.value


def test_null_handles():
    L = O.lib()
    assert L.slowmo_orthogonalize(None, None, None, None) == B.SLOWMO_ERR_ARG
    assert L.slowmo_momentum_orthogonalize(None, None, None, None, 0.9, 1, None) == B.SLOWMO_ERR_ARG
    assert L.slowmo_orth_destroy(None) == B.SLOWMO_OK


def test_coefficients_that_let_singular_values_grow_are_refused():
    """X is held as halves times 2^13: its elements have to stay below 8."""
    three = lambda *abc: (C.c_float * 15)(*(abc * 5))  # noqa: E731
    assert _bytes(_config(coefficients=three(3.4445, -4.7750, 2.0315))) > 0
    assert _bytes(_config(coefficients=three(1.5, -0.5, 0.0))) > 0
    assert _bytes(_config(coefficients=three(2.0, 0.0, 0.0))) == 0        # 2^5 times as large
    assert "grow" in P.slowmo_last_error(None)
    assert _bytes(_config(coefficients=three(1.0, 1.0, 1.0))) == 0
    assert _bytes(_config(coefficients=three(-3e38, 3e38, 3e38))) == 0
    h = C.c_void_p()
    assert O.lib().slowmo_orth_create(C.byref(h), _config(coefficients=three(2.0, 0.0, 0.0)), 1, _i64(64), _i64(32),
                                      None, 0x10000, 1 << 30, None) == B.SLOWMO_ERR_ARG
    assert not h.value
