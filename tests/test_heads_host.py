"""The heads' C entry points without a GPU: every bad argument is refused before
the device is touched, and the library exports what the header declares."""
import ctypes as C
import os
import re

import pytest

import paper_1910_00643_amd as P
from paper_1910_00643_amd import binding as B
from paper_1910_00643_amd import operators as O

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_header_and_binding_agree():
    header = open(os.path.join(ROOT, "include", "slowmo_operators.h")).read()
    code = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(slowmo_[a-z_]+)\s*\(", code))
    assert declared == set(O.EXPORTS)
    lib = C.CDLL(B.LIB_PATH)
    for name in declared:
        assert hasattr(lib, name), name
    assert C.sizeof(O.slowmo_head_config) == 88 and C.sizeof(O.slowmo_heads) == 32


def _config(**kw):
    base = dict(dtype=B.SLOWMO_BF16, head_dim=64, rotary_dim=64, interleaved=0, norm=1, eps=1e-6, n_axes=1,
                table=0x10000, table_rows=8, positions=0x20000)
    base.update(kw)
    return O.slowmo_head_config(**base)


def _heads(data, heads=2, token=None, head=64):
    return O.slowmo_heads(data, heads, heads * 64 if token is None else token, head)


GOOD = dict(q=_heads(0x100000), k=_heads(0x200000), q_out=_heads(0x300000), k_out=_heads(0x400000))


def _forward(cfg, tokens=4, slots=None, rows=0, **kw):
    h = dict(GOOD, **kw)
    return O.lib().slowmo_head_norm_rotary(cfg, tokens, h["q"], h["k"], h["q_out"], h["k_out"], slots, rows,
                                           None)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(head_dim=0), dict(head_dim=513), dict(rotary_dim=66),
                                dict(rotary_dim=3), dict(rotary_dim=-2), dict(interleaved=2), dict(norm=-1),
                                dict(eps=float("nan")), dict(eps=-1.0), dict(n_axes=0), dict(n_axes=5),
                                dict(table=None), dict(positions=None), dict(table_rows=-1),
                                dict(n_axes=2, position_stride=3)])
def test_bad_configurations(kw):
    assert _forward(_config(**kw)) == B.SLOWMO_ERR_ARG
    assert P.slowmo_last_error(None)


def test_bad_pair_axis():
    axis = (C.c_uint8 * 32)(*([0] * 31 + [1]))
    assert _forward(_config(pair_axis=C.addressof(axis))) == B.SLOWMO_ERR_ARG
    assert "axis" in P.slowmo_last_error(None)


@pytest.mark.parametrize("kw,status", [
    (dict(q=_heads(None)), B.SLOWMO_ERR_ARG),
    (dict(q=_heads(0x100001)), B.SLOWMO_ERR_ALIGN),
    (dict(q=_heads(0x100000, heads=3)), B.SLOWMO_ERR_ARG),
    (dict(k=_heads(0x200000, heads=-1)), B.SLOWMO_ERR_ARG),
    (dict(k=_heads(0x200000, token=-1)), B.SLOWMO_ERR_ARG),
    (dict(q_out=_heads(0x300000, head=63)), B.SLOWMO_ERR_ARG),        # heads run into one another
    (dict(q_out=_heads(0x300000, token=0)), B.SLOWMO_ERR_ARG),
    (dict(q_out=_heads(0x300000, token=96)), B.SLOWMO_ERR_ARG),
    (dict(q_out=_heads(0x400040)), B.SLOWMO_ERR_ARG),                 # over k_out
    (dict(k_out=_heads(0x100000)), B.SLOWMO_ERR_ARG),                 # over the other input
    (dict(q_out=_heads(0x100002)), B.SLOWMO_ERR_ARG),                 # over q, but not q
])
def test_bad_arrays(kw, status):
    assert _forward(_config(), **kw) == status
    assert P.slowmo_last_error(None)


def test_slots_and_weights():
    assert _forward(_config(), slots=0x1004, rows=9) == B.SLOWMO_ERR_ALIGN
    assert _forward(_config(), slots=0x1000, rows=-1) == B.SLOWMO_ERR_ARG
    assert _forward(_config(), slots=0x1000, rows=9, k_out=_heads(0x200000)) == B.SLOWMO_ERR_ARG
    assert _forward(_config(q_weight=0x1002)) == B.SLOWMO_ERR_ALIGN
    assert _forward(_config(), tokens=-1) == B.SLOWMO_ERR_ARG
    assert O.lib().slowmo_head_norm_rotary(None, 1, None, None, None, None, None, 0, None) == B.SLOWMO_ERR_ARG


def test_nothing_to_do_is_no_error():
    assert _forward(_config(), tokens=0) == B.SLOWMO_OK


def _backward(cfg, tokens=4, space=0x900000, nbytes=1 << 24, dwq=0x800000, **kw):
    h = dict(gq=_heads(0x100000), gk=_heads(0x200000), q=_heads(0x300000), k=_heads(0x400000),
             dq=_heads(0x500000), dk=_heads(0x600000))
    h.update(kw)
    return O.lib().slowmo_head_norm_rotary_backward(cfg, tokens, h["gq"], h["gk"], h["q"], h["k"], h["dq"],
                                                    h["dk"], dwq, None, space, nbytes, None)


def test_backward_refusals():
    need = O.lib().slowmo_head_backward_bytes(_config(), 4, 2, 2)
    assert need > 0 and O.lib().slowmo_head_backward_bytes(_config(norm=0), 4, 2, 2) == 0
    assert _backward(_config(), nbytes=0) == B.SLOWMO_ERR_NOMEM
    assert _backward(_config(), space=None) == B.SLOWMO_ERR_ARG
    assert _backward(_config(), space=0x900008) == B.SLOWMO_ERR_ALIGN
    assert _backward(_config(norm=0)) == B.SLOWMO_ERR_ARG
    assert _backward(_config(), dq=_heads(0x300000)) == B.SLOWMO_ERR_ARG       # over q
    assert _backward(_config(), dq=_heads(0x600000)) == B.SLOWMO_ERR_ARG       # over dk
    assert _backward(_config(), dk=_heads(0x100000)) == B.SLOWMO_ERR_ARG       # over the other gradient
    assert _backward(_config(), gq=_heads(0x100000, heads=1)) == B.SLOWMO_ERR_ARG
    assert _backward(_config(), dwq=0x800002) == B.SLOWMO_ERR_ALIGN
