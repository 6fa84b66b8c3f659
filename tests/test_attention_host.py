"""The attention's C entry points without a GPU: every bad argument is refused before the device is touched, and the
library exports what the header declares."""
import ctypes as C
import os
import re

import pytest

import paper_1910_00643_amd as P
from paper_1910_00643_amd import attention as A
from paper_1910_00643_amd import binding as B
from paper_1910_00643_amd.operators import slowmo_heads

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ARG, ALIGN, NOMEM = B.SLOWMO_ERR_ARG, B.SLOWMO_ERR_ALIGN, B.SLOWMO_ERR_NOMEM


def test_header_and_binding_agree():
    header = open(os.path.join(ROOT, "include", "slowmo_attention.h")).read()
    code = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(slowmo_[a-z_]+)\s*\(", code))
    assert declared == set(A.EXPORTS)
    lib = C.CDLL(B.LIB_PATH)
    for name in declared:
        assert hasattr(lib, name), name
    assert C.sizeof(A.slowmo_attention_config) == 40 and C.sizeof(A.slowmo_cache) == 48
    assert C.sizeof(A.slowmo_pages) == 40 and C.sizeof(A.slowmo_append_config) == 40
    assert A._CACHES.size == 96 and A._PAGES.size == 40 and A._HEADS[8].size == 8 * 32


def _config(**kw):
    return A.slowmo_attention_config(**dict(dict(dtype=B.SLOWMO_BF16, head_dim=64, causal=1, clear_rest=0, scale=0.125, window=0,
                                                 sinks=0), **kw))


def _heads(data, heads=2, token=None, head=64):
    return slowmo_heads(data, heads, heads * 64 if token is None else token, head)


def _forward(cfg=None, batch=1, q_offsets=0x1000, k_offsets=None, tokens=4, keys=4, lse=0x8000, **kw):
    h = dict(dict(q=_heads(0x100000, 4), k=_heads(0x200000), v=_heads(0x300000), out=_heads(0x400000, 4)), **kw)
    return A.lib().slowmo_attention(_config() if cfg is None else cfg, batch, q_offsets, k_offsets, tokens, keys, h["q"], h["k"],
                                    h["v"], h["out"], lse, None)


BAD_CONFIGS = [dict(dtype=2), dict(dtype=-1), dict(head_dim=0), dict(head_dim=257), dict(causal=2), dict(clear_rest=-1),
               dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38),
               dict(window=-1), dict(sinks=-1)]


@pytest.mark.parametrize("kw", BAD_CONFIGS, ids=str)
def test_bad_configurations(kw):
    assert _forward(_config(**kw)) == ARG and P.slowmo_last_error(None)
    assert _paged(_config(**kw)) == ARG
    assert _backward(_config(**kw)) == ARG
    assert A.lib().slowmo_attention_backward_bytes(_config(**kw), 1, 4, 4, 4, 2) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), ARG), (dict(batch=(1 << 20) + 1), ARG), (dict(q_offsets=None), ARG), (dict(q_offsets=0x1004), ALIGN),
    (dict(k_offsets=0x1002), ALIGN), (dict(tokens=-1), ARG), (dict(tokens=(1 << 30) + 1, k_offsets=0x2000), ARG),
    (dict(keys=5), ARG),                                                 # as many keys as tokens without k_offsets
    (dict(lse=0x8002), ALIGN), (dict(lse=0x100010), ARG),
    (dict(q=_heads(None, 4)), ARG), (dict(q=_heads(0x100001, 4)), ALIGN), (dict(q=_heads(0x100000, 3)), ARG),
    (dict(q=_heads(0x100000, 0)), ARG), (dict(k=_heads(0x200000, 0)), ARG), (dict(v=_heads(0x300000, 4)), ARG),
    (dict(out=_heads(0x400000, 2)), ARG), (dict(out=_heads(0x100040, 4)), ARG), (dict(out=_heads(0x200000, 4)), ARG),
    (dict(out=_heads(0x400000, 4, head=63)), ARG), (dict(out=_heads(0x400000, 4, token=128)), ARG),
    (dict(out=_heads(0x400000, 4, token=0)), ARG), (dict(k=_heads(0x200000, token=-1)), ARG),
    (dict(k=_heads(0x200000, token=1 << 41)), ARG), (dict(q=_heads(0x100000, 2 * 4097), out=_heads(0x4000000, 2 * 4097)), ARG),
    (dict(q=None), ARG),
], ids=str)
def test_bad_calls(kw, status):
    assert _forward(**kw) == status
    assert P.slowmo_last_error(None)


def test_more_rows_than_2_36_are_refused():
    many = _heads(0x100000, 1 << 12, token=1 << 20, head=64)
    assert _forward(tokens=(1 << 24) + 1, keys=4, k_offsets=0x2000, q=many, out=_heads(0x40000000000000, 1 << 12, token=1 << 20),
                    k=_heads(0x200000, 1), v=_heads(0x300000, 1), lse=None) == ARG
    assert "2^36" in P.slowmo_last_error(None)


def test_nothing_to_do_is_no_error():
    none = _heads(None, 4)
    assert _forward(tokens=0, keys=0, q=none, out=none, k=_heads(None), v=_heads(None), lse=None) == B.SLOWMO_OK
    assert _forward(batch=0, tokens=0, keys=0, q=none, out=none, k=_heads(None), v=_heads(None), lse=None) == B.SLOWMO_OK


def test_side_by_side_arrays_do_not_overlap():
    """q, k and v in one projection's output, dq, dk and dv in one tensor, keys and values in one cache: refused
    would be what reaches past them."""
    at, token = 0x100000, 8 * 64
    q, k, v = (slowmo_heads(at + 2 * 64 * i, n, token, 64) for i, n in ((0, 4), (4, 2), (6, 2)))
    out = slowmo_heads(at + 2 * 64 * 6, 2, token, 64)
    assert _forward(q=q, k=k, v=v, out=_heads(0x400000, 4), tokens=0, keys=0) == B.SLOWMO_OK
    assert _forward(q=slowmo_heads(at, 2, token, 64), k=k, v=v, out=out) == ARG      # over v
    assert "overlap" in P.slowmo_last_error(None)


def _backward(cfg=None, batch=1, q_offsets=0x1000, k_offsets=None, tokens=4, keys=4, lse=0x8000, space=0x900000, nbytes=1 << 24,
              **kw):
    h = dict(g=_heads(0x100000, 4), q=_heads(0x200000, 4), k=_heads(0x300000), v=_heads(0x400000), out=_heads(0x500000, 4),
             dq=_heads(0x600000, 4), dk=_heads(0x700000), dv=_heads(0x800000))
    h.update(kw)
    return A.lib().slowmo_attention_backward(_config() if cfg is None else cfg, batch, q_offsets, k_offsets, tokens, keys, h["g"],
                                             h["q"], h["k"], h["v"], h["out"], lse, h["dq"], h["dk"], h["dv"], space, nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(nbytes=0), NOMEM), (dict(space=None), ARG), (dict(space=0x900008), ALIGN), (dict(lse=None), ARG),
    (dict(lse=0x8001), ALIGN), (dict(dq=_heads(0x200000, 4)), ARG), (dict(dk=_heads(0x300000)), ARG),
    (dict(dv=_heads(0x700000)), ARG), (dict(g=_heads(0x100000, 2)), ARG), (dict(dq=_heads(0x600000, 2)), ARG),
    (dict(dk=_heads(0x700000, 4)), ARG), (dict(out=_heads(0x500000, 2)), ARG), (dict(space=0x600000), ARG),
    (dict(dv=_heads(0x900000)), ARG), (dict(dk=_heads(0x700000, head=10)), ARG), (dict(q_offsets=None), ARG), (dict(batch=-1), ARG),
    (dict(lse=0x600000), ARG), (dict(dq=_heads(0x600002 - 1, 4)), ALIGN),
], ids=str)
def test_backward_refusals(kw, status):
    need = A.lib().slowmo_attention_backward_bytes(_config(), 1, 4, 4, 4, 2)
    assert 0 < need <= 1 << 24
    assert _backward(**kw) == status
    assert P.slowmo_last_error(None)


def _cache(data, heads=2, page=16, pages=8, page_stride=None, token=None, head=64):
    token = heads * 64 if token is None else token
    return A.slowmo_cache(data, heads, page, pages, page * token if page_stride is None else page_stride, token, head)


def _pages(batch=1, columns=4, stride=4, pages=0x1000, lengths=0x2000, offsets=0x3000):
    return A.slowmo_pages(batch, columns, stride, pages, lengths, offsets)


def _paged(cfg=None, pages=None, tokens=4, lse=None, space=0x9000000, nbytes=1 << 28, **kw):
    h = dict(q=_heads(0x100000, 4), out=_heads(0x200000, 4), k=_cache(0x300000), v=_cache(0x400000))
    h.update(kw)
    return A.lib().slowmo_paged_attention(_config() if cfg is None else cfg, _pages() if pages is None else pages, tokens, h["q"],
                                          h["k"], h["v"], h["out"], lse, space, nbytes, None)


BAD_PAGES = [(dict(batch=-1), ARG), (dict(batch=1 << 21), ARG), (dict(columns=-1), ARG), (dict(columns=(1 << 30) + 1, stride=1 << 31), ARG),
             (dict(stride=3), ARG), (dict(pages=None), ARG), (dict(lengths=None), ARG), (dict(offsets=None), ARG),
             (dict(pages=0x1002), ALIGN), (dict(lengths=0x2004), ALIGN), (dict(offsets=0x3004), ALIGN)]
BAD_CACHES = [(dict(heads=0), ARG), (dict(page=3), ARG), (dict(page=0), ARG), (dict(page=1 << 17), ARG), (dict(pages=-1), ARG),
              (dict(pages=1 << 31), ARG), (dict(data=None), ARG), (dict(data=0x300001), ALIGN), (dict(token=-1), ARG),
              (dict(page_stride=1 << 41), ARG)]


@pytest.mark.parametrize("kw,status", BAD_PAGES, ids=str)
def test_bad_pages(kw, status):
    assert _paged(pages=_pages(**kw)) == status
    assert _append(pages=_pages(**kw)) == status


@pytest.mark.parametrize("kw,status", BAD_CACHES, ids=str)
def test_bad_caches(kw, status):
    bad = _cache(**dict(dict(data=0x300000), **kw))
    assert _paged(k=bad) == status
    assert _append(k_cache=bad) == status


@pytest.mark.parametrize("kw,status", [
    (dict(v=_cache(0x400000, heads=1)), ARG), (dict(v=_cache(0x400000, page=32)), ARG), (dict(v=_cache(0x400000, pages=9)), ARG),
    (dict(q=_heads(0x100000, 3), out=_heads(0x200000, 3)), ARG), (dict(out=_heads(0x200000, 2)), ARG), (dict(out=_heads(0x100000, 4)), ARG),
    (dict(out=_heads(0x300000, 4)), ARG), (dict(lse=0x200010), ARG), (dict(lse=0x200001), ALIGN), (dict(tokens=-1), ARG),
], ids=str)
def test_paged_refusals(kw, status):
    assert _paged(**kw) == status
    assert P.slowmo_last_error(None)


def test_paged_workspace():
    long = _pages(columns=100000, stride=100000)
    need = A.lib().slowmo_paged_attention_bytes(_config(), long, 4, 4, _cache(0x300000))
    assert need > 0 and A.lib().slowmo_paged_attention_bytes(_config(), _pages(), 4, 4, _cache(0x300000)) == 0
    assert _paged(pages=long, nbytes=need - 1) == NOMEM
    assert _paged(pages=long, space=None) == ARG
    assert _paged(pages=long, space=0x9000008) == ALIGN
    assert _paged(pages=long, space=0x200000) == ARG                 # over out
    for bad in (dict(heads=0), dict(page=0)):
        assert A.lib().slowmo_paged_attention_bytes(_config(), long, 4, 4, _cache(0x300000, **bad)) == 0


def _append(cfg=None, pages=None, tokens=4, **kw):
    cfg = dict(dict(dtype=B.SLOWMO_BF16, head_dim=64, rotary_dim=64, interleaved=0, clear_rest=0, table=0x10000, table_rows=8),
               **(cfg or {}))
    h = dict(k=_heads(0x100000), v=_heads(0x200000), k_cache=_cache(0x300000), v_cache=_cache(0x400000), q=_heads(0x500000, 4),
             q_out=_heads(0x600000, 4))
    h.update(kw)
    return A.lib().slowmo_cache_append(A.slowmo_append_config(**cfg), _pages() if pages is None else pages, tokens, h["k"], h["v"],
                                       h["k_cache"], h["v_cache"], h["q"], h["q_out"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(cfg=dict(dtype=2)), ARG), (dict(cfg=dict(head_dim=0)), ARG), (dict(cfg=dict(head_dim=513)), ARG),
    (dict(cfg=dict(rotary_dim=66)), ARG), (dict(cfg=dict(rotary_dim=3)), ARG), (dict(cfg=dict(rotary_dim=-2)), ARG),
    (dict(cfg=dict(interleaved=2)), ARG), (dict(cfg=dict(clear_rest=2)), ARG), (dict(cfg=dict(table=None)), ARG),
    (dict(cfg=dict(table=0x10002)), ALIGN), (dict(cfg=dict(table_rows=-1)), ARG), (dict(q=None), ARG), (dict(q_out=None), ARG),
    (dict(q_out=_heads(0x600000, 2)), ARG), (dict(q_out=_heads(0x500040, 4)), ARG), (dict(q_out=_heads(0x100000, 4)), ARG),
    (dict(k=_heads(0x100000, 1)), ARG), (dict(v=_heads(0x200000, 1)), ARG), (dict(k=None), ARG),
    (dict(k_cache=_cache(0x100000)), ARG), (dict(v_cache=_cache(0x300000)), ARG), (dict(v_cache=_cache(0x400000, page=32)), ARG),
    (dict(k_cache=_cache(0x300000, token=64)), ARG), (dict(k_cache=_cache(0x300000, page_stride=128)), ARG),
    (dict(k_cache=_cache(0x600000)), ARG), (dict(tokens=-1), ARG), (dict(tokens=(1 << 30) + 1), ARG),
], ids=str)
def test_append_refusals(kw, status):
    assert _append(**kw) == status
    assert P.slowmo_last_error(None)


def test_append_of_nothing():
    assert _append(tokens=0) == B.SLOWMO_OK
    assert _append(pages=_pages(batch=0)) == B.SLOWMO_OK
    # keys and values beside each other in every row, and in every page, of one array
    for k, v in ((_cache(0x300000, token=256, page_stride=16 * 256), _cache(0x300000 + 256, token=256, page_stride=16 * 256)),
                 (_cache(0x300000, page_stride=2 * 16 * 128), _cache(0x300000 + 16 * 256, page_stride=2 * 16 * 128))):
        assert _append(k_cache=k, v_cache=v, pages=_pages(batch=0)) == B.SLOWMO_OK


def test_outputs_beside_inputs_in_one_array_pass():
    """Rows of q, k, v and out in turn.  What is refused is the lse, which lies in out's last row, behind the inputs, and is
    looked at after them."""
    at, token, tokens = 0x100000, 10 * 64, 100
    q, k, v, out = (slowmo_heads(at + 2 * 64 * i, n, token, 64) for i, n in ((0, 4), (4, 1), (5, 1), (6, 4)))
    lse = at + 2 * (token * (tokens - 1) + 6 * 64)
    assert _forward(q=q, k=k, v=v, out=out, tokens=tokens, keys=tokens, lse=lse) == ARG
    assert P.slowmo_last_error(None) == "out and lse overlap"
    # one element nearer, out reaches into v
    assert _forward(q=q, k=k, v=v, out=slowmo_heads(out.data - 2, 4, token, 64), tokens=tokens, keys=tokens, lse=None) == ARG
    assert P.slowmo_last_error(None) == "an output overlaps an input"
    # rows of another length are not beside them
    assert _forward(q=q, k=k, v=v, out=slowmo_heads(out.data, 4, token + 64, 64), tokens=tokens, keys=tokens, lse=None) == ARG
    assert P.slowmo_last_error(None) == "an output overlaps an input"
