"""Which coefficients the orthogonalising call takes, on both sides of its bound, without a GPU: a
singular value of 0..1 may come to 7.5, with 1/1024 of |a| s + |b| s^3 + |c| s^5 a step for rounding."""
import ctypes as C

import pytest

import paper_1910_00643_amd as P
from paper_1910_00643_amd import binding as B
from paper_1910_00643_amd import operators as O

# quintics that are each the best approximation of 1 on what the one before leaves of 1e-3..1
FAST = [(8.4703, -25.1081, 18.6293), (4.1832, -3.1091, 0.5807), (3.9623, -2.9537, 0.5627), (3.2912, -2.4691, 0.5082),
        (2.2767, -1.6464, 0.4159), (1.8890, -1.2654, 0.3765)]
SAFE = [(a / 1.01, b / 1.01 ** 3, c / 1.01 ** 5) for a, b, c in FAST]
DEFAULT = (3.4445, -4.7750, 2.0315)


def _taken(triples, out):
    flat = [v for t in triples for v in t]
    cfg = O.slowmo_orth_config(in_dtype=B.SLOWMO_F32, out_dtype=out, steps=len(triples), scale=0, eps=1e-7,
                               coefficients=(C.c_float * len(flat))(*flat))
    one = (C.c_int64 * 1)(300)
    return O.lib().slowmo_orth_bytes(cfg, 1, one, one, None) > 0


@pytest.mark.parametrize("out", [B.SLOWMO_F32, B.SLOWMO_BF16])
@pytest.mark.parametrize("triples,taken", [
    ([(7.48, 0, 0)], True), ([(7.51, 0, 0)], False), ([(7.74, 0, 0)], False),
    ([(-7.48, 0, 0)], True), ([(-7.51, 0, 0)], False),
    ([(1, 0, 0)] * 15 + [(6, 0, 0)], True),            # 6 and the rounding of 16 steps: 6.1
    ([(1, 0, 0)] * 15 + [(7.3, 0, 0)], True), ([(1, 0, 0)] * 15 + [(7.45, 0, 0)], False),
    ([(2, 0, 0), (3.7, 0, 0)], True), ([(2, 0, 0), (3.8, 0, 0)], False),
    ([(0, 0, 7.4)], True), ([(0, 0, 7.6)], False),
    ([(25, -30, 0)], False),                           # 8.8 at 0.53, though -5 at 1
    ([(20, -30, 0), (1, 0, 0)], False),                # 10 at 1 with the other sign
    ([DEFAULT] * 5, True), ([DEFAULT] * 16, True), ([(1.5, -0.5, 0)] * 16, True), ([(1.875, -1.25, 0.375)] * 16, True),
    (SAFE, True), (SAFE[:3], True), (FAST, False),
    ([(3e38, -3e38, 3e38)] * 16, False), ([(0, 0, 0)] * 16, True),
], ids=lambda v: str(v)[:40])
def test_both_sides_of_the_bound(triples, taken, out):
    assert _taken(triples, out) == taken
    if not taken:
        assert "7.5" in P.slowmo_last_error(None)
