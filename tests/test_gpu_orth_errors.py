"""How far orthogonalised updates are from 64 bits, as close as the arithmetic lets it be said, and the
same matrix by itself and in a list that sends it another way.

Tolerances, on the Frobenius norm.  bf16 results: the roundings that the kernels' comment names -- X, A and P to
halves times powers of two, X's next 11 bits kept for a X, a on P's diagonal in the last two steps -- are done
to the definition in 64 bits, and what they make of this very matrix is allowed 1.25 times (it is the mean of n k
roundings, but singular values near each other may share them), beside the result's own rounding, which is known.
fp32 results: a rounding to p bits is 2^-p * 0.41 of a value (2^-p / sqrt(3), and 1 / sqrt(2) for where its
mantissa lies).  Near 1, A's rounding enters b + 2 c A = -0.7 times, P's and that of the factor X |b + c| = 2.7 times
each, sqrt(0.7^2 + 2 * 2.7^2) = 3.9; the step after multiplies by a + 3 b + 5 c = -0.7, so that all steps have
1.45 of one's, and sqrt(2) is left for singular values elsewhere: 8 roundings of p = 22, with the product of the lower
halves left out (2^-24) and fp32 sums of 3 k / 16 terms with a rounding each, 2^-24 * 0.41 * sqrt(3 k / 16)."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_orth import ABC, DEV, _P, _exact, _matrix  # noqa: E402

T = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True, scope="module")
def _memory_goes_back():
    """Later tests look at allocations of their own."""
    yield
    torch.cuda.empty_cache()


def _in_halves(u):
    a, b, c = ABC
    one = 2.0 ** 13
    x = u.double() / (torch.linalg.vector_norm(u.double()) + 1e-7)
    x = (x.t().contiguous() if u.shape[0] > u.shape[1] else x) * one
    for step in range(5):
        hi = x.half().double()
        both = hi + (x - hi).half().double()
        gram = (hi @ hi.t().contiguous() / one).half().double() / one
        p = b * gram + c * (gram @ gram)
        if step < 3:
            x = a * both + (p * one).half().double() / one @ hi
        else:
            p.diagonal().add_(a)
            x = (p * one).half().double() / one @ hi
    x = x / one
    return x.t() if u.shape[0] > u.shape[1] else x


def _allowed(u, want, out):
    if out == "bf16":
        own = float((want.bfloat16().double() - want).norm())
        return math.hypot(own, 1.25 * float((_in_halves(u) - want).norm()))
    sums = 2.0 ** -24 * 0.41 * math.sqrt(3 * max(want.shape) / 16)
    return 8 * (2.0 ** -22 * 0.41 + 2.0 ** -24 + sums) * float(want.norm())


def _run(sizes, x, out):
    got = [torch.full(s, float("nan"), device=DEV, dtype=T[out]) for s in sizes]
    _P().Orthogonalizer(sizes, dtype="f32", out_dtype=out).orthogonalize(x, got)
    return got


@pytest.mark.parametrize("kind", ["gradient", "flat"])
@pytest.mark.parametrize("size", [(60, 100), (128, 96), (250, 120), (300, 1000), (512, 2048), (700, 700), (2048, 8192)], ids=str)
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_distance_from_64_bits(out, size, kind):
    x = _matrix(*size, 6, kind)
    want = _exact(x)
    err = float((_run([size], [x], out)[0].double() - want).norm())
    assert err <= _allowed(x, want, out), (err / float(want.norm()), _allowed(x, want, out) / float(want.norm()))


@pytest.mark.parametrize("size", [(64, 64), (100, 128), (130, 100), (100, 2000), (1100, 1024)], ids=str)
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_alone_and_beside_others(size, out):
    """64 x 64 and, for bf16 results, 100 x 128 by one workgroup alone and in tiles beside a longer matrix; the
    others with their sums cut in other places."""
    sizes = [(700, 900), size, (300, 1300)]
    x = [_matrix(*s, 6 + i) for i, s in enumerate(sizes)]
    alone, beside = _run([size], [x[1]], out)[0], _run(sizes, x, out)[1]
    want = _exact(x[1])
    for v in (alone, beside):
        assert float((v.double() - want).norm()) <= _allowed(x[1], want, out)
    assert float((alone.double() - beside.double()).norm()) <= 2 * _allowed(x[1], want, out)
