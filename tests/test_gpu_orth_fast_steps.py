"""A schedule of steps that take singular values from 1e-3..1 to 1 in six, whose quintics are steep at
the largest values that reach them.  Against 64 bits.  Tolerance: what the definition itself, in 64
bits, makes of a relative change of every element of X, of the size of 2^-18 for fp32 results (the pairs' 2^-22 and
fp32 sums of up to 2048 terms, 2^-24 * 45 = 2^-18.5) and 2^-9 for bf16 ones (three roundings of 2^-11 to a product
that share no sign), in front of every step; twice that, and the result's own rounding."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_orth import DEV, _P, _matrix  # noqa: E402
from test_orth_coefficients import SAFE  # noqa: E402


@pytest.fixture(autouse=True, scope="module")
def _memory_goes_back():
    """Later tests look at allocations of their own."""
    yield
    torch.cuda.empty_cache()


def _steps(u, change, seed=5):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = u.double()
    x = x / (torch.linalg.vector_norm(x) + 1e-7)
    if x.shape[0] > x.shape[1]:
        x = x.t().contiguous()
    for a, b, c in SAFE:
        x = x * (1 + change * (2 * torch.rand(x.shape, device=DEV, generator=g, dtype=torch.float64) - 1))
        s = x @ x.t().contiguous()
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.t() if u.shape[0] > u.shape[1] else x


@pytest.mark.parametrize("kind", ["gradient", "flat"])
@pytest.mark.parametrize("size", [(20, 30), (60, 100), (120, 90), (300, 1000), (700, 650)], ids=str)
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_fast_steps(out, size, kind):
    x = _matrix(*size, 3, kind)
    got = torch.full(size, float("nan"), device=DEV, dtype=torch.float32 if out == "f32" else torch.bfloat16)
    _P().Orthogonalizer([size], dtype="f32", out_dtype=out, steps=6, coefficients=SAFE).orthogonalize([x], [got])
    want = _steps(x, 0.0)
    change = 2.0 ** -18 if out == "f32" else 2.0 ** -9
    allowed = 2 * (_steps(x, change) - want).norm() + (2.0 ** -8 if out == "bf16" else 2.0 ** -23) * want.norm()
    assert (got.double() - want).norm() <= allowed, (float((got.double() - want).norm()), float(allowed))
