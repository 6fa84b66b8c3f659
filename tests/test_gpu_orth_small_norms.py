"""Orthogonalised updates of matrices whose norm is far below eps: X_0 = U / (|U| + eps) is
small then, and the steps multiply it by a until it is not.  Against 64 bits, with the tolerances of
test_gpu_orth.py: while X is small a step is a X, so that relative errors only add up."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_orth import DEV, _P, _exact, _matrix, _near  # noqa: E402

T = {"f32": torch.float32, "bf16": torch.bfloat16}
TYPES = [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")]
# 64 bits throughout; one workgroup each; tiles, without and with the first two steps as one
LISTS = {"tiny": [(20, 30), (5, 700)], "small": [(60, 100), (100, 64)], "tiles": [(700, 700), (130, 128)],
         "pairs": [(300, 1000), (2000, 140)]}


@pytest.fixture(autouse=True, scope="module")
def _memory_goes_back():
    """Later tests look at allocations of their own."""
    yield
    torch.cuda.empty_cache()


def _of_norm(size, seed, norm, dtype):
    x = _matrix(*size, seed, "flat").double()
    return (x * (norm / x.norm())).to(dtype)


@pytest.mark.parametrize("ratio", [0.3, 1e-2, 1e-4, 1e-8, 1e-20])
@pytest.mark.parametrize("types", TYPES, ids=str)
@pytest.mark.parametrize("which", sorted(LISTS))
def test_norms_below_eps(which, types, ratio):
    P = _P()
    din, dout = types
    sizes = LISTS[which]
    x = [_of_norm(s, 3 + i, ratio * 1e-7, T[din]) for i, s in enumerate(sizes)]
    out = [torch.full(s, float("nan"), device=DEV, dtype=T[dout]) for s in sizes]
    o = P.Orthogonalizer(sizes, dtype=din, out_dtype=dout, scale="rms")
    o.orthogonalize(x, out)
    eps = float(torch.tensor(1e-7))
    for v, w, s in zip(x, out, sizes):
        _near(w, _exact(v, eps=eps) * 0.2 * max(s) ** 0.5, dout)


@pytest.mark.parametrize("which", sorted(LISTS))
@pytest.mark.parametrize("steps", [1, 2, 12])
@pytest.mark.parametrize("types", [("bf16", "bf16"), ("f32", "f32")], ids=str)
def test_few_and_many_steps(types, steps, which):
    """12 steps of a = 1.875 bring a norm of 1e-3 eps to 1.9 or near it, through every size in between."""
    P = _P()
    din, dout = types
    sizes, abc = LISTS[which], (1.875, -1.25, 0.375)
    x = [_of_norm(s, 3 + i, 1e-3, T[din]) for i, s in enumerate(sizes)]
    out = [torch.full(s, float("nan"), device=DEV, dtype=T[dout]) for s in sizes]
    P.Orthogonalizer(sizes, dtype=din, out_dtype=dout, steps=steps, eps=1.0, coefficients=abc).orthogonalize(x, out)
    for v, w in zip(x, out):
        _near(w, _exact(v, steps, eps=1.0, coefficients=abc), dout)


@pytest.mark.parametrize("which", sorted(LISTS))
def test_one_list_of_many_norms(which):
    """Each matrix has its own; zeros and NaN among them stay where they are."""
    P = _P()
    sizes = [s for s in LISTS[which] for _ in range(4)]
    x = [_of_norm(s, i, 10.0 ** -(3 * i), torch.float32) for i, s in enumerate(sizes)]
    x[1].zero_()
    x[6][0, 0] = float("nan")
    out = [torch.empty(s, device=DEV) for s in sizes]
    P.Orthogonalizer(sizes, dtype="f32", eps=1e-2).orthogonalize(x, out)
    eps = float(torch.tensor(1e-2))
    for i, (v, w) in enumerate(zip(x, out)):
        if i == 1:
            assert (w == 0).all()
        elif i == 6:
            assert w.isnan().all()
        else:
            _near(w, _exact(v, eps=eps), "f32")


def test_momentum_below_eps():
    P = _P()
    sizes = [(300, 200), (40, 90)]
    o = P.Orthogonalizer(sizes, dtype="f32")
    g = [_of_norm(s, 3, 1e-13, torch.float32) for s in sizes]
    m = [torch.zeros(s, device=DEV) for s in sizes]
    out = [torch.empty(s, device=DEV) for s in sizes]
    o.momentum_orthogonalize(g, m, out, 0.5)
    for v, w in zip(g, out):
        _near(w, _exact(1.5 * v.double(), eps=float(torch.tensor(1e-7))), "f32")
