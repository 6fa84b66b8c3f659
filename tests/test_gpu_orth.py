"""Orthogonalised updates against the definition in 64 bits.

Tolerances, on the Frobenius norm of the difference over that of the result.  bf16
results: the result's own rounding is at most 2^-9 of every element.  The products are
formed of halves (a rounding is at most 2^-12 of an element, 2^-12 / sqrt(3) in the mean):
per step A, P and the factor X are rounded, and what a step adds is multiplied by at most
a = 3.45 in each later one; X itself, where it enters linearly, is kept to 2^-23.  The early
steps' roundings enter through b A + c A A, which is small while the singular values are, so
that of 3 roundings a step times 3.45^(4-j) about 20 are left: 2^-9 + 20 * 2^-12 = 6.9e-3.
fp32 results: the same with pairs of halves, 2^-22 (the product of the two lower halves is left
out: one more) and fp32 sums over up to k terms, 2^-24 sqrt(k) each: 40 * 2^-22 + 20 * 2^-24 sqrt(k).
One element may be off by 12 times the mean error allowed."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DEV = "cuda:0"
ABC = (3.4445, -4.7750, 2.0315)


def _P():
    import paper_1910_00643_amd as P
    return P


def _exact(u, steps=5, eps=1e-7, coefficients=ABC):
    triples = [coefficients] * steps if not isinstance(coefficients[0], tuple) else coefficients
    x = u.double()
    x = x / (torch.linalg.vector_norm(x) + eps)
    if x.shape[0] > x.shape[1]:
        x = x.t().contiguous()
    for a, b, c in triples:
        g = x @ x.t().contiguous()
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.t() if u.shape[0] > u.shape[1] else x


def _near(got, want, out):
    k = max(want.shape)
    tol = 2.0 ** -9 + 20 * 2.0 ** -12 if out == "bf16" else 40 * 2.0 ** -22 + 20 * 2.0 ** -24 * math.sqrt(k)
    norm = want.norm()
    err = got.double() - want
    assert err.norm() <= tol * norm, float(err.norm() / norm)
    assert err.abs().max() <= 12 * tol * norm / math.sqrt(want.numel()) + 2.0 ** -8 * want.abs().max() * (out == "bf16")


def _matrix(rows, cols, seed, kind="gradient"):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = torch.randn(rows, cols, device=DEV, generator=g)
    if kind == "flat":
        return n
    r = max(1, min(rows, cols) // 8)
    low = torch.randn(rows, r, device=DEV, generator=g) @ torch.randn(r, cols, device=DEV, generator=g) / r ** 0.5
    return 1e-3 * (low + 0.2 * n) if kind == "gradient" else low


SIZES = [(1, 1), (1, 7), (9, 1), (2, 3), (33, 20), (64, 64), (64, 147), (127, 129), (128, 128), (129, 64),
         (300, 1000), (1000, 300), (511, 513), (700, 700), (257, 4100), (4100, 130)]


@pytest.mark.parametrize("kind", ["gradient", "flat", "deficient"])
@pytest.mark.parametrize("types", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")], ids=str)
def test_one_list_of_many_sizes(types, kind):
    P = _P()
    din, dout = types
    t = {"f32": torch.float32, "bf16": torch.bfloat16}
    x = [_matrix(r, c, 10 + i, kind).to(t[din]) for i, (r, c) in enumerate(SIZES)]
    out = [torch.full(s, float("nan"), device=DEV, dtype=t[dout]) for s in SIZES]
    o = P.Orthogonalizer(SIZES, dtype=din, out_dtype=dout)
    keep = [v.clone() for v in x]
    o.orthogonalize(x, out)
    for v, w, k in zip(x, out, keep):
        assert torch.equal(v, k)
        _near(w, _exact(v), dout)
    again = [torch.empty_like(v) for v in out]
    o.orthogonalize(x, again)                     # the same bits each time
    assert all(torch.equal(a, b) for a, b in zip(out, again))


@pytest.mark.parametrize("size", [(64, 64), (130, 100), (100, 2000), (1100, 1024)], ids=str)
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_alone_and_in_a_list_give_the_same_values(size, out):
    P = _P()
    x = _matrix(*size, 3)
    alone = torch.empty(size, device=DEV, dtype=torch.float32 if out == "f32" else torch.bfloat16)
    P.Orthogonalizer([size], dtype="f32", out_dtype=out).orthogonalize([x], [alone])
    _near(alone, _exact(x), out)


@pytest.mark.parametrize("scale,factor", [("none", lambda r, c: 1.0), ("shape", lambda r, c: max(1, r / c) ** 0.5),
                                          ("rms", lambda r, c: 0.2 * max(r, c) ** 0.5)])
def test_scales_steps_and_coefficients(scale, factor):
    P = _P()
    cubic = [(1.5, -0.5, 0.0)] * 3 + [(1.875, -1.25, 0.375)] * 4
    for size in ((40, 70), (300, 128)):
        x = _matrix(*size, 4, "flat")
        got = torch.empty(size, device=DEV)
        P.Orthogonalizer([size], dtype="f32", scale=scale, steps=7, coefficients=cubic).orthogonalize([x], [got])
        _near(got, _exact(x, 7, coefficients=cubic) * factor(*size), "f32")
        P.Orthogonalizer([size], dtype="f32", scale=scale, steps=1, eps=3.0).orthogonalize([x], [got])
        _near(got, _exact(x, 1, eps=3.0) * factor(*size), "f32")


def test_results_are_nearly_orthogonal():
    """With convergent coefficients the rows of the result are orthonormal."""
    P = _P()
    x = _matrix(96, 200, 4, "flat")
    got = torch.empty_like(x)
    P.Orthogonalizer([(96, 200)], dtype="f32", steps=14, coefficients=(1.875, -1.25, 0.375)).orthogonalize([x], [got])
    gram = got.double() @ got.double().t()
    assert (gram - torch.eye(96, device=DEV, dtype=torch.float64)).abs().max() < 1e-4


def test_stacks_row_strides_and_in_place():
    P = _P()
    g = torch.Generator(device=DEV).manual_seed(9)
    wide = torch.randn(3, 50, 120, device=DEV, generator=g)
    x = wide[:, :, 7:87]                                  # [3, 50, 80], rows 120 apart
    y = torch.randn(90, 40, device=DEV, generator=g)
    o = P.Orthogonalizer([(3, 50, 80), (90, 40)], dtype="f32", ld=[120, None])
    before, want = wide.clone(), [_exact(m) for m in x] + [_exact(y)]
    o.orthogonalize([x, y], [x, y])
    for a, b in zip(list(x) + [y], want):
        _near(a, b, "f32")
    wide[:, :, 7:87] = before[:, :, 7:87]
    assert torch.equal(wide, before)                      # nothing beside the rows was touched


def test_zeros_and_special_values_stay_in_their_matrix():
    P = _P()
    sizes = [(70, 90)] * 5
    x = [_matrix(70, 90, i, "flat") for i in range(5)]
    o = P.Orthogonalizer(sizes, dtype="f32")
    clean = [torch.empty_like(v) for v in x]
    o.orthogonalize(x, clean)
    bad = [v.clone() for v in x]
    bad[0].zero_()
    bad[2][3, 4] = float("inf")
    bad[3][69, 89] = float("nan")
    got = [torch.empty_like(v) for v in x]
    o.orthogonalize(bad, got)
    assert (got[0] == 0).all() and got[2].isnan().all() and got[3].isnan().all()
    assert torch.equal(got[1], clean[1]) and torch.equal(got[4], clean[4])
    o.orthogonalize(x, got)                               # nothing of it is left in the workspace
    assert all(torch.equal(a, b) for a, b in zip(got, clean))


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e12, 1e30])
def test_very_small_and_very_large_matrices(scale):
    P = _P()
    x = _matrix(60, 80, 1, "flat") * scale
    got = torch.empty_like(x)
    P.Orthogonalizer([(60, 80)], dtype="f32", eps=0.0).orthogonalize([x], [got])
    _near(got, _exact(x, eps=0.0), "f32")


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("din", ["f32", "bf16"])
def test_momentum_over_several_steps(din, nesterov):
    """M <- mu M + G in fp32: two roundings a step, 2^-23 of the terms' sizes, over 4 steps."""
    P = _P()
    sizes = [(80, 200), (2, 300, 64), (5, 5)]
    o = P.Orthogonalizer(sizes, dtype=din, out_dtype="f32")
    m = [torch.zeros(s, device=DEV) for s in sizes]
    m64 = [v.double() for v in m]
    for step in range(4):
        g = [torch.randn(s, device=DEV, generator=torch.Generator(device=DEV).manual_seed(7 * step + i))
             .to(torch.float32 if din == "f32" else torch.bfloat16) for i, s in enumerate(sizes)]
        out = [torch.empty(s, device=DEV) for s in sizes]
        o.momentum_orthogonalize(g, m, out, 0.9, nesterov=nesterov)
        for i, s in enumerate(sizes):
            m64[i] = float(torch.tensor(0.9)) * m64[i] + g[i].double()
            assert (m[i].double() - m64[i]).abs().max() <= 8 * 2.0 ** -24 * 12
            u = g[i].double() + float(torch.tensor(0.9)) * m64[i] if nesterov else m64[i]
            for a, b in zip(out[i].reshape(-1, *s[-2:]), u.reshape(-1, *s[-2:])):
                _near(a, _exact(b), "f32")


def test_many_matrices_and_another_stream():
    P = _P()
    sizes = [(16 + i % 5, 24 + i % 7) for i in range(150)]
    x = [_matrix(*s, i) for i, s in enumerate(sizes)]
    o = P.Orthogonalizer(sizes, dtype="f32", out_dtype="bf16")
    out = [torch.empty(s, device=DEV, dtype=torch.bfloat16) for s in sizes]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o.orthogonalize(x, out)
    torch.cuda.current_stream().wait_stream(side)
    for v, w in zip(x, out):
        _near(w, _exact(v), "bf16")


def test_a_graph_replays_with_new_inputs():
    P = _P()
    sizes = [(300, 200), (4, 64, 100)]
    o = P.Orthogonalizer(sizes, dtype="bf16")
    x = [torch.randn(s, device=DEV).bfloat16() for s in sizes]
    m = [torch.zeros(s, device=DEV) for s in sizes]
    out = [torch.empty_like(v) for v in x]
    o.momentum_orthogonalize(x, m, out, 0.95)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o.momentum_orthogonalize(x, m, out, 0.95)
    for _ in range(3):
        for v in x:
            v.copy_(torch.randn(v.shape, device=DEV))
        m2, out2 = [v.clone() for v in m], [torch.empty_like(v) for v in out]
        graph.replay()
        torch.cuda.synchronize()
        o.momentum_orthogonalize(x, m2, out2, 0.95)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out + m, out2 + m2))


def test_long_thin_and_empty_matrices():
    P = _P()
    sizes = [(65536, 3), (0, 5), (2, 60000), (7, 0)]
    x = [_matrix(*s, 5, "flat") if min(s) else torch.empty(s, device=DEV) for s in sizes]
    out = [torch.empty(s, device=DEV) for s in sizes]
    P.Orthogonalizer(sizes, dtype="f32").orthogonalize(x, out)
    for v, w in zip(x, out):
        if v.numel():
            _near(w, _exact(v), "f32")


def test_directions_feed_the_local_step():
    """Two workers' directions as the gradients of a Slow Momentum round: x <- x - lr (O + wd x),
    then the average; against the same in 64 bits."""
    P = _P()
    sizes, m, lr, wd = [(48, 64), (100, 30)], 2, 0.02, 0.1
    params = [[_matrix(*s, 3 + i, "flat") * 0.05 for i, s in enumerate(sizes)] for _ in range(m)]
    x64 = [[p.double() for p in params[0]] for _ in range(m)]
    opt = P.SlowMo(params, P.make_config(m=m, tau=2, alpha=1.0, beta=0.5, momentum=0.0, weight_decay=wd))
    o = P.Orthogonalizer(sizes * m, dtype="f32", out_dtype="f32", scale="rms")
    mom = [torch.zeros(s, device=DEV) for s in sizes * m]
    mom64 = [v.double() for v in mom]
    out = [[torch.empty(s, device=DEV) for s in sizes] for _ in range(m)]
    for step in range(2):
        g = [_matrix(*s, 100 * step + i, "flat") for i, s in enumerate(sizes * m)]
        o.momentum_orthogonalize(g, mom, [t for w in out for t in w], 0.95)
        opt.local_step(out, lr)
        for i in range(m):
            for j, s in enumerate(sizes):
                at = i * len(sizes) + j
                mom64[at] = 0.95 * mom64[at] + g[at].double()
                d = _exact(g[at].double() + 0.95 * mom64[at]) * 0.2 * max(s) ** 0.5
                x64[i][j] = x64[i][j] - lr * (d + wd * x64[i][j])
    opt.outer_step(lr)
    for j in range(len(sizes)):
        mean = (x64[0][j] + x64[1][j]) / 2                # u_0 = 0, alpha = 1: x <- x0 - (x0 - mean)
        for i in range(m):
            assert (params[i][j].double() - mean).abs().max() < 2e-5
    opt.close()
