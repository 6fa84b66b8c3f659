"""Orthogonalised updates on the lists that go their own ways: small matrices alone, large
ones in large tiles, wide ones, sums in shares, many matrices, addresses that are aligned to
an element only, offsets past 32 bits.  Against 64 bits, with the tolerances of
test_gpu_orth.py (the same arithmetic)."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_orth import DEV, _P, _exact, _matrix, _near  # noqa: E402

T = {"f32": torch.float32, "bf16": torch.bfloat16}
TYPES = [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")]

# each alone in its list: up to 64 and up to 128 a side, up to 256 long, tiny ones beside
SMALL = {
    "up_to_64": [(64, 64), (33, 256), (256, 33), (64, 40), (40, 64), (50, 255), (64, 129), (4, 4), (3, 200)],
    "up_to_128": [(128, 128), (65, 256), (256, 128), (128, 255), (100, 101), (127, 66), (40, 250), (1, 1), (20, 2)],
}


@pytest.mark.parametrize("kind", ["gradient", "flat", "deficient"])
@pytest.mark.parametrize("types", TYPES, ids=str)
@pytest.mark.parametrize("which", sorted(SMALL))
def test_small_matrices_alone(which, types, kind):
    P = _P()
    din, dout = types
    sizes = SMALL[which]
    x = [_matrix(r, c, 40 + i, kind).to(T[din]) for i, (r, c) in enumerate(sizes)]
    out = [torch.full(s, float("nan"), device=DEV, dtype=T[dout]) for s in sizes]
    o = P.Orthogonalizer(sizes, dtype=din, out_dtype=dout, scale="rms")
    o.orthogonalize(x, out)
    for v, w, s in zip(x, out, sizes):
        _near(w, _exact(v) * 0.2 * max(s) ** 0.5, dout)
    again = [torch.empty_like(v) for v in out]
    o.orthogonalize(x, again)
    assert all(torch.equal(a, b) for a, b in zip(out, again))


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("types", TYPES, ids=str)
def test_small_matrices_with_momentum(types, nesterov):
    """M <- mu M + G: one fused or two single roundings of fp32 a step."""
    P = _P()
    din, dout = types
    sizes = [(60, 100), (64, 64), (100, 60), (8, 8)] + ([(128, 200), (200, 90)] if dout == "bf16" else [])
    o = P.Orthogonalizer(sizes, dtype=din, out_dtype=dout)
    m = [_matrix(*s, 4 + i, "flat") for i, s in enumerate(sizes)]
    mu = float(torch.tensor(0.9))
    for step in range(2):
        g = [_matrix(*s, 50 + 10 * step + i, "flat").to(T[din]) for i, s in enumerate(sizes)]
        m64 = [mu * a.double() + b.double() for a, b in zip(m, g)]
        out = [torch.empty(s, device=DEV, dtype=T[dout]) for s in sizes]
        o.momentum_orthogonalize(g, m, out, 0.9, nesterov=nesterov)
        for a, b, c, w in zip(m, m64, g, out):
            assert (a.double() - b).abs().max() <= 2 * 2.0 ** -24 * 16
            _near(w, _exact(c.double() + mu * b if nesterov else b), dout)


@pytest.mark.parametrize("types", TYPES, ids=str)
def test_small_matrices_by_rows_apart_and_in_place(types):
    P = _P()
    din, dout = types
    sizes, n = [(60, 100), (100, 60), (5, 9)], 128 * 130
    store = torch.randn(3, n, device=DEV, generator=torch.Generator(device=DEV).manual_seed(3)).to(T[din])
    # one element past the start of a row of 16 bytes
    x = [torch.as_strided(store[i], s, (111, 1), i * n + 1) for i, s in enumerate(sizes)]
    o = P.Orthogonalizer(sizes, dtype=din, out_dtype=dout, ld=[111] * 3)
    want = [_exact(v) for v in x]
    if din == dout:
        before = store.clone()
        o.orthogonalize(x, x)
        for v, w in zip(x, want):
            _near(v, w, dout)
        for v, i in zip(x, range(3)):
            v.copy_(torch.as_strided(before[i], v.shape, (111, 1), i * n + 1))
        assert torch.equal(store, before)
    else:
        room = torch.zeros(3, n, device=DEV, dtype=T[dout])
        out = [torch.as_strided(room[i], s, (111, 1), i * n + 1) for i, s in enumerate(sizes)]
        o.orthogonalize(x, out)
        for v, w in zip(out, want):
            _near(v, w, dout)
            v.zero_()
        assert (room == 0).all()


def test_special_values_among_small_matrices():
    P = _P()
    sizes = [(64, 90)] * 4 + [(6, 6)] * 3
    o = P.Orthogonalizer(sizes, dtype="f32", out_dtype="bf16")
    x = [_matrix(*s, i, "flat") for i, s in enumerate(sizes)]
    clean = [torch.empty(s, device=DEV, dtype=torch.bfloat16) for s in sizes]
    o.orthogonalize(x, clean)
    bad = [v.clone() for v in x]
    bad[0].zero_()
    bad[4].zero_()
    bad[1][63, 89] = float("inf")
    bad[5][0, 0] = float("nan")
    got = [torch.empty_like(v) for v in clean]
    o.orthogonalize(bad, got)
    assert (got[0] == 0).all() and (got[4] == 0).all() and got[1].isnan().all() and got[5].isnan().all()
    assert all(torch.equal(got[i], clean[i]) for i in (2, 3, 6))


@pytest.mark.parametrize("size", [(64, 90), (300, 200), (20, 30)], ids=str)
@pytest.mark.parametrize("types", TYPES, ids=str)
def test_subnormal_matrices(types, size):
    """The norm's inverse is past fp32's range; the elements are what the input type holds."""
    P = _P()
    din, dout = types
    x = (_matrix(*size, 1, "flat") * 2e-39).to(T[din])
    assert float(x.double().norm()) > 0
    got = torch.empty(size, device=DEV, dtype=T[dout])
    o = P.Orthogonalizer([size], dtype=din, out_dtype=dout, eps=0.0)
    o.orthogonalize([x], [got])
    _near(got, _exact(x, eps=0.0), dout)


@pytest.mark.parametrize("size", [(300, 200), (100, 100), (20, 30)], ids=str)
def test_special_values_in_bf16(size):
    P = _P()
    sizes = [size] * 5
    x = [_matrix(*s, i, "flat").bfloat16() for i, s in enumerate(sizes)]
    o = P.Orthogonalizer(sizes, dtype="bf16")
    clean = [torch.empty_like(v) for v in x]
    o.orthogonalize(x, clean)
    bad = [v.clone() for v in x]
    bad[0].zero_()
    bad[1][1, 2] = float("-inf")
    bad[2][0, 0] = float("nan")
    got = [torch.empty_like(v) for v in clean]
    o.orthogonalize(bad, got)
    assert (got[0] == 0).all() and got[1].isnan().all() and got[2].isnan().all()
    assert all(torch.equal(got[i], clean[i]) for i in (3, 4))
    o.orthogonalize(x, got)
    assert all(torch.equal(a, b) for a, b in zip(got, clean))


def test_more_small_matrices_than_travel_with_a_launch():
    P = _P()
    sizes = [(33 + i % 31, 40 + i % 17) for i in range(140)]
    x = [_matrix(*s, i) for i, s in enumerate(sizes)]
    out = [torch.empty(s, device=DEV) for s in sizes]
    P.Orthogonalizer(sizes, dtype="f32").orthogonalize(x, out)
    for v, w in zip(x, out):
        _near(w, _exact(v), "f32")


def test_more_matrices_in_tiles_than_travel_with_a_launch():
    P = _P()
    sizes = [(130 + i % 31, 140 + i % 17) for i in range(130)] + [(0, 4), (3, 3)]
    x = [_matrix(*s, i) for i, s in enumerate(sizes)]
    out = [torch.empty(s, device=DEV, dtype=torch.bfloat16) for s in sizes]
    P.Orthogonalizer(sizes, dtype="f32", out_dtype="bf16").orthogonalize(x, out)
    for v, w in zip(x, out):
        if v.numel():
            _near(w, _exact(v), "bf16")


@pytest.mark.parametrize("types", [("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16")], ids=str)
@pytest.mark.parametrize("sizes", [[(2049, 8250)], [(8250, 2049), (2300, 2049)], [(2100, 8300), (300, 1000), (64, 64), (5, 5)],
                                   [(640, 16384)] * 3, [(1024, 1024)] * 40, [(130, 65536)], [(1000, 512)] * 21],
                         ids=["large", "tall", "mixed", "wide", "many", "long", "shares"])
def test_kinds_of_tiles(sizes, types):
    P = _P()
    din, dout = types
    x = [_matrix(r, c, 70 + i).to(T[din]) for i, (r, c) in enumerate(sizes)]
    out = [torch.full(s, float("nan"), device=DEV, dtype=T[dout]) for s in sizes]
    o = P.Orthogonalizer(sizes, dtype=din, out_dtype=dout)
    o.orthogonalize(x, out)
    for v, w in zip(x, out):
        _near(w, _exact(v), dout)
    again = [torch.empty_like(v) for v in out]
    o.orthogonalize(x, again)
    assert all(torch.equal(a, b) for a, b in zip(out, again))


@pytest.mark.parametrize("types", TYPES, ids=str)
def test_addresses_aligned_to_an_element(types):
    P = _P()
    din, dout = types
    sizes, lds = [(300, 401), (520, 260)], [403, 261]
    o = P.Orthogonalizer(sizes, dtype=din, out_dtype=dout, ld=lds)
    g = torch.Generator(device=DEV).manual_seed(8)
    from_, to, mom = [], [], []
    for (r, c), ld in zip(sizes, lds):
        from_.append(torch.as_strided(torch.randn(r * ld + 1, device=DEV, generator=g).to(T[din]), (r, c), (ld, 1), 1))
        to.append(torch.as_strided(torch.zeros(r * ld + 1, device=DEV, dtype=T[dout]), (r, c), (ld, 1), 1))
        mom.append(torch.as_strided(torch.zeros(r * ld + 1, device=DEV), (r, c), (ld, 1), 1))
    o.orthogonalize(from_, to)
    for v, w in zip(from_, to):
        _near(w, _exact(v), dout)
    o.momentum_orthogonalize(from_, mom, to, 0.9)
    for v, w, k in zip(from_, to, mom):
        assert torch.equal(k, v.float())
        _near(w, _exact(v), dout)                    # U = 1.9 G


def test_rows_far_apart():
    """The last row begins 2^32 elements behind the first."""
    P = _P()
    ld = 1 << 28
    store = torch.empty(16 * ld + 8192, device=DEV, dtype=torch.bfloat16)
    for size in ((17, 300), (17, 90)):
        x = torch.as_strided(store, size, (ld, 1))
        x.copy_(_matrix(*size, 3, "flat"))
        out = torch.as_strided(store, size, (ld, 1), 4096)
        out.zero_()
        P.Orthogonalizer([size, (130, 140)], dtype="bf16", ld=[ld, 140]).orthogonalize(
            [x, torch.ones(130, 140, device=DEV, dtype=torch.bfloat16)], [out, torch.empty(130, 140, device=DEV, dtype=torch.bfloat16)])
        _near(out, _exact(x), "bf16")
    del store
    torch.cuda.empty_cache()


def test_a_workspace_past_32_bits():
    """16384 x 65536: three arrays of 2^30 halves for X alone."""
    P = _P()
    n, k = 16384, 65536
    x = torch.randn(n, k, device=DEV, dtype=torch.bfloat16, generator=torch.Generator(device=DEV).manual_seed(2))
    out = torch.empty_like(x)
    o = P.Orthogonalizer([(n, k)], dtype="bf16", steps=3)
    o.orthogonalize([x], [out])
    o.close()
    torch.cuda.empty_cache()
    want = x.double()
    want /= torch.linalg.vector_norm(want) + 1e-7
    a, b, c = 3.4445, -4.7750, 2.0315
    for _ in range(3):
        g = want @ want.t()
        p = c * (g @ g)
        p += b * g
        del g
        p.diagonal().add_(a)
        want = p @ want
        del p
    want -= out
    norm = float(torch.linalg.vector_norm(want))
    size = float(torch.linalg.vector_norm(out.double()))
    assert norm <= (2.0 ** -9 + 20 * 2.0 ** -12) * size, norm / size
    del want
    torch.cuda.empty_cache()
