"""The gradient of attention over packed sequences against its formula in 64 bits (attention_utils.py has the
tolerances), against differences, through autograd and in graphs."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import attention_utils as U  # noqa: E402
from test_gpu_attention import CASES, DEV, _each, _inputs, _P  # noqa: E402


@pytest.fixture(autouse=True)
def _free_gpu_memory():
    yield
    torch.cuda.empty_cache()


def _grad(q, dtype, g):
    return torch.randn(q.shape, device=DEV, generator=g).to(U.TD[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES + [
    ([600], None, 16, 1, 64, True, None, 0, 0, 0),       # few keys, many rows: pieces
    ([64, 900], [900, 64], 3, 1, 128, False, None, 0, 0, 0),
    ([1200], None, 2, 2, 128, True, 200, 4, 0, 0),
    ([0], [50], 2, 1, 64, True, None, 0, 0, 0),          # keys without queries
], ids=str)
def test_backward(case, dtype):
    op, q, k, v, at, k_at, g = _inputs(case, dtype)
    gout = _grad(q, dtype, g)
    out, lse = op.forward(q, k, v, at, k_at)
    got = dict(zip(("dq", "dk", "dv"), op.backward(gout, q, k, v, out, lse, at, k_at)))
    again = op.backward(gout, q, k, v, out, lse, at, k_at)
    assert all(torch.equal(a, b) for a, b in zip(got.values(), again))
    for a, b in _each(case):
        want, tol = U.dense(q[a], k[b], v[b], dtype, causal=case[5], window=case[6], sinks=case[7], g=gout[a])
        U.near(got["dq"][a], want["dq"], tol["dq"], "dq")
        U.near(got["dk"][b], want["dk"], tol["dk"], "dk")
        U.near(got["dv"][b], want["dv"], tol["dv"], "dv")


@pytest.mark.parametrize("dim", [32, 128, 256])
@pytest.mark.parametrize("times", [1.0, 4.0])
def test_rows_of_few_keys(dim, times):
    """Where few keys have a row's weight, g V^T and g . out all but cancel: what the rounding of `out` leaves of them is
    not what dQ and dK are made of."""
    lengths = [2, 3, 1, 5, 17, 2, 64, 100]
    g = torch.Generator(device=DEV).manual_seed(41)
    n, at = sum(lengths), U.offsets_of(lengths)
    q = U.rows(g, n, 4, dim, "bf16", times=times)
    k, v, gout = (U.rows(g, n, h, dim, "bf16") for h in (2, 2, 4))
    op, offsets = _P().Attention(dim), torch.tensor(at, device=DEV)
    out, lse = op.forward(q, k, v, offsets)
    got = dict(zip(("dq", "dk", "dv"), op.backward(gout, q, k, v, out, lse, offsets)))
    for i, m in enumerate(lengths):
        s = slice(at[i], at[i + 1])
        want, tol = U.dense(q[s], k[s], v[s], "bf16", g=gout[s], mended=True)
        for name, x in got.items():
            U.near(x[s], want[name], tol[name], name)


@pytest.mark.parametrize("window,sinks", [(None, 0), (20, 3)])
def test_against_differences(window, sinks):
    """The derivative along a direction, from the definition in 64 bits on either side."""
    case = ([70, 33], None, 4, 2, 64, True, window, sinks, 0, 0)
    op, q, k, v, at, _, g = _inputs(case, "f32")
    gout = _grad(q, "f32", g)
    out, lse = op.forward(q, k, v, at)
    got = op.backward(gout, q, k, v, out, lse, at)

    def loss(x):
        total = 0.0
        for a, b in _each(case):
            total += (U.dense(x[0][a], x[1][b], x[2][b], "f32", window=window, sinks=sinks)[0]["out"] * gout[a].double()).sum()
        return total

    x = [t.double() for t in (q, k, v)]
    for i, name in enumerate(("dq", "dk", "dv")):
        d = torch.randn(x[i].shape, device=DEV, generator=g, dtype=torch.float64)
        step = 1e-5
        up, down = ([t + (step * s * d if j == i else 0) for j, t in enumerate(x)] for s in (1, -1))
        slope = (loss(up) - loss(down)) / (2 * step)
        allowed = 0.0
        for a, b in _each(case):
            tol = U.dense(q[a], k[b], v[b], "f32", window=window, sinks=sinks, g=gout[a])[1]
            allowed += (tol[name] * d[a if i == 0 else b].abs()).sum()
        # the differences themselves: steps of 1e-5 leave 1e-10 of third derivatives, 64 bits 1e-11 of the loss
        assert (slope - (got[i].double() * d).sum()).abs() <= allowed + 1e-6 * (1 + slope.abs()), name


def test_autograd():
    case = ([40, 33], None, 4, 2, 64, True, None, 0, 0, 0)
    op, q, k, v, at, _, g = _inputs(case, "f32", rest=9)
    q, k, v = (t.contiguous().requires_grad_() for t in (q, k, v))
    gout = _grad(q, "f32", g)
    y = op(q, k, v, at)
    y.backward(gout)
    out, lse = op.forward(q.detach(), k.detach(), v.detach(), at)
    want = op.backward(gout, q.detach(), k.detach(), v.detach(), out, lse, at)
    assert torch.equal(y.detach(), out)
    for t, w in zip((q, k, v), want):
        assert torch.equal(t.grad, w) and (t.grad[73:] == 0).all()


def test_autograd_of_a_broadcast_gradient_and_shared_tensors():
    """A gradient of stride 0, and keys that are the values too."""
    case = ([50], None, 2, 2, 64, True, None, 0, 0, 0)
    op, q, k, _, at, _, _ = _inputs(case, "f32")
    q, k = q.contiguous().requires_grad_(), k.contiguous().requires_grad_()
    op(q, k, k, at).sum().backward()
    want, tol = U.dense(q.detach(), k.detach(), k.detach(), "f32", g=torch.ones_like(q))
    U.near(q.grad, want["dq"], tol["dq"], "dq")
    U.near(k.grad, want["dk"] + want["dv"], tol["dk"] + tol["dv"], "dk + dv")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_not_seen_has_no_part(dtype):
    """Wild keys and values, and wild gradients, reach no gradient of what does not see them."""
    case = ([200], None, 4, 2, 64, True, 40, 0, 0, 0)
    op, q, k, v, at, _, g = _inputs(case, dtype)
    gout = _grad(q, dtype, g)
    out, lse = op.forward(q, k, v, at)
    clean = op.backward(gout, q, k, v, out, lse, at)
    k2, v2, g2 = k.clone(), v.clone(), gout.clone()
    k2[100] = float("nan")
    v2[101, 0, 3] = float("inf")
    g2[104, :, 7] = float("nan")
    out2, lse2 = op.forward(q, k2, v2, at)
    dq, dk, dv = op.backward(g2, q, k2, v2, out2, lse2, at)
    sees = U.visible(200, 200, True, 40, 0)
    touched_q = sees[:, 100] | sees[:, 101]
    touched_q[104] = True
    touched_k = sees[touched_q].any(0)
    assert (~touched_q).any() and (~touched_k).any()
    assert torch.equal(dq[~touched_q], clean[0][~touched_q])
    assert torch.equal(dk[~touched_k], clean[1][~touched_k]) and torch.equal(dv[~touched_k], clean[2][~touched_k])
    assert not dq[sees[:, 100]].isfinite().any()


def test_rows_behind_the_last_sequence():
    case = ([40, 33], None, 2, 1, 64, True, None, 0, 0, 0)
    op, q, k, v, at, _, g = _inputs(case, "bf16", rest=77)
    for t in (q, k, v):
        t[73:] = float("nan")
    gout = _grad(q, "bf16", g)
    gout[73:] = float("nan")
    out, lse = op.forward(q, k, v, at)
    for d in op.backward(gout, q, k, v, out, lse, at):
        assert (d[73:] == 0).all() and d[:73].isfinite().all()


@pytest.mark.parametrize("dim,dtype", [(64, "bf16"), (128, "bf16"), (128, "f32"), (256, "bf16")])
def test_a_captured_step_is_replayed(dim, dtype):
    """Forward and backward in a graph, on offsets that change between replays, beside an eager graph of the same leaves."""
    case = ([90, 60, 50], None, 4, 2, dim, True, 33, 2, 0, 0)
    op, q, k, v, at, _, g = _inputs(case, dtype)
    leaves = [t.contiguous().requires_grad_() for t in (q, k, v)]
    gout = _grad(q, dtype, g)
    held = op(*leaves, at)                      # an eager graph that stays alive

    def step():
        with torch.no_grad():
            out, lse = op.forward(*leaves, at)
            return (out, *op.backward(gout, *leaves, out, lse, at))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    for turn, lengths in enumerate(([90, 60, 50], [200, 0, 0], [1, 2, 150], [64, 65, 71])):
        at.copy_(torch.tensor(U.offsets_of(lengths), device=DEV))
        gout.copy_(_grad(q, dtype, g))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in kept]
        for a, b in zip(got, step()):
            assert torch.equal(a, b), turn
    assert held.isfinite().all()


def test_two_streams_at_once():
    case = ([700, 300], None, 8, 2, 128, True, None, 0, 0, 0)
    op, q, k, v, at, _, g = _inputs(case, "bf16")
    gout = [_grad(q, "bf16", g) for _ in range(2)]
    out, lse = op.forward(q, k, v, at)
    want = [op.backward(x, q, k, v, out, lse, at) for x in gout]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s, x in zip(streams, gout):
        with torch.cuda.stream(s):
            got.append(op.backward(x, q, k, v, out, lse, at))
    torch.cuda.synchronize()
    for w, y in zip(want, got):
        assert all(torch.equal(a, b) for a, b in zip(w, y))


@pytest.mark.parametrize("window", [None, 70])
@pytest.mark.parametrize("dim", [32, 64, 128, 192])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_key_whose_score_is_minus_infinity(dtype, dim, window):
    """It has no weight: the element that holds the infinity gets 0 times it, and every other gradient is that of a key far
    below the others."""
    case = ([200], None, 4, 2, dim, True, window, 0, 0, 0)
    op, q, k, v, at, _, g = _inputs(case, dtype)
    gout = _grad(q, dtype, g)
    q[:, :, 6] = q[:, :, 6].abs() + 1
    k[100, :, 6] = -1e5
    out, lse = op.forward(q, k, v, at)
    want = op.backward(gout, q, k, v, out, lse, at)
    k[100, :, 6] = -float("inf")
    assert all(torch.equal(a, b) for a, b in zip(op.forward(q, k, v, at), (out, lse)))
    dq, dk, dv = op.backward(gout, q, k, v, out, lse, at)
    rest = [d for d in range(dim) if d != 6]
    assert torch.equal(dq[:, :, rest], want[0][:, :, rest]) and torch.equal(dk, want[1]) and torch.equal(dv, want[2])
    seen = U.visible(200, 200, True, window, 0)[:, 100]
    assert dq[seen][:, :, 6].isnan().all() and torch.equal(dq[~seen], want[0][~seen])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_everything_side_by_side_in_two_arrays(dtype):
    """Through the C entries: q, k, v and out in the rows of one array, dq, dk and dv in those of another, with a head between
    that stays as it was."""
    from paper_1910_00643_amd import attention as A
    case = ([70, 140], None, 4, 2, 64, True, None, 0, 0, 0)
    op, q, k, v, at, _, g = _inputs(case, dtype)
    gout = _grad(q, dtype, g)
    out, lse = op.forward(q, k, v, at)
    want = op.backward(gout, q, k, v, out, lse, at)
    n = 210
    one = torch.full((n, 4 + 1 + 2 + 2 + 4, 64), 7.0, device=DEV, dtype=U.TD[dtype])
    two = torch.full((n, 4 + 2 + 1 + 2, 64), 7.0, device=DEV, dtype=U.TD[dtype])
    q1, k1, v1, out1 = one[:, :4], one[:, 5:7], one[:, 7:9], one[:, 9:]
    dq1, dk1, dv1 = two[:, :4], two[:, 4:6], two[:, 7:]
    for x, y in ((q1, q), (k1, k), (v1, v)):
        x.copy_(y)

    def heads(x):
        return A.slowmo_heads(x.data_ptr(), x.shape[1], x.stride(0), x.stride(1))

    lib, cfg, stream = A.lib(), op._kept, torch.cuda.current_stream().cuda_stream or None
    lse1 = torch.empty_like(lse)
    assert lib.slowmo_attention(cfg, 2, at.data_ptr(), None, n, n, heads(q1), heads(k1), heads(v1), heads(out1), lse1.data_ptr(),
                                stream) == 0
    assert torch.equal(out1, out) and torch.equal(lse1, lse) and (one[:, 4] == 7).all() and torch.equal(k1, k)
    need = lib.slowmo_attention_backward_bytes(cfg, 2, n, n, 4, 2)
    space = torch.empty(need, dtype=torch.uint8, device=DEV)
    assert lib.slowmo_attention_backward(cfg, 2, at.data_ptr(), None, n, n, heads(gout), heads(q1), heads(k1), heads(v1), heads(out1),
                                         lse1.data_ptr(), heads(dq1), heads(dk1), heads(dv1), space.data_ptr(), need, stream) == 0
    assert all(torch.equal(a, b) for a, b in zip((dq1, dk1, dv1), want))
    assert (two[:, 6] == 7).all() and (one[:, 4] == 7).all() and torch.equal(q1, q) and torch.equal(v1, v)
