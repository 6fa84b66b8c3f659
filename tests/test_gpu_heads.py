"""The norm of queries and keys with the position rotation, forward, backward and
for single tokens with a cache, against the definition in 64 bits.

Tolerances.  Inside a row of D elements the kernel rounds fp32 values: the sum of
squares (D / lanes + log2 lanes additions, halved by the square root), the root, three
products and the two of the rotation.  For D <= 512 that is under 64 roundings of
2^-24 relative to the row's largest |w x^|, so 4e-6 of it; a bf16 result adds its
own rounding, 2^-8 of the value.  The gradient has two such sums over the row and
terms as large as 1/r max(|g w|) and their product with x^, so 3e-5 of max |g w| r max(1, x^2).
Weight gradients: a sum of N terms in fp32, any order: 2^-24 * (log2 N + 40) * sum |terms|,
where 40 covers a lane's own chain of additions and the terms' roundings."""
import ctypes as C

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DEV = "cuda:0"


def _P():
    import paper_1910_00643_amd as P
    return P


def _turn64(y, table, positions, pair_axis, interleaved, back=False):
    """The rotation as its definition: pair by pair, in 64 bits."""
    pairs = table.shape[2]
    y = y.clone()
    for i in range(pairs):
        rows = positions[pair_axis[i]]
        still = rows == -1
        c = table[rows.clamp(min=0), 0, i].double().masked_fill(still, 1.0)[:, None]
        s = table[rows.clamp(min=0), 1, i].double().masked_fill(still, 0.0)[:, None]
        if back:
            s = -s
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
        u, v = y[..., a].clone(), y[..., b].clone()
        y[..., a], y[..., b] = u * c - v * s, u * s + v * c
    return y


def _norm64(x, w, eps):
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    return x * r, r, (w.double() if w is not None else torch.ones(x.shape[-1], dtype=torch.float64, device=DEV))


def _inputs(seed, tokens, hq, hk, dim, rot, dtype, axes, rows=61, pad=0, offset=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    width = (hq + hk) * dim + pad
    flat = torch.randn(tokens * width + offset, device=DEV, generator=g).mul_(2).to(dtype)[offset:]
    both = flat.view(tokens, width)[:, :(hq + hk) * dim].unflatten(1, (hq + hk, dim))
    table = _P().rotary_table(rows, [rot // 2 - (axes - 1) * (rot // 2 // axes)] +
                              [rot // 2 // axes] * (axes - 1), device=DEV) if rot else None
    positions = torch.randint(-1, rows, (axes, tokens), device=DEV, generator=g)
    n = rot // 2
    pair_axis = [(i * 7 // 3) % axes for i in range(n)]      # pieces of one axis and mixed ones
    wq = torch.randn(dim, device=DEV, generator=g)
    wk = torch.randn(dim, device=DEV, generator=g)
    return both[:, :hq], both[:, hq:], table, positions, pair_axis, wq, wk


CASES = [  # tokens, hq, hk, dim, rot, axes, pad, offset
    (1, 1, 1, 128, 128, 1, 0, 0),
    (1, 5, 0, 64, 32, 1, 0, 0),
    (3, 0, 2, 64, 64, 1, 0, 0),
    (7, 4, 2, 64, 64, 1, 0, 0),
    (130, 9, 3, 128, 64, 3, 0, 0),
    (33, 2, 1, 256, 256, 2, 0, 0),
    (5, 3, 3, 512, 512, 1, 0, 0),
    (65, 3, 3, 72, 72, 2, 0, 0),
    (17, 2, 2, 80, 40, 4, 8, 0),
    (19, 2, 2, 96, 32, 1, 3, 0),       # rows of odd strides
    (19, 2, 2, 64, 64, 1, 0, 1),       # data off by one element
    (9, 3, 2, 33, 20, 2, 0, 0),        # an odd head
    (6, 2, 1, 1, 0, 1, 0, 0),
    (6, 2, 1, 2, 2, 1, 0, 0),
    (4, 2, 2, 511, 510, 1, 0, 0),
    (9000, 1, 1, 64, 64, 1, 0, 0),     # more tokens than waves
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward_and_backward(case, norm, interleaved, dtype):
    tokens, hq, hk, dim, rot, axes, pad, offset = case
    td = torch.float32 if dtype == "f32" else torch.bfloat16
    q, k, table, positions, pair_axis, wq, wk = _inputs(5, tokens, hq, hk, dim, rot, td, axes, pad=pad,
                                                        offset=offset)
    op = _P().HeadNormRotary(dim, table, dtype=dtype, norm=norm, interleaved=interleaved,
                             pair_axis=pair_axis if rot else None)
    yq, yk = op.forward(q, k, positions, wq if norm else None, wk if norm else None)
    g = torch.Generator(device=DEV).manual_seed(6)
    gq = torch.randn(q.shape, device=DEV, generator=g).to(td)
    gk = torch.randn(k.shape, device=DEV, generator=g).to(td)
    dq, dk, dwq, dwk = op.backward(gq, gk, q, k, positions, wq if norm else None, wk if norm else None)
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    for x, w, y, gy, dx, dw in ((q, wq, yq, gq, dq, dwq), (k, wk, yk, gk, dk, dwk)):
        if not x.shape[1]:
            if norm:
                assert (dw == 0).all()
            continue
        x64 = x.double()
        xh, r, w64 = _norm64(x64, w, 1e-6)
        if not norm:
            xh, r, w64 = x64, torch.ones_like(r), torch.ones_like(w64)
        want = _turn64(xh * w64, table, positions, pair_axis, interleaved) if rot else xh * w64
        big = (xh * w64).abs().amax(-1, keepdim=True)
        assert ((y.double() - want).abs() <= 4e-6 * big + half * want.abs()).all()
        gr = _turn64(gy.double(), table, positions, pair_axis, interleaved, back=True) if rot else gy.double()
        gw = gr * w64
        if norm:
            wdx = r * (gw - xh * (gw * xh).mean(-1, keepdim=True))
            big = gw.abs().amax(-1, keepdim=True) * r * (xh * xh).amax(-1, keepdim=True).clamp(min=1)
            terms = gr * xh
            n = tokens * x.shape[1]
            bound = 2.0 ** -24 * (n.bit_length() + 40) * terms.abs().sum((0, 1)) * 1.5
            assert ((dw.double() - terms.sum((0, 1))).abs() <= bound).all()
        else:
            wdx, big = gw, gw.abs().amax(-1, keepdim=True) * 2
            assert dw is None
        assert ((dx.double() - wdx).abs() <= 3e-5 * big + half * wdx.abs()).all()


def test_gradient_against_differences():
    """Central differences of the forward call in fp32: step h = 2^-6 on one element at a time.
    The forward value is good to 4e-6 * 4 (rows of magnitude up to about 4), so the quotient to
    2 * 1.6e-5 / (2 h) * sqrt(D) summed over the row, 4e-3; the cubic term of a norm with
    |x| around 2 and h = 1/64 adds under 2e-3."""
    q, k, table, positions, pair_axis, wq, wk = _inputs(1, 3, 2, 1, 16, 16, torch.float32, 2)
    op = _P().HeadNormRotary(16, table, dtype="f32", pair_axis=pair_axis)
    g = torch.Generator(device=DEV).manual_seed(2)
    gq, gk = torch.randn(q.shape, device=DEV, generator=g), torch.randn(k.shape, device=DEV, generator=g)

    def loss(q, k, wq, wk):
        a, b = op.forward(q, k, positions, wq, wk)
        return float((a.double() * gq.double()).sum() + (b.double() * gk.double()).sum())

    grads = op.backward(gq, gk, q, k, positions, wq, wk)
    h = 2.0 ** -6
    for at, (x, dx) in enumerate(zip((q, k, wq, wk), grads)):
        for e in range(0, x.numel(), 5):
            moved = []
            for sign in (1, -1):
                args = [v.clone().contiguous() for v in (q, k, wq, wk)]
                args[at].view(-1)[e] += sign * h
                moved.append(loss(*args))
            assert abs((moved[0] - moved[1]) / (2 * h) - float(dx.reshape(-1)[e])) < 6e-3 * 4


def test_autograd_reaches_weights_and_inputs():
    q, k, table, positions, pair_axis, wq, wk = _inputs(1, 12, 4, 2, 64, 64, torch.float32, 1)
    op = _P().HeadNormRotary(64, table, dtype="f32")
    leaves = [t.detach().clone().requires_grad_() for t in (q, k, wq, wk)]
    a, b = op(leaves[0], leaves[1], positions[0], leaves[2], leaves[3])
    (a.square().sum() + b.sum()).backward()
    want = op.backward(2 * a.detach(), torch.ones_like(b), q, k, positions, wq, wk)
    for t, w in zip(leaves, want):
        assert torch.equal(t.grad, w)


def test_single_tokens_reach_their_rows_of_the_cache():
    q, k, table, positions, pair_axis, wq, wk = _inputs(3, 6, 8, 2, 128, 128, torch.bfloat16, 1)
    op = _P().HeadNormRotary(128, table)
    cache = torch.full((2, 9, 2, 128), 7.0, device=DEV, dtype=torch.bfloat16)
    slots = torch.tensor([3, -1, 0, 8, 9, 5], device=DEV)      # one without a row, one past the end
    yq, yk = op.forward(q, k, positions, wq, wk)
    got, same = op.forward(q, k, positions, wq, wk, k_out=cache[1], k_slots=slots)
    assert torch.equal(got, yq) and same.data_ptr() == cache[1].data_ptr()
    want = torch.full_like(cache, 7.0)
    for t, row in enumerate(slots.tolist()):
        if 0 <= row < 9:
            want[1, row] = yk[t]
    assert torch.equal(cache, want)


def test_in_place_layouts_and_shared_rows():
    """Results over the inputs; head-major layouts; inputs whose heads are one broadcast head."""
    q, k, table, positions, pair_axis, wq, wk = _inputs(4, 50, 3, 3, 64, 64, torch.bfloat16, 1)
    op = _P().HeadNormRotary(64, table)
    yq, yk = op.forward(q, k, positions, wq, wk)
    major = torch.empty(3, 50, 64, device=DEV, dtype=torch.bfloat16).transpose(0, 1)
    got, _ = op.forward(q.transpose(0, 1).contiguous().transpose(0, 1), k, positions, wq, wk, q_out=major)
    assert torch.equal(got, yq)
    shared = q[:, :1].expand(50, 3, 64)
    a, _ = op.forward(shared, k, positions, wq, wk)
    assert torch.equal(a, yq[:, :1].expand(50, 3, 64))
    op.forward(q, k, positions, wq, wk, q_out=q, k_out=k)
    assert torch.equal(q, yq) and torch.equal(k, yk)


def test_rows_of_zeros_and_special_values_stay_in_their_rows():
    q, k, table, positions, pair_axis, wq, wk = _inputs(4, 40, 3, 1, 64, 64, torch.float32, 1)
    op = _P().HeadNormRotary(64, table, dtype="f32")
    q = q.contiguous().clone()
    clean, _ = op.forward(q, k, positions, wq, wk)
    q[3, 1] = 0
    q[7, 2, 5] = float("inf")
    q[9, 0, 1] = float("nan")
    pos = positions.clone()
    pos[0, 11], pos[0, 12] = 61, -2                       # past the table, and before it
    y, yk = op.forward(q, k, pos, wq, wk)
    assert (y[3, 1] == 0).all() and y[9, 0].isnan().all() and y[7, 2, 5].isnan()
    assert y[11].isnan().all() and y[12].isnan().all() and yk[11].isnan().all()
    keep = torch.ones(40, 3, dtype=torch.bool, device=DEV)
    keep[3, 1] = keep[7, 2] = keep[9, 0] = False
    keep[11] = keep[12] = False
    assert torch.equal(y[keep], clean[keep])
    dq, dk, dwq, dwk = op.backward(torch.ones_like(y), torch.ones_like(yk), clean * 0, k, positions, wq, wk)
    assert dq.isfinite().all() and (dwq == 0).all()


def test_no_tokens_and_no_heads():
    op = _P().HeadNormRotary(64, _P().rotary_table(4, 32, device=DEV))
    q = torch.empty(0, 2, 64, device=DEV, dtype=torch.bfloat16)
    pos = torch.empty(0, device=DEV, dtype=torch.int64)
    a, b = op.forward(q, q, pos)
    assert a.shape == q.shape
    dq, dk, dwq, dwk = op.backward(q, q, q, q, pos)
    assert (dwq == 0).all() and (dwk == 0).all()


def test_another_stream_and_a_graph():
    q, k, table, positions, pair_axis, wq, wk = _inputs(8, 300, 4, 2, 128, 128, torch.bfloat16, 1)
    op = _P().HeadNormRotary(128, table)
    want = op.forward(q, k, positions, wq, wk)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = op.forward(q, k, positions, wq, wk)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    x, y = q.contiguous().clone(), k.contiguous().clone()
    outs = [torch.empty_like(x), torch.empty_like(y)]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        op.forward(x, y, positions, wq, wk, q_out=outs[0], k_out=outs[1])
    for seed in range(3):
        fresh = _inputs(20 + seed, 300, 4, 2, 128, 128, torch.bfloat16, 1)
        x.copy_(fresh[0])
        y.copy_(fresh[1])
        graph.replay()
        torch.cuda.synchronize()
        want = op.forward(x, y, positions, wq, wk)
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


def test_offsets_past_32_bits():
    """A cache whose rows lie past 2^31 elements."""
    rows = 2 ** 31 // 128 + 10
    cache = torch.zeros(rows, 1, 128, device=DEV, dtype=torch.bfloat16)
    q, k, table, positions, pair_axis, wq, wk = _inputs(8, 4, 1, 1, 128, 128, torch.bfloat16, 1)
    op = _P().HeadNormRotary(128, table)
    slots = torch.tensor([rows - 1, 2, rows - 5, 0], device=DEV)
    _, yk = op.forward(q, k, positions, wq, wk)
    op.forward(q, k, positions, wq, wk, k_out=cache, k_slots=slots)
    assert torch.equal(cache[slots], yk)
    assert int((cache != 0).any(-1).sum()) == 4
