"""Attention's calls on long lists of sequences, ragged ones, and edges of its plans: what one launch shape must not
take from another."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import attention_utils as U  # noqa: E402

DEV = U.DEV


@pytest.fixture(autouse=True)
def _free_gpu_memory():
    yield
    torch.cuda.empty_cache()


def _P():
    import paper_1910_00643_amd as P
    return P


LISTS = [  # lengths, hq, hk, dim, window, sinks
    ([0] * 300 + [70] + [0] * 300, 2, 1, 64, None, 0),             # sequences of nothing around one
    ([3] * 255 + [130], 1, 1, 64, None, 0),                        # as many as one look covers
    ([3] * 256 + [130], 1, 1, 64, None, 0),
    ([1] * 600, 4, 4, 32, None, 0),
    ([1] * 1023 + [90], 1, 1, 32, None, 0),                        # more than a thousand sequences
    ([2, 0, 5] * 1000 + [90, 0, 0, 3], 2, 1, 32, None, 0),
    ([0] * 1500 + [70] + [1] * 1500, 1, 1, 64, 9, 1),
    ([1, 1, 1, 1900], 4, 1, 64, None, 0),                          # one far longer than the average
    ([1, 1, 1, 1900], 4, 1, 64, 100, 2),
    ([2100], 2, 1, 128, 1000, 1500),                               # more sinks than window
    ([500], 3, 1, 64, 1 << 40, 1 << 40),                           # a window and sinks past every length
    ([65, 64, 63], 1, 1, 64, 64, 1),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", LISTS, ids=lambda c: f"{len(c[0])}x{max(c[0])} {c[1:]}")
def test_lists_of_sequences(case, dtype):
    lengths, hq, hk, dim, window, sinks = case
    g = torch.Generator(device=DEV).manual_seed(31)
    n = sum(lengths)
    q = U.rows(g, n, hq, dim, dtype, times=2.0)
    k, v, gout = (U.rows(g, n, h, dim, dtype) for h in (hk, hk, hq))
    at = U.offsets_of(lengths)
    offsets = torch.tensor(at, device=DEV)
    op = _P().Attention(dim, dtype=dtype, window=window, sinks=sinks)
    out, lse = op.forward(q, k, v, offsets)
    got = op.backward(gout, q, k, v, out, lse, offsets)
    checked = {}
    for i, m in enumerate(lengths):
        if not m or checked.setdefault(m, 0) > 3:       # a few of equal ones
            continue
        checked[m] += 1
        s = slice(at[i], at[i + 1])
        want, tol = U.dense(q[s], k[s], v[s], dtype, window=window, sinks=sinks, g=gout[s])
        for name, x in zip(("out", "lse", "dq", "dk", "dv"), (out, lse, *got)):
            U.near(x[s], want[name], tol[name], name)
    assert all(x.isfinite().all() for x in (out, *got))


@pytest.mark.parametrize("offsets", [[0, 90, 40, 130], [-50, 20, 20, 10 ** 15], [10 ** 12, 10 ** 13, 0, 5], [0, -1, -2, -3]], ids=str)
def test_offsets_of_no_meaning_reach_nothing_outside(offsets):
    """What they give is of no meaning; rows beside the arrays stay as they were."""
    g = torch.Generator(device=DEV).manual_seed(32)
    whole = [torch.full((330, 2, 64), 5.0, device=DEV) for _ in range(4)]
    q, k, v = (torch.randn(130, 2, 64, device=DEV, generator=g) for _ in range(3))
    at = torch.tensor(offsets, device=DEV)
    op = _P().Attention(64, dtype="f32", window=30, sinks=1)
    out, lse = op.forward(q, k, v, at, out=whole[0][100:230])
    op.backward(q, q, k, v, out, lse, at)
    pages = torch.randint(-3, 40, (3, 9), dtype=torch.int32, device=DEV, generator=g)
    lengths = torch.tensor([10 ** 15, -7, 2 ** 31], device=DEV)
    kc, vc = (torch.randn(20, 16, 2, 64, device=DEV, generator=g) for _ in range(2))
    paged = _P().PagedAttention(64, _P().rotary_table(64, 32, device=DEV), dtype="f32")
    paged.append(k, v, kc, vc, pages, torch.tensor([70, 3, 200], device=DEV), at, q=q, q_out=whole[1][100:230])
    window = _P().PagedAttention(64, dtype="f32", window=40)
    window.forward(q, kc, vc, pages, torch.tensor([70, -7, 200], device=DEV), at, out=whole[2][100:230])
    window.forward(q[:2], kc, vc, pages, lengths, at.clamp(0, 2), out=whole[3][100:102])
    torch.cuda.synchronize()
    for x, used in zip(whole, (130, 130, 130, 2)):
        assert (x[:100] == 5).all() and (x[100 + used:] == 5).all()


def test_thousands_of_running_sequences():
    """Append and a step of single tokens, some of whose keys are cut into pieces."""
    g = torch.Generator(device=DEV).manual_seed(35)
    batch, page = 2500, 16
    new = [1 if i % 3 else 0 for i in range(batch)]
    lengths = [3000 if i == 1700 else 1 + i % 40 for i in range(batch)]
    held = [-(-m // page) for m in lengths]
    order = torch.randperm(sum(held), device=DEV, generator=g).int()
    pages = torch.full((batch, max(held)), -1, dtype=torch.int32, device=DEV)
    row = torch.repeat_interleave(torch.arange(batch), torch.tensor(held)).to(DEV)
    column = torch.cat([torch.arange(m) for m in held]).to(DEV)
    pages[row, column] = order
    kc, vc = (torch.randn(sum(held), page, 1, 64, device=DEV, generator=g) for _ in range(2))
    q, k, v = (torch.randn(sum(new), h, 64, device=DEV, generator=g) for h in (2, 1, 1))
    n, at = torch.tensor(lengths, device=DEV), torch.tensor(U.offsets_of(new), device=DEV)
    op = _P().PagedAttention(64, dtype="f32")
    op.append(k, v, kc, vc, pages, n, at)
    out = op.forward(q, kc, vc, pages, n, at)
    for b in [i for i in range(batch) if new[i] and (i < 5 or i > batch - 6 or i % 200 == 100 or i == 1700)]:
        j, s = torch.arange(lengths[b], device=DEV), slice(int(at[b]), int(at[b]) + 1)
        place = pages[b, j // page].long()
        assert torch.equal(kc[place[-1], (lengths[b] - 1) % page], k[s][0])
        want, tol = U.dense(q[s], kc[place, j % page], vc[place, j % page], "f32")
        U.near(out[s], want["out"], tol["out"] * 1.01, "out")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_transposed_heads_and_broadcast_keys(dtype):
    """[heads][tokens] in memory, and keys of one head for all tokens at stride 0."""
    g = torch.Generator(device=DEV).manual_seed(33)
    q = torch.randn(4, 100, 64, device=DEV, generator=g).to(U.TD[dtype]).transpose(0, 1)
    k = torch.randn(2, 100, 64, device=DEV, generator=g).to(U.TD[dtype]).transpose(0, 1)
    v = torch.randn(1, 2, 64, device=DEV, generator=g).to(U.TD[dtype]).expand(100, 2, 64)
    op, at = _P().Attention(64, dtype=dtype), torch.tensor([0, 100], device=DEV)
    out, lse = op.forward(q, k, v, at)
    gout = torch.randn(100, 4, 64, device=DEV, generator=g).to(U.TD[dtype])
    dq, dk, dv = op.backward(gout, q, k, v, out, lse, at)
    want, tol = U.dense(q, k, v, dtype, g=gout)
    for name, x in zip(("out", "lse", "dq", "dk", "dv"), (out, lse, dq, dk, dv)):
        U.near(x, want[name], tol[name], name)


def test_two_graphs_replayed_side_by_side():
    """Captured calls have workspaces of their own."""
    g = torch.Generator(device=DEV).manual_seed(34)
    op = _P().PagedAttention(64)
    n, at = torch.tensor([5000, 70], device=DEV), torch.tensor([0, 1, 2], device=DEV)
    pages = torch.arange(640, dtype=torch.int32, device=DEV).view(2, 320)
    kc, vc = (torch.randn(640, 16, 2, 64, device=DEV, generator=g).bfloat16() for _ in range(2))
    qs = [torch.randn(2, 8, 64, device=DEV, generator=g).bfloat16() for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = [op.forward(q, kc, vc, pages, n, at) for q in qs]
    torch.cuda.current_stream().wait_stream(side)
    graphs, held = [], []
    for q in qs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held.append(op.forward(q, kc, vc, pages, n, at))
        graphs.append(graph)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("at,tokens,keys", [
    ([0, 100], 100, 50), ([0, 30, 100], 100, 40), ([0, 30, 100], 50, 100), ([0, 30, 100], 130, 100), ([0, 30, 100], 20, 25),
    ([0, 900], 900, 40), ([0, 900], 40, 900), ([0, 50], 0, 50), ([0, 50], 50, 0),
], ids=str)
def test_one_list_over_unequal_numbers_of_rows(at, tokens, keys, dtype):
    """The same tensor as both lists: each is cut by its own number of rows, and the rows behind them, NaN here, are not
    read."""
    g = torch.Generator(device=DEV).manual_seed(36)

    def inside(n, heads):
        x = torch.full((n + 1000, heads, 64), float("nan"), device=DEV, dtype=U.TD[dtype])
        x[:n] = torch.randn(n, heads, 64, device=DEV, generator=g)
        return x[:n]

    q, k, v, gout = inside(tokens, 4), inside(keys, 2), inside(keys, 2), inside(tokens, 4)
    op, offsets = _P().Attention(64, dtype=dtype), torch.tensor(at, device=DEV)
    out, lse = op.forward(q, k, v, offsets, offsets)
    got = op.backward(gout, q, k, v, out, lse, offsets, offsets)
    for name, x in zip(("out", "dq", "dk", "dv"), (out, *got)):
        assert x.isfinite().all(), name
    for lo, hi in zip(at, at[1:]):
        a, b = slice(min(lo, tokens), min(hi, tokens)), slice(min(lo, keys), min(hi, keys))
        want, tol = U.dense(q[a], k[b], v[b], dtype, g=gout[a])
        for name, x, s in zip(("out", "lse", "dq", "dk", "dv"), (out, lse, *got), (a, a, a, b, b)):
            U.near(x[s], want[name], tol[name], name)
