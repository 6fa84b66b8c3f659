"""The paged cache: what append writes and leaves, and attention of the newest tokens over it, against the
definitions in 64 bits (attention_utils.py has attention's tolerances).  Append: two products and a sum in
fp32, 3 * 2^-24 of |u| + |v|, and the result's own rounding."""
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


def _paged(g, lengths, page, spare=3, columns=None):
    held = [-(-max(n, 0) // page) for n in lengths]
    order = torch.randperm(sum(held) + spare, device=DEV, generator=g).int()
    pages = torch.full((len(lengths), max(held + [1]) if columns is None else columns), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(held):
        pages[b, :n] = order[at:at + n]
        at += n
    return pages, sum(held) + spare


def _gathered(cache, pages, length):
    page = cache.shape[1]
    j = torch.arange(length, device=DEV)
    return cache[pages[j // page].long(), j % page]


CASES = [  # new tokens, lengths, hq, hk, dim, page, window, sinks
    ([1], [1], 1, 1, 64, 16, None, 0),
    ([1], [1000], 8, 2, 128, 16, None, 0),
    ([1, 1, 1], [5, 700, 64], 4, 4, 64, 64, None, 0),
    ([1, 0, 3, 40], [130, 50, 3, 90], 4, 2, 128, 32, None, 0),
    ([1, 1], [3000, 257], 4, 1, 96, 1, None, 0),             # pages of one position
    ([1, 1], [3000, 257], 4, 1, 64, 1024, None, 0),
    ([1, 2], [3000, 257], 4, 1, 72, 16, 100, 0),
    ([1, 70], [3000, 1257], 4, 1, 128, 16, 100, 4),
    ([33], [2050], 2, 2, 80, 128, 500, 70),
    ([129], [129], 2, 1, 256, 64, None, 0),
    ([1], [4001], 2, 1, 192, 64, None, 0),
    ([2], [4001], 71, 1, 64, 64, None, 0),
    ([5], [300], 2, 1, 33, 16, None, 0),
    ([1] * 70, [i * 7 + 1 for i in range(70)], 2, 1, 64, 16, None, 0),
    ([9], [4], 2, 1, 64, 16, None, 0),                       # more new tokens than positions: the first see nothing
    ([3, 2], [0, 900], 2, 1, 64, 16, None, 0),
    ([1], [20000], 2, 1, 128, 16, None, 0),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward(case, dtype):
    new, lengths, hq, hk, dim, page, window, sinks = case
    g = torch.Generator(device=DEV).manual_seed(11)
    pages, total = _paged(g, lengths, page)
    kc, vc = (torch.randn(total, page, hk, dim, device=DEV, generator=g).to(U.TD[dtype]) for _ in range(2))
    q = U.rows(g, sum(new), hq, dim, dtype, times=2.0)
    op = _P().PagedAttention(dim, dtype=dtype, window=window, sinks=sinks)
    at = U.offsets_of(new)
    out, lse = op.forward(q, kc, vc, pages, torch.tensor(lengths, device=DEV), torch.tensor(at, device=DEV), return_lse=True)
    for b, m in enumerate(lengths):
        if not new[b]:
            continue
        mine = slice(at[b], at[b + 1])
        k, v = _gathered(kc, pages[b], m), _gathered(vc, pages[b], m)
        want, tol = U.dense(q[mine], k, v, dtype, window=window, sinks=sinks)
        # pieces of the keys are joined: a rounding more for each
        U.near(out[mine], want["out"], tol["out"] * 1.01, "out")
        U.near(lse[mine], want["lse"], tol["lse"], "lse")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pages_outside_the_cache(dtype):
    """What a query sees of them is no number; what none sees is not looked at."""
    g = torch.Generator(device=DEV).manual_seed(12)
    lengths, page = [400, 400, 400, 400], 16
    pages, total = _paged(g, lengths, page)
    kc, vc = (torch.randn(total, page, 2, 64, device=DEV, generator=g).to(U.TD[dtype]) for _ in range(2))
    q = U.rows(g, 40, 4, 64, dtype)
    n, at = torch.tensor(lengths, device=DEV), torch.tensor([0, 10, 20, 30, 40], device=DEV)
    op = _P().PagedAttention(64, dtype=dtype, window=50, sinks=3)
    want = op.forward(q, kc, vc, pages, n, at)
    assert want.isfinite().all()
    bad = pages.clone()
    bad[0, 5:15] = total            # no query sees positions 80 to 239
    bad[1, 10] = 2 ** 31 - 1
    bad[2, 24] = -5                 # the last 16 positions: queries from 384 on see them, which are all but none
    bad[3, 0] = total               # the sinks
    got = op.forward(q, kc, vc, bad, n, at)
    assert torch.equal(got[:20], want[:20])
    assert got[20:30].isnan().all() and got[30:40].isnan().all()
    # a length that the table's row does not reach
    short = op.forward(q, kc, vc, pages[:, :24].contiguous(), n, at)
    assert short.isnan().all()


@pytest.mark.parametrize("window,sinks", [(None, 0), (90, 0), (90, 3), (90, 1 << 40)])
def test_lengths_far_past_the_table(window, sinks):
    """Queries at positions without pages have NaN, and no more is walked than the table holds."""
    g = torch.Generator(device=DEV).manual_seed(20)
    kc, vc = (torch.randn(20, 16, 1, 64, device=DEV, generator=g).bfloat16() for _ in range(2))
    pages = torch.arange(20, dtype=torch.int32, device=DEV).view(1, 20)
    q = U.rows(g, 300, 4, 64, "bf16")
    op = _P().PagedAttention(64, window=window, sinks=sinks)
    at = torch.tensor([0, 300], device=DEV)
    for length in (2 ** 29 + 7, 2 ** 62, 10 ** 6, 650):
        assert op.forward(q, kc, vc, pages, torch.tensor([length], device=DEV), at).isnan().all()
    # the first 20 of these are at positions 300 to 319, which have pages
    out = op.forward(q, kc, vc, pages, torch.tensor([600], device=DEV), at)
    want, tol = U.dense(q[:20], _gathered(kc, pages[0], 320), _gathered(vc, pages[0], 320), "bf16", window=window, sinks=sinks)
    U.near(out[:20], want["out"], tol["out"] * 1.01, "out")
    assert out[20:].isnan().all()


def test_one_bad_page_leaves_the_queries_before_it():
    g = torch.Generator(device=DEV).manual_seed(13)
    pages, total = _paged(g, [64], 16)
    kc, vc = (torch.randn(total, 16, 1, 64, device=DEV, generator=g) for _ in range(2))
    q = U.rows(g, 64, 1, 64, "f32")
    op = _P().PagedAttention(64, dtype="f32")
    n, at = torch.tensor([64], device=DEV), torch.tensor([0, 64], device=DEV)
    want = op.forward(q, kc, vc, pages, n, at)
    pages[0, 2] = -1
    got = op.forward(q, kc, vc, pages, n, at)
    assert torch.equal(got[:32], want[:32]) and got[32:].isnan().all()


def test_what_lies_behind_a_sequence_in_its_page_has_no_part():
    g = torch.Generator(device=DEV).manual_seed(14)
    pages, total = _paged(g, [37, 900], 64)
    kc, vc = (torch.randn(total, 64, 2, 128, device=DEV, generator=g).bfloat16() for _ in range(2))
    q = U.rows(g, 6, 8, 128, "bf16")
    op = _P().PagedAttention(128)
    n, at = torch.tensor([37, 900], device=DEV), torch.tensor([0, 5, 6], device=DEV)
    want = op.forward(q, kc, vc, pages, n, at)
    for c in (kc, vc):
        c[pages[0, 0], 37:] = float("nan")
        c[pages[1, 14], 4:] = float("inf")
        c[-1] = c[-1]
    assert torch.equal(op.forward(q, kc, vc, pages, n, at), want)


def _turned(x, table, position, interleaved):
    x = x.double()
    r = 2 * table.shape[2]
    rows = table.double()[position.clamp(0, table.shape[0] - 1)]
    c, s = rows[:, 0][:, None], rows[:, 1][:, None]
    gone = ((position < 0) | (position >= table.shape[0]))[:, None, None]
    u, v = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    a, b = (u * c - v * s).masked_fill(gone, float("nan")), (u * s + v * c).masked_fill(gone, float("nan"))
    size = (u.abs() + v.abs())
    both, sizes = (torch.stack([a, b], -1).flatten(-2), torch.stack([size, size], -1).flatten(-2)) if interleaved else \
        (torch.cat([a, b], -1), torch.cat([size, size], -1))
    return torch.cat([both, x[..., r:]], -1), torch.cat([sizes, torch.zeros_like(x[..., r:])], -1)


APPENDS = [  # new tokens, lengths, hq, hk, hv, dim, rot, page, pad, offset
    ([1], [1], 1, 1, 1, 64, 64, 16, 0, 0),
    ([1, 1, 1, 1], [17, 300, 64, 65], 8, 2, 2, 128, 128, 16, 0, 0),
    ([0, 5, 0, 130, 1], [9, 5, 0, 200, 1], 4, 2, 2, 128, 64, 64, 0, 0),
    ([40, 3], [40, 90], 2, 1, 2, 72, 72, 1, 0, 0),
    ([40, 3], [40, 90], 2, 2, 1, 80, 0, 32, 8, 0),
    ([40, 3], [40, 90], 3, 3, 3, 33, 20, 16, 0, 0),
    ([40, 3], [40, 90], 2, 1, 1, 64, 32, 16, 3, 0),
    ([40, 3], [40, 90], 2, 1, 1, 64, 64, 16, 0, 1),
    ([7], [5], 2, 1, 1, 64, 64, 16, 0, 0),                  # two positions below zero
    ([700], [1500], 2, 1, 1, 256, 256, 128, 0, 0),          # past the table's end
    ([1] * 200, list(range(1, 201)), 1, 1, 1, 32, 32, 16, 0, 0),
    ([2] + [0] * 100 + [2], [2] + [0] * 100 + [5], 1, 1, 1, 8, 8, 4, 0, 0),
    ([3], [40], 1, 1, 1, 1, 0, 16, 0, 0),
]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", APPENDS, ids=str)
def test_append(case, dtype, interleaved):
    new, lengths, hq, hk, hv, dim, rot, page, pad, offset = case
    g = torch.Generator(device=DEV).manual_seed(15)
    pages, total = _paged(g, lengths, page)
    kc = torch.randn(total, page, hk, dim, device=DEV, generator=g).to(U.TD[dtype])
    vc = torch.randn(total, page, hv, dim, device=DEV, generator=g).to(U.TD[dtype])
    tokens, rest = sum(new), 5
    q, k, v = (U.rows(g, tokens + rest, h, dim, dtype, pad, offset) for h in (hq, hk, hv))
    table = _P().rotary_table(1400, rot // 2, device=DEV) if rot else None
    op = _P().PagedAttention(dim, table, dtype=dtype, interleaved=interleaved)
    at = U.offsets_of(new)
    position = torch.cat([torch.arange(m - n, m, device=DEV) for n, m in zip(new, lengths)])
    want_k, want_v = kc.double(), vc.double()
    tol_k = torch.zeros_like(want_k)
    own = 0.0 if dtype == "f32" else U.H["bf16"]

    def turned(x):
        if not rot:
            return x.double(), torch.zeros_like(x, dtype=torch.float64)
        y, size = _turned(x, table, position, interleaved)
        return y, 3 * 2.0 ** -24 * size + own * y.abs() * (size > 0)

    yk, ek = turned(k[:tokens])
    for t in range(tokens):
        b = max(i for i in range(len(new)) if at[i] <= t and new[i])
        p = int(position[t])
        if p < 0:
            continue
        row = int(pages[b, p // page])
        want_k[row, p % page], want_v[row, p % page] = yk[t], v[t].double()
        tol_k[row, p % page] = ek[t]
    got_q = op.append(k, v, kc, vc, pages, torch.tensor(lengths, device=DEV), torch.tensor(at, device=DEV), q=q)
    U.near(kc, want_k, tol_k, "k_cache")
    assert torch.equal(vc.double(), want_v)
    yq, eq = turned(q[:tokens])
    U.near(got_q[:tokens], yq, eq, "q")
    assert (got_q[tokens:] == 0).all()
    kept = torch.full_like(q, 3.0)
    assert op.append(k, v, kc, vc, pages, torch.tensor(lengths, device=DEV), torch.tensor(at, device=DEV), q=q, q_out=kept) is kept
    assert (kept[tokens:] == 3).all() and torch.equal(kept[:tokens].nan_to_num(9), got_q[:tokens].nan_to_num(9))


def test_append_in_place_and_to_bad_pages():
    g = torch.Generator(device=DEV).manual_seed(16)
    pages, total = _paged(g, [64, 64, 64], 16)
    table = _P().rotary_table(64, 32, device=DEV)
    op = _P().PagedAttention(64, table)
    # keys and values beside each other in one array
    both = torch.randn(total, 2, 16, 2, 64, device=DEV, generator=g).bfloat16()
    before = both.clone()
    kc, vc = both[:, 0], both[:, 1]
    q, k, v = (U.rows(g, 6, h, 64, "bf16") for h in (4, 2, 2))
    pages[1, 3], pages[2, 3] = total, -1
    n, at = torch.tensor([64, 64, 65], device=DEV), torch.tensor([0, 2, 4, 6], device=DEV)
    fresh = op.append(k, v, kc, vc, pages, n, at, q=q)
    written = both.clone()
    assert op.append(k, v, kc, vc, pages, n, at, q=q, q_out=q) is q and torch.equal(q.nan_to_num(9), fresh.nan_to_num(9))
    assert torch.equal(both, written)
    row = pages[0, 3].item()
    assert torch.equal(vc[row, 14:], v[:2])
    written[row, :, 14:] = before[row, :, 14:]
    assert torch.equal(written, before)


def test_a_serving_run_equals_attention_over_the_whole_text():
    """Prompts in chunks, then single tokens: append and paged attention step by step give what attention
    over the packed texts gives."""
    g = torch.Generator(device=DEV).manual_seed(17)
    P, hq, hk, dim, page = _P(), 8, 2, 64, 16
    lengths = [150, 83, 201]
    table = P.rotary_table(256, dim // 2, device=DEV)
    flat = torch.randn(sum(lengths), hq + 2 * hk, dim, device=DEV, generator=g)
    q, k, v = flat.split([hq, hk, hk], 1)
    at = U.offsets_of(lengths)
    positions = torch.cat([torch.arange(n, device=DEV) for n in lengths])
    rotate = P.HeadNormRotary(dim, table, dtype="f32", norm=False)
    tq, tk = rotate.forward(q, k, positions)
    whole = P.Attention(dim, dtype="f32", window=60, sinks=2)
    want, _ = whole.forward(tq, tk, v, torch.tensor(at, device=DEV))
    op = P.PagedAttention(dim, table, dtype="f32", window=60, sinks=2)
    pages, total = _paged(g, lengths, page)
    kc, vc = (torch.full((total, page, hk, dim), float("nan"), device=DEV) for _ in range(2))
    got = torch.empty_like(want)
    done = [0, 0, 0]
    for step in range(200):
        new = [min(n - d, 70 if step == 0 else 33 if step == 1 and b else 1) for b, (n, d) in enumerate(zip(lengths, done))]
        if not any(new):
            break
        rows = torch.cat([torch.arange(at[b] + done[b], at[b] + done[b] + new[b], device=DEV) for b in range(3)])
        done = [d + n for d, n in zip(done, new)]
        n, o = torch.tensor(done, device=DEV), torch.tensor(U.offsets_of(new), device=DEV)
        turned = op.append(k[rows], v[rows], kc, vc, pages, n, o, q=q[rows])
        got[rows] = op.forward(turned, kc, vc, pages, n, o)
    for b, n in enumerate(lengths):
        mine = slice(at[b], at[b + 1])
        _, tol = U.dense(tq[mine], tk[mine], v[mine], "f32", window=60, sinks=2)
        # both sides are off, and so are the turned queries and keys: 3 roundings of each score's factors
        U.near(got[mine], want[mine].double(), 3 * tol["out"], "out")


@pytest.mark.parametrize("dtype", ["bf16"])
def test_captured_steps_are_replayed(dtype):
    """Append and attention of single tokens in a graph, on lengths and pages that change between replays."""
    g = torch.Generator(device=DEV).manual_seed(18)
    P = _P()
    op = P.PagedAttention(128, P.rotary_table(4096, 64, device=DEV), dtype=dtype)
    lengths = [3000, 17, 900]
    pages, total = _paged(g, [4000] * 3, 16)
    kc, vc = (torch.randn(total, 16, 2, 128, device=DEV, generator=g).to(U.TD[dtype]) for _ in range(2))
    q, k, v = (torch.randn(3, h, 128, device=DEV, generator=g).to(U.TD[dtype]) for h in (8, 2, 2))
    n, o = torch.tensor(lengths, device=DEV), torch.arange(4, device=DEV)

    def step():
        return op.forward(op.append(k, v, kc, vc, pages, n, o, q=q), kc, vc, pages, n, o)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for turn in range(4):
        n += 1
        k.copy_(torch.randn(k.shape, device=DEV, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        got = held.clone()
        assert torch.equal(got, step()), turn


def test_an_offset_past_32_bits():
    """The last pages of a cache of more than 2^32 bytes, and of more than 2^32 elements."""
    page, hk, dim = 1024, 8, 128
    total = (2 ** 32) // (page * hk * dim) + 3
    kc = torch.empty(total, page, hk, dim, dtype=torch.bfloat16, device=DEV)
    vc = torch.empty_like(kc)
    g = torch.Generator(device=DEV).manual_seed(19)
    ids = [total - 1, 0, total - 2, 2 ** 31 // (page * hk * dim) + 1]
    for c in (kc, vc):
        for i in ids:
            c[i] = torch.randn(page, hk, dim, device=DEV, generator=g)
    pages = torch.tensor([ids], dtype=torch.int32, device=DEV)
    q, k, v = (torch.randn(2, h, dim, device=DEV, generator=g).bfloat16() for h in (8, 8, 8))
    n, o = torch.tensor([2050], device=DEV), torch.tensor([0, 2], device=DEV)
    op = _P().PagedAttention(dim)
    op.append(k, v, kc, vc, pages, n, o)
    assert torch.equal(kc[total - 2, :2], k) and torch.equal(vc[total - 2, :2], v)
    out = op.forward(q, kc, vc, pages, n, o)
    want, tol = U.dense(q, _gathered(kc, pages[0], 2050), _gathered(vc, pages[0], 2050), "bf16")
    U.near(out, want["out"], tol["out"] * 1.01, "out")


def _far_apart(dtype, seqs, times, seed=21):
    """Sequences whose keys are cut into 40 pieces (one sequence) or 24: one key of each, at position 100 i + 5000, has a
    score far above the others."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    length = 20000 if seqs == 1 else 12000
    pages, total = _paged(g, [length] * seqs, 16)
    kc, vc = (torch.randn(total, 16, 1, 64, device=DEV, generator=g).to(U.TD[dtype]) for _ in range(2))
    q = U.rows(g, seqs, 4, 64, dtype)
    q[:] = q[:, :1]                       # all heads of a token ask for the same key
    for i in range(seqs):
        at = 5000 + 100 * i
        kc[pages[i, at // 16], at % 16] = times * q[i, 0]
    n, at = torch.full((seqs,), length, device=DEV), torch.arange(seqs + 1, device=DEV)
    from paper_1910_00643_amd import attention as A
    cfg = A.slowmo_attention_config(dtype=A._DTYPE[dtype], head_dim=64, causal=1, clear_rest=0, scale=0.125)
    assert A.lib().slowmo_paged_attention_bytes(cfg, A.slowmo_pages(seqs, pages.shape[1], pages.shape[1]), seqs, 4,
                                                A.slowmo_cache(None, 1, 16, total)) > 0
    return q, kc, vc, pages, n, at, total


@pytest.mark.parametrize("times", [0.0, 60.0])   # scores of up to 1 and of some 300 beside it: weights underflow
@pytest.mark.parametrize("seqs", [1, 40])        # many pieces, joined by a workgroup a row, and few, by a wave
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_page_missing_in_one_of_several_pieces(dtype, seqs, times):
    q, kc, vc, pages, n, at, total = _far_apart(dtype, seqs, times)
    op = _P().PagedAttention(64, dtype=dtype)
    want, want_lse = op.forward(q, kc, vc, pages, n, at, return_lse=True)
    assert want.isfinite().all() and want_lse.isfinite().all()
    bad = pages.clone()
    gone = torch.arange(seqs, device=DEV) % 3 == 0
    for i in range(0, seqs, 3):
        bad[i, (i * 31) % 600] = total if i % 2 else -1
    got, lse = op.forward(q, kc, vc, bad, n, at, return_lse=True)
    assert got[gone].isnan().all() and lse[gone].isnan().all()
    assert torch.equal(got[~gone], want[~gone]) and torch.equal(lse[~gone], want_lse[~gone])
    # the table ends before the sequence: the positions without a column are the last ones
    got, lse = op.forward(q, kc, vc, pages[:, :-1].contiguous(), n, at, return_lse=True)
    assert got.isnan().all() and lse.isnan().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_missing_page_marks_the_queries_that_see_it(dtype):
    """And their lse, in one piece or several: no other row."""
    g = torch.Generator(device=DEV).manual_seed(22)
    pages, total = _paged(g, [9000], 16)
    kc, vc = (torch.randn(total, 16, 2, 64, device=DEV, generator=g).to(U.TD[dtype]) for _ in range(2))
    q = U.rows(g, 300, 4, 64, dtype)
    n, at = torch.tensor([9000], device=DEV), torch.tensor([0, 300], device=DEV)
    position = torch.arange(8700, 9000, device=DEV)
    for window, sinks, column in ((None, 0, 550), (None, 0, 3), (100, 0, 548), (4000, 20, 1), (4000, 20, 300)):
        op = _P().PagedAttention(64, dtype=dtype, window=window, sinks=sinks)
        want, want_lse = op.forward(q, kc, vc, pages, n, at, return_lse=True)
        bad = pages.clone()
        bad[0, column] = -1
        j = torch.arange(column * 16, column * 16 + 16, device=DEV)[None]
        p = position[:, None]
        gone = ((j <= p) & ((p - j < (window or 1 << 30)) | (j < sinks))).any(1)
        got, lse = op.forward(q, kc, vc, bad, n, at, return_lse=True)
        assert got[gone].isnan().all() and lse[gone].isnan().all(), (window, sinks, column)
        assert torch.equal(got[~gone], want[~gone]) and torch.equal(lse[~gone], want_lse[~gone]), (window, sinks, column)


@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")], ids=str)
@pytest.mark.parametrize("times", [0.0, 60.0])
@pytest.mark.parametrize("seqs", [1, 40])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_wild_value_in_one_of_several_pieces(dtype, seqs, times, what):
    """A value that a query sees has a part in its result, however small its probability; no other element has."""
    q, kc, vc, pages, n, at, total = _far_apart(dtype, seqs, times)
    op = _P().PagedAttention(64, dtype=dtype)
    want, want_lse = op.forward(q, kc, vc, pages, n, at, return_lse=True)
    for i in range(0, seqs, 3):
        vc[pages[i, (i * 31) % 600], 5, 0, 7 + i % 50] = what
        want[i, :, 7 + i % 50] = what
    got, lse = op.forward(q, kc, vc, pages, n, at, return_lse=True)
    assert torch.equal(got.nan_to_num(1e30), want.nan_to_num(1e30)) and torch.equal(got.isnan(), want.isnan())
    assert torch.equal(lse, want_lse)


@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 0), (60, 5)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_without_a_causal_mask(dtype, window, sinks):
    """Through the C entry, which takes it: new tokens that see each other, in one piece and in several."""
    from paper_1910_00643_amd import attention as A
    g = torch.Generator(device=DEV).manual_seed(23)
    new, lengths = [40, 0, 3, 1], [100, 7, 9000, 50]
    pages, total = _paged(g, lengths, 16)
    kc, vc = (torch.randn(total, 16, 2, 64, device=DEV, generator=g).to(U.TD[dtype]) for _ in range(2))
    q = U.rows(g, 44, 4, 64, dtype)
    at = U.offsets_of(new)
    n, o = torch.tensor(lengths, device=DEV), torch.tensor(at, device=DEV)
    out, lse = torch.empty_like(q), torch.empty(44, 4, device=DEV)
    cfg = A.slowmo_attention_config(dtype=A._DTYPE[dtype], head_dim=64, causal=0, clear_rest=0, scale=0.125, window=window, sinks=sinks)
    table = A.slowmo_pages(4, pages.shape[1], pages.shape[1], pages.data_ptr(), n.data_ptr(), o.data_ptr())
    k, v = (A.slowmo_cache(c.data_ptr(), 2, 16, total, 16 * 128, 128, 64) for c in (kc, vc))
    rows = [A.slowmo_heads(x.data_ptr(), 4, 256, 64) for x in (q, out)]
    need = A.lib().slowmo_paged_attention_bytes(cfg, table, 44, 4, k)
    space = torch.empty(need, dtype=torch.uint8, device=DEV)
    assert A.lib().slowmo_paged_attention(cfg, table, 44, rows[0], k, v, rows[1], lse.data_ptr(), space.data_ptr() if need else None,
                                          need, torch.cuda.current_stream().cuda_stream or None) == 0
    for b, m in enumerate(lengths):
        s = slice(at[b], at[b + 1])
        want, tol = U.dense(q[s], _gathered(kc, pages[b], m), _gathered(vc, pages[b], m), dtype, causal=False, window=window or None,
                            sinks=sinks)
        U.near(out[s], want["out"], tol["out"] * 1.01, "out")
        U.near(lse[s], want["lse"], tol["lse"], "lse")


@pytest.mark.parametrize("columns", [300, 8192])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_table_far_wider_than_its_sequences(dtype, columns):
    """As a program has it that captures its steps for the longest text it accepts: how the keys are cut follows the table's
    width."""
    g = torch.Generator(device=DEV).manual_seed(24)
    new, lengths = [1, 1, 0, 1, 30, 1], [4700, 17, 5, 1, 900, 2048]
    pages, total = _paged(g, lengths, 16, columns=columns)
    kc, vc = (torch.randn(total, 16, 2, 128, device=DEV, generator=g).to(U.TD[dtype]) for _ in range(2))
    q = U.rows(g, sum(new), 8, 128, dtype, times=2.0)
    at = U.offsets_of(new)
    for window, sinks in ((None, 0), (700, 4)):
        op = _P().PagedAttention(128, dtype=dtype, window=window, sinks=sinks)
        out, lse = op.forward(q, kc, vc, pages, torch.tensor(lengths, device=DEV), torch.tensor(at, device=DEV), return_lse=True)
        for b, m in enumerate(lengths):
            s = slice(at[b], at[b + 1])
            if not new[b]:
                continue
            want, tol = U.dense(q[s], _gathered(kc, pages[b], m), _gathered(vc, pages[b], m), dtype, window=window, sinks=sinks)
            U.near(out[s], want["out"], tol["out"] * 1.01, "out")
            U.near(lse[s], want["lse"], tol["lse"], "lse")
