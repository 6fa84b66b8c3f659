"""Attention over packed sequences, forward, against its definition in 64 bits (attention_utils.py has the
tolerances)."""
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


CASES = [  # query lengths, key lengths (None: the same), hq, hk, dim, causal, window, sinks, pad, offset
    ([1], None, 1, 1, 64, True, None, 0, 0, 0),
    ([1, 2, 3], None, 2, 1, 32, True, None, 0, 0, 0),
    ([0, 5, 0, 64, 0], None, 2, 2, 64, True, None, 0, 0, 0),
    ([63, 64, 65], None, 4, 2, 128, True, None, 0, 0, 0),
    ([130], None, 3, 1, 96, True, None, 0, 0, 0),
    ([257, 31], None, 2, 2, 72, False, None, 0, 0, 0),
    ([200], None, 2, 1, 80, True, 17, 0, 0, 0),
    ([200, 333], None, 2, 1, 64, True, 17, 3, 0, 0),
    ([300], None, 1, 1, 128, True, 64, 100, 0, 0),       # sinks past several tiles
    ([150], None, 1, 1, 64, False, 20, 5, 0, 0),
    ([150], None, 1, 1, 64, False, 20, 120, 0, 0),       # sinks ahead of queries
    ([70], None, 2, 2, 192, True, 1, 0, 0, 0),           # a query sees itself alone
    ([70], None, 2, 1, 256, True, None, 0, 0, 0),
    ([70], None, 2, 1, 160, True, 33, 1, 0, 0),
    ([5, 70], [9, 200], 2, 1, 64, True, None, 0, 0, 0),  # more keys than queries
    ([90, 40], [30, 0], 2, 1, 64, True, None, 0, 0, 0),  # queries that see nothing
    ([90, 7], [30, 300], 2, 1, 64, False, 25, 0, 0, 0),
    ([90, 7], [30, 300], 2, 1, 64, False, 25, 2, 0, 0),
    ([33, 50], None, 3, 3, 33, True, None, 0, 0, 0),     # odd heads
    ([33, 50], None, 2, 1, 1, True, 9, 1, 0, 0),
    ([40], None, 2, 1, 100, True, None, 0, 0, 0),
    ([66], None, 2, 2, 64, True, None, 0, 3, 0),         # rows of odd strides
    ([66], None, 2, 2, 64, True, None, 0, 0, 1),         # data off by one element
    ([66], None, 2, 2, 64, True, None, 0, 8, 0),
    ([12] * 130, None, 2, 1, 64, True, None, 0, 0, 0),   # more sequences than lanes
    ([11, 23], None, 71, 1, 64, True, None, 0, 0, 0),    # one key head for many
    ([1000], None, 7, 1, 64, True, None, 0, 0, 0),
    ([19], None, 9, 3, 128, True, None, 0, 0, 0),
]


def _inputs(case, dtype, seed=3, rest=0):
    lengths, k_lengths, hq, hk, dim, causal, window, sinks, pad, offset = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    n, m = sum(lengths) + rest, sum(k_lengths or lengths) + rest
    q = U.rows(g, n, hq, dim, dtype, pad, offset, 2.0)
    k, v = (U.rows(g, m, hk, dim, dtype, pad, offset) for _ in range(2))
    at = torch.tensor(U.offsets_of(lengths), device=DEV)
    k_at = None if k_lengths is None else torch.tensor(U.offsets_of(k_lengths), device=DEV)
    op = _P().Attention(dim, dtype=dtype, causal=causal, window=window, sinks=sinks)
    return op, q, k, v, at, k_at, g


def _each(case):
    lengths, k_lengths = case[0], case[1] or case[0]
    a, b = U.offsets_of(lengths), U.offsets_of(k_lengths)
    for i in range(len(lengths)):
        yield slice(a[i], a[i + 1]), slice(b[i], b[i + 1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward(case, dtype):
    op, q, k, v, at, k_at, _ = _inputs(case, dtype)
    out, lse = op.forward(q, k, v, at, k_at)
    for a, b in _each(case):
        if a.start == a.stop:
            continue
        want, tol = U.dense(q[a], k[b], v[b], dtype, causal=case[5], window=case[6], sinks=case[7])
        U.near(out[a], want["out"], tol["out"], "out")
        U.near(lse[a], want["lse"], tol["lse"], "lse")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_behind_the_last_sequence(dtype):
    case = ([40, 33], None, 2, 1, 64, True, None, 0, 0, 0)
    op, q, k, v, at, _, _ = _inputs(case, dtype, rest=77)
    q[73:], k[73:], v[73:] = float("nan"), float("nan"), float("nan")
    out, lse = op.forward(q, k, v, at)
    assert (out[73:] == 0).all() and (lse[73:] == float("-inf")).all() and out[:73].isfinite().all()
    kept = torch.full_like(q, 7.0)
    same, lse2 = op.forward(q, k, v, at, out=kept)
    assert same is kept and (kept[73:] == 7).all() and torch.equal(kept[:73], out[:73]) and torch.equal(lse, lse2)


@pytest.mark.parametrize("wild", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("window,sinks", [(None, 0), (40, 2)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_not_seen_has_no_part(dtype, window, sinks, wild):
    """A wild value leaves the queries that do not see its key as they were."""
    case = ([150, 90], None, 2, 1, 64, True, window, sinks, 0, 0)
    op, q, k, v, at, _, _ = _inputs(case, dtype)
    clean, clean_lse = op.forward(q, k, v, at)
    v[100, 0, 5] = wild
    k[101, 0, 6] = float("nan")
    out, lse = op.forward(q, k, v, at)
    sees = U.visible(150, 150, True, window, sinks)
    v_seen, k_seen = sees[:, 100], sees[:, 101]
    none = ~(v_seen | k_seen)
    assert none.any() and torch.equal(out[:150][none], clean[:150][none]) and torch.equal(lse[:150][none], clean_lse[:150][none])
    assert torch.equal(out[150:], clean[150:])
    only = v_seen & ~k_seen
    assert not out[:150][only][:, :, 5].isfinite().any()
    rest = [d for d in range(64) if d != 5]
    assert torch.equal(out[:150][only][:, :, rest], clean[:150][only][:, :, rest])
    assert out[:150][k_seen].isnan().all()


def test_large_scores():
    """Scores of 300 and more apart: the sums neither overflow nor lose the largest."""
    g = torch.Generator(device=DEV).manual_seed(5)
    q, k, v = (torch.randn(300, 1, 64, device=DEV, generator=g) for _ in range(3))
    q, k = q * 12, k * 12
    op = _P().Attention(64, dtype="f32")
    out, lse = op.forward(q, k, v, torch.tensor([0, 300], device=DEV))
    want, tol = U.dense(q, k, v, "f32")
    assert want["lse"].abs().max() > 300
    U.near(out, want["out"], tol["out"], "out")
    U.near(lse, want["lse"], tol["lse"], "lse")


def test_two_calls_give_the_same_bits():
    case = ([700, 3, 255], None, 8, 2, 128, True, 100, 4, 0, 0)
    op, q, k, v, at, _, _ = _inputs(case, "bf16")
    a, b = op.forward(q, k, v, at), op.forward(q, k, v, at)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_another_stream():
    case = ([300, 40], None, 2, 1, 64, True, None, 0, 0, 0)
    op, q, k, v, at, _, _ = _inputs(case, "bf16")
    want = op.forward(q, k, v, at)[0]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = op.forward(q, k, v, at)[0]
    side.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("times", [1.0, 60.0])      # 60: a later score is some 300 higher, by which the sums are brought down
@pytest.mark.parametrize("where", [0, 3, 100, 290])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_an_infinite_value_that_is_seen_stays_one(dtype, where, times):
    case = ([300], None, 2, 1, 64, True, None, 0, 0, 0)
    op, q, k, v, at, _, _ = _inputs(case, dtype)
    q[:] = q[250, 0]
    k[200] = times * q[250, 0]
    want, want_lse = op.forward(q, k, v, at)
    v[where, 0, 5], v[where, 0, 40] = float("inf"), -float("inf")
    want[where:, :, 5], want[where:, :, 40] = float("inf"), -float("inf")
    out, lse = op.forward(q, k, v, at)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
