"""Gradients of rows of hundreds to thousands of keys whose g V^T and g . out all but cancel: keys and values that have
something in common, and rows whose weight lies on few keys.  bf16, against 64 bits.

Tolerances, in the terms of attention_utils.py (h = 2^-24, es and ep its errors of a score and a probability).  g . out is to be
that of the unrounded probabilities: with d0 what `out`, rounded, gives of it, off by r = |g| . (sum P |v| 2^-8 + 2^-8 |out|),
it is d0 + sum P (g . v - d0), which is off by
    ed = sum P e1 + (ep + keys h) sum P (|g . v - g . out| + r),   e1 = (D + 2) h (|g| |v| + |g| |out|),
so that dS is off by P (e1 + ed) + |dS| ep before it is rounded to bf16.  These sum up as they are, twice over.  The roundings of dS
are within 2^-8 |dS| each and independent of each other, so that a sum of them passes 8 times 2^-8 sqrt(sum (dS k)^2) with a
probability of 2 exp(-32), 3e-14 (Hoeffding's bound); their sum in the worst case, sqrt(keys) times as much, would let pass
what this is about."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import attention_utils as U  # noqa: E402

DEV = U.DEV


@pytest.fixture(autouse=True)
def _free_gpu_memory():
    yield
    torch.cuda.empty_cache()


def _want(q, k, v, g, window, sinks):
    """{"dq", "dk"} and {name: tolerance} of one sequence."""
    n, hq, d = q.shape
    m, hk, _ = k.shape
    group, scale, h, own = hq // hk, d ** -0.5, 2.0 ** -24, 2.0 ** -8
    hidden = ~U.visible(n, m, True, window, sinks)
    q, k, v, g = (x.double().transpose(0, 1).contiguous() for x in (q, k, v, g))
    k, v = k.repeat_interleave(group, 0), v.repeat_interleave(group, 0)
    kt, vt = (x.transpose(1, 2).contiguous() for x in (k, v))
    s = torch.bmm(q, kt) * scale
    es = (scale * (d + 2) * h * torch.bmm(q.abs(), kt.abs()) + 3 * h * s.abs()).masked_fill(hidden, 0.0)
    p = torch.softmax(s.masked_fill(hidden, -math.inf), -1)
    ep = es + es.amax(-1, keepdim=True) + (m + 6) * h
    out, dp = torch.bmm(p, v), torch.bmm(g, vt)
    delta = (g * out).sum(-1, keepdim=True)
    ds = p * (dp - delta)
    r = (g.abs() * (torch.bmm(p, v.abs()) + out.abs())).sum(-1, keepdim=True) * own
    e1 = (d + 2) * h * (torch.bmm(g.abs(), vt.abs()) + (g.abs() * out.abs()).sum(-1, keepdim=True))
    ed = (p * e1).sum(-1, keepdim=True) + ((ep + m * h) * p * ((dp - delta).abs() + r)).sum(-1, keepdim=True)
    eds = p * (e1 + ed) + ds.abs() * ep

    def shared(x):
        return x.unflatten(0, (hk, group)).sum(1).transpose(0, 1)

    dst, edst = (x.transpose(1, 2).contiguous() for x in (ds, eds))
    rows = group * n
    got = {"dq": scale * torch.bmm(ds, k).transpose(0, 1), "dk": scale * shared(torch.bmm(dst, q))}
    eq = torch.bmm(eds + (m + 4) * h * ds.abs(), k.abs()).transpose(0, 1)
    ek = shared(torch.bmm(edst + (rows + 4) * h * dst.abs(), q.abs()))
    tol = {"dq": 2 * (scale * eq + (own + h) * got["dq"].abs()) +
           8 * own * scale * torch.bmm(ds.square(), k.square()).sqrt().transpose(0, 1),
           "dk": 2 * (scale * ek + (own + h) * got["dk"].abs()) +
           8 * own * scale * shared(torch.bmm(dst.square(), q.square())).sqrt()}
    return got, tol


CASES = [  # query lengths, key lengths (None: the same), hq, hk, dim, window, sinks
    ([2000], None, 2, 1, 128, None, 0),
    ([300, 700, 1300], None, 2, 2, 64, None, 0),
    ([257, 321, 2], None, 4, 1, 96, None, 0),            # a tile more than four, and four
    ([1500], None, 2, 1, 128, 700, 4),
    ([700], [1900], 2, 1, 72, None, 0),
    ([900], None, 2, 1, 32, None, 0),
    ([800], None, 2, 1, 192, None, 0),
    ([800], None, 2, 1, 256, None, 0),
    ([600], None, 3, 1, 33, None, 0),
]


@pytest.mark.parametrize("times,of_k,of_v", [(1.7, 5.0, 3.0), (1.7, 0.0, 3.0), (1.0, 1.0, 1.0), (4.0, 0.0, 0.0), (8.0, 2.0, 0.0)])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_rows_that_cancel(case, times, of_k, of_v):
    lengths, k_lengths, hq, hk, dim, window, sinks = case
    g = torch.Generator(device=DEV).manual_seed(51)
    n, m = sum(lengths), sum(k_lengths or lengths)
    q, gout = U.rows(g, n, hq, dim, "bf16", times=times), U.rows(g, n, hq, dim, "bf16")
    k, v = ((torch.randn(m, hk, dim, device=DEV, generator=g) + by * torch.randn(1, hk, dim, device=DEV, generator=g)).bfloat16()
            for by in (of_k, of_v))
    import paper_1910_00643_amd as P
    op, at = P.Attention(dim, window=window, sinks=sinks), U.offsets_of(lengths)
    k_at = U.offsets_of(k_lengths or lengths)
    lists = [torch.tensor(x, device=DEV) for x in (at, k_at)]
    out, lse = op.forward(q, k, v, *lists)
    got = dict(zip(("dq", "dk"), op.backward(gout, q, k, v, out, lse, *lists)))
    for i in range(len(lengths)):
        a, b = slice(at[i], at[i + 1]), slice(k_at[i], k_at[i + 1])
        want, tol = _want(q[a], k[b], v[b], gout[a], window, sinks)
        U.near(got["dq"][a], want["dq"], tol["dq"], "dq")
        U.near(got["dk"][b], want["dk"], tol["dk"], "dk")
