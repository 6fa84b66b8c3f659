"""Attention by its definition in 64 bits, for the tests, with what fp32 and bf16 may be off.

Tolerances, element by element.  A rounding is off by at most half a step: h = 2^-24 of the value in fp32,
2^-8 in bf16.  A score is a sum of D products, its factors exact in fp32 (bf16 products are): D + 2 roundings of at most
sum |q k| each, and 3 of its own size on the way to the exponent (the scale, its conversion to base 2, the fused
subtraction):  es = scale (D + 2) h sum |q k| + 3 h |s|.  A probability is off by its score's error, by the
row's sum's (at most the largest of the row's es, and a rounding per key) and 6 roundings more (exponential 2, logarithm,
quotient, sums joined):  ep = es + max es + (keys + 6) h, relative, and, where it goes through bf16, 2^-8 more.
    out:  sum P |v| (ep + keys h)            + the result's own rounding
    lse:  max es + (keys + 6) h + 3 h |lse|
    dV:   sum P |g| (ep + queries h)         + its own rounding
    dS:   P (D + 2) h (sum |g v| + sum |g out|) + P sum |g| eo + |dS| ep, eo: what `out`, which is read
          again, is off;  dQ, dK: the products of that with |K|, |Q|, a rounding per term, and their own rounding.
Each is taken twice over (terms of second order, the order of sums)."""
import math

import torch

DEV = "cuda:0"
H = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
TD = {"f32": torch.float32, "bf16": torch.bfloat16}


def visible(n, m, causal, window, sinks, device=DEV):
    p = torch.arange(m - n, m, device=device)[:, None]
    j = torch.arange(m, device=device)[None]
    ok = torch.ones(n, m, dtype=torch.bool, device=device)
    if causal:
        ok &= j <= p
    if window:
        ok &= ((p - j).abs() < window) | (j < sinks)
    return ok


def dense(q, k, v, dtype, *, scale=None, causal=True, window=None, sinks=0, g=None, mended=False):
    """One sequence: {"out", "lse"[, "dq", "dk", "dv"]} and {name: tolerance}.  q [n, hq, D], k and v [m, hk, D]."""
    n, hq, d = q.shape
    m, hk, _ = k.shape
    group, scale = hq // hk, d ** -0.5 if scale is None else scale
    h, own = 2.0 ** -24, 0.0 if dtype == "f32" else H["bf16"]
    ok = visible(n, m, causal, window, sinks, q.device)
    q, k, v = (x.double().transpose(0, 1).contiguous() for x in (q, k, v))
    k, v = k.repeat_interleave(group, 0), v.repeat_interleave(group, 0)
    kt = k.transpose(1, 2).contiguous()
    s = torch.bmm(q, kt) * scale
    es = scale * (d + 2) * h * torch.bmm(q.abs(), kt.abs()) + 3 * h * s.abs()
    es = es.masked_fill(~ok, 0.0)
    s = s.masked_fill(~ok, -math.inf)
    lse = torch.logsumexp(s, -1, keepdim=True) if m else torch.full((hq, n, 1), -math.inf, dtype=torch.float64, device=q.device)
    p = torch.exp(s - lse.masked_fill(lse == -math.inf, 0.0))
    top = es.amax(-1, keepdim=True) if m else torch.zeros_like(lse)
    ep = es + top + (m + 6) * h
    out = torch.bmm(p, v)
    got = {"out": out.transpose(0, 1), "lse": lse[..., 0].t()}
    eo = torch.bmm(p * (ep + own + m * h), v.abs())
    tol = {"out": (2 * (eo + (own + h) * out.abs())).transpose(0, 1),
           "lse": (2 * (top + (m + 6) * h + 3 * h * lse.abs().nan_to_num(0, 0, 0)))[..., 0].t()}
    if g is None:
        return got, tol
    g = g.double().transpose(0, 1).contiguous()
    vt = v.transpose(1, 2).contiguous()
    ds = p * (torch.bmm(g, vt) - (g * out).sum(-1, keepdim=True))
    eo = eo + (own + h) * out.abs()
    # rows of few keys: g . out is mended by the sum of dS, to 2^-12 of the sum of |dS|
    left = ds.abs().sum(-1, keepdim=True) * 2.0 ** -12 if mended else (g.abs() * eo).sum(-1, keepdim=True)
    eds = p * ((d + 2) * h * (torch.bmm(g.abs(), vt.abs()) + (g.abs() * out.abs()).sum(-1, keepdim=True)) + left) + \
        ds.abs() * (ep + own)

    def shared(x):
        return x.unflatten(0, (hk, group)).sum(1).transpose(0, 1)

    pt, dst, edst = (x.transpose(1, 2).contiguous() for x in (p, ds, eds))
    dq = scale * torch.bmm(ds, k)
    got.update(dq=dq.transpose(0, 1), dk=shared(scale * torch.bmm(dst, q)), dv=shared(torch.bmm(pt, g)))
    rows = group * n
    eq = scale * torch.bmm(eds + (m + 4) * h * ds.abs(), k.abs())
    ek = shared(scale * torch.bmm(edst + (rows + 4) * h * dst.abs(), q.abs()))
    ev = shared(torch.bmm((p * (ep + own + (rows + 4) * h)).transpose(1, 2).contiguous(), g.abs()))
    tol["dq"] = 2 * (eq.transpose(0, 1) + (own + h) * got["dq"].abs())
    tol["dk"] = 2 * (ek + (own + h) * got["dk"].abs())
    tol["dv"] = 2 * (ev + (own + h) * got["dv"].abs())
    return got, tol


def near(x, want, tol, what):
    x = x.double()
    same = (x == want) | (torch.isnan(x) & torch.isnan(want))
    off = (x - want).abs()
    bad = ~(same | (off <= tol + 1e-30))
    if bad.any():
        at = tuple(int(i) for i in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, the first at {at}: {x[at].item()} for "
                             f"{want[at].item()}, tolerance {tol[at].item() if tol.shape == x.shape else tol}")


def offsets_of(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def rows(g, tokens, heads, dim, dtype, pad=0, offset=0, times=1.0):
    """[tokens, heads, dim] inside wider rows, its data off by `offset` elements."""
    width = heads * dim + pad
    flat = torch.randn(tokens * width + offset, device=DEV, generator=g).mul_(times).to(TD[dtype])[offset:]
    return flat.view(tokens, width)[:, :heads * dim].unflatten(1, (heads, dim))
