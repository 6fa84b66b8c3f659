"""Performance cases of attention: over packed sequences, as training and prompts run
it (forward, and forward with backward), and over a paged cache of keys and values, as
running sequences read it; and of what fills that cache, the append of new keys and
values with the position rotation applied on the way.

`run` is one call of an operator (a training case: forward and backward).  Where `own`
is false it is computed from elementary torch operations in 32 bits, rounded once at
the end; where it is true by the framework's kernels.

Attention.  For each sequence, its query i lies at position p = i + (keys - queries) of
its keys; query heads share key heads in groups of hq / hk.  Key j is visible if
    (j <= p or not causal) and (j < sinks or |p - j| < window, window = 0: any distance),
    s_ij = scale q_i . k_j,   out_i = sum_j e^(s_ij - lse_i) v_j,   lse_i = log sum_j e^(s_ij)
over the visible ones.  Backward, with P = e^(s - lse) and g the output's gradient:
    dV = P^T g,   dS = P (g V^T - rowsum(P g V^T)),   dQ = scale dS K,   dK = scale dS^T Q.

Paged cache.  Position j of sequence b lies in row j mod `page` of page pages[b, j / page];
lengths[b] counts the positions, those of the call's new tokens, the last ones, included.
Append: the first `rot` elements of a new key (and query) head, in pairs (i, i + rot / 2),
are turned by the angle of the token's position, u' = u cos - v sin, v' = u sin + v cos,
and the key and the value go to their place; all other places stay as they are.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEVICE = "cuda:0"
BASE = 10000.0
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


# ---- the listed cases ---------------------------------------------------------

def listed():
    return [
        # Training step of the Transformer-big decoder (16 heads of 64) on a batch of sentences.
        _packed("train_sentences", "train", batch=160, shortest=5, longest=100, hq=16, hk=16, dim=64),
        # The smallest training step: the example's (32 sequences of 48 tokens, 4 heads of 32, fp32).
        _packed("train_example_f32", "train", batch=32, shortest=48, longest=48, hq=4, hk=4, dim=32, dtype="f32"),
        # Training on one long text, key heads shared by four.
        _packed("train_long", "train", batch=1, shortest=8192, longest=8192, hq=16, hk=4, dim=128),
        # Training on texts of many lengths with a window and first tokens that stay visible,
        # heads of 96, shared by three.
        _packed("train_window_ragged", "train", batch=7, shortest=301, longest=4001, hq=12, hk=4, dim=96,
                window=512, sinks=3),
        # One long prompt, all of it visible.
        _packed("forward_prompt", "forward", batch=1, shortest=8192, longest=8192, hq=32, hk=8, dim=128),
        # A longer one with a window.
        _packed("forward_prompt_window", "forward", batch=1, shortest=16384, longest=16384, hq=8, hk=2, dim=128,
                window=2048, sinks=4),
        # Patches of images (14 x 14 and one token more, 61 images), every one sees every one, fp32.
        _packed("forward_images_f32", "forward", batch=61, shortest=197, longest=197, hq=16, hk=16, dim=72,
                dtype="f32", causal=False),
        # The new tokens of 48 running sequences, one each, to their places: the smallest call.
        _cached("append_token_step", "append", batch=48, new_shortest=1, new_longest=1, shortest=60, longest=1500),
        # Prompts of 24 new sequences.
        _cached("append_prompts", "append", batch=24, new_shortest=17, new_longest=2100, shortest=0, longest=0),
        # One step of 48 running sequences, a token each.
        _cached("paged_token_step", "paged", batch=48, new_shortest=1, new_longest=1, shortest=101, longest=16000),
        # One sequence alone, its cache long.
        _cached("paged_token_long", "paged", batch=1, new_shortest=1, new_longest=1, shortest=131069, longest=131069,
                page=16),
        # Chunks of prompts beside single tokens, with a window and first tokens that stay visible.
        _cached("paged_chunks_window", "paged", batch=6, new_shortest=1, new_longest=512, shortest=700,
                longest=19999, hq=16, hk=4, window=4096, sinks=4),
    ]


def _packed(name, op, **more):
    c = {"op": op, "batch": 1, "shortest": 1, "longest": 1, "hq": 1, "hk": 1, "dim": 64, "dtype": "bf16",
         "causal": True, "window": 0, "sinks": 0}
    c.update(more)
    return {"name": name, **c} if name else c


def _cached(name, op, **more):
    """new_shortest..new_longest new tokens of each sequence behind shortest..longest cached ones."""
    c = {"op": op, "batch": 1, "new_shortest": 1, "new_longest": 1, "shortest": 0, "longest": 0, "hq": 32, "hk": 8,
         "dim": 128, "rot": 128, "dtype": "bf16", "causal": True, "window": 0, "sinks": 0, "page": 64}
    c.update(more)
    return {"name": name, **c} if name else c


def _between(case, lo, hi, salt):
    """The lengths of a case's sequences: spread evenly between lo and hi, in an order of no meaning."""
    n = case["batch"]
    out = [lo + (hi - lo) * i // (n - 1) for i in range(n)] if n > 1 else [hi]
    random.Random(1000003 * n + 17 * hi + salt).shuffle(out)
    return out


def _lengths(case):
    """(new tokens, all keys) of every sequence."""
    if case["op"] in ("train", "forward"):
        n = _between(case, case["shortest"], case["longest"], 0)
        return n, n
    new = _between(case, case["new_shortest"], case["new_longest"], 1)
    return new, [a + b for a, b in zip(new, _between(case, case["shortest"], case["longest"], 2))]


MOST_SCORES, MOST_KEYS, MOST_FLOPS = 2_200_000_000, 120_000_000, 6.0e11


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sequences of one token to some 10 000, one to 200 of them; caches of
    up to 130 000 tokens behind one new token to 2000; heads of 32 to 256, one to 32, shared
    by one to eight."""
    while True:
        op = rng.choice(["train", "forward", "append", "paged", "paged"])
        hk = _log_int(rng, 1, 16)
        more = {"hk": hk, "hq": hk * rng.choice([1, 1, 2, 4, 7, 8]),
                "dim": rng.choice([32, 64, 64, 72, 80, 96, 128, 128, 128, 160, 192, 256]),
                "dtype": rng.choice(["bf16", "bf16", "f32"]), "batch": _log_int(rng, 1, 200)}
        if rng.random() < 0.4:
            more.update(window=_log_int(rng, 16, 8192), sinks=rng.choice([0, 1, 4, 100]))
        if op in ("train", "forward"):
            hi = _log_int(rng, 1, 12000)
            c = _packed(None, op, shortest=rng.choice([hi, max(1, hi // 10)]), longest=hi,
                        causal=rng.random() < 0.75, **more)
        else:
            single = rng.random() < 0.5
            hi = _log_int(rng, 16, 130000)
            c = _cached(None, op, new_shortest=1, new_longest=1 if single else _log_int(rng, 1, 2000),
                        shortest=rng.choice([hi, hi // 10, hi // 10]), longest=hi, page=rng.choice([16, 32, 64, 128]),
                        **more)
            c["rot"] = rng.choice([c["dim"], c["dim"], c["dim"] // 2])
        new, keys = _lengths(c)
        scores = c["batch"] * c["hq"] * max(new) * max(keys) * (1 if op != "train" else 2)
        rows = c["batch"] * max(keys) * c["hk"] * c["dim"]
        tokens = sum(new) * (c["hq"] + c["hk"]) * c["dim"]
        if op == "append":
            scores, rows = 0, 2 * rows
        most = {"flops": MOST_FLOPS / (1 if c["dtype"] == "bf16" else 8)}
        if scores <= MOST_SCORES and rows <= MOST_KEYS and tokens <= MOST_KEYS and work(c)["flops"] <= most["flops"]:
            return c


# ---- what a program has in hand -------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    c = dict(case)
    new, keys = _lengths(c)
    dt, d, tokens = DTYPE[c["dtype"]], c["dim"], sum(new)
    offsets = [0]
    for n in new:
        offsets.append(offsets[-1] + n)
    s = {"case": c, "new": new, "keys": keys, "offsets": torch.tensor(offsets, device=DEVICE)}
    # queries, keys and values lie beside each other in one projection's output; scores have a
    # deviation of 1.7, so that a row has a few large weights and a broad rest
    flat = torch.randn(tokens, c["hq"] + 2 * c["hk"], d, device=DEVICE, generator=g)
    flat[:, :c["hq"]] *= 1.7
    flat = flat.to(dt)
    s["q"], s["k"], s["v"] = flat.split([c["hq"], c["hk"], c["hk"]], 1)
    window = c["window"] or None
    if c["op"] in ("train", "forward"):
        if c["op"] == "train":
            s["g"] = torch.randn(tokens, c["hq"], d, device=DEVICE, generator=g).to(dt)
        if own:     # the layer's settings, as a program keeps them
            from paper_1910_00643_amd import Attention
            s["handle"] = Attention(d, dtype=c["dtype"], causal=c["causal"], window=window, sinks=c["sinks"])
        return s
    page = c["page"]
    held = [-(-n // page) for n in keys]
    total = sum(held) + 3
    order = torch.randperm(total, device=DEVICE, generator=g)
    pages = torch.full((c["batch"], max(held)), -1, dtype=torch.int32)
    row = torch.cat([torch.full((n,), b) for b, n in enumerate(held)])
    column = torch.cat([torch.arange(n) for n in held])
    pages = pages.to(DEVICE)
    pages[row.to(DEVICE), column.to(DEVICE)] = order[:sum(held)].int()
    s["pages"], s["lengths"] = pages, torch.tensor(keys, device=DEVICE)
    for name in ("k_cache", "v_cache"):
        s[name] = torch.randn(total, page, c["hk"], d, device=DEVICE, generator=g).to(dt)
    table = None
    if c["op"] == "append":
        pairs = c["rot"] // 2
        freq = BASE ** (-torch.arange(pairs, dtype=torch.float64, device=DEVICE) / pairs)
        angle = torch.arange(max(keys), dtype=torch.float64, device=DEVICE)[:, None] * freq
        table = s["table"] = torch.stack([angle.cos(), angle.sin()], 1).float().contiguous()
    if own:
        from paper_1910_00643_amd import PagedAttention
        s["handle"] = PagedAttention(d, table, dtype=c["dtype"], window=window, sinks=c["sinks"])
    return s


# ---- one pass -------------------------------------------------------------------

def run(s):
    c = s["case"]
    op = c["op"]
    if own:
        h = s["handle"]
        if op == "append":
            q = h.append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["pages"], s["lengths"], s["offsets"], q=s["q"])
            return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
        if op == "paged":
            return {"out": h.forward(s["q"], s["k_cache"], s["v_cache"], s["pages"], s["lengths"], s["offsets"])}
        out, lse = h.forward(s["q"], s["k"], s["v"], s["offsets"])
        if op == "forward":
            return {"out": out, "lse": lse}
        dq, dk, dv = h.backward(s["g"], s["q"], s["k"], s["v"], out, lse, s["offsets"])
        return {"out": out, "dq": dq, "dk": dk, "dv": dv}
    if op == "append":
        return _plain_append(s)
    return _plain_attention(s)


# ---- the plain forms ------------------------------------------------------------

def _plain_rows(s):
    """For every new token: its sequence, its place in it, its position."""
    t = torch.arange(s["q"].shape[0], device=DEVICE)
    b = torch.searchsorted(s["offsets"], t, right=True) - 1
    i = t - s["offsets"][b]
    new = s["offsets"][1:] - s["offsets"][:-1]
    at = i if s["case"]["op"] in ("train", "forward") else i + s["lengths"][b] - new[b]
    return b, i, at


def _plain_append(s):
    c = s["case"]
    b, _, at = _plain_rows(s)
    page = c["page"]
    where = s["pages"][b, at // page] * page + at % page
    cos, sin = s["table"][at, 0][:, None], s["table"][at, 1][:, None]
    r = c["rot"]

    def turn(x):
        u, v = x[..., :r // 2].float(), x[..., r // 2:r].float()
        return torch.cat([u * cos - v * sin, u * sin + v * cos, x[..., r:].float()], -1).to(x.dtype)

    s["k_cache"].view(-1, c["hk"], c["dim"]).index_copy_(0, where, turn(s["k"]))
    s["v_cache"].view(-1, c["hk"], c["dim"]).index_copy_(0, where, s["v"])
    return {"q": turn(s["q"]), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attention(s):
    """Sequences side by side, padded to the longest."""
    c = s["case"]
    hk, group, d, batch = c["hk"], c["hq"] // c["hk"], c["dim"], c["batch"]
    longest, keys = max(s["new"]), max(s["keys"])
    b, i, at = _plain_rows(s)

    def padded(x, heads):       # [tokens, heads * group, d] -> [batch, hk, group, longest, d]
        y = torch.zeros(batch, longest, *x.shape[1:], device=DEVICE)
        y[b, i] = x.float()
        return y.view(batch, longest, hk, heads // hk, d).permute(0, 2, 3, 1, 4).contiguous()

    q = padded(s["q"], c["hq"]).view(batch, hk, group * longest, d)
    if c["op"] == "paged":
        j = torch.arange(keys, device=DEVICE)
        place = s["pages"][:, j // c["page"]].clamp(min=0)
        k, v = (s[n][place, j % c["page"]].float().permute(0, 2, 1, 3).contiguous() for n in ("k_cache", "v_cache"))
        n_keys = s["lengths"]
    else:
        k, v = (padded(s[n], hk).view(batch, hk, keys, d) for n in ("k", "v"))
        n_keys = s["offsets"][1:] - s["offsets"][:-1]
    n_new = s["offsets"][1:] - s["offsets"][:-1]
    p = (torch.arange(longest, device=DEVICE) + (n_keys - n_new)[:, None])[:, :, None]     # [batch, longest, 1]
    j = torch.arange(keys, device=DEVICE)[None, None]
    seen = j < n_keys[:, None, None]
    if c["causal"]:
        seen = seen & (j <= p)
    if c["window"]:
        seen = seen & ((j < c["sinks"]) | ((p - j).abs() < c["window"]))
    scale = d ** -0.5
    w = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale).view(batch, hk, group, longest, keys)
    w.masked_fill_(~seen[:, None, None], float("-inf"))
    top = w.amax(-1, keepdim=True).clamp_(min=-1e30)
    w.sub_(top).exp_()
    total = w.sum(-1, keepdim=True)
    w.div_(total.clamp(min=1e-30))
    w = w.view(batch, hk, group * longest, keys)

    def packed(x):              # back to [tokens, hq or hk, d]
        x = x.view(batch, hk, -1, longest, d).permute(0, 3, 1, 2, 4).reshape(batch, longest, -1, d)
        return x[b, i].to(s["q"].dtype)

    out = packed(torch.matmul(w, v))
    if c["op"] == "paged":
        return {"out": out}
    if c["op"] == "forward":
        lse = (total.log() + top).view(batch, c["hq"], longest).transpose(1, 2)
        return {"out": out, "lse": lse[b, i]}
    g = padded(s["g"], c["hq"]).view(batch, hk, group * longest, d)
    dv = torch.matmul(w.transpose(2, 3).contiguous(), g)
    ds = torch.matmul(g, v.transpose(2, 3).contiguous())
    ds.sub_((w * ds).sum(-1, keepdim=True)).mul_(w).mul_(scale)
    return {"out": out, "dq": packed(torch.matmul(ds, k)),
            "dk": packed(torch.matmul(ds.transpose(2, 3).contiguous(), q)), "dv": packed(dv)}


# ---- what a pass cannot do without ------------------------------------------------

def _visible(n, keys, c):
    """(visible pairs, keys that some query sees) of a sequence."""
    if not n:
        return 0, 0
    far, w = keys - n, c["window"] or 1 << 40
    pairs = seen = 0
    if c["causal"] and not c["window"]:
        return n * far + n * (n + 1) // 2, keys
    for p in range(far, keys):
        lo, hi = max(0, p - w + 1), p + 1 if c["causal"] else min(keys, p + w)
        pairs += hi - lo + min(c["sinks"], lo) + max(0, min(c["sinks"], keys if not c["causal"] else p + 1) - max(hi, 0))
    first = max(0, far - w + 1)
    seen = keys - first + min(c["sinks"], first)
    return pairs, seen


def work(case):
    c = case
    new, keys = _lengths(c)
    d, e, tokens = c["dim"], SIZE[c["dtype"]], sum(new)
    if c["op"] == "append":
        rows = tokens * (c["hq"] + 2 * c["hk"]) * d
        table = min(tokens, max(keys)) * c["rot"] * 4
        return {"bytes": float(2 * rows * e + table + 8 * tokens), "flops": float(3 * tokens * (c["hq"] + c["hk"]) * c["rot"])}
    both = [_visible(n, m, c) for n, m in zip(new, keys)]
    pairs, seen = sum(p for p, _ in both), sum(m for _, m in both)
    rows = tokens * c["hq"] * d
    if c["op"] == "train":
        # two products forward, five backward; out is written and read again
        return {"bytes": float(e * (5 * rows + 4 * seen * c["hk"] * d) + 8 * tokens * c["hq"]),
                "flops": float(14 * pairs * c["hq"] * d)}
    lse = 4 * tokens * c["hq"] if c["op"] == "forward" else 0
    return {"bytes": float(e * (2 * rows + 2 * seen * c["hk"] * d) + lse), "flops": float(4 * pairs * c["hq"] * d)}


# ---- the definitions in 64 bits ---------------------------------------------------

def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    c = s["case"]
    if c["op"] == "append":
        return _exact_append(s)
    group, starts = c["hq"] // c["hk"], s["offsets"].tolist()
    shape = s["q"].shape
    out = torch.empty(shape, dtype=torch.float64, device=DEVICE)
    lse = torch.empty(shape[:2], dtype=torch.float64, device=DEVICE)
    dq, dk, dv = (torch.zeros(s[n].shape, dtype=torch.float64, device=DEVICE) for n in ("q", "k", "v"))
    for b, (n, keys) in enumerate(zip(s["new"], s["keys"])):
        at = slice(starts[b], starts[b] + n)
        if c["op"] == "paged":
            held = s["pages"][b, :-(-keys // c["page"])]
            k, v = (s[x][held].flatten(0, 1)[:keys].double() for x in ("k_cache", "v_cache"))
        else:
            k, v = s["k"][at].double(), s["v"][at].double()
        q = s["q"][at].double()
        place = torch.arange(keys, device=DEVICE)
        # heads side by side as far as memory goes, queries in pieces of at most 4096
        heads = max(1, min(c["hk"], 100_000_000 // max(1, group * min(n, 4096) * keys)))
        for h in range(0, c["hk"], heads):
            mine = slice(h, min(h + heads, c["hk"]))
            theirs = slice(mine.start * group, mine.stop * group)
            kt, vt = (x[:, mine].transpose(0, 1).contiguous().repeat_interleave(group, 0) for x in (k, v))
            for first in range(0, n, 4096):
                last = min(first + 4096, n)
                p = torch.arange(keys - n + first, keys - n + last, device=DEVICE)[:, None]
                hidden = torch.zeros(last - first, keys, dtype=torch.bool, device=DEVICE)
                if c["causal"]:
                    hidden |= place > p
                if c["window"]:
                    hidden |= (place >= c["sinks"]) & ((place - p >= c["window"]) | (p - place >= c["window"]))
                rows = slice(at.start + first, at.start + last)
                qt = q[first:last, theirs].transpose(0, 1).contiguous()
                score = torch.bmm(qt, kt.transpose(1, 2).contiguous()) / math.sqrt(c["dim"])
                score = score.masked_fill(hidden, float("-inf"))
                norm = torch.logsumexp(score, -1, keepdim=True)
                prob = torch.exp(score - norm)
                got = torch.bmm(prob, vt)
                out[rows, theirs] = got.transpose(0, 1)
                lse[rows, theirs] = norm[..., 0].t()
                if c["op"] != "train":
                    continue
                g = s["g"][rows, theirs].double().transpose(0, 1).contiguous()
                # d loss / d score through the softmax: prob (g . v - g . out)
                back = prob * (torch.bmm(g, vt.transpose(1, 2).contiguous()) - (g * got).sum(-1, keepdim=True))
                back = back / math.sqrt(c["dim"])
                dq[rows, theirs] = torch.bmm(back, kt).transpose(0, 1)
                for total, x in ((dk, torch.bmm(back.transpose(1, 2).contiguous(), qt)),
                                 (dv, torch.bmm(prob.transpose(1, 2).contiguous(), g))):
                    total[at, mine] += x.unflatten(0, (-1, group)).sum(1).transpose(0, 1)
    if c["op"] == "train":
        return {"out": out, "dq": dq, "dk": dk, "dv": dv}
    return {"out": out, "lse": lse} if c["op"] == "forward" else {"out": out}


def _exact_append(s):
    """The rotation as a complex product, sequence by sequence."""
    c, r = s["case"], s["case"]["rot"]
    starts, table = s["offsets"].tolist(), s["table"].double()
    angle = torch.complex(table[:, 0], table[:, 1])

    def turned(x, first):
        x = x.double()
        z = torch.complex(x[..., :r // 2], x[..., r // 2:r]) * angle[first:first + x.shape[0], None]
        return torch.cat([z.real, z.imag, x[..., r:]], -1)

    q = torch.empty(s["q"].shape, dtype=torch.float64, device=DEVICE)
    caches = [s["k_cache"].double(), s["v_cache"].double()]
    for b, (n, keys) in enumerate(zip(s["new"], s["keys"])):
        at = slice(starts[b], starts[b] + n)
        q[at] = turned(s["q"][at], keys - n)
        place = torch.arange(keys - n, keys, device=DEVICE)
        page, row = s["pages"][b, place // c["page"]], place % c["page"]
        caches[0][page, row] = turned(s["k"][at], keys - n)
        caches[1][page, row] = s["v"][at].double()
    return {"q": q, "k_cache": caches[0], "v_cache": caches[1]}
