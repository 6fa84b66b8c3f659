"""Performance cases of the operators a worker's local step needs around a
Transformer's matrices: orthogonalising an update by Newton-Schulz products (by
itself, and after the momentum of the SGD row of Table C.1), and the norm of
queries and keys for each head with the position rotation, forward and backward,
with one axis of positions or several.

`run` is one call of an operator.  Where `own` is false it is computed from
elementary torch operations in 32 bits, rounded once at the end; where it is true
by the framework's kernels.

Orthogonalising.  n <= k are the shorter and the longer side of a matrix U:
    X_0 = U / (|U|_F + eps),   A = X X^T (n x n),   X <- a X + (b A + c A A) X,  5 times,
    O = s X_5,  s by the matrix's shape.
With momentum:  M <- mu M + G,  U = G + mu M  (Nesterov).

Norm and rotation.  For each token and head, x of length D:
    y = w x / sqrt(mean(x^2) + eps)   (left out where a case has no norm),
then the first R elements in pairs (u, v) are turned by the angle of the pair's row
of the table: u' = u cos - v sin, v' = u sin + v cos.  The row is the token's
position along the axis the pair belongs to.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS = 5
NORM_EPS = 1e-7
HEAD_EPS = 1e-6
MU = 0.95
BASE = 10000.0
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- the listed cases ---------------------------------------------------------

def listed():
    return [
        # One small matrix, alone: a call is all launches and dependent products.
        _orth("orth_one_small", "128x96"),
        # The matrices of one encoder block of the Transformer-big configuration.
        _orth("orth_transformer_block", "4*1024x1024,4096x1024,1024x4096"),
        # ResNet-50's convolutions as matrices (output channels by inputs times window),
        # fp32 in and out: many sizes, most of them small, 147 columns at the odd end.
        _orth("orth_resnet50_f32", "resnet50", dtype="f32", out="f32"),
        # The experts of a mixture layer, equal matrices in one stacked tensor.
        _orth("orth_experts", "32*768x2560", scale="rms"),
        # The largest: one square matrix, fp32 gradients.
        _orth("orth_one_large", "8192x8192", dtype="f32", scale="rms"),
        # Local step of 4 workers on two encoder blocks of the Transformer-big
        # configuration, bf16 gradients as its benchmark has them.
        _orth("momentum_transformer_workers", "32*1024x1024,8*4096x1024,8*1024x4096",
              op="momentum", scale="rms"),
        # Local step of 8 workers on ResNet-18's convolutions and head, fp32.
        _orth("momentum_resnet18_workers_f32", "resnet18", op="momentum", copies=8, dtype="f32",
              out="f32"),
        # Training forward, Transformer-big heads (16 of 64), a batch of text.
        _head("head_forward_text", tokens=8192, hq=16, hk=16, dim=64, rot=64),
        # Training backward on long sequences with shared key heads.
        _head("head_backward_long", op="head_backward", tokens=32768, hq=32, hk=8, dim=128, rot=128),
        # Single tokens of 48 running sequences, keys written to their places in a cache.
        _head("head_token_step", op="head_token", tokens=48, hq=32, hk=8, dim=128, rot=128,
              rows=65536, cache=16384),
        # Patches of images: two axes, rotation without a norm, fp32, neighbouring pairs,
        # an odd number of tokens (14 x 14 patches and one token more, 61 images).
        _head("axes_forward_image_f32", tokens=61 * 197, hq=16, hk=16, dim=72, rot=72, dtype="f32",
              axes=2, norm=False, interleaved=True, rows=64),
        # Patches of video: three axes, part of the head rotated, backward.
        _head("axes_backward_video", op="head_backward", tokens=24 * 33 * 17, hq=24, hk=24, dim=128,
              rot=96, axes=3, rows=256),
    ]


def _orth(name, sizes, **more):
    c = {"op": "orthogonalize", "sizes": sizes, "copies": 1, "dtype": "bf16", "out": "bf16",
         "scale": "shape"}
    c.update(more)
    return {"name": name, **c} if name else c


def _head(name, **more):
    c = {"op": "head_forward", "tokens": 1, "hq": 1, "hk": 1, "dim": 64, "rot": 64, "dtype": "bf16",
         "axes": 1, "norm": True, "interleaved": False, "rows": 32768, "cache": 0}
    c.update(more)
    return {"name": name, **c} if name else c


LARGEST_FLOPS = 8.0e12


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: lists of one to four shapes from 16 to 8192 a side, stacks of one
    to 64, or heads of 32 to 256 over one token to 65 536."""
    if rng.random() < 0.5:
        while True:
            parts = []
            for _ in range(rng.randint(1, 4)):
                parts.append("%d*%dx%d" % (_log_int(rng, 1, 64), _log_int(rng, 16, 8192),
                                           _log_int(rng, 16, 8192)))
            dtype = rng.choice(["f32", "bf16"])
            c = _orth(None, ",".join(parts), op=rng.choice(["orthogonalize", "momentum"]),
                      dtype=dtype, out=rng.choice([dtype, "bf16"]),
                      scale=rng.choice(["none", "shape", "rms"]))
            w = work(c)
            # products of fp32 results take several times as long
            if w["flops"] * (4 if c["out"] == "f32" else 1) <= LARGEST_FLOPS and w["bytes"] <= 8e9:
                return c
    op = rng.choice(["head_forward", "head_backward", "head_token"])
    dim = rng.choice([32, 64, 72, 80, 96, 128, 160, 192, 256])
    hk = _log_int(rng, 1, 16)
    c = _head(None, op=op, hk=hk, hq=hk * rng.choice([1, 1, 2, 4, 7]), dim=dim,
              rot=rng.choice([dim, dim, dim // 2]), dtype=rng.choice(["f32", "bf16", "bf16"]),
              axes=rng.choice([1, 1, 2, 3]), norm=rng.random() < 0.75,
              interleaved=rng.random() < 0.4, rows=_log_int(rng, 16, 65536))
    if op == "head_token":
        c["tokens"] = _log_int(rng, 1, 300)
        c["cache"] = c["tokens"] * rng.randint(1, 60) + rng.randint(0, 9)
    else:
        most = 400_000_000 // ((c["hq"] + c["hk"]) * dim)
        c["tokens"] = _log_int(rng, 1, min(65536, most))
    return c


# ---- what a program has in hand -------------------------------------------------

def _resnet(blocks, bottleneck):
    """(output channels, inputs times window) of every convolution and the head."""
    got, cin = [(64, 147)], 64
    for width, count in zip((64, 128, 256, 512), blocks):
        cout = 4 * width if bottleneck else width
        for b in range(count):
            if bottleneck:
                got += [(width, cin), (width, 9 * width), (cout, width)]
            else:
                got += [(width, 9 * cin), (width, 9 * width)]
            if b == 0 and cin != cout:
                got.append((cout, cin))
            cin = cout
    return got + [(1000, cin)]


def _stacks(c):
    """[(count, rows, cols)]: equal matrices lie in one stacked tensor."""
    if c["sizes"] in ("resnet18", "resnet50"):
        every = _resnet((2, 2, 2, 2), False) if c["sizes"] == "resnet18" else _resnet((3, 4, 6, 3), True)
        shapes = sorted(set(every))
        return [(every.count(s) * c["copies"], *s) for s in shapes]
    out = []
    for part in c["sizes"].split(","):
        count, _, shape = part.rpartition("*")
        rows, cols = shape.split("x")
        out.append((int(count or 1) * c["copies"], int(rows), int(cols)))
    return out


def _scale(c, rows, cols):
    return {"none": 1.0, "shape": math.sqrt(max(1.0, rows / cols)),
            "rms": 0.2 * math.sqrt(max(rows, cols))}[c["scale"]]


def _gradient(count, rows, cols, g, dtype):
    """A few strong directions above broad noise, as gradients of weight matrices have."""
    r = max(1, min(rows, cols) // 16)
    left = torch.randn(count, rows, r, device=DEVICE, generator=g)
    right = torch.randn(count, r, cols, device=DEVICE, generator=g)
    noise = torch.randn(count, rows, cols, device=DEVICE, generator=g)
    return (1e-3 * (left @ right / math.sqrt(r) + 0.25 * noise)).to(dtype)


def _sections(pairs, axes):
    """Pairs per axis, the first one taking what is left over."""
    return [pairs - (axes - 1) * (pairs // axes)] + [pairs // axes] * (axes - 1)


def _table(rows, sections):
    """cos and sin of position times frequency, [rows, 2, pairs]; each axis has its own
    range of frequencies."""
    freq = torch.cat([BASE ** (-torch.arange(n, dtype=torch.float64) / n) for n in sections])
    angle = torch.arange(rows, dtype=torch.float64, device=DEVICE)[:, None] * freq.to(DEVICE)
    return torch.stack([angle.cos(), angle.sin()], 1).float().contiguous()


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    c = dict(case)
    if c["op"] in ("orthogonalize", "momentum"):
        stacks = _stacks(c)
        s = {"case": c, "x": [_gradient(*st, g, DTYPE[c["dtype"]]) for st in stacks],
             "out": [torch.empty(st, device=DEVICE, dtype=DTYPE[c["out"]]) for st in stacks]}
        if c["op"] == "momentum":
            s["m"] = [3.0 * _gradient(*st, g, torch.float32) for st in stacks]
        if own:     # the handle with its workspace, as a training program keeps it
            from paper_1910_00643_amd import Orthogonalizer
            s["handle"] = Orthogonalizer(stacks, dtype=c["dtype"], out_dtype=c["out"],
                                         scale=c["scale"], steps=STEPS, eps=NORM_EPS,
                                         coefficients=COEFFICIENTS, device=DEVICE)
        return s
    dt, t, d = DTYPE[c["dtype"]], c["tokens"], c["dim"]
    pairs = c["rot"] // 2
    sections = _sections(pairs, c["axes"])
    # queries and keys lie beside each other in one projection's output
    both = torch.randn(t, c["hq"] + c["hk"], d, device=DEVICE, generator=g) * 1.7
    both = both.to(dt)
    s = {"case": c, "q": both[:, :c["hq"]], "k": both[:, c["hq"]:],
         "wq": None, "wk": None, "table": _table(c["rows"], sections),
         "pair_axis": [a for a, n in enumerate(sections) for _ in range(n)],
         "positions": torch.randint(0, c["rows"], (c["axes"], t), device=DEVICE, generator=g)}
    if c["norm"]:
        s["wq"] = 1.0 + 0.3 * torch.randn(d, device=DEVICE, generator=g)
        s["wk"] = 1.0 + 0.3 * torch.randn(d, device=DEVICE, generator=g)
    if c["op"] == "head_backward":
        s["gq"] = torch.randn(t, c["hq"], d, device=DEVICE, generator=g).to(dt)
        s["gk"] = torch.randn(t, c["hk"], d, device=DEVICE, generator=g).to(dt)
    if c["op"] == "head_token":
        s["cache"] = torch.randn(c["cache"], c["hk"], d, device=DEVICE, generator=g).to(dt)
        s["slots"] = torch.randperm(c["cache"], device=DEVICE, generator=g)[:t].contiguous()
    if own:         # the layer's settings and table, as a program keeps them
        from paper_1910_00643_amd import HeadNormRotary
        s["handle"] = HeadNormRotary(d, s["table"], dtype=c["dtype"], norm=c["norm"], eps=HEAD_EPS,
                                     interleaved=c["interleaved"], pair_axis=s["pair_axis"])
    return s


# ---- one pass -------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if op in ("orthogonalize", "momentum"):
        if op == "momentum":
            if own:
                s["handle"].momentum_orthogonalize(s["x"], s["m"], s["out"], MU, nesterov=True)
            else:
                for m, x, o in zip(s["m"], s["x"], s["out"]):
                    u = x.float()
                    m.mul_(MU).add_(u)
                    o.copy_(_plain_orthogonalize(s["case"], u + MU * m))
            return {"out": s["out"], "momentum": s["m"]}
        if own:
            s["handle"].orthogonalize(s["x"], s["out"])
        else:
            for x, o in zip(s["x"], s["out"]):
                o.copy_(_plain_orthogonalize(s["case"], x.float()))
        return {"out": s["out"]}
    c = s["case"]
    if own:
        h = s["handle"]
        if op == "head_backward":
            dq, dk, dwq, dwk = h.backward(s["gq"], s["gk"], s["q"], s["k"], s["positions"], s["wq"], s["wk"])
            return {"dq": dq, "dk": dk, **({"dwq": dwq, "dwk": dwk} if c["norm"] else {})}
        if op == "head_token":
            q, k = h.forward(s["q"], s["k"], s["positions"], s["wq"], s["wk"], k_out=s["cache"],
                             k_slots=s["slots"])
            return {"q": q, "cache": k}
        q, k = h.forward(s["q"], s["k"], s["positions"], s["wq"], s["wk"])
        return {"q": q, "k": k}
    cos, sin = _plain_rows(s)
    if op == "head_backward":
        dq, dwq = _plain_head_backward(c, s["gq"], s["q"], s["wq"], cos, sin)
        dk, dwk = _plain_head_backward(c, s["gk"], s["k"], s["wk"], cos, sin)
        return {"dq": dq, "dk": dk, **({"dwq": dwq, "dwk": dwk} if c["norm"] else {})}
    q = _plain_head(c, s["q"], s["wq"], cos, sin)
    k = _plain_head(c, s["k"], s["wk"], cos, sin)
    if op == "head_token":
        s["cache"].index_copy_(0, s["slots"], k)
        return {"q": q, "cache": s["cache"]}
    return {"q": q, "k": k}


# ---- the plain forms ------------------------------------------------------------

def _plain_orthogonalize(c, u):
    rows, cols = u.shape[-2:]
    a, b, cc = COEFFICIENTS
    x = u.transpose(1, 2).contiguous() if rows > cols else u
    x = x / ((x * x).sum((1, 2), keepdim=True).sqrt() + NORM_EPS)
    for _ in range(STEPS):
        gram = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * gram + cc * torch.matmul(gram, gram), x)
    x = x * _scale(c, rows, cols)
    return x.transpose(1, 2) if rows > cols else x


def _plain_rows(s):
    """cos and sin for each token and pair, [tokens, 1, pairs]."""
    pairs = s["table"].shape[2]
    axis = torch.tensor(s["pair_axis"], device=DEVICE)
    rows = s["positions"][axis].t()                       # [tokens, pairs]
    column = torch.arange(pairs, device=DEVICE)
    return s["table"][rows, 0, column][:, None], s["table"][rows, 1, column][:, None]


def _turn(c, y, cos, sin):
    r = c["rot"]
    if c["interleaved"]:
        u, v = y[..., 0:r:2], y[..., 1:r:2]
        turned = torch.stack([u * cos - v * sin, u * sin + v * cos], -1).flatten(-2)
    else:
        u, v = y[..., :r // 2], y[..., r // 2:r]
        turned = torch.cat([u * cos - v * sin, u * sin + v * cos], -1)
    return torch.cat([turned, y[..., r:]], -1)


def _plain_head(c, x, w, cos, sin):
    y = x.float()
    if c["norm"]:
        y = y * ((y * y).mean(-1, keepdim=True) + HEAD_EPS).rsqrt() * w
    return _turn(c, y, cos, sin).to(x.dtype)


def _plain_head_backward(c, gy, x, w, cos, sin):
    gr = _turn(c, gy.float(), cos, -sin)
    if not c["norm"]:
        return gr.to(x.dtype), None
    xf = x.float()
    rstd = ((xf * xf).mean(-1, keepdim=True) + HEAD_EPS).rsqrt()
    xh = xf * rstd
    gw = gr * w
    return (rstd * (gw - xh * (gw * xh).mean(-1, keepdim=True))).to(x.dtype), (gr * xh).sum((0, 1))


# ---- what a pass cannot do without ------------------------------------------------

def work(case):
    c = case
    size = {"f32": 4, "bf16": 2}
    if c["op"] in ("orthogonalize", "momentum"):
        elements = flops = 0
        for count, rows, cols in _stacks(c):
            n, k = min(rows, cols), max(rows, cols)
            elements += count * rows * cols
            # products: X X^T and A A are symmetric (half of each), P X is not
            flops += count * STEPS * (n * (n + 1) * k + n * n * (n + 1) + 2 * n * n * k)
        per = size[c["dtype"]] + size[c["out"]] + (8 if c["op"] == "momentum" else 0)
        return {"bytes": float(elements * per), "flops": float(flops)}
    rows = c["tokens"] * (c["hq"] + c["hk"])
    e = rows * c["dim"]
    passes = 3 if c["op"] == "head_backward" else 2
    table = min(c["tokens"], c["rows"]) * c["rot"] * 4 + c["tokens"] * c["axes"] * 8
    flops = e * ((8 if c["norm"] else 3) if passes == 2 else (15 if c["norm"] else 3))
    return {"bytes": float(e * passes * size[c["dtype"]] + table), "flops": float(flops)}


# ---- the definitions in 64 bits ---------------------------------------------------

def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    c = s["case"]
    if c["op"] in ("orthogonalize", "momentum"):
        outs, moms = [], []
        for j, x in enumerate(s["x"]):
            out = torch.empty(x.shape, dtype=torch.float64, device=DEVICE)
            mom = torch.empty_like(out) if c["op"] == "momentum" else None
            for e in range(x.shape[0]):
                u = x[e].double()
                if mom is not None:
                    mom[e] = MU * s["m"][j][e].double() + u
                    u = u + MU * mom[e]
                out[e] = _exact_orthogonalize(c, u)
            outs.append(out)
            moms.append(mom)
        return {"out": outs, "momentum": moms} if c["op"] == "momentum" else {"out": outs}
    q, dwq = _exact_head(s, "q", "wq", "gq")
    k, dwk = _exact_head(s, "k", "wk", "gk")
    if c["op"] == "head_backward":
        return {"dq": q, "dk": k, **({"dwq": dwq, "dwk": dwk} if c["norm"] else {})}
    if c["op"] == "head_token":
        cache = s["cache"].double()
        cache[s["slots"]] = k
        return {"q": q, "cache": cache}
    return {"q": q, "k": k}


def _exact_orthogonalize(c, u):
    """The polynomial of the singular values, on whichever Gram matrix is smaller."""
    a, b, cc = COEFFICIENTS
    rows, cols = u.shape
    x = u / (torch.linalg.vector_norm(u) + NORM_EPS)
    for _ in range(STEPS):
        if rows <= cols:
            gram = torch.mm(x, x.t())
            turned = torch.mm(gram, x)
            x = a * x + b * turned + cc * torch.mm(gram, turned)
        else:
            gram = torch.mm(x.t(), x)
            turned = torch.mm(x, gram)
            x = a * x + b * turned + cc * torch.mm(turned, gram)
    return x * _scale(c, rows, cols)


def _exact_head(s, name, weight, grad):
    """The rotation as a complex product; the gradient from the formula of the norm."""
    c, x = s["case"], s[name].double()
    r = c["rot"]
    table = s["table"].double()
    angle = torch.complex(table[:, 0], table[:, 1])                     # [rows, pairs]
    turn = torch.stack([angle[s["positions"][a], i] for i, a in enumerate(s["pair_axis"])], 1)[:, None]

    def rotate(y, by):
        z = torch.complex(y[..., :r].unflatten(-1, (-1, 2))[..., 0], y[..., :r].unflatten(-1, (-1, 2))[..., 1]) \
            if c["interleaved"] else torch.complex(*y[..., :r].chunk(2, -1))
        z = z * by
        head = torch.view_as_real(z).flatten(-2) if c["interleaved"] else torch.cat([z.real, z.imag], -1)
        return torch.cat([head, y[..., r:]], -1)

    w = s[weight].double() if c["norm"] else None
    length = torch.sqrt((x ** 2).sum(-1, keepdim=True) / c["dim"] + HEAD_EPS) if c["norm"] else None
    if c["op"] != "head_backward":
        return rotate(x / length * w if c["norm"] else x, turn), None
    g = rotate(s[grad].double(), turn.conj())
    if not c["norm"]:
        return g, None
    inner = (g * w * x).sum(-1, keepdim=True) / c["dim"]
    return g * w / length - x * inner / length ** 3, (g * x / length).sum((0, 1))
