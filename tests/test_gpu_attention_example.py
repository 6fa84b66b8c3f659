"""The example's answers, token by token over a paged cache, are what its training path computes of the whole
sequences, and its gradients are those of the same model in 64 bits."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import orthogonal_attention as E
    finally:
        sys.path.pop(0)
    return E


def _model64(E, p, tokens):
    """The model from elementary operations, one sequence."""
    t = tokens.numel()
    x = p["embed"][tokens]
    q, k, v = ((x @ p[n].t()).view(t, E.HEADS, E.DIM) for n in ("wq", "wk", "wv"))
    angle = torch.arange(t, device=tokens.device, dtype=x.dtype)[:, None] * \
        10000.0 ** (-torch.arange(E.DIM // 2, device=tokens.device, dtype=x.dtype) / (E.DIM // 2))
    c, s = angle.cos()[:, None], angle.sin()[:, None]

    def normed(y, w):
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6) * w
        a, b = y.chunk(2, -1)
        return torch.cat([a * c - b * s, a * s + b * c], -1).transpose(0, 1)

    scores = normed(q, p["q_norm"]) @ normed(k, p["k_norm"]).transpose(1, 2).contiguous() * E.SCALE
    later = torch.ones(t, t, dtype=torch.bool, device=tokens.device).triu(1)
    mixed = torch.softmax(scores.masked_fill(later, float("-inf")), -1) @ v.transpose(0, 1)
    return (x + mixed.transpose(0, 1).reshape(t, E.WIDTH) @ p["wo"].t()) @ p["head"].t()


# Both sides are fp32 sums of at most WIDTH = 128 terms one after the other, through five layers of them; scores of at
# most 4 / sqrt(32) * 32 = 23 carry 23 * 130 * 2^-24 = 2e-4 of a probability, and the logits are of the size of 100.
TOL = 2e-2


def test_answers_are_those_of_the_whole_sequences():
    E = _example()
    p = E.make_worker("cuda:0", 3)
    g = torch.Generator(device="cuda:0").manual_seed(4)
    lengths, n = [5, 1, 33, 16], 6
    texts = [torch.randint(0, E.VOCAB, (m + n,), device="cuda:0", generator=g) for m in lengths]
    first, rest = E.answer(p, [t[:m] for t, m in zip(texts, lengths)], torch.stack([t[m:] for t, m in zip(texts, lengths)]))
    p64 = {k: v.detach().double() for k, v in p.items()}
    at = 0
    for i, (t, m) in enumerate(zip(texts, lengths)):
        want = _model64(E, p64, t)
        assert (first[at:at + m] - want[:m]).abs().max() < TOL and (rest[i] - want[m:]).abs().max() < TOL
        at += m


def test_gradients_are_those_of_the_model():
    E = _example()
    p = E.make_worker("cuda:0", 5)
    g = torch.Generator(device="cuda:0").manual_seed(6)
    tokens = torch.randint(0, E.VOCAB, (3, 21), device="cuda:0", generator=g)
    rotate = E.HeadNormRotary(E.DIM, E.rotary_table(21, E.DIM // 2, device="cuda:0"), dtype="f32")
    E.loss_of(p, tokens, rotate, E.Attention(E.DIM, dtype="f32", scale=E.SCALE)).backward()
    p64 = {k: v.detach().double().requires_grad_() for k, v in p.items()}
    logits = torch.stack([_model64(E, p64, t) for t in tokens])
    torch.nn.functional.cross_entropy(logits[:, 2:].reshape(-1, E.VOCAB), tokens[:, :-2].reshape(-1)).backward()
    for name in p:
        want = p64[name].grad
        # 2e-4 of a probability, as above, and as much again through the sums of the products around it
        assert (p[name].grad - want).norm() <= 1e-3 * want.norm(), name
