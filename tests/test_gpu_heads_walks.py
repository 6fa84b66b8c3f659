"""The norm of queries and keys with the position rotation on sizes whose waves take several
turns or walk over several blocks of tokens, whose rows stream past the caches, and whose lanes share
an axis that is not the first.  Against the definition in 64 bits, with the tolerances of
test_gpu_heads.py; a weight's gradient is summed in chains here, one to a lane over its wave's whole
walk: at most rows / 3072 + 64 additions (3072 waves of a full walk, rounded up for both sides), then
4 waves, 12 and 64 sums: 2^-24 * (rows / 3072 + 200) * sum |terms|."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_heads import DEV, _P, _inputs, _norm64, _turn64  # noqa: E402

T = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True, scope="module")
def _memory_goes_back():
    """Later tests look at allocations of their own."""
    yield
    torch.cuda.empty_cache()


def _check(tokens, hq, hk, dim, rot, dtype, axes=1, pair_axis=None, norm=True, interleaved=False, pad=0):
    q, k, table, positions, mixed, wq, wk = _inputs(11, tokens, hq, hk, dim, rot, T[dtype], axes, pad=pad)
    pair_axis = mixed if pair_axis is None else pair_axis
    op = _P().HeadNormRotary(dim, table, dtype=dtype, norm=norm, interleaved=interleaved, pair_axis=pair_axis)
    weights = (wq, wk) if norm else (None, None)
    y = op.forward(q, k, positions, *weights)
    g = torch.Generator(device=DEV).manual_seed(12)
    gy = [torch.randn(x.shape, device=DEV, generator=g).to(T[dtype]) for x in (q, k)]
    grads = op.backward(*gy, q, k, positions, *weights)
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    for i, (x, w) in enumerate(((q, wq), (k, wk))):
        xh, r, w64 = _norm64(x.double(), w, 1e-6)
        if not norm:
            xh, r, w64 = x.double(), torch.ones_like(r), torch.ones_like(w64)
        big = (xh * w64).abs().amax(-1, keepdim=True)
        want = _turn64(xh * w64, table, positions, pair_axis, interleaved)
        assert ((y[i].double() - want).abs() <= 4e-6 * big + half * want.abs()).all()
        del want
        gr = _turn64(gy[i].double(), table, positions, pair_axis, interleaved, back=True)
        gw = gr * w64
        if norm:
            terms = gr * xh
            bound = 2.0 ** -24 * (tokens * (hq + hk) / 3072 + 200) * terms.abs().sum((0, 1))
            assert ((grads[2 + i].double() - terms.sum((0, 1))).abs() <= bound).all()
            del terms
            big = gw.abs().amax(-1, keepdim=True) * r * (xh * xh).amax(-1, keepdim=True).clamp(min=1)
            gw = r * (gw - xh * (gw * xh).mean(-1, keepdim=True))
        else:
            big = gw.abs().amax(-1, keepdim=True) * 2
        assert ((grads[i].double() - gw).abs() <= 3e-5 * big + half * gw.abs()).all()


# tokens x turns past the waves that fill the card: a wave takes all turns, every second, every third
@pytest.mark.parametrize("tokens", [9000, 3500, 2100])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_several_turns_of_a_token(tokens, dtype):
    _check(tokens, 40, 3, 128, 128, dtype)


@pytest.mark.parametrize("hq,hk,dim,tokens", [(1, 1, 64, 100003), (5, 2, 64, 30011), (3, 0, 33, 40001),
                                              (40, 8, 128, 5003)], ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_walks_over_several_blocks(hq, hk, dim, tokens, dtype):
    """More blocks of tokens than a full walk has waves, the last one short."""
    _check(tokens, hq, max(hk, 1), dim, dim // 2 * 2, dtype)


# lanes of 8 pairs, of 4, and single ones; 768 MiB of traffic both ways and more
@pytest.mark.parametrize("dim,pad", [(128, 0), (72, 0), (72, 1)], ids=str)
@pytest.mark.parametrize("norm,interleaved", [(True, False), (False, True)], ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_stream_past_the_caches(dtype, norm, interleaved, dim, pad):
    elements = (768 << 20) / 2 / (4 if dtype == "f32" else 2)
    tokens = int(elements / (20 * dim)) + 13
    _check(tokens, 16, 4, dim, dim, dtype, norm=norm, interleaved=interleaved, pad=pad)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("norm,interleaved", [(True, False), (True, True), (False, False), (False, True)], ids=str)
@pytest.mark.parametrize("sections", [(32, 32), (24, 24, 16), (36, 28), (28, 20, 16), (8, 4, 40, 12)], ids=str)
def test_sections_of_whole_lanes(sections, norm, interleaved, dtype):
    """Every axis's pairs beside each other, their edges at multiples of 8 and of 4."""
    pair_axis = [a for a, n in enumerate(sections) for _ in range(n)]
    _check(501, 6, 2, 128, 128, dtype, axes=len(sections), pair_axis=pair_axis, norm=norm, interleaved=interleaved)
