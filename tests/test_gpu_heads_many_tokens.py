"""More tokens than one grid has waves for (less than 2^32 threads, a wave to a token): one row for
all of them, keys into a small cache."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DEV = "cuda:0"


@pytest.fixture(autouse=True, scope="module")
def _memory_goes_back():
    """Later tests look at allocations of their own."""
    yield
    torch.cuda.empty_cache()


def test_more_tokens_than_a_grid_has_waves():
    import paper_1910_00643_amd as P
    tokens, dim, rows = (1 << 26) + 1001, 512, 97
    g = torch.Generator(device=DEV).manual_seed(1)
    op = P.HeadNormRotary(dim, P.rotary_table(rows, 32, device=DEV))
    row = torch.randn(1, 1, dim, device=DEV, generator=g).bfloat16()
    positions = torch.arange(tokens, device=DEV) % rows
    # data off by one element: a row takes a whole wave
    cache = torch.full((9 * dim + 1,), 7.0, device=DEV, dtype=torch.bfloat16)[1:].view(9, 1, dim)
    slots = torch.full((tokens,), -1, device=DEV, dtype=torch.int64)
    of = [0, 1 << 25, (1 << 25) - 1, 1 << 26, (1 << 26) - 1, tokens - 1]
    for i, t in enumerate(of):
        slots[t] = 8 - i
    none = torch.empty(tokens, 0, dim, device=DEV, dtype=torch.bfloat16)
    op.forward(none, row.expand(tokens, 1, dim), positions, k_out=cache, k_slots=slots)
    want = torch.full_like(cache, 7.0)
    few = positions[of].contiguous()
    want[[8 - i for i in range(len(of))]] = op.forward(none[:len(of)], row.expand(len(of), 1, dim).contiguous(), few)[1]
    # rows of a wave and rows of half a wave add their squares in other orders: 2^-24 * 10, and a bf16's last bit
    assert ((cache.double() - want.double()).abs() <= 2.0 ** -7 * want.double().abs()).all()
    assert (cache[:3] == 7).all()
