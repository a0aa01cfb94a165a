"""Calls of more threads than one launch takes (HIP: below 2^32 along an axis),
and of more than the library puts into one (2^28)."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory(device):
    """Tens of gigabytes, given back afterwards."""
    if torch.cuda.get_device_properties(device).total_memory < 200 << 30:
        pytest.skip("needs the memory of an MI355X")
    yield
    torch.cuda.empty_cache()


def test_lookup_of_many_tokens(device):
    """2^24 tokens and more, 256 threads each."""
    import paper_1511_00175_amd as fc
    rows, dim, n = 1000, 1032, (1 << 24) + 3
    g = torch.Generator(device=device)
    g.manual_seed(1)
    table = torch.randn(rows, dim, generator=g, device=device).half()
    tokens = torch.randint(-10, rows, (n,), generator=g, device=device, dtype=torch.int32)
    out = torch.full((n, dim), float("nan"), dtype=torch.float16, device=device)
    fc.Embedding(rows, dim, 1).lookup(table, tokens, out, scale=0.5)
    with_zeros = torch.cat([table * 0.5, torch.zeros_like(table[:1])])  # a power of two: exact
    for at in range(0, n, 1 << 20):
        t = tokens[at:at + (1 << 20)].long()
        assert torch.equal(out[at:at + (1 << 20)], with_zeros[torch.where(t < 0, rows, t)]), at


def test_zeros_for_a_large_gradient_without_tokens(device):
    """2^32 elements of dw."""
    import paper_1511_00175_amd as fc
    rows, dim = 1 << 20, 4096
    w = torch.zeros(rows, dim, dtype=torch.float16, device=device)
    dw = torch.full_like(w, 3.0)
    none = torch.zeros(0, device=device)
    fc.CrossEntropy(rows, dim, 1).loss_grad(none.half().view(0, dim), w, none.long(), none, None, dw)
    assert not bool(dw.any())


def test_copies_of_a_large_vocabulary(device):
    """More than 2^28 vectors of a w whose rows are copied (513 of 8 elements each)."""
    import paper_1511_00175_amd as fc
    rows, dim, n = (1 << 19) + 7, 4097, 3
    g = torch.Generator(device=device)
    g.manual_seed(2)
    w = torch.randn(rows, dim, generator=g, device=device, dtype=torch.float16)
    x = (torch.randn(n, dim, generator=g, device=device) * dim ** -0.5).half()
    y = torch.tensor([5, rows - 1, -1], device=device)
    loss = torch.full((n,), float("nan"), device=device)
    fc.CrossEntropy(rows, dim, n).loss(x, w, y, loss)
    logits = torch.cat([x.float() @ w[at:at + 65536].float().t() for at in range(0, rows, 65536)], 1).double()
    want = torch.logsumexp(logits, 1) - logits[torch.arange(n, device=device), y.clamp(min=0)]
    # logits of about 1: (dim + 2) 2^-24 of the terms' absolute sum, about 0.64 dim^0.5, in both
    assert float((loss.double() - want)[:2].abs().max()) <= 4 * (dim + 2) * 2.0 ** -24 * dim ** 0.5 and float(loss[2]) == 0


@pytest.mark.parametrize("rows", [7, 1000])
def test_gradient_of_many_tokens(device, rows):
    """More than 2^20 chunks of the sorted list, with rows that run over them."""
    import paper_1511_00175_amd as fc
    dim, n = 4, (1 << 25) + 4000
    g = torch.Generator(device=device)
    g.manual_seed(3)
    tokens = torch.randint(0, rows, (n,), generator=g, device=device, dtype=torch.int32)
    dy = torch.randint(-3, 4, (n, dim), generator=g, device=device).half()
    out = torch.full((rows, dim), float("nan"), device=device)
    fc.Embedding(rows, dim, n).grad(dy, tokens, out)
    if rows < 10:
        want = torch.stack([dy[tokens == r].double().sum(0) for r in range(rows)])
    else:
        want = torch.zeros(rows, dim, dtype=torch.float64, device=device).index_add_(0, tokens.long(), dy.double())
    # whole numbers below 2^24 in every partial sum (3 n / 7 = 1.4e7): exact
    assert torch.equal(out.double(), want)
