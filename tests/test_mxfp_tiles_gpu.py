"""Products in 4 bits by every kernel and tile size, more tokens than one launch takes,
and scales from the least to the largest; the bounds are test_mxfp_gpu.py's."""
import pytest

torch = pytest.importorskip("torch")

from block_formats import decode, quantise  # noqa: E402
from product_shapes import LINEARS, PRODUCTS  # noqa: E402
from test_mxfp_gpu import product_case  # noqa: E402

pytestmark = pytest.mark.gpu

CHUNK = 1 << 18  # tokens of one launch


@pytest.fixture(scope="module")
def fc(device):
    import paper_1511_00175_amd as m
    return m


@pytest.mark.parametrize("kind,split,n,rows,dim,dtype,to,pad,shift,accumulate", PRODUCTS + LINEARS[len(PRODUCTS) - 2:])
def test_products(fc, device, kind, split, n, rows, dim, dtype, to, pad, shift, accumulate):
    product_case(fc, device, n, rows, dim, dtype, to, pad, shift, accumulate, scale=0.625)


@pytest.mark.parametrize("n,rows,dim,pad,accumulate", [(CHUNK + 77, 70, 64, 0, False), (CHUNK + 77, 70, 64, 3, True), (CHUNK + 30000, 600, 40, 0, False),
                                                       (CHUNK + 1, 40, 600, 1, True)])
def test_more_tokens_than_a_launch_takes(fc, device, n, rows, dim, pad, accumulate):
    """The second launch's inputs, scales and results, with tiles of the first's size and of another."""
    product_case(fc, device, n, rows, dim, "f16", "f32", pad, pad, accumulate)


def test_inputs_packed_in_several_launches(fc, device):
    """2^18 tokens of 8200: past 2^28 threads they are packed by launches of their own, the weight's scales by another."""
    n, rows, dim = CHUNK, 600, 8200
    g = torch.Generator(device=device)
    g.manual_seed(3)
    x = torch.empty(n, dim, dtype=torch.float16, device=device)
    for a in range(0, n, 1 << 15):
        x[a:a + (1 << 15)].normal_(generator=g)
    w = torch.randn(rows, dim, generator=g, device=device)
    plan = fc.Mxfp4(rows, dim, n)
    b, out = plan.empty(rows), torch.empty(n, rows, device=device)
    plan.pack(w, *b)
    plan.linear(x, *b, out)
    bv = decode(*b, "e2m1", dim)
    border = (1 << 28) // (4 * 257)  # rows of a launch
    for first in (0, border - 50, n - 100):
        av = quantise(x[first:first + 100], "e2m1")[0]
        want, size = av @ bv.t(), av.abs() @ bv.t().abs()
        assert bool(((out[first:first + 100].double() - want).abs() <= 2 * ((dim / 16 + 68) * 2.0 ** -24 * size + 2.0 ** -24 * want.abs())).all()), first


def test_columns_packed_in_several_launches(fc, device):
    """More columns than a launch's blocks take along one axis."""
    most, dim = 128 * 32768, 40
    n = most + 300
    x = torch.empty(dim, n, dtype=torch.float16, device=device)
    x.normal_(generator=torch.Generator(device=device).manual_seed(4))
    plan = fc.Mxfp4(1, dim, 0)
    codes, scales = plan.empty(n)
    plan.pack(x, codes, scales, transpose=True)
    for first in (0, most - 150, n - 200):
        value, byte = quantise(x[:, first:first + 200].t().contiguous(), "e2m1")
        part = codes[first:first + 200], scales[first:first + 200]
        assert torch.equal(part[1][:, :2], byte) and torch.equal(decode(*part, "e2m1", dim), value), first


@pytest.mark.parametrize("call,n,rows", [("linear", 3, 700), ("linear", 71, 123), ("product", 71, 123), ("product", 199, 8315), ("product", 2580, 3233)])
def test_least_and_largest_scales(fc, device, call, n, rows):
    """Scales of bytes 0 and 253 in every kernel, beside ones that bring the product back in range: every term is a power
    of two and every sum a whole number of them, which fp32 holds."""
    dim = 64
    g = torch.Generator(device=device)
    g.manual_seed(n)

    def rows_of(k, sizes):
        x = torch.tensor(sizes, dtype=torch.float32, device=device).repeat(-(-k // len(sizes)))[:k, None].expand(k, dim)
        return torch.where(torch.rand(k, dim, generator=g, device=device) < 0.4, -x, x)

    most = torch.finfo(torch.float32).max  # rounds to 2^128
    x, w = rows_of(n, (most, 2.0 ** -127, 1.0)), rows_of(rows, (most, 2.0 ** -127, 2.0 ** -100, 2.0 ** 100))
    plan = fc.Mxfp4(rows, dim, n)
    a, b, out = plan.empty(n), plan.empty(rows), torch.empty(n, rows, device=device)
    plan.pack(x, *a)
    plan.pack(w, *b)
    assert a[1][:3, 0].tolist() == [253, 0, 125] and b[1][:4, 0].tolist() == [253, 0, 25, 225]
    if call == "linear":
        plan.linear(x, *b, out)
    else:
        plan.product(*a, *b, out)
    want = decode(*a, "e2m1", dim) @ decode(*b, "e2m1", dim).t()
    size = decode(*a, "e2m1", dim).abs() @ decode(*b, "e2m1", dim).abs().t()
    held = (size < 2.0 ** 127) & (size > 2.0 ** -110)
    # of the 12 pairs of sizes the 6 of about 1 are: 2^128 with 2^-127 both ways and 2^-100, 2^-127 with 2^100, 1 with 2^-100 and 2^100
    assert held[:3, :4].tolist() == [[False, True, True, False], [True, False, False, True], [False, False, True, True]]
    assert torch.equal(out[held].double(), want[held])
