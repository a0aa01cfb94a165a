"""Matrices of more than 2^31 elements: what lies past the first 2^32 bytes and 2^31
elements is computed as it is alone."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fc(device):
    import paper_1511_00175_amd as m
    return m


def rows(n, dim, device, dtype=torch.float16, seed=0):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    t = torch.empty(n, dim, dtype=dtype, device=device)
    for a in range(0, n, 1 << 15):
        t[a:a + (1 << 15)].normal_(generator=g)
    return t


def test_norm(fc, device):
    n, dim, last = 270000, 8192, 3
    h, b, dy = (rows(n, dim, device, seed=k) for k in range(3))
    out, y, dh, db = (torch.empty_like(h) for _ in range(4))
    dw = torch.empty(dim, device=device)
    plan, small = fc.Norm(dim, n, "f16", "f16"), fc.Norm(dim, last, "f16", "f16")
    plan.between(h, b, out, y)
    plan.between_grad(out, b, dy, dh, db, dout=h, dweight=dw)
    want = [torch.empty_like(h[:last]) for _ in range(4)]
    small.between(h[-last:], b[-last:], *want[:2])
    small.between_grad(want[0], b[-last:], dy[-last:], *want[2:], dout=h[-last:])
    for got, ref in zip((out, y, dh, db), want):
        assert torch.equal(got[-last:], ref)
    total = torch.zeros(dim, dtype=torch.float64, device=device)
    for a in range(0, n, 1 << 14):
        x = b[a:a + (1 << 14)].float()
        x *= (x.square().mean(1, keepdim=True) + 1e-6).rsqrt()
        total += (dh[a:a + (1 << 14)].float() * x).sum(0, dtype=torch.float64)
    # dh is rounded to fp16 here: 270000 independent errors of 2^-12 of terms of size 1 to 2
    assert float((dw.double() - total).abs().max()) < 8 * 270000 ** 0.5 * 2.0 ** -11


def test_checkpoint(fc, device):
    n, dim, outs = 33000, 65536, 8
    x = rows(n, dim, device)
    plan = fc.Checkpoint(dim, n, outs)
    codes, scales = plan.empty(n)
    plan.pack(x, codes, scales)
    back = torch.empty_like(x)
    plan.unpack(codes, scales, back)
    small = fc.Checkpoint(dim, 2)
    c2, s2 = small.empty(2)
    b2 = torch.empty_like(x[:2])
    small.pack(x[-2:], c2, s2)
    small.unpack(c2, s2, b2)
    assert torch.equal(codes[-2:], c2) and torch.equal(scales[-2:], s2) and torch.equal(back[-2:], b2)
    dy, dw = rows(n, outs, device, seed=1), torch.empty(outs, dim, device=device)
    plan.grad(dy, codes, scales, dw)
    want = torch.zeros(outs, dim, dtype=torch.float64, device=device)
    for a in range(0, n, 4096):
        want += dy[a:a + 4096].double().t() @ back[a:a + 4096].double()
    # sums of 33000 products, of which fp32 keeps n / 4 roundings at the most, of terms of size 1
    assert float((dw.double() - want).abs().max()) < 2.0 ** -24 * (n / 4 + 66) * n ** 0.5 * 8


def test_product(fc, device):
    n, wide, dim = 70000, 32768, 256
    plan, small = fc.Mxfp4(wide, dim, n), fc.Mxfp4(wide, dim, 100)
    x, w = rows(n, dim, device), rows(wide, dim, device, seed=1)
    b = plan.empty(wide)
    plan.pack(w, *b)
    out, want = (torch.empty(k, wide, dtype=torch.bfloat16, device=device) for k in (n, 100))
    plan.linear(x, *b, out)
    small.linear(x[-100:], *b, want)
    assert torch.equal(out[-100:], want)  # two sums of 128 exact products each, in either tile
    plan.linear(x, *b, out, accumulate=True)
    assert torch.equal(out[-100:], (want.float() + want.float()).bfloat16())
