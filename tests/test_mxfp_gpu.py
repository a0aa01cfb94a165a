"""Matrices in microscaled 4-bit floating point and their products on the GPU.

Codes and scales are what the definition gives in 64 bits, exactly.  A product's terms
are exact in fp32; its sum of k terms is taken 128 at a time with at most 8 roundings
each, in up to 64 parts: |err| <= (k / 16 + 66) 2^-24 sum |terms|, one more with `scale`
and one with `accumulate`, and the result's own rounding U |out|; doubled for the terms
of second order."""
import pytest

torch = pytest.importorskip("torch")

from block_formats import DT, decode, quantise, rounded, samples, strided  # noqa: E402

pytestmark = pytest.mark.gpu

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 1e-37, torch.float16: 2.0 ** -24, torch.bfloat16: 1e-37}


@pytest.fixture(scope="module")
def fc(device):
    import paper_1511_00175_amd as m
    return m


def same(a, b):
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(torch.nan_to_num(a.float(), 0, 1e30, -1e30), torch.nan_to_num(b.float(), 0, 1e30, -1e30))


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("n,d,pad,shift", [(1, 1, 0, 0), (0, 5, 0, 0), (3, 31, 0, 0), (40, 32, 0, 0), (40, 33, 0, 0), (17, 64, 8, 0), (20, 257, 3, 1),
                                           (63, 1001, 5, 3), (65, 255, 0, 0), (700, 96, 0, 0), (130, 513, 1, 0)])
def test_round_trip(fc, device, dtype, transpose, n, d, pad, shift):
    t = DT[dtype]
    plain = samples(n, d, t, device, n + 3 * d)
    plan = fc.Mxfp4(1, d, 0)
    r, c = (d, n) if transpose else (n, d)
    x = strided(r, c, t, device, pad, shift, fill=float("nan"))
    x.copy_(plain.t() if transpose else plain)
    codes = strided(n, plan.widths[0], torch.uint8, device, 16 * (pad > 0), 0)
    scales = strided(n, plan.widths[1], torch.uint8, device, 8 * (pad > 0), 0)
    plan.pack(x, codes, scales, transpose=transpose)
    value, byte = quantise(plain, "e2m1")
    assert torch.equal(scales[:, :byte.shape[1]], byte) and bool((scales[:, byte.shape[1]:] == 0).all())
    assert same(decode(codes, scales, "e2m1", d), value)
    assert same(decode(codes, scales, "e2m1", 32 * byte.shape[1])[:, d:].nan_to_num(0), torch.zeros(n, -d % 32, device=device))
    for o in DT.values():
        out = strided(n, d, o, device, pad, shift)
        plan.unpack(codes, scales, out)
        assert same(out, rounded(value, o)), o
    if pad and n > 1:  # between the rows nothing is written
        for m, w in ((codes, 16), (scales, 8)):
            assert bool((torch.as_strided(m, (n - 1, w), (m.stride(0), 1), m.storage_offset() + m.shape[1]) == 7).all())


def product_case(fc, device, n, rows, dim, dtype="f16", to="f32", pad=0, shift=0, accumulate=False, scale=1.0, plan=None):
    t, o = DT[dtype], DT[to]
    g = torch.Generator(device=device)
    g.manual_seed(n + 7 * dim + rows)
    plan = plan or fc.Mxfp4(rows, dim, n)
    x = strided(n, dim, t, device, pad, shift, fill=float("nan"))
    x.copy_(samples(n, dim, torch.float32, device, n + dim, special=False).clamp(-1e4, 1e4))
    w = (torch.randn(rows, dim, generator=g, device=device) * dim ** -0.5 * torch.exp(torch.randn(rows, 1, generator=g, device=device))).to(t)
    a, b = plan.empty(n), plan.empty(rows)
    plan.pack(x, *a)
    plan.pack(w, *b)
    old = torch.randn(n, rows, generator=g, device=device).to(o)
    out = strided(n, rows, o, device, pad, shift)
    got = []
    for k in range(3):
        out.copy_(old if accumulate else torch.full_like(old, float("nan")))
        if k == 2:
            plan.linear(x, *b, out, scale=scale, accumulate=accumulate)
        else:
            plan.product(*a, *b, out, scale=scale, accumulate=accumulate)
        got.append(out.clone())
    assert torch.equal(got[0], got[1])  # the same bits again
    av, bv = decode(*a, "e2m1", dim), decode(*b, "e2m1", dim)
    want, size = scale * av @ bv.t(), abs(scale) * av.abs() @ bv.t().abs()
    if accumulate:
        want, size = want + old.double(), size + old.double().abs()
    bound = 2 * ((dim / 16 + 68) * 2.0 ** -24 * size + U[o] * want.abs()) + TINY[o]
    for v in got[1:]:
        bad = (v.double() - want).abs() > bound
        assert not bool(bad.any()), (int(bad.sum()), float(((v.double() - want).abs() / bound).max()))
    if pad and n > 1:
        assert bool((torch.as_strided(out, (n - 1, pad), (rows + pad, 1), out.storage_offset() + rows) == 7).all())


@pytest.mark.parametrize("n,rows,dim", [(1, 1, 1), (1, 16, 32), (1, 100, 256), (2, 17, 33), (3, 700, 9216), (5, 5, 31), (15, 1000, 520), (16, 64, 4096),
                                        (17, 48, 1000), (33, 130, 257), (64, 64, 512), (65, 63, 520), (128, 128, 256), (129, 127, 255), (200, 72, 9216),
                                        (257, 300, 1024), (1003, 1001, 520), (2100, 2500, 300), (4096, 4096, 520)])
def test_product_sizes(fc, device, n, rows, dim):
    product_case(fc, device, n, rows, dim)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("to", list(DT))
@pytest.mark.parametrize("n", [1, 9, 90])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_product_types_strides_alignment(fc, device, dtype, to, n, pad, shift):
    product_case(fc, device, n, 77, 300, dtype, to, pad, shift)


@pytest.mark.parametrize("dtype,to", [("f32", "f16"), ("f16", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
@pytest.mark.parametrize("n,rows,dim", [(90, 77, 700), (40, 130, 576), (40, 130, 577), (1000, 1024, 552), (1000, 1030, 552), (17, 16300, 40), (17, 16400, 40)])
def test_inputs_packed_within_the_product_and_before_it(fc, device, dtype, to, pad, shift, n, rows, dim):
    """Both sides of the widths and tiles up to which one launch packs and multiplies."""
    product_case(fc, device, n, rows, dim, dtype, to, pad, shift, accumulate=pad > 0)


@pytest.mark.parametrize("to", list(DT))
@pytest.mark.parametrize("n,rows,dim", [(1, 90, 700), (12, 50, 9000), (70, 66, 9000), (300, 200, 96)])
def test_product_accumulates(fc, device, to, n, rows, dim):
    product_case(fc, device, n, rows, dim, to=to, accumulate=True, scale=-1.75)


@pytest.mark.parametrize("n,rows,dim", [(5000, 4400, 520), (4700, 4500, 200), (8193, 4300, 256)])
def test_more_tiles_than_blocks(fc, device, n, rows, dim):
    """Blocks go through several tiles, of three steps and of one, with the next one's loads under way."""
    product_case(fc, device, n, rows, dim, to="bf16")


def test_fewer_tokens_than_the_plan(fc, device):
    plan = fc.Mxfp4(130, 600, 700)
    for n in (700, 1, 65, 16, 300):
        product_case(fc, device, n, 130, 600, plan=plan)


def test_nothing(fc, device):
    plan = fc.Mxfp4(24, 40, 8)
    b = plan.empty(24)
    plan.pack(torch.ones(24, 40, device=device), *b)
    plan.product(*plan.empty(0), *b, torch.empty(0, 24, device=device))
    plan.linear(torch.empty(0, 40, device=device), *b, torch.empty(0, 24, device=device))


def test_nan_stays_in_its_row(fc, device):
    """A block that holds an infinity or NaN spoils the products of its row, and no other's."""
    for n, rows, dim in ((7, 40, 300), (90, 70, 300)):
        torch.manual_seed(n)
        plan = fc.Mxfp4(rows, dim, n)
        x, w = torch.randn(n, dim, device=device), torch.randn(rows, dim, device=device)
        b = plan.empty(rows)
        clean, out = (torch.empty(n, rows, device=device) for _ in range(2))
        plan.pack(w, *b)
        plan.linear(x, *b, clean)
        x[3, 299], w[5, 0] = float("inf"), float("nan")
        plan.pack(w, *b)
        plan.linear(x, *b, out)
        spoilt = torch.zeros(n, rows, dtype=torch.bool, device=device)
        spoilt[3], spoilt[:, 5] = True, True
        assert bool(out[spoilt].isnan().all()) and torch.equal(out[~spoilt], clean[~spoilt])


def test_scales_at_the_ends_of_their_range(fc, device):
    """Products of the largest and the smallest scales, 2^100 and 2^-120 apart from 1, are exact powers of two."""
    plan = fc.Mxfp4(2, 64, 2)
    x = torch.tensor([2.0 ** 60, 2.0 ** -60], device=device)[:, None].expand(2, 64).contiguous()
    w = torch.tensor([2.0 ** 60, 2.0 ** -60], device=device)[:, None].expand(2, 64).contiguous()
    b, out = plan.empty(2), torch.empty(2, 2, device=device)
    plan.pack(w, *b)
    plan.linear(x, *b, out)
    assert out.tolist() == [[2.0 ** 126, 64.0], [64.0, 2.0 ** -114]]


def test_layer_forward_and_backward(fc, device):
    """y = x w^T and dx = dy w with one weight packed both ways: <dx, v> is y's change along v, for the 4-bit numbers that
    each direction keeps."""
    n, rows, dim = 70, 96, 160
    g = torch.Generator(device=device)
    g.manual_seed(3)
    x, w, dy = (torch.randn(s, generator=g, device=device) for s in ((n, dim), (rows, dim), (n, rows)))
    ahead, back = fc.Mxfp4(rows, dim, n), fc.Mxfp4(dim, rows, n)
    wa, wb = ahead.empty(rows), back.empty(dim)
    ahead.pack(w, *wa)
    back.pack(w, *wb, transpose=True)
    y, dx = torch.empty(n, rows, device=device), torch.empty(n, dim, device=device)
    ahead.linear(x, *wa, y)
    back.linear(dy, *wb, dx)
    xq, dyq = quantise(x, "e2m1")[0], quantise(dy, "e2m1")[0]
    wq, wtq = quantise(w, "e2m1")[0], quantise(w.t().contiguous(), "e2m1")[0]
    assert float((y.double() - xq @ wq.t()).norm()) <= 1e-5 * float(y.double().norm())
    assert float((dx.double() - dyq @ wtq.t()).norm()) <= 1e-5 * float(dx.double().norm())
    # a rounding to one bit after the first is off by at most a fifth (1.25 of 1), by half a step of 0.5 below 1
    assert float((y.double() - x.double() @ w.double().t()).norm()) < 0.4 * float((x.double() @ w.double().t()).norm())


def test_streams_and_graph(fc, device):
    n, rows, dim = 300, 130, 2100
    plan = fc.Mxfp4(rows, dim, n)
    g = torch.Generator(device=device)
    g.manual_seed(2)
    w, b = torch.randn(rows, dim, generator=g, device=device), plan.empty(rows)
    plan.pack(w, *b)
    for m in (n, 1, 11):  # large, single, few
        sets = [torch.randn(m, dim, generator=g, device=device) for _ in range(3)]
        want, got = ([torch.empty(m, rows, device=device) for _ in sets] for _ in range(2))
        for x, o in zip(sets, want):
            plan.linear(x, *b, o)
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        for k in range(3):
            for i, x in enumerate(sets):
                plan.linear(x, *b, got[i], stream=streams[(i + k) % 2])
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        x, out = sets[0], torch.empty(m, rows, device=device)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            plan.pack(w, *b)
            plan.linear(x, *b, out)
        for k in range(4):
            w.copy_(torch.randn(rows, dim, generator=g, device=device))
            x.copy_(torch.randn(m, dim, generator=g, device=device))
            out.fill_(5.0)
            graph.replay()
            torch.cuda.synchronize()
            first = out.clone()
            plan.linear(sets[1], *b, got[1])  # the program's own calls between
            plan.pack(w, *b)
            plan.linear(x, *b, out)
            assert torch.equal(first, out), (m, k)


def test_refusals(fc, device):
    plan = fc.Mxfp4(24, 40, 8)
    x, w, out = torch.zeros(8, 40, device=device), torch.zeros(24, 40, device=device), torch.zeros(8, 24, device=device)
    a, b = plan.empty(8), plan.empty(24)
    plan.pack(x, *a)
    plan.pack(w, *b)
    plan.pack(w.t().contiguous(), *b, transpose=True)
    plan.product(*a, *b, out)
    for bad in (lambda: plan.pack(x.double(), *a), lambda: plan.pack(x, *b), lambda: plan.pack(w, *b, transpose=True), lambda: plan.pack(x[0], *a),
                lambda: plan.pack(x.tolist(), *a), lambda: plan.pack(x, a[0].view(torch.int8), a[1]), lambda: plan.pack(x, a[0], a[1][:, :2]),
                lambda: plan.unpack(*a, out), lambda: plan.product(*a, *b, out[:, :23]), lambda: plan.product(*a, *a, out), lambda: plan.linear(x, *b, out.double()),
                lambda: plan.linear(x.repeat(2, 1), *b, out.repeat(2, 1)), lambda: plan.linear(x.cpu(), *b, out), lambda: plan.linear(x[:, :39], *b, out)):
        with pytest.raises(ValueError):
            bad()
    odd = torch.zeros(24 * 48, dtype=torch.uint8, device=device)
    for code, bad in ((-2, lambda: plan.pack(w, odd[8:8 + 24 * 32].view(24, 32), b[1])), (-2, lambda: plan.pack(w, odd[:24 * 40].view(24, 40)[:, :32], b[1])),
                      (-2, lambda: plan.pack(w, b[0], odd[4:4 + 24 * 8].view(24, 8))), (-2, lambda: plan.linear(x, b[0], odd[:24 * 12].view(24, 12)[:, :8], out)),
                      (-3, lambda: plan.linear(x, *b, b[0].view(-1)[:768].view(torch.float32).view(8, 24))), (-3, lambda: plan.pack(w, b[0], b[0].view(-1)[:192].view(24, 8)))):
        with pytest.raises(fc.FcError) as e:
            bad()
        assert e.value.code == code
    for args in ((0, 1, 1), (1, 0, 1), ((1 << 21) + 1, 1, 1), (1, (1 << 21) + 1, 1), (8, 8, -1), (8, 8, 1 << 31)):
        with pytest.raises(fc.FcError) as e:
            fc.Mxfp4(*args)
        assert e.value.code == -1


def test_fresh_workspaces_may_hold_anything(fc, device):
    junk = [torch.full((1 << 24,), float("nan"), device=device) for _ in range(8)]
    torch.cuda.synchronize()
    del junk
    torch.cuda.empty_cache()
    for n in (1, 13, 70, 300):
        product_case(fc, device, n, 129, 2000)
