"""Activations in 8 bits and weights' gradients from them on the GPU.

Codes and scales are what the definition gives in 64 bits, exactly, and so are
unpacked values, rounded once.  A gradient's products are exact in fp32 (11 and 8
bits at most); its sum of n terms is taken 32 at a time with at most 8 roundings
each, and in up to 64 parts: |err| <= (n / 4 + 64) 2^-24 sum |terms|, one more with
the scale and one with `accumulate`, and the result's own rounding U |dw|; doubled
for the terms of second order."""
import pytest

torch = pytest.importorskip("torch")

from block_formats import BLOCK, DT, decode, quantise, rounded, samples, strided  # noqa: E402

pytestmark = pytest.mark.gpu

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 1e-37, torch.float16: 2.0 ** -24, torch.bfloat16: 1e-37}
KEPT = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}


@pytest.fixture(scope="module")
def fc(device):
    import paper_1511_00175_amd as m
    return m


def same(a, b):
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(torch.nan_to_num(a.float(), 0, 1e30, -1e30), torch.nan_to_num(b.float(), 0, 1e30, -1e30))


def round_trip(fc, device, kind, n, d, dtype, pad=0, shift=0):
    t = DT[dtype]
    x = strided(n, d, t, device, pad, shift, fill=float("nan"))
    x.copy_(samples(n, d, t, device, n + 3 * d))
    plan = fc.Checkpoint(d, 0, format=kind)
    blocks = -(-d // BLOCK)
    codes = strided(n, BLOCK * blocks, KEPT[kind], device, 16 * (pad > 0), 0)
    scales = strided(n, blocks, torch.uint8, device, pad, shift)
    plan.pack(x, codes, scales)
    value, byte = quantise(x, kind)
    assert torch.equal(scales, byte)
    assert same(decode(codes, scales, kind, d), value)
    assert bool((codes.float()[:, d:] == 0).all())
    for o in DT.values():
        out = strided(n, d, o, device, pad, shift)
        plan.unpack(codes, scales, out)
        assert same(out, rounded(value, o)), o
        if pad and n > 1:
            assert bool((torch.as_strided(out, (n - 1, pad), (d + pad, 1), out.storage_offset() + d) == 7).all())
    if pad and n > 1:  # between the rows nothing is written
        assert bool((torch.as_strided(scales, (n - 1, pad), (blocks + pad, 1), scales.storage_offset() + blocks) == 7).all())


@pytest.mark.parametrize("kind", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("n,d,pad,shift", [(1, 1, 0, 0), (0, 5, 0, 0), (3, 31, 0, 0), (40, 32, 0, 0), (40, 33, 0, 0), (17, 64, 8, 0), (20, 257, 3, 1),
                                           (40, 1001, 5, 3), (700, 96, 0, 0), (33, 4100, 0, 0)])
def test_round_trip(fc, device, kind, dtype, n, d, pad, shift):
    round_trip(fc, device, kind, dtype=dtype, n=n, d=d, pad=pad, shift=shift)


def grad_case(fc, device, n, d, outs, kind="i8", dtype="f16", to="f32", pad=0, shift=0, accumulate=False, scale=1.0, max_outs=None, plan=None):
    t, o = DT[dtype], DT[to]
    g = torch.Generator(device=device)
    g.manual_seed(n + 7 * d + outs)
    plan = plan or fc.Checkpoint(d, n, outs if max_outs is None else max_outs, dtype, format=kind)
    codes, scales = plan.empty(n)
    plan.pack(samples(n, d, t, device, n + d, special=False), codes, scales)
    dy = strided(n, outs, t, device, pad, shift, fill=float("nan"))
    dy.copy_(torch.randn(n, outs, generator=g, device=device))
    old = torch.randn(outs, d, generator=g, device=device).to(o)
    dw = strided(outs, d, o, device, pad, shift)
    got = []
    for _ in range(2):
        dw.copy_(old if accumulate else torch.full_like(old, float("nan")))
        plan.grad(dy, codes, scales, dw, scale=scale, accumulate=accumulate)
        got.append(dw.clone())
    assert torch.equal(*got)  # the same bits again
    x = decode(codes, scales, kind, d)
    assert same(x.to(t).double(), x)  # exact in dy's type
    want, size = scale * dy.double().t() @ x, abs(scale) * dy.double().t().abs() @ x.abs()
    if accumulate:
        want, size = want + old.double(), size + old.double().abs()
    bound = 2 * ((n / 4 + 66) * 2.0 ** -24 * size + U[o] * want.abs()) + TINY[o]
    bad = (got[0].double() - want).abs() > bound
    assert not bool(bad.any()), (int(bad.sum()), float(((got[0].double() - want).abs() / bound).max()))
    if pad and outs > 1:
        assert bool((torch.as_strided(dw, (outs - 1, pad), (d + pad, 1), dw.storage_offset() + d) == 7).all())


@pytest.mark.parametrize("kind", ["i8", "e4m3"])
@pytest.mark.parametrize("n,d,outs", [(1, 1, 1), (1, 40, 16), (2, 33, 7), (31, 64, 64), (64, 100, 130), (65, 257, 96), (300, 520, 129), (1003, 129, 300),
                                      (5000, 64, 72), (20000, 40, 24), (130, 1500, 2100), (256, 3000, 2600)])
def test_gradient_sizes(fc, device, kind, n, d, outs):
    grad_case(fc, device, n, d, outs, kind)


@pytest.mark.parametrize("kind", ["i8", "e4m3"])
@pytest.mark.parametrize("n,d,outs,dtype,to,pad,shift,accumulate", [
    (1, 1100, 1100, "f16", "f32", 0, 0, False), (70, 1300, 1031, "bf16", "f16", 3, 1, True), (300, 2049, 777, "f16", "bf16", 0, 0, False),
    (77, 1200, 1040, "bf16", "f32", 8, 0, True), (700, 520, 2503, "f16", "f32", 5, 3, False), (4097, 300, 130, "bf16", "f32", 1, 1, True)])
def test_gradients_of_more_tiles(fc, device, kind, n, d, outs, dtype, to, pad, shift, accumulate):
    """Past what goes in one launch: more tiles than compute units, or so many tokens that k is split."""
    grad_case(fc, device, n, d, outs, kind, dtype, to, pad, shift, accumulate=accumulate)


def test_largest_activations_stay_in_range(fc, device):
    """fp16's largest number rounds to 65536 in 8 bits, which is taken as the largest again, by gradients of few tiles and many."""
    for outs in (64, 4096):
        plan = fc.Checkpoint(300, 80, outs)
        x = torch.full((80, 300), 65504.0, dtype=torch.float16, device=device)
        codes, scales = plan.empty(80)
        plan.pack(x, codes, scales)
        dw = torch.empty(outs, 300, device=device)
        dy = torch.zeros(80, outs, dtype=torch.float16, device=device)
        dy[33] = 0.5
        plan.grad(dy, codes, scales, dw)
        kept = torch.empty_like(x)
        plan.unpack(codes, scales, kept)
        assert torch.equal(dw, (kept[33].float() * 0.5).expand(outs, 300))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("to", list(DT))
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (3, 1)])
def test_gradient_types_strides_alignment(fc, device, dtype, to, pad, shift):
    grad_case(fc, device, 77, 120, 65, "e4m3", dtype, to, pad, shift)  # 65 outputs: dy may lie anywhere
    if shift == 0:
        grad_case(fc, device, 77, 121, 64, "i8", dtype, to, pad, shift)


@pytest.mark.parametrize("to", list(DT))
@pytest.mark.parametrize("n,d,outs", [(40, 70, 50), (9000, 40, 33)])
def test_gradient_accumulates(fc, device, to, n, d, outs):
    grad_case(fc, device, n, d, outs, to=to, accumulate=True, scale=-0.375)


def test_fewer_outputs_than_the_plan(fc, device):
    plan = fc.Checkpoint(96, 500, 201, "bf16")
    for n, outs in ((500, 201), (3, 8), (499, 64), (77, 7)):
        grad_case(fc, device, n, 96, outs, dtype="bf16", plan=plan)


def test_no_tokens(fc, device):
    plan = fc.Checkpoint(40, 8, 16)
    codes, scales = plan.empty(0)
    for accumulate in (True, False):
        dw = torch.full((16, 40), 3.0, device=device)
        plan.grad(torch.empty(0, 16, dtype=torch.float16, device=device), codes, scales, dw, accumulate=accumulate)
        assert bool((dw == (3.0 if accumulate else 0.0)).all())
    codes, scales = plan.empty(4)
    plan.pack(torch.ones(4, 40, device=device), codes, scales)
    plan.grad(torch.empty(4, 0, dtype=torch.float16, device=device), codes, scales, torch.empty(0, 40, device=device))


def test_nan_stays_in_its_columns(fc, device):
    """A block of NaN spoils the gradient of its 32 inputs, and no other's; activations at fp16's largest stay finite."""
    torch.manual_seed(7)
    plan = fc.Checkpoint(100, 50, 24)
    x = torch.randn(50, 100, device=device).half()
    x[7, 40] = float("inf")
    x[9, 99] = 65504.0
    codes, scales = plan.empty(50)
    plan.pack(x, codes, scales)
    dy = torch.randn(50, 24, device=device).half()
    dw = torch.empty(24, 100, device=device)
    plan.grad(dy, codes, scales, dw)
    spoilt = torch.zeros(100, dtype=torch.bool, device=device)
    spoilt[32:64] = True
    assert bool(dw[:, spoilt].isnan().all()) and bool(dw[:, ~spoilt].isfinite().all())


def test_gradient_is_that_of_the_product(fc, device):
    """<dw, v> = <dy, x v^T> along a random direction v: both sums of the same exact products, fp32 rounding apart."""
    n, d, outs = 200, 96, 56
    torch.manual_seed(8)
    plan = fc.Checkpoint(d, n, outs)
    x = torch.randn(n, d, device=device)
    codes, scales = plan.empty(n)
    plan.pack(x, codes, scales)
    kept = torch.empty_like(x)
    plan.unpack(codes, scales, kept)
    dy, v = torch.randn(n, outs, device=device).half(), torch.randn(outs, d, device=device).double()
    dw = torch.empty(outs, d, device=device)
    plan.grad(dy, codes, scales, dw)
    left, right = (dw.double() * v).sum(), (dy.double() * (kept.double() @ v.t())).sum()
    size = (dy.double().abs() * (kept.double().abs() @ v.abs().t())).sum()
    assert abs(float(left - right)) <= (n / 4 + 66) * 2.0 ** -24 * float(size)
    # i8: half a step.  The largest magnitude is 64 to 127.5 steps, or from 63.75 on where it would round to 128 at
    # half the step: half a step is at most 1 / 127.5 of it
    most = torch.nn.functional.pad(x, (0, -d % 32)).view(n, -1, 32).abs().amax(2).repeat_interleave(32, 1)[:, :d]
    assert bool(((kept - x).abs() <= most / 127.5).all())


def test_streams_and_graph(fc, device):
    """Calls on two streams in turn use the workspace one after the other; captured calls give the eager ones' bits."""
    n, d, outs = 900, 200, 203
    plan = fc.Checkpoint(d, n, outs, "bf16", format="e4m3")
    g = torch.Generator(device=device)
    g.manual_seed(2)
    sets = [(torch.randn(n, d, generator=g, device=device), torch.randn(n, outs, generator=g, device=device).bfloat16(), *plan.empty(n)) for _ in range(3)]
    want, got = ([torch.empty(outs, d, device=device) for _ in sets] for _ in range(2))

    def call(s, out, stream=None):
        plan.pack(s[0], s[2], s[3], stream=stream)
        plan.grad(s[1], s[2], s[3], out, stream=stream)

    for s, o in zip(sets, want):
        call(s, o)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for k in range(3):
        for i, s in enumerate(sets):
            call(s, got[i], streams[(i + k) % 2])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    s, out, back = sets[0], torch.empty(outs, d, device=device), torch.empty(n, d, device=device)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(s, out)
        plan.unpack(s[2], s[3], back)
    for k in range(4):
        s[0].copy_(torch.randn(n, d, generator=g, device=device))
        s[1].copy_(torch.randn(n, outs, generator=g, device=device))
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        a, b = out.clone(), back.clone()
        call(sets[1], got[1])  # the program's own calls between
        call(s, out)
        plan.unpack(s[2], s[3], back)
        assert torch.equal(a, out) and torch.equal(b, back), k


def test_refusals(fc, device):
    plan = fc.Checkpoint(40, 8, 16)
    x, (codes, scales) = torch.zeros(8, 40, device=device), plan.empty(8)
    plan.pack(x, codes, scales)
    dy, dw = torch.zeros(8, 16, dtype=torch.float16, device=device), torch.zeros(16, 40, device=device)
    plan.grad(dy, codes, scales, dw)
    for bad in (lambda: plan.pack(x.double(), codes, scales), lambda: plan.pack(x[:7], codes, scales), lambda: plan.pack(x, codes.view(torch.uint8), scales),
                lambda: plan.pack(x, codes[:, :40], scales), lambda: plan.pack(x, codes, scales.int()), lambda: plan.pack(x, codes, scales[:, :1]),
                lambda: plan.pack(x.cpu(), codes, scales), lambda: plan.pack(x.tolist(), codes, scales), lambda: plan.pack(x[0], codes, scales),
                lambda: plan.unpack(codes, scales, x.t()), lambda: plan.unpack(codes[:1].expand(8, 64), scales, x),
                lambda: plan.grad(dy.bfloat16(), codes, scales, dw), lambda: plan.grad(dy[:, :15], codes, scales, dw),
                lambda: plan.grad(dy.repeat(2, 1), *plan.empty(16), dw), lambda: plan.grad(dy.repeat(1, 2), codes, scales, dw.repeat(2, 1))):
        with pytest.raises(ValueError):
            bad()
    wide = torch.zeros(8, 80, dtype=torch.int8, device=device)
    flat = torch.zeros(8 * 24 + 8, dtype=torch.float16, device=device)
    first = codes.view(-1)
    other, small = fc.Checkpoint(8, 1, 8), torch.zeros(1, 16, dtype=torch.float16, device=device)
    for code, bad in ((-3, lambda: plan.pack(first[:80].view(torch.float16).view(1, 40), codes[:1], scales[:1])),
                      (-3, lambda: plan.unpack(codes[:1], scales[:1], first[:160].view(torch.float32).view(1, 40))),
                      (-3, lambda: plan.pack(x, codes, first[:16].view(torch.uint8).view(8, 2))),
                      (-3, lambda: other.grad(small[:, :1], *other.empty(1), small.view(torch.float32))),
                      (-2, lambda: plan.pack(x, wide[:, 8:72], scales)),
                      (-2, lambda: plan.pack(x, torch.zeros(8 * 72, dtype=torch.int8, device=device).view(8, 72)[:, :64], scales)),
                      (-2, lambda: plan.grad(flat[1:1 + 8 * 16].view(8, 16), codes, scales, dw)),
                      (-2, lambda: plan.grad(flat[:8 * 20].view(8, 20)[:, :16], codes, scales, dw))):
        with pytest.raises(fc.FcError) as e:
            bad()
        assert e.value.code == code
    for args in ((0, 1), ((1 << 21) + 1, 1), (8, -1), (8, 1 << 31), (8, 1, -1), (8, 1, (1 << 21) + 1)):
        with pytest.raises(fc.FcError) as e:
            fc.Checkpoint(*args)
        assert e.value.code == -1
    for kw in ({"dtype": "f32"}, {"format": "e5m2"}):
        with pytest.raises(ValueError):
            fc.Checkpoint(8, 1, **kw)


def test_fresh_workspaces_may_hold_anything(fc, device):
    junk = [torch.full((1 << 24,), float("nan"), device=device) for _ in range(8)]
    torch.cuda.synchronize()
    del junk
    torch.cuda.empty_cache()
    grad_case(fc, device, 70, 129, 67)
    grad_case(fc, device, 6000, 45, 39)
