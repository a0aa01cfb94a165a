"""Vocabulary cross entropy on the GPU against the definition in 64 bits.

Bounds, from the operations (u32 = 2^-24, u = 2^-11 for fp16 and 2^-8 for bf16,
the unit roundoffs; A[t] = the largest over r of sum |x[t, d] w[r, d]|):
  logits   |err| <= E[t] = (dim + 2) u32 A[t]: an fp32 sum of dim exact products
  loss     the two logits' errors and the exponentials': a factor exp(l - m) is
           off by 2 u32 |l - m| + 4 u32 relative, |l - m| <= 2 A[t], and the sum
           and its logarithm by less than 64 u32 (pieces, joined pairwise) and
           2 u32 |loss|:  |err| <= 2 E + 4 u32 A + 80 u32 + 4 u32 |lse|
  d        relative error g = 2 u + 2 E + 6 u32 A + 80 u32 of the softmax part
           (two roundings; the exponents' errors), u of the whole entry, and the
           stored type's smallest steps: 2^-25 of a piece's largest numerator,
           and 2^-24 / 2^15 (fp16; nothing for bf16)
  dx, dw   the sum over the entries' errors, the fp32 sum's (terms + 4) u32 of
           the terms' absolute sum, and the output's rounding u_out |y|."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 1e-37, "f16": 2.0 ** -24, "bf16": 1e-37}


@pytest.fixture(scope="module")
def fc(device):
    import paper_1511_00175_amd as m
    return m


def inputs(device, rows, dim, n, dtype, seed=0, pad=0, gain=1.0, masked=0.1):
    g = torch.Generator(device=device)
    g.manual_seed(seed * 1000 + rows + 3 * dim + 7 * n)
    w = torch.zeros(rows, dim + pad, dtype=DT[dtype], device=device)[:, :dim]
    x = torch.zeros(n, dim + pad, dtype=DT[dtype], device=device)[:, :dim]
    w.copy_(torch.randn(rows, dim, generator=g, device=device) * dim ** -0.5)
    y = torch.randint(0, rows, (n,), generator=g, device=device)
    x.copy_(gain * (torch.randn(n, dim, generator=g, device=device) + 2 * w[y].float()))
    y = torch.where(torch.rand(n, generator=g, device=device) < masked, -100, y)
    return x, w, y


def check(fc, device, x, w, y, dtype, scale=0.75, out_x=None, out_w=None, chunk=0, plan=None, dx=None, dw=None):
    rows, dim = w.shape
    n = x.shape[0]
    out_x, out_w = out_x or dtype, out_w or dtype
    plan = plan or fc.CrossEntropy(rows, dim, n, dtype, chunk)
    nan = float("nan")
    loss = torch.full((n,), nan, device=device)
    dx = torch.full((n, dim), nan, dtype=DT[out_x], device=device) if dx is None else dx
    dw = torch.full((rows, dim), nan, dtype=DT[out_w], device=device) if dw is None else dw
    plan.loss_grad(x, w, y, loss, dx, dw, scale=scale)
    alone = torch.full((n,), nan, device=device)
    plan.loss(x, w, y, alone)
    assert torch.equal(loss, alone)

    live = (y >= 0) & (y < rows)
    u32, u = U["f32"], U[dtype]
    X, W, Y = x[live].double(), w.double(), y[live]
    L = X @ W.t()
    A = (X.abs() @ W.abs().t()).amax(1) if len(Y) else torch.zeros(0, device=device, dtype=torch.float64)
    E = (dim + 2) * u32 * A
    lse = torch.logsumexp(L, 1)
    at = torch.arange(len(Y), device=device)
    want = lse - L[at, Y]
    assert bool((loss[~live] == 0).all())
    assert bool(((loss[live].double() - want).abs() <= 2 * E + 4 * u32 * A + 80 * u32 + 4 * u32 * lse.abs()).all())

    P = torch.exp(L - lse[:, None])
    D = P.clone()
    D[at, Y] -= 1
    rel = (2 * u + 2 * E + 6 * u32 * A + 80 * u32)[:, None]
    eD = rel * P + u * D.abs()
    if dtype == "f16":  # numerators and d have a smallest step
        eD += 2.0 ** -25 * P.amax(1, keepdim=True) + 2.0 ** -40
    for got, other, d, ed, o in ((dx[live], W, D, eD, out_x), (dw, X, D.t(), eD.t(), out_w)):
        ref = d @ other
        bound = scale * (ed @ other.abs() + (d.shape[1] + 4) * u32 * (d.abs() @ other.abs())) + U[o] * scale * ref.abs()
        err = (got.double() - scale * ref).abs()
        assert bool((err <= 1.01 * bound + TINY[o]).all()), float((err / (bound + TINY[o])).max())
    assert bool((dx[~live] == 0).all())
    # the same bits again
    a, b, c = loss.clone(), dx.clone(), dw.clone()
    plan.loss_grad(x, w, y, loss, dx, dw, scale=scale)
    assert torch.equal(a, loss) and torch.equal(b, dx) and torch.equal(c, dw)
    return plan, loss, dx, dw


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows,dim,n", [(1, 8, 1), (7, 64, 3), (1000, 72, 64), (1001, 264, 65), (130, 1000, 129), (2500, 96, 300),
                                        (3001, 520, 7), (64, 64, 64), (33, 8, 1000)])
def test_sizes(fc, device, rows, dim, n, dtype):
    check(fc, device, *inputs(device, rows, dim, n, dtype), dtype)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_large_tiles(fc, device, dtype):
    """Enough tokens, rows and columns for every product's large tiles."""
    check(fc, device, *inputs(device, 17000, 1032, 1100, dtype), dtype)
    check(fc, device, *inputs(device, 260, 4100, 4200, dtype), dtype)
    check(fc, device, *inputs(device, 20001, 520, 1003, dtype), dtype)
    check(fc, device, *inputs(device, 4097, 1290, 4100, dtype), dtype)


@pytest.mark.parametrize("dtype,n,dim", [("f16", 5, 4104), ("bf16", 64, 4097)])
def test_weights_larger_than_the_caches(fc, device, dtype, n, dim):
    """At least 2^28 bytes of w for few tokens."""
    check(fc, device, *inputs(device, 32801, dim, n, dtype), dtype)


@pytest.mark.parametrize("dim", [1, 3, 63, 130, 1001])
def test_odd_dimensions(fc, device, dim):
    check(fc, device, *inputs(device, 777, dim, 200, "bf16"), "bf16")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("chunk", [1, 64, 100, 256])
def test_chunks(fc, device, dtype, chunk):
    """Tokens in several chunks: dw is summed over them in fp32."""
    check(fc, device, *inputs(device, 1500, 128, 515 if chunk > 1 else 5, dtype), dtype, chunk=chunk)


@pytest.mark.parametrize("out_x", list(DT))
@pytest.mark.parametrize("out_w", list(DT))
def test_output_types_and_strides(fc, device, out_x, out_w):
    for dtype in ("f16", "bf16"):
        x, w, y = inputs(device, 515, 72, 90, dtype, pad=24)
        dx = torch.full((90, 72 + 5), 3.0, dtype=DT[out_x], device=device)
        dw = torch.full((515 * (72 + 3) + 1,), 3.0, dtype=DT[out_w], device=device)[1:].view(515, 75)
        check(fc, device, x, w, y.to(torch.int32), dtype, out_x=out_x, out_w=out_w, dx=dx[:, 1:73], dw=dw[:, :72])
        assert bool((dx[:, 0] == 3).all()) and bool((dx[:, 73:] == 3).all()) and bool((dw[:, 72:] == 3).all())


@pytest.mark.parametrize("gain", [0.0, 30.0])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_flat_and_sharp_distributions(fc, device, gain, dtype):
    """Logits all alike (probabilities of 1 / rows) and far apart (almost all
    probability on a row)."""
    check(fc, device, *inputs(device, 9000, 64, 150, dtype, gain=gain), dtype)


def test_padding_may_hold_anything(fc, device):
    x, w, y = inputs(device, 600, 128, 100, "bf16", masked=0.0)
    y[::3] = torch.tensor([-1, 600, -2 ** 31, 2 ** 40], device=device).repeat(9)[:34]
    clean = check(fc, device, x, w, y, "bf16")
    x[::6] = float("nan")
    x[3::6] = float("inf")
    dirty = check(fc, device, x, w, y, "bf16")
    for a, b in zip(clean[1:], dirty[1:]):
        assert torch.equal(a, b)
    y.fill_(-1)  # no token left
    plan = fc.CrossEntropy(600, 128, 100, "bf16")
    loss, dx, dw = torch.ones(100, device=device), torch.ones_like(x), torch.ones_like(w)
    plan.loss_grad(x, w, y, loss, dx, dw)
    assert not loss.any() and not dx.any() and not dw.any()
    w[5] = float("nan")  # nor does a padding token meet what w holds
    dx.fill_(1)
    plan.loss_grad(x, w, y, loss, dx, None)
    assert not loss.any() and not dx.any()


def test_infinite_inputs_are_not_hidden(fc, device):
    """A token with an infinite logit or a NaN has no finite loss; the others
    keep theirs."""
    x, w, y = inputs(device, 300, 64, 80, "f16", masked=0.0)
    plan, loss, _, _ = check(fc, device, x, w, y, "f16")
    x2 = x.clone()
    x2[7, 3] = float("nan")
    x2[9, 5] = float("inf")
    got = torch.zeros_like(loss)
    plan.loss(x2, w, y, got)
    keep = torch.ones(80, dtype=torch.bool, device=device)
    keep[[7, 9]] = False
    assert torch.equal(got[keep], loss[keep]) and not bool(torch.isfinite(got[~keep]).any())
    w2 = w.clone()
    w2[:, 0] = 0
    w2[11] = 0
    w2[11, 0] = float("-inf")  # one row that no token can choose: exp(-inf) = 0
    x3 = x.clone()
    x3[:, 0] = 1
    y3 = torch.where(y == 11, 12, y)
    plan.loss(x3, w2, y3, got)
    L = x3.double() @ w2.double().t()
    want = torch.logsumexp(L, 1) - L[torch.arange(80, device=device), y3]
    assert bool(((got.double() - want).abs() < 1e-4).all())


def test_gradients_against_differences(fc, device):
    """Central differences of the fp32 losses, in a random direction of x and of
    w: the step's cubic term and the losses' roundings bound the difference."""
    rows, dim, n = 400, 64, 50
    x, w, y = inputs(device, rows, dim, n, "f16")
    plan = fc.CrossEntropy(rows, dim, n, "f16")
    loss, dx, dw = torch.zeros(n, device=device), torch.zeros(n, dim, device=device), torch.zeros(rows, dim, device=device)
    plan.loss_grad(x, w, y, loss, dx, dw)
    g = torch.Generator(device=device)
    g.manual_seed(1)
    for which, grad in ((0, dx), (1, dw)):
        base = (x, w)[which]
        step = torch.randn(base.shape, generator=g, device=device) * 2.0 ** -6
        up, down = (base.float() + step).half(), (base.float() - step).half()
        ends = []
        for moved in (up, down):
            args = [x, w]
            args[which] = moved
            plan.loss(args[0], args[1], y, loss)
            ends.append(loss.double().sum())
        moved = up.double() - down.double()
        left, right = float(ends[0] - ends[1]), float((grad.double() * moved).sum())
        assert abs(left - right) <= 0.02 * float((grad.double() * moved).abs().sum())


def test_one_gradient_alone(fc, device):
    x, w, y = inputs(device, 900, 128, 150, "f16")
    plan, loss, dx, dw = check(fc, device, x, w, y, "f16")
    a, b = torch.zeros_like(dx), torch.zeros_like(dw)
    plan.loss_grad(x, w, y, loss, a, None, scale=0.75)
    plan.loss_grad(x, w, y, loss, None, b, scale=0.75)
    assert torch.equal(a, dx) and torch.equal(b, dw)


def test_no_tokens(fc, device):
    x, w, y = inputs(device, 50, 16, 0, "f16")
    plan = fc.CrossEntropy(50, 16, 8, "f16")
    dw = torch.ones_like(w)
    plan.loss_grad(x, w, y, torch.zeros(0, device=device), torch.zeros_like(x), dw)
    assert not dw.any()


def test_streams_are_ordered(fc, device):
    sets = [inputs(device, 4000, 256, 300, "f16", seed=k) for k in range(4)]
    plan = fc.CrossEntropy(4000, 256, 300, "f16")
    outs = [(torch.zeros(300, device=device), torch.zeros_like(x), torch.zeros_like(w)) for x, w, _ in sets]
    want = []
    for (x, w, y), o in zip(sets, outs):
        plan.loss_grad(x, w, y, *o)
        want.append([t.clone() for t in o])
        for t in o:
            t.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for i, ((x, w, y), o) in enumerate(zip(sets, outs)):
        plan.loss_grad(x, w, y, *o, stream=streams[i % 2])
    torch.cuda.synchronize()
    for o, t in zip(outs, want):
        assert all(torch.equal(p, q) for p, q in zip(o, t))


def test_graph(fc, device):
    x, w, y = inputs(device, 1200, 128, 200, "bf16")
    plan = fc.CrossEntropy(1200, 128, 200, "bf16")
    loss, dx, dw = torch.zeros(200, device=device), torch.zeros_like(x), torch.zeros_like(w)
    plan.loss_grad(x, w, y, loss, dx, dw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.loss_grad(x, w, y, loss, dx, dw)
    for k in range(4):
        x2, w2, y2 = inputs(device, 1200, 128, 200, "bf16", seed=k + 1)
        x.copy_(x2), w.copy_(w2), y.copy_(y2)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (loss, dx, dw)]
        plan.loss_grad(x, w, y, loss, dx, dw)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, (loss, dx, dw))), k


def test_refusals(fc, device):
    x, w, y = inputs(device, 100, 64, 16, "f16")
    plan = fc.CrossEntropy(100, 64, 16, "f16")
    loss = torch.zeros(16, device=device)
    for bad in (lambda: plan.loss(x.bfloat16(), w, y, loss), lambda: plan.loss(x.float(), w, y, loss),
                lambda: plan.loss(x, w[:99], y, loss), lambda: plan.loss(x, w, y.float(), loss),
                lambda: plan.loss(x, w, y, loss.half()), lambda: plan.loss(x, w, y, loss[:15]),
                lambda: plan.loss(x.repeat(2, 1), w, y.repeat(2), loss.repeat(2)), lambda: plan.loss(x, w, y[:15], loss),
                lambda: plan.loss_grad(x, w, y, loss, x.double(), None), lambda: fc.CrossEntropy(100, 64, 16, "f32")):
        with pytest.raises(ValueError):
            bad()
    odd = torch.zeros(100 * 64 + 4, dtype=torch.float16, device=device)[4:].view(100, 64)
    for bad, code in ((lambda: plan.loss_grad(x, w, y, loss, x, None), -3), (lambda: plan.loss_grad(x, w, y, loss, None, w), -3),
                      (lambda: plan.loss(x, odd, y, loss), -2), (lambda: fc.CrossEntropy(0, 64, 16), -1),
                      (lambda: fc.CrossEntropy(1 << 22, 64, 16), -1), (lambda: fc.CrossEntropy(10, 64, 16, chunk=-1), -1)):
        with pytest.raises(fc.FcError) as e:
            bad()
        assert e.value.code == code


@pytest.mark.parametrize("rows", [1500, 33, 1001, 130, 4000])
@pytest.mark.parametrize("n", [3, 64, 70, 600])
def test_fresh_workspaces_may_hold_anything(fc, device, rows, n):
    """Plans made where other memory was: what their workspaces hold before a
    call does not matter."""
    junk = [torch.full((1 << 24,), float("nan"), device=device) for _ in range(8)]
    torch.cuda.synchronize()
    del junk
    torch.cuda.empty_cache()
    for dtype in ("f16", "bf16"):
        x, w, y = inputs(device, rows, 264, n, dtype)
        check(fc, device, x, w, y, dtype, plan=fc.CrossEntropy(rows, 264, n, dtype, chunk=0 if n < 100 else 64))
