"""Gates from far below zero to far above it: a(g) and its slope keep their leading bits
where they are small, and are not lost to 1 - a(g).

Bounds, u = 2^-24, relative: t = exp(-|g|) carries the exponential's step (2 u), its
argument's low part (1) and one multiplication (1), 4 u; 1 + t at most 3 more, its
reciprocal 2; the sigmoid of a negative gate, t / (1 + t), 4 + 3 + 2 + 1 = 10, its slope
t / (1 + t)^2 = 4 + 2 (3 + 2) + 2 = 16.  SiLU's value has one more multiplication; its
slope s (1 + g (1 - s)) is off by 10 + 12 + 2 of s (1 + |g| (1 - s)), the sum of its two
terms' sizes.  Then the products with what the gate multiplies (the norm of a row of a
constant magnitude, whose statistics are 16 u off, the weight, the scale, the sum of one
row): 24.  All is doubled for the terms of second order.  A t below 2^-126, |g| above 87.3,
may become 0: with SiLU's factor g, 87.4 there, and the products' largest, 0.75 dw's, less
than 66 2^-126 < 2^-119 is lost."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = 1e-6


@pytest.fixture(scope="module")
def fc(device):
    import paper_1511_00175_amd as m
    return m


def gates(dim, device):
    """Both signs, from 1e-3 to past the exponential's range, each once, and 0."""
    half = torch.cat((torch.logspace(-3, 1, dim // 4, dtype=torch.float64), torch.linspace(10, 100, dim // 2 - dim // 4, dtype=torch.float64)))
    g = torch.cat((half, -half, torch.zeros(dim - 2 * (dim // 2), dtype=torch.float64)))
    return g.float().to(device)


def act_of(g, act):
    """a(g), its slope, and the sizes that their errors are relative to, in 64 bits."""
    g = g.double()
    t = torch.exp(-g.abs())
    up = g >= 0
    s, rest = torch.where(up, 1 / (1 + t), t / (1 + t)), torch.where(up, t / (1 + t), 1 / (1 + t))
    if act == "sigmoid":
        return s, s * rest, s, s * rest
    return g * s, s * (1 + g * rest), (g * s).abs(), s * (1 + g.abs() * rest)


def close(got, want, size):
    err, bound = (got.double() - want).abs(), 2 * (24 + 24) * U * size + 2.0 ** -119
    assert bool((err <= bound).all()), float((err / bound).max())


@pytest.mark.parametrize("form", ["vector", "matrix"])
@pytest.mark.parametrize("act", ["sigmoid", "silu"])
@pytest.mark.parametrize("dim", [4, 60, 1001, 9216])
def test_saturated_gates(fc, device, dim, act, form):
    plan = fc.Norm(dim, 1, "f32", "f32", eps=EPS, gate=act)
    g = gates(dim, device)
    b = torch.where(torch.arange(dim, device=device) % 3 == 0, -0.75, 0.75)[None]
    h, dout, w = torch.zeros(1, dim, device=device), torch.full((1, dim), 1.5, device=device), torch.full((dim,), 0.875, device=device)
    nb = b.double() * (0.75 ** 2 + EPS) ** -0.5
    a, slope, size, size_slope = act_of(g, act)
    out, db, dg = torch.empty_like(h), torch.empty_like(b), torch.empty(dim, device=device)
    dw = torch.empty(dim, device=device)
    given = g if form == "vector" else g[None].clone()
    dgate = dg if form == "vector" else dg[None]
    plan.after(h, b, out, weight=w, gate=given, scale=0.5)
    close(out[0], 0.5 * a * 0.875 * nb[0], (0.5 * size * 0.875 * nb[0]).abs())
    plan.after_grad(b, dout, db, weight=w, dweight=dw, gate=given, dgate=dgate, scale=0.5)
    close(dg, 0.75 * slope * 0.875 * nb[0], (0.75 * size_slope * 0.875 * nb[0]).abs())
    close(dw, 0.75 * a * nb[0], (0.75 * size * nb[0]).abs())


@pytest.mark.parametrize("act", ["sigmoid", "silu"])
@pytest.mark.parametrize("dim", [60, 1001, 9216])
def test_saturated_gates_in_16_bits(fc, device, dim, act):
    """The argument's rounding, 1.5 |g| u, is at most 131 u more where t is above 2^-126, and all is below 2^-16; what
    is stored in bf16 is rounded once, 2^-8."""
    plan = fc.Norm(dim, 1, "bf16", "f32", eps=EPS, gate=act)
    g = gates(dim, device).bfloat16()[None]
    b = torch.where(torch.arange(dim, device=device) % 3 == 0, -0.75, 0.75).bfloat16()[None]
    h, dout = torch.zeros(1, dim, device=device), torch.full((1, dim), 1.5, device=device)
    nb = b.double() * (0.75 ** 2 + EPS) ** -0.5
    a, slope, size, size_slope = act_of(g, act)
    out, db, dg = torch.empty_like(h), torch.empty_like(b), torch.empty_like(b)
    plan.after(h, b, out, gate=g, scale=0.5)
    plan.after_grad(b, dout, db, gate=g, dgate=dg, scale=0.5)
    for got, want, by, rounding in ((out, 0.5 * a * nb, (0.5 * size * nb).abs(), 0.0), (dg, 0.75 * slope * nb, (0.75 * size_slope * nb).abs(), 2.0 ** -8)):
        err, bound = (got.double() - want).abs(), 2 * 2.0 ** -16 * by + rounding * want.abs() + 2.0 ** -119
        assert bool((err <= bound).all()), float((err / bound).max())


def test_gates_without_a_number(fc, device):
    """A gate of NaN gives NaN in its place alone; infinite gates are the ends of a sigmoid."""
    inf, nan = float("inf"), float("nan")
    g = torch.tensor([[inf, -inf, nan, 0.0, 200.0, -200.0, 1.0, -1.0]], device=device)
    b = torch.ones(1, 8, device=device)
    h, out, db, dg = torch.zeros(1, 8, device=device), torch.empty(1, 8, device=device), torch.empty(1, 8, device=device), torch.empty(1, 8, device=device)
    plan = fc.Norm(8, 1, "f32", "f32", eps=EPS, gate="sigmoid")
    plan.after(h, b, out, gate=g)
    assert out.isnan().tolist() == [[k == 2 for k in range(8)]]
    assert out[0, 1] == 0 and out[0, 5] == 0 and out[0, 0] == out[0, 4] and abs(float(out[0, 0]) - 1) < 1e-5
    plan.after_grad(b, b, db, gate=g, dgate=dg)
    assert dg.isnan().tolist() == [[k == 2 for k in range(8)]] and dg[0, [0, 1, 4, 5]].tolist() == [0, 0, 0, 0]
