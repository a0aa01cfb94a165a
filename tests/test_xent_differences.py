"""The cross entropy's gradients against central differences of its losses, in
directions along the gradients, where the difference is as large as its terms.

Inputs and steps are multiples of 2^-8 below 4, so that fp16 holds base, base +
step and base - step exactly and the difference's second-order term is zero.  With
f(s) the losses' sum at base + s step:
  f(1) - f(-1) = 2 f'(0) + f'''(z) / 3, and |f'''| <= the sum over tokens of (2 D)^3
  sqrt(3) / 18, the largest third central moment in an interval of 2 D, D the largest
  change of a token's logits (the target's part is linear);
  each loss is off by 2 E + 4 u32 A + 80 u32 + 4 u32 |lse|, E = (dim + 2) u32 A,
  u32 = 2^-24, A[t] = the largest over r of sum |x[t, d] w[r, d]|;
  a gradient's entries are off by 3 u (softmax's part + the target's part in size), u = 2^-11."""
import pytest

torch = pytest.importorskip("torch")

ROWS, DIM = 400, 64
U, U32 = 2.0 ** -11, 2.0 ** -24


def inputs(n, seed):
    g = torch.Generator()
    g.manual_seed(seed)

    def on_grid(t, steps):
        return (t.clamp(-3.9, 3.9) * steps).round() / steps

    w = on_grid(torch.randn(ROWS, DIM, generator=g) * DIM ** -0.5, 256)
    y = torch.randint(0, ROWS, (n,), generator=g)
    x = on_grid(torch.randn(n, DIM, generator=g) + 2 * w[y], 128)
    return x.double(), w.double(), y, g


def parts(x, w, y):
    """(softmax's part, the target's part) of the gradients by x and by w, in 64 bits."""
    p = (x @ w.t()).softmax(1)
    t = torch.zeros_like(p)
    t[torch.arange(len(y)), y] = 1
    return {"x": (p @ w, t @ w), "w": (p.t() @ x, t.t() @ x)}, p + t


def failures(n, seed, losses, gradients):
    """(which, direction, difference over tolerance) where losses(x, w, y) and
    gradients(x, w, y) -> {"x", "w"} disagree."""
    x, w, y, g = inputs(n, seed)
    got = gradients(x, w, y)
    both, size = parts(x, w, y)
    bad = []
    for which in "xw":
        soft, target = both[which]
        # along the gradient; along softmax's part, which the target's then offsets
        for name, along in (("gradient", soft - target), ("softmax", soft)):
            step = along.sign() * 2.0 ** -8 * torch.randint(1, 3, along.shape, generator=g)
            places = [(x + s * step, w) if which == "x" else (x, w + s * step) for s in (1, -1)]
            assert all(torch.equal(t.half().double(), t) for t in (x, w, *places[0], *places[1]))
            ends = [losses(*p, y) for p in places]
            left, right = float(ends[0] - ends[1]), float((got[which] * 2 * step).sum())
            change = (step @ w.t() if which == "x" else x @ step.t()).abs().amax(1)
            a = (x.abs() @ w.abs().t()).amax(1) + change
            lse = torch.logsumexp(x @ w.t(), 1).abs() + change
            each = 2 * (DIM + 2) * U32 * a + 4 * U32 * a + 80 * U32 + 4 * U32 * lse
            terms = size @ w.abs() if which == "x" else size.t() @ x.abs()
            tolerance = float(((2 * change) ** 3 * 3 ** 0.5 / 18 / 3).sum() + 2 * each.sum() + 3 * U * (terms * 2 * step.abs()).sum())
            if not abs(left - right) <= tolerance:
                bad.append((which, name, abs(left - right) / tolerance))
    return bad


def plain_losses(x, w, y):
    return torch.nn.functional.cross_entropy(x @ w.t(), y, reduction="sum")


def plain_gradients(x, w, y):
    return {k: s - t for k, (s, t) in parts(x, w, y)[0].items()}


@pytest.mark.parametrize("n", [50, 200])
def test_the_check_finds_wrong_gradients(n):
    """In 64 bits on the CPU: the gradients pass, and every one with a term left
    out, a factor or a sign that is wrong fails in both operands."""
    assert not failures(n, 1, plain_losses, plain_gradients)
    for wrong in (lambda s, t: -t, lambda s, t: s, lambda s, t: t - s, lambda s, t: s + t, lambda s, t: 1.5 * (s - t),
                  lambda s, t: 2 * (s - t), lambda s, t: 0.5 * (s - t), lambda s, t: 0 * s):
        bad = failures(n, 1, plain_losses, lambda x, w, y: {k: wrong(*v) for k, v in parts(x, w, y)[0].items()})
        assert {which for which, _, _ in bad} == {"x", "w"}, bad


@pytest.mark.gpu
@pytest.mark.parametrize("n", [50, 200])
@pytest.mark.parametrize("seed", [1, 2])
def test_gradients_against_differences(device, n, seed):
    import paper_1511_00175_amd as fc
    plan = fc.CrossEntropy(ROWS, DIM, n, "f16")

    def args(x, w, y):
        return x.half().to(device), w.half().to(device), y.to(device), torch.zeros(n, device=device)

    def losses(x, w, y):
        a = args(x, w, y)
        plan.loss(*a)
        return a[3].double().sum().cpu()

    def gradients(x, w, y):
        dx, dw = torch.zeros(n, DIM, device=device), torch.zeros(ROWS, DIM, device=device)
        plan.loss_grad(*args(x, w, y), dx, dw)
        return {"x": dx.double().cpu(), "w": dw.double().cpu()}

    assert not failures(n, seed, losses, gradients)
