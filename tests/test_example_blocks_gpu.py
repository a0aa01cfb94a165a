"""The example with residual blocks: one step's gradients are those of the same model
in 64 bits whose blocks' products and kept inputs are rounded to the same formats, and
a step runs with every update.

What separates the two is the example's fp16 (y, b, dy, db and the two gradients of
the loss; 8 roundings of 2^-11 between a weight and its gradient), and the elements
whose value beside a border between two 4-bit or 8-bit numbers falls to the other side
for it.  4-bit numbers are at least a sixth of their size apart, so that a shift of 8 *
2^-11 moves at most 6 * 8 * 2^-11 of them, by a third of their size at most: the root
of 0.024 times a third, 5% of a product's norm, added up over the two blocks' two
products each as independent errors: 10%."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

from block_formats import quantise  # noqa: E402

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EPS = 1e-6


@pytest.fixture(scope="module")
def lm_blocks(device):
    spec = importlib.util.spec_from_file_location("lm_blocks", os.path.join(ROOT, "examples", "lm_blocks.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


class Product(torch.autograd.Function):
    """y W^T of 4-bit numbers; the gradients as the example takes them: dW from y in 8 bits, dy from 4-bit ones."""

    @staticmethod
    def forward(ctx, y, w):
        ctx.save_for_backward(y, w)
        return quantise(y, "e2m1")[0] @ quantise(w, "e2m1")[0].t()

    @staticmethod
    def backward(ctx, d):
        y, w = ctx.saved_tensors
        return quantise(d, "e2m1")[0] @ quantise(w.t(), "e2m1")[0].t(), d.t() @ quantise(y, "i8")[0]


def norm(x):
    return x * (x.square().mean(1, keepdim=True) + EPS).rsqrt()


def test_gradients(lm_blocks, device):
    model = lm_blocks.Model(vocab=300, dim=96, blocks=2, workers=2, tokens=500, seed=3)
    g = torch.Generator(device=device)
    g.manual_seed(4)
    for name, (at, shape) in model.places.items():  # vectors away from where they begin
        if len(shape) == 1:
            model.part(model.w, name).add_(0.3 * torch.randn(shape, generator=g, device=device))
    w = model.w.double().requires_grad_()
    p = {n: model.part(w, n) for n in model.places}
    data = lm_blocks.batches(model, 5)
    want = 0
    for tokens, targets in data:
        h = p["E"][tokens]
        y = norm(h) * p["v"]
        for i in range(model.blocks):
            b = Product.apply(y, p[f"W{i}"])
            h = h + lm_blocks.SCALE * torch.sigmoid(p[f"g{i}"]) * p[f"v{i}"] * norm(b)
            y = norm(h) * p[f"u{i}"]
        want = want + torch.nn.functional.cross_entropy(y @ p["U"].t(), targets, ignore_index=-1, reduction="sum")
    want.backward()
    loss = torch.cat([model.gradients(k, *b) for k, b in enumerate(data)])
    assert abs(float(loss.double().sum() - want.detach())) < 1e-2 * float(want.detach())
    model.reduce.tree_reduce(model.replicas, model.sum)
    for n in model.places:
        got, ref = model.part(model.sum, n).double(), model.part(w.grad, n)
        assert float((got - ref).norm()) <= 0.1 * float(ref.norm()), n


def test_a_step_changes_every_weight(lm_blocks, device):
    model = lm_blocks.Model(blocks=3)
    before = model.w.clone()
    losses = [float(model.step(lm_blocks.batches(model, k))) for k in range(3)]
    assert all(v == v and v < 20 for v in losses) and bool(model.w.isfinite().all())
    for n in model.places:
        moved = model.part(model.w, n) != model.part(before, n)
        assert bool(moved.float().mean() > 0.9), n
