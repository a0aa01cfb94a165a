"""The example's training step: its loss falls, and one step's gradients are
those of the same model in 64 bits.

The example's activations and products are fp16 with fp32 sums; each of the at
most 6 roundings between weights and gradients (the 16-bit copies of E, U and M,
h M, d, the two products of dz) is 2^-11 of its operand, so gradients agree to
8 * 2^-11 of their norm."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lm_step(device):
    spec = importlib.util.spec_from_file_location("lm_step", os.path.join(ROOT, "examples", "lm_step.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_gradients(lm_step, device):
    model = lm_step.Model(vocab=300, dim=64, workers=3, tokens=500)
    w = model.w.double().requires_grad_()
    E, U, M = (model.part(w, n) for n in ("E", "U", "M"))
    data = lm_step.batches(model, 5)
    want = 0
    for tokens, targets in data:
        logits = (E[tokens] @ M) @ U.t()
        want = want + torch.nn.functional.cross_entropy(logits, targets, ignore_index=-1, reduction="sum")
    want.backward()
    loss = torch.cat([model.gradients(k, *b) for k, b in enumerate(data)])
    assert abs(float(loss.double().sum() - want.detach())) < 1e-3 * float(want.detach())
    model.reduce.tree_reduce(model.replicas, model.sum)
    for n in ("E", "U", "M"):
        got, ref = model.part(model.sum, n).double(), model.part(w.grad, n)
        assert float((got - ref).norm()) <= 8 * 2.0 ** -11 * float(ref.norm()), n


def test_loss_falls(lm_step, device):
    model = lm_step.Model()
    losses = [float(model.step(lm_step.batches(model, k))) for k in range(60)]
    assert losses[0] > 5.5 and losses[-1] < 0.6 * losses[0], losses
