"""The bounds by which the norms' gradients are judged (norm_gradients.py): fp32's own
arithmetic is within them, and what leaves a term out is not."""
import pytest

torch = pytest.importorskip("torch")

from norm_gradients import CASES, EPS, SCALE, Normed, excess, gradients, inputs  # noqa: E402


def arrange(n, dim, offset):
    return inputs(n, dim, torch.float32, torch.float32, "matrix", "cpu", n + dim, offset)


@pytest.mark.parametrize("n,dim,kind,offset", CASES)
def test_a_missing_term_fails(n, dim, kind, offset):
    s = arrange(n, dim, offset)
    want = gradients(s, kind, EPS, "silu", SCALE, "between")
    mistakes = ["no part along"] + (["no mean"] + (["uncentred"] if offset else []) if kind == "layer" else [])
    for wrong in mistakes:
        for name, (v, _) in gradients(s, kind, EPS, "silu", SCALE, "between", wrong).items():
            if name in ("dh", "db") or wrong == "uncentred":
                over = excess(v, *want[name], dtype=torch.float32)
                assert float((over > 1).double().mean()) > 0.5, (wrong, name, float(over.max()))
    for name, (v, err) in want.items():
        over = excess(torch.zeros_like(v), v, err, dtype=torch.float32)
        assert float((over > 10).double().mean()) > 0.9, (name, float(over.median()))


@pytest.mark.parametrize("n,dim,kind,offset", CASES)
def test_plain_arithmetic_in_32_bits_is_within(n, dim, kind, offset):
    s = arrange(n, dim, offset)
    x, u = s["out"], s["dy"] * s["next"]
    c = x - x.mean(1, keepdim=True) if kind == "layer" else x
    r = 1 / (c.square().mean(1, keepdim=True) + EPS).sqrt()
    xh = c * r
    got = s["dout"] + r * (u - (u.mean(1, keepdim=True) if kind == "layer" else 0) - xh * (u * xh).mean(1, keepdim=True))
    assert float(excess(got, *gradients(s, kind, EPS, "silu", SCALE, "before")["dh"]).max()) <= 1


def test_normed_rows_have_no_mean():
    n = Normed(300 + torch.randn(5, 64), "layer", EPS)
    assert float(n.xh.mean(1).abs().max()) < 1e-12 and float((n.xh.square().mean(1) - 1).abs().max()) < 1e-4
