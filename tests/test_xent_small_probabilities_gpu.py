"""Rows of small probability that share a piece of the vocabulary with one that
holds almost all of it: their gradients keep the bounds of their own size.

Bounds as in test_xent_gpu.py: an entry d[t, r] with r not the target is off by
(2 u + 2 E + 6 u32 A + 80 u32) d, and by the smallest steps of what is stored: half of
2^-39 of the row's largest probability for the numerator (fp16 times 2^15) and 2^-40
for d.  Of the sums only those over such rows are looked at: dw of these rows, and
dx in columns where the other rows of w are zero."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
U = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}
U32 = 2.0 ** -24


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("gain", [8.0, 14.0, 20.0])
@pytest.mark.parametrize("rows,n", [(520, 40), (520, 300), (5000, 1100)])
def test_rows_beside_a_dominant_one(device, rows, n, gain, dtype):
    import paper_1511_00175_amd as fc
    dim, big, other = 64, 5, rows - 100
    g = torch.Generator(device=device)
    g.manual_seed(rows + n)
    w = torch.randn(rows, dim, generator=g, device=device) * dim ** -0.5
    w[[big, other], dim // 2:] = 0
    w[big] /= w[big].norm()
    x = torch.randn(n, dim, generator=g, device=device) + gain * w[big]
    w, x = w.to(DT[dtype]), x.to(DT[dtype])
    y = torch.where(torch.arange(n, device=device) % 2 == 0, big, other)
    loss, dx, dw = torch.zeros(n, device=device), torch.zeros(n, dim, device=device), torch.zeros(rows, dim, device=device)
    fc.CrossEntropy(rows, dim, n, dtype).loss_grad(x, w, y, loss, dx, dw)

    X, W = x.double(), w.double()
    L = X @ W.t()
    P = L.softmax(1)
    A = (X.abs() @ W.abs().t()).amax(1)
    rel = (2 * U[dtype] + 2 * (dim + 2) * U32 * A + 6 * U32 * A + 80 * U32)[:, None]
    eD = rel * P + 2.0 ** -40 * P.amax(1, keepdim=True) + 2.0 ** -40
    keep = torch.ones(rows, dtype=torch.bool, device=device)
    keep[[big, other]] = False
    D, eD = P[:, keep], eD[:, keep]
    for got, d, ed, v in ((dw[keep], D.t(), eD.t(), X), (dx[:, dim // 2:], D, eD, W[keep][:, dim // 2:])):
        bound = ed @ v.abs() + (d.shape[1] + 6) * U32 * (d @ v.abs())
        err = (got.double() - d @ v).abs()
        assert bool((err <= 1.01 * bound).all()), float((err / bound).max())
