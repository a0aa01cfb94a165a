"""Gradients in fp32 of plans whose chunks hold at most 64 tokens: d is kept to
twice its type's bits whatever the number of tokens.

Bounds as in test_xent_gpu.py with both roundings to 16 bits replaced: the numerator
is fp32 (u32 more), d is the sum of two 16-bit numbers (u^2 |d|, and half the smallest
step of the lower one, 2^-40 for fp16), and dw's sum goes over n terms and the chunks."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
U = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}
U32 = 2.0 ** -24


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,dim,n,chunk", [(700, 72, 300, 64), (3001, 130, 129, 33), (260, 520, 1000, 64), (900, 64, 64, 0)])
def test_fine_gradients(device, rows, dim, n, chunk, dtype):
    import paper_1511_00175_amd as fc
    g = torch.Generator(device=device)
    g.manual_seed(rows + n)
    w = (torch.randn(rows, dim, generator=g, device=device) * dim ** -0.5).to(DT[dtype])
    y = torch.randint(0, rows, (n,), generator=g, device=device)
    x = (torch.randn(n, dim, generator=g, device=device) + 2 * w[y].float()).to(DT[dtype])
    y[::7] = -1
    loss, dx, dw = torch.zeros(n, device=device), torch.zeros(n, dim, device=device), torch.zeros(rows, dim, device=device)
    fc.CrossEntropy(rows, dim, n, dtype, chunk=chunk).loss_grad(x, w, y, loss, dx, dw)
    live = y >= 0
    X, W, Y = x[live].double(), w.double(), y[live]
    P = (X @ W.t()).softmax(1)
    D = P.clone()
    D[torch.arange(len(Y), device=device), Y] -= 1
    A = (X.abs() @ W.abs().t()).amax(1)
    rel = (2 * (dim + 2) * U32 * A + 6 * U32 * A + 81 * U32)[:, None]
    eD = rel * P + (U[dtype] ** 2 + 2 * U32) * D.abs() + (2.0 ** -40 if dtype == "f16" else 0)
    for got, d, ed, v in ((dx[live], D, eD, W), (dw, D.t(), eD.t(), X)):
        ref = d @ v
        bound = ed @ v.abs() + (2 * d.shape[1] + n + 8) * U32 * (d.abs() @ v.abs()) + U32 * ref.abs()
        err = (got.double() - ref).abs()
        assert bool((err <= 1.01 * bound).all()), float((err / bound).max())
