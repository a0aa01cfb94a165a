"""Few tokens over a w that is read past the caches: from 5 * 2^26 bytes on for
losses alone, from 2^29 on with dx.  Between the two, loss_grad and loss read w in
different ways, and `check` asks for the same losses, bit for bit."""
import pytest

from test_xent_gpu import check, fc, inputs  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,rows,dim,n", [("f16", 42001, 4104, 16), ("bf16", 42001, 4101, 64), ("bf16", 66001, 4104, 7),
                                              ("f16", 66001, 4101, 63)])
def test_weights_beyond_the_caches(fc, device, dtype, rows, dim, n):  # noqa: F811
    check(fc, device, *inputs(device, rows, dim, n, dtype), dtype)
