"""Weights' gradients from 8-bit activations by every tile size, with the tokens in one
part and in several, written and added to; the bounds are test_ckpt_gpu.py's."""
import pytest

torch = pytest.importorskip("torch")

from product_shapes import GRADIENTS  # noqa: E402
from test_ckpt_gpu import grad_case  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fc(device):
    import paper_1511_00175_amd as m
    return m


@pytest.mark.parametrize("format", ["i8", "e4m3"])
@pytest.mark.parametrize("kind,split,n,outs,dim,dtype,to,pad,shift,accumulate", GRADIENTS)
def test_gradients(fc, device, kind, split, n, outs, dim, dtype, to, pad, shift, accumulate, format):
    grad_case(fc, device, n, dim, outs, format, dtype, to, pad, shift, accumulate, scale=0.625)
