"""Norm, Checkpoint and Mxfp4 without a GPU: their checks of buffers come before any
call of the library, and plans of impossible sizes are refused before a device is
touched."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

HALF, FULL = torch.float16, torch.float32


@pytest.fixture(scope="module")
def fc():
    import paper_1511_00175_amd as m
    return m


def bare(cls, reached, **fields):
    """An object of the class with no plan behind it; the library's calls are noted."""
    plan = object.__new__(cls)
    plan.device = torch.device("cpu")
    for name, value in fields.items():
        setattr(plan, name, value)
    plan._call = lambda name, *args: reached.append((name, args))
    from paper_1511_00175_amd import lm
    lm._types()
    return plan


def refused(*calls):
    for bad in calls:
        with pytest.raises(ValueError):
            bad()


def test_norm_checks_its_buffers(fc):
    reached = []
    plan = bare(fc.Norm, reached, dim=8, max_tokens=4, block=HALF, residual=FULL, vector=FULL)
    h, b, v = torch.zeros(3, 8), torch.zeros(3, 8, dtype=HALF), torch.zeros(8)
    wide = torch.zeros(3, 12)[:, 2:10]
    plan.before(wide, b, weight=v, stream=0)
    assert reached[-1][0] == "fc_norm_before" and reached[-1][1][1] == 12  # the row stride
    plan.after(h, b, wide, gate=v, stream=0)
    assert reached[-1][1][6] == 0  # a vector's stride
    plan.after(h, b, wide, gate=b.clone(), stream=0)
    assert reached[-1][1][6] == 8
    plan.between(h, b, wide, b.clone(), weight=v, gate=v, next_weight=v, stream=0)
    plan.before_grad(h, b, h.clone(), dout=h, dweight=v.half(), stream=0)
    plan.after_grad(b, h, b.clone(), gate=v, dgate=v.bfloat16(), dweight=v.bfloat16(), stream=0)
    plan.after_grad(b, h, b.clone(), gate=b, dgate=b.clone(), dweight=v.half(), stream=0)
    plan.between_grad(h, b, b, h.clone(), b.clone(), gate=v, dgate=v.clone(), dnext=v.clone(), stream=0)
    count = len(reached)
    refused(lambda: plan.before(b, b, stream=0), lambda: plan.before(h, h, stream=0), lambda: plan.before(h, b[:2], stream=0),
            lambda: plan.before(h, b, weight=v.half(), stream=0), lambda: plan.before(h, b, weight=v[:7], stream=0),
            lambda: plan.before(h, b, weight=torch.zeros(16)[::2], stream=0), lambda: plan.before([0.0], b, stream=0),
            lambda: plan.before(torch.tensor(0.0), b, stream=0), lambda: plan.before(h[0], b, stream=0),
            lambda: plan.after(h, b, h.t().contiguous().t(), stream=0), lambda: plan.after(h, b, h[:1].expand(3, 8), stream=0),
            lambda: plan.after(h, b, wide, gate=h, stream=0), lambda: plan.after(h, b, wide, gate=b[:2], stream=0),
            lambda: plan.before_grad(torch.zeros(5, 8), torch.zeros(5, 8, dtype=HALF), torch.zeros(5, 8), stream=0),
            lambda: plan.after_grad(b, h, b.clone(), dgate=v, stream=0), lambda: plan.after_grad(b, h, b.clone(), gate=v, dgate=b, stream=0),
            lambda: plan.after_grad(b, h, b.clone(), gate=v, dgate=v, dweight=v.half(), stream=0),
            lambda: plan.after_grad(b, h, b.clone(), dweight=v.double(), stream=0), lambda: plan.after_grad(b, h, b.clone(), dweight=[1.0], stream=0))
    assert len(reached) == count


def test_checkpoint_checks_its_buffers(fc):
    reached = []
    plan = bare(fc.Checkpoint, reached, dim=40, max_tokens=4, max_outs=16, blocks=2, dtype=HALF, types=(torch.int8, torch.uint8))
    x, (codes, scales) = torch.zeros(3, 40), plan.empty(3)
    assert codes.shape == (3, 64) and scales.shape == (3, 2)
    dy, dw = torch.zeros(3, 16, dtype=HALF), torch.zeros(16, 40)
    plan.pack(x.bfloat16(), codes, scales, stream=0)
    plan.unpack(codes, scales, x.half(), stream=0)
    plan.grad(dy, codes, scales, dw.half(), stream=0)
    plan.grad(dy[:1, :7], codes[:1], scales[:1], dw[:7], stream=0)
    assert reached[-1][1][1] == 8  # one row's stride is what the call wants
    assert [n for n, _ in reached] == ["fc_ckpt_pack", "fc_ckpt_unpack", "fc_ckpt_grad", "fc_ckpt_grad"]
    refused(lambda: plan.pack(x.double(), codes, scales, stream=0), lambda: plan.pack(x[:2], codes, scales, stream=0),
            lambda: plan.pack(x, codes.view(torch.uint8), scales, stream=0), lambda: plan.pack(x, codes[:, :40], scales, stream=0),
            lambda: plan.pack(x, codes, scales.int(), stream=0), lambda: plan.pack(None, codes, scales, stream=0),
            lambda: plan.unpack(codes, scales, x[:, :39], stream=0), lambda: plan.grad(dy.float(), codes, scales, dw, stream=0),
            lambda: plan.grad(dy, codes, scales, dw[:15], stream=0), lambda: plan.grad(torch.zeros(5, 16, dtype=HALF), *plan.empty(5), dw, stream=0),
            lambda: plan.grad(torch.zeros(3, 17, dtype=HALF), codes, scales, torch.zeros(17, 40), stream=0))
    assert len(reached) == 4


def test_mxfp_checks_its_buffers(fc):
    reached = []
    plan = bare(fc.Mxfp4, reached, rows=24, dim=40, max_tokens=4, widths=(32, 8), type=torch.uint8)
    x, w, out = torch.zeros(3, 40), torch.zeros(24, 40), torch.zeros(3, 24)
    a, b = plan.empty(3), plan.empty(24)
    plan.pack(w, *b, stream=0)
    plan.pack(w.t().contiguous(), *b, transpose=True, stream=0)
    plan.unpack(*b, w.half(), stream=0)
    plan.product(*a, *b, out, stream=0)
    plan.linear(x.half(), *b, out.bfloat16(), accumulate=True, stream=0)
    assert [n for n, _ in reached] == ["fc_mxfp_pack", "fc_mxfp_pack", "fc_mxfp_unpack", "fc_mxfp_product", "fc_mxfp_linear"]
    refused(lambda: plan.pack(w, *a, stream=0), lambda: plan.pack(w, *b, transpose=True, stream=0), lambda: plan.pack(w[0], *b, stream=0),
            lambda: plan.pack(w, b[0].view(torch.int8), b[1], stream=0), lambda: plan.pack(w, b[0], b[1][:, :2], stream=0),
            lambda: plan.pack(w, 5, b[1], stream=0), lambda: plan.product(*a, *a, out, stream=0), lambda: plan.product(*a, *b, out[:, :23], stream=0),
            lambda: plan.linear(torch.zeros(5, 40), *b, torch.zeros(5, 24), stream=0), lambda: plan.linear(x.double(), *b, out, stream=0),
            lambda: plan.linear(x, *b, out.t(), stream=0))
    assert len(reached) == 5


def test_plans_of_impossible_sizes():
    from paper_1511_00175_amd._fc_lm import lib
    h = ctypes.c_void_p()
    big = 1 << 31
    for make, sizes in ((lib.fc_norm_create, [(0, 1, 1, 1, 0, 1e-6, 0), (16385, 1, 1, 1, 0, 1e-6, 0), (8, big, 1, 1, 0, 1e-6, 0), (8, 1, 3, 3, 0, 1e-6, 0),
                                              (8, 1, 1, 2, 0, 1e-6, 0), (8, 1, 1, 1, 2, 1e-6, 0), (8, 1, 1, 1, 0, 0.0, 0), (8, 1, 1, 1, 0, 1e-6, 3)]),
                        (lib.fc_ckpt_create, [(0, 1, 1, 1, 0), ((1 << 21) + 1, 1, 1, 1, 0), (8, (1 << 30) + 1, 8, 1, 0), (8, 1, (1 << 21) + 1, 1, 0),
                                              (8, 1, 8, 0, 0), (8, 1, 8, 1, 2)]),
                        (lib.fc_mxfp_create, [(0, 1, 1), (1, 0, 1), ((1 << 21) + 1, 1, 1), (1, (1 << 21) + 1, 1), (1, 1, big), (1, 1, -1)])):
        for args in sizes:
            assert make(ctypes.byref(h), *args) == -1 and not h.value, (make.__name__, args)
