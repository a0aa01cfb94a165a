"""The operators' C ABI and binding without a GPU: the library exports what
include/fc_lm.h declares, the header is plain C, and calls that need no device
are refused as documented."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "fc_lm.h")


@pytest.fixture(scope="module")
def lm():
    import paper_1511_00175_amd as m
    from paper_1511_00175_amd import _fc_lm
    assert m.Embedding
    return _fc_lm


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(fc_[a-z_]+)\s*\(", text)))


def test_library_exports_every_declared_symbol(lm):
    names = declared()
    assert len(names) >= 4
    for n in names:
        assert ctypes.cast(getattr(lm.lib, n), ctypes.c_void_p).value, n
        assert getattr(lm.lib, n).argtypes is not None, n


def test_header_is_plain_c(tmp_path):
    src = tmp_path / "use.c"
    src.write_text('#include "fc_lm.h"\nint main(void) { return FC_BF16 == 2 ? 0 : 1; }\n')
    r = subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-fsyntax-only",
                        f"-I{os.path.join(ROOT, 'include')}", str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def test_calls_without_a_plan(lm):
    """Every call with every argument null or zero: FC_EINVAL, and destroying
    no plan does nothing."""
    for n in declared():
        f = getattr(lm.lib, n)
        args = [None if a in (ctypes.c_void_p,) or issubclass(a, ctypes._Pointer) else a(0) for a in f.argtypes]
        rc = f(*args)
        assert rc == (None if n.endswith("_destroy") else -1), n


def test_embedding_checks_its_buffers():
    """The binding's checks come before any call of the library."""
    torch = pytest.importorskip("torch")
    import paper_1511_00175_amd as fc
    plan = object.__new__(fc.Embedding)
    plan.device, plan.rows, plan.dim, plan.max_tokens = torch.device("cpu"), 10, 8, 4
    table, tok, out = torch.zeros(10, 8), torch.zeros(3, dtype=torch.int32), torch.zeros(3, 8)
    reached = []
    plan._call = lambda name, *args: reached.append(name)
    import paper_1511_00175_amd as m
    plan.lookup(table, tok, out, stream=0)
    plan.grad(out, tok, table, stream=0)
    plan.grad(torch.zeros(3, 12)[:, 2:10].half(), tok.long(), table.bfloat16(), stream=0)
    assert reached == ["fc_embed_lookup", "fc_embed_grad", "fc_embed_grad"]
    for bad in (lambda: plan.lookup(table, tok, out.double(), stream=0), lambda: plan.lookup(table, tok, out.t(), stream=0),
                lambda: plan.grad(torch.zeros(5, 8), torch.zeros(5, dtype=torch.int32), table, stream=0),
                lambda: plan.lookup(table, tok[None], out, stream=0), lambda: plan.lookup(table[:, ::2], tok, out, stream=0)):
        with pytest.raises(ValueError):
            bad()
    assert len(reached) == 3 and m.Embedding is fc.Embedding


def test_cross_entropy_checks_its_buffers():
    torch = pytest.importorskip("torch")
    import paper_1511_00175_amd as fc
    plan = object.__new__(fc.CrossEntropy)
    plan.device, plan.rows, plan.dim, plan.max_tokens, plan.code = torch.device("cpu"), 10, 8, 4, 1
    reached = []
    plan._call = lambda name, *args: reached.append(name)
    x, w, y, loss = torch.zeros(3, 8).half(), torch.zeros(10, 8).half(), torch.zeros(3, dtype=torch.int64), torch.zeros(3)
    plan.loss(x, w, y, loss, stream=0)
    plan.loss_grad(x, w, y, loss, x.float(), None, stream=0)
    assert reached == ["fc_xent_loss", "fc_xent_loss_grad"]
    for bad in (lambda: plan.loss(x.bfloat16(), w, y, loss, stream=0), lambda: plan.loss(x, w, y, loss.double(), stream=0),
                lambda: plan.loss_grad(x, w, y, loss, x[:2], None, stream=0), lambda: plan.loss(x, w.t(), y, loss, stream=0)):
        with pytest.raises(ValueError):
            bad()
    assert len(reached) == 2


def test_muon_checks_its_buffers():
    torch = pytest.importorskip("torch")
    import paper_1511_00175_amd as fc
    plan = object.__new__(fc.Muon)
    plan.device, plan.extent, plan.code = torch.device("cpu"), 64, 2
    reached = []
    plan._call = lambda name, *args: reached.append(name)
    g, out = torch.zeros(64), torch.zeros(80, dtype=torch.bfloat16)
    plan.orthogonalize(g.half(), out, stream=0)
    plan.step(g, g.clone(), g.clone(), 0.1, 0.9, 0.0, 8, stream=0)
    assert reached == ["fc_muon_orthogonalize", "fc_muon_step"]
    for bad in (lambda: plan.orthogonalize(g, g, stream=0), lambda: plan.orthogonalize(g[:63], out, stream=0),
                lambda: plan.orthogonalize(torch.zeros(128)[::2], out, stream=0),
                lambda: plan.step(g, g.half(), g, 0.1, 0.9, 0.0, 8, stream=0)):
        with pytest.raises(ValueError):
            bad()
    for bad in ([(0, 8)], [(0, 8, 8, 1.0, 1.0, 1.0)], [(-4, 8, 8)]):
        with pytest.raises(ValueError):
            fc.Muon(bad)
    assert len(reached) == 2
