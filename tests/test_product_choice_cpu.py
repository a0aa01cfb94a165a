"""Every way in which the operators' products are computed (fc_choice.h) is taken by a
shape of the GPU tests (product_shapes.py), as the shape says."""
import os
import shutil
import subprocess

import pytest

from product_shapes import GRADIENTS, LINEARS, PRODUCTS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ways(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    exe = tmp_path_factory.mktemp("choice") / "choice_check"
    r = subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-fsanitize=address,undefined",
                        f"-I{os.path.join(ROOT, 'paper_1511_00175_amd', 'csrc')}",
                        os.path.join(ROOT, "tests", "c", "choice_check.cpp"), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def ask(lines):
        r = subprocess.run([str(exe)], input="\n".join(lines), capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr
        got = [(line.split()[0], int(line.split()[1])) for line in r.stdout.splitlines()]
        assert len(got) == len(lines)
        return got
    return ask


def test_gradients_take_every_way(ways):
    got = ways([f"ckpt {n} {outs} {dim} {n} {outs}" for _, _, n, outs, dim, *_ in GRADIENTS])
    assert [(kind, parts > 1) for kind, parts in got] == [c[:2] for c in GRADIENTS]
    assert {c[:2] for c in GRADIENTS} == {(k, s) for k in ("LARGE", "BROAD", "MIDDLE", "TINY") for s in (False, True)} | {("FEW", False)}
    for kind in ("LARGE", "BROAD", "MIDDLE"):  # sums in one part and in several, written and added to
        assert {(c[1], c[-1]) for c in GRADIENTS if c[0] == kind} >= {(False, False), (False, True), (True, True)}


@pytest.mark.parametrize("op,cases,others", [("product", PRODUCTS, set()), ("linear", LINEARS, {("SMALL", False), ("FEW", False)})])
def test_products_take_every_way(ways, op, cases, others):
    got = ways([f"{op} {rows} {dim} {n} {n}" for _, _, n, rows, dim, *_ in cases])
    assert [(kind, parts > 1) for kind, parts in got] == [c[:2] for c in cases]
    assert {c[:2] for c in cases} == {(k, s) for k in ("WIDE4", "HALF4", "SMALL4") for s in (False, True)} | others
    for kind in ("WIDE4", "HALF4"):
        assert {(c[1], c[-1]) for c in cases if c[0] == kind} == {(a, b) for a in (False, True) for b in (False, True)}
