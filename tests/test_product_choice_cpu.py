"""Every way in which the operators' products are computed (fc_choice.h) is taken by a
shape of the GPU tests (product_shapes.py), as the shape says."""
import math
import os
import random
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
        got = [(line.split()[0], *(int(v) for v in line.split()[1:])) for line in r.stdout.splitlines()]
        assert len(got) == len(lines)
        return got
    return ask


def test_gradients_take_every_way(ways):
    got = ways([f"ckpt {n} {outs} {dim} {n} {outs}" for _, _, n, outs, dim, *_ in GRADIENTS])
    assert [(kind, parts > 1) for kind, parts, *_ in got] == [c[:2] for c in GRADIENTS]
    assert {c[:2] for c in GRADIENTS} == {(k, s) for k in ("LARGE", "BROAD", "MIDDLE", "TINY") for s in (False, True)} | {("FEW", False)}
    for kind in ("LARGE", "BROAD", "MIDDLE"):  # sums in one part and in several, written and added to
        assert {(c[1], c[-1]) for c in GRADIENTS if c[0] == kind} >= {(False, False), (False, True), (True, True)}


@pytest.mark.parametrize("op,cases,others", [("product", PRODUCTS, set()), ("linear", LINEARS, {("SMALL", False), ("FEW", False)})])
def test_products_take_every_way(ways, op, cases, others):
    got = ways([f"{op} {rows} {dim} {n} {n}" for _, _, n, rows, dim, *_ in cases])
    assert [(kind, parts > 1) for kind, parts, *_ in got] == [c[:2] for c in cases]
    assert {c[:2] for c in cases} == {(k, s) for k in ("WIDE4", "HALF4", "SMALL4") for s in (False, True)} | others
    for kind in ("WIDE4", "HALF4"):
        assert {(c[1], c[-1]) for c in cases if c[0] == kind} == {(a, b) for a in (False, True) for b in (False, True)}


def test_partial_sums_fit_their_room(ways):
    """Whatever a plan's sizes and a call's within them."""
    r = random.Random(5)

    def upto(most, least=1):
        return int(round(math.exp(r.uniform(math.log(least), math.log(most)))))

    lines = []
    for _ in range(20000):
        tokens, outs, dim = upto(300000), upto(20000), upto(20000)
        lines.append(f"ckpt {tokens} {outs} {dim} {r.choice((tokens, upto(tokens)))} {r.choice((outs, upto(outs)))}")
        lines.append(f"product {outs} {dim} {tokens} {r.choice((tokens, upto(tokens)))}")
        lines.append(f"product {upto(5000)} {upto(60000)} {min(tokens, 100)} {upto(min(tokens, 100))}")
        lines.append(f"ckpt {tokens} {upto(300)} {upto(300)} {r.choice((tokens, upto(tokens)))} 1")
    got = ways(lines)
    assert sum(1 for g in got if g[1] > 1) > 4000
    for line, (kind, parts, floats, room) in zip(lines, got):
        assert floats <= room <= 1 << 25, (line, kind, parts, floats, room)


def test_no_room_is_made_for_what_is_never_written(ways):
    few, one, short, wide = ways(["product 4096 9216 1 1", "ckpt 128 512 512 128 512", "product 4096 512 4096 4096", "product 4096 9216 64 64"])
    assert few[3] <= 18 * 4096 and one[3] == 0 and short[3] == 0  # 36 steps in 18 parts at most; two steps of tokens; two of dim
    assert wide[3] <= 18 * 64 * 4096
