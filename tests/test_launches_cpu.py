"""Work of more threads than a launch takes is cut into parts (fc_launches.h)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_parts_cover_the_work_once_and_fit_a_launch(tmp_path):
    exe = tmp_path / "launches_check"
    r = subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-fsanitize=address,undefined",
                        f"-I{os.path.join(ROOT, 'paper_1511_00175_amd', 'csrc')}",
                        os.path.join(ROOT, "tests", "c", "launches_check.cpp"), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr
