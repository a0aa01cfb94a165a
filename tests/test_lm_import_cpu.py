"""The operators' library is needed by the operators alone: without it the
package is imported and its Plan used as before, and the operators' names say
what is missing."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_1511_00175_amd")


def run(code, cwd):
    return subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=cwd, timeout=300)


@pytest.fixture(scope="module")
def without(tmp_path_factory):
    """A copy of the package that lacks libfc_lm.so."""
    root = tmp_path_factory.mktemp("tree")
    shutil.copytree(PKG, root / "paper_1511_00175_amd",
                    ignore=shutil.ignore_patterns("libfc_lm.so*", "_build", "csrc", "__pycache__"))
    return root


def test_the_package_without_the_operators_library(without):
    r = run("import paper_1511_00175_amd as fc\n"
            "from paper_1511_00175_amd import *\n"
            "import os; assert os.path.dirname(fc.__file__) == os.path.join(os.getcwd(), 'paper_1511_00175_amd')\n"
            "assert fc.Plan is Plan and fc_strerror(0) is not None\n"
            "for n in ('Embedding', 'CrossEntropy', 'Muon'):\n"
            "    try:\n"
            "        getattr(fc, n)\n"
            "    except ImportError as e:\n"
            "        assert 'libfc_lm.so is not built' in str(e)\n"
            "    else:\n"
            "        raise AssertionError(n)\n"
            "print('fine')", without)
    assert r.returncode == 0 and "fine" in r.stdout, r.stderr


def test_the_operators_library_is_loaded_when_it_is_used():
    r = run("import paper_1511_00175_amd as fc\n"
            "maps = lambda: open('/proc/self/maps').read()\n"
            "assert 'libfc_lm.so' not in maps() and 'Muon' in dir(fc) and 'Muon' in fc.__all__\n"
            "assert not hasattr(fc, 'Nothing') and fc.lm.Muon is fc.Muon\n"
            "from paper_1511_00175_amd import Muon, CrossEntropy\n"
            "from paper_1511_00175_amd import *\n"
            "assert Muon is fc.Muon and Embedding is fc.lm.Embedding and 'libfc_lm.so' in maps()\n"
            "print('fine')", ROOT)
    assert r.returncode == 0 and "fine" in r.stdout, r.stderr
