"""build() writes where it is told to: a build with another output (other flags,
say) leaves the package's own libraries as they are."""
import importlib.util
import os
import types

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load():
    spec = importlib.util.spec_from_file_location("_build_under_test", os.path.join(ROOT, "paper_1511_00175_amd", "build.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_both_libraries_go_where_the_output_is(tmp_path, monkeypatch):
    m = load()
    pkg, other = tmp_path / "pkg", tmp_path / "other"
    pkg.mkdir(), other.mkdir()
    for name in ("libfc.so", "libfc_lm.so"):
        (pkg / name).write_text("kept")
    linked = []

    def link(cmd, check):
        linked.append(cmd)
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write("new")

    monkeypatch.setattr(m, "PKG", str(pkg))
    monkeypatch.setattr(m, "RESOURCES", str(pkg / "resources.txt"))
    monkeypatch.setattr(m, "LIB", str(pkg / "libfc.so"))
    if hasattr(m, "LIB_LM"):
        monkeypatch.setattr(m, "LIB_LM", str(pkg / "libfc_lm.so"))
    monkeypatch.setattr(m, "_compile", lambda src, obj, extra: {})
    monkeypatch.setattr(m, "subprocess", types.SimpleNamespace(run=link))
    assert m.build(str(other / "variant.so"), ["-DX"]) == str(other / "variant.so")
    assert len(linked) == 2
    assert sorted(os.listdir(other)) == ["libfc_lm.so", "variant.so"]
    assert [(pkg / n).read_text() for n in ("libfc.so", "libfc_lm.so")] == ["kept"] * 2
    m.build(str(pkg / "libfc.so"))
    assert [(pkg / n).read_text() for n in ("libfc.so", "libfc_lm.so")] == ["new"] * 2
