"""What the package exports, and what of it needs which built file."""
import os
import shutil
import subprocess
import sys

import pytest

import paper_1511_05950_b200 as P
from paper_1511_05950_b200 import build as lib_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_server_needs_no_extension(tmp_path):
    """A checkout with the library but without _marshal.so: the server's names work, those of learn raise, others are no attributes."""
    pkg = tmp_path / "paper_1511_05950_b200"
    pkg.mkdir()
    src = os.path.join(ROOT, "paper_1511_05950_b200")
    for fn in os.listdir(src):
        if fn.endswith(".py") or fn == "libsoftsync_ps.so":
            shutil.copy(os.path.join(src, fn), pkg / fn)
    code = ("import paper_1511_05950_b200 as P\n"
            "server = P.ParameterServer(0, 2, 1, 0.1)\n"
            "assert server.timestamps() == (0, 0) and P.PS_OK == 0 and P.binding.lib is P.lib\n"
            "assert not hasattr(P, 'no_such_name')\n"
            "for name in ('AdamW', 'policy_loss', 'learn'):\n"
            "    try:\n        getattr(P, name)\n"
            "    except RuntimeError as e:\n        assert 'not built' in str(e)\n"
            "    else:\n        raise AssertionError(name)\n"
            "print('fine')\n")
    out = subprocess.run([sys.executable, "-c", code], cwd=tmp_path, capture_output=True, text=True, env={**os.environ, "PYTHONPATH": str(tmp_path)})
    assert out.returncode == 0 and "fine" in out.stdout, out.stderr


def test_everything_of_learn_is_reachable():
    defined = {n for n, x in vars(P.learn).items() if getattr(x, "__module__", None) == P.learn.__name__ and not n.startswith("_")} | {"INPLACE"}
    assert defined == P._LEARN
    for name in defined:
        assert getattr(P, name) is getattr(P.learn, name)
    assert P.ParameterServer is P.binding.ParameterServer


def test_a_failed_build_of_the_extension_leaves_the_library(monkeypatch):
    def fails(force=False):
        raise subprocess.CalledProcessError(1, "g++")

    monkeypatch.setattr(lib_build, "build_marshal", fails)
    with pytest.warns(UserWarning, match="could not be built"):
        assert lib_build.ensure_built() == lib_build.LIB
    with pytest.raises(subprocess.CalledProcessError):
        lib_build.build()


def test_an_extension_of_other_sources_does_not_outlive_a_failed_build(monkeypatch, tmp_path):
    for name in ("MARSHAL", "MARSHAL_STAMP"):
        path = tmp_path / name
        path.write_text("of other sources")
        monkeypatch.setattr(lib_build, name, str(path))
    (tmp_path / "broken.cpp").write_text("this is no C++\n")
    monkeypatch.setattr(lib_build, "MARSHAL_SOURCES", [str(tmp_path / "broken.cpp")])
    with pytest.raises(subprocess.CalledProcessError):
        lib_build.build_marshal()
    assert sorted(os.listdir(tmp_path)) == ["broken.cpp"]
