"""What the package needs where only its C library is wanted: neither torch nor another compiler than hipcc."""
import os
import subprocess
import sys
import types

from paper_2312_16733_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_library_builds_without_torch(monkeypatch, tmp_path):
    ran = []
    monkeypatch.setattr(build, "OBJ", str(tmp_path / "obj"))
    monkeypatch.setattr(build.subprocess, "run", lambda cmd, **k: ran.append(cmd) or types.SimpleNamespace(returncode=0, stdout="", stderr=""))
    for name in [n for n in sys.modules if n == "torch" or n.startswith("torch.")]:
        monkeypatch.delitem(sys.modules, name)
    monkeypatch.setitem(sys.modules, "torch", None)                    # an import of it fails
    assert build.build_library(verbose=False) == build.LIB
    assert len(ran) == len(build.sources()) + 1 and all(cmd[0] == build.HIPCC for cmd in ran)
    assert ran[-1][ran[-1].index("-o") + 1] == build.LIB


def test_every_public_name_of_the_package_comes_without_torch():
    """And without the library being loaded, or built."""
    code = ("import sys; sys.modules['torch'] = None\n"
            "from paper_2312_16733_amd import *\n"
            "import paper_2312_16733_amd as sna\n"
            "assert Supernet is sna.Supernet and sna.binding._lib is None\n"
            "assert {'PagedCache', 'PagedBatch', 'kv_append', 'paged_attention', 'verify_draft'} <= set(dir(sna))\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
