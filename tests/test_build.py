"""What the build needs: hipcc for the library, torch only for the binding's module (CPU only)."""
import os
import subprocess
import sys

import paper_2511_22481_amd.build as build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# An interpreter without torch: it cannot be imported, and nothing is known of its version.
NO_TORCH = """
import importlib.metadata, sys
sys.modules["torch"] = None
version = importlib.metadata.version
def without(name):
    if name == "torch":
        raise importlib.metadata.PackageNotFoundError(name)
    return version(name)
importlib.metadata.version = without
"""


def _run(code):
    res = subprocess.run([sys.executable, "-c", NO_TORCH + code], capture_output=True, text=True, cwd=ROOT)
    assert res.returncode == 0, res.stderr[-2000:]
    return res.stdout.split()


def test_the_library_loads_without_torch():
    import paper_2511_22481_amd as oa
    oa.load_library()   # (built, if it was not)
    assert _run("""
import paper_2511_22481_amd as oa
from paper_2511_22481_amd.build import is_stale
print(is_stale(), oa.load_library().omniattn_strerror(0).decode().split()[0], oa.omniattn_ring_pages(128, 2048))
""")[0] == "False"


def test_the_library_is_built_without_torch(tmp_path):
    """Everything but the compiler itself."""
    said = _run(f"""
import subprocess
import paper_2511_22481_amd.build as build
build.LIB, build.STAMP = {str(tmp_path / "a.so")!r}, {str(tmp_path / "a.so.stamp")!r}
ran = []
def run(cmd, **kw):
    ran.append(cmd)
    open(build.LIB, "w").close()
    return subprocess.CompletedProcess(cmd, 0, "", "")
build.subprocess.run, build.subprocess.Popen = run, None
build.check_generated_code = lambda verbose: None
build.build()
print(len(ran), "hipcc" in ran[0][0], build.is_stale())
""")
    assert said == ["1", "True", "False"]


def test_a_module_of_another_torch_is_built_again(tmp_path, monkeypatch):
    import torch
    build.build_marshal(force=False)
    assert not build.marshal_is_stale()
    monkeypatch.setattr(torch, "__version__", "0.0")
    assert build.marshal_is_stale()
    monkeypatch.undo()
    monkeypatch.setattr(build, "MARSHAL_STAMP", str(tmp_path / "none"))
    assert build.marshal_is_stale()
