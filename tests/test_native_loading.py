"""When the compiled parts are loaded and rebuilt (CPU)."""
import os
import shutil
import subprocess
import sys

from paper_2309_06973_b200 import build as build_mod

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PACKAGE = "paper_2309_06973_b200"


def run(code, cwd):
    return subprocess.run([sys.executable, "-c", code], cwd=cwd, env=dict(os.environ, PYTHONPATH=str(cwd)), capture_output=True, text=True, timeout=300)


def test_importing_the_runtime_loads_no_library(tmp_path):
    """In a tree where nothing is built yet the runtime can be imported (the tests do, before their fixture builds), and in a built
    one importing it maps no file that a build may still replace."""
    shutil.copytree(os.path.join(ROOT, PACKAGE), tmp_path / PACKAGE, ignore=shutil.ignore_patterns("*.so", "__pycache__", "csrc"))
    for tree in (tmp_path, ROOT):
        out = run(f"import os\nimport {PACKAGE}.runtime as R\nassert os.path.dirname(R.__file__) == {os.path.join(str(tree), PACKAGE)!r}\n"
                  "print([l for l in open('/proc/self/maps') if 'libdnns' in l or '_native' in l])", tree)
        assert out.returncode == 0, out.stderr[-1000:]
        assert out.stdout.strip() == "[]"
    out = run(f"from {PACKAGE} import runtime as R\nR._native.rows(1, 2)", tmp_path)
    assert out.returncode != 0 and "ImportError" in out.stderr


def test_first_use_loads_the_compiled_calls():
    out = run(f"from {PACKAGE} import runtime as R\nR._native.rows(16, 16, 16, 0, 0, 2, 3, 0)\n"
              "print(type(R._native).__name__, sorted(l.split('/')[-1].strip() for l in open('/proc/self/maps') if 'libdnns' in l or '_native.so' in l)[0])", ROOT)
    assert out.returncode == 0, out.stderr[-1000:]
    assert out.stdout.split() == ["module", "_native.so"]


def test_compiled_calls_are_rebuilt_for_another_torch(tmp_path, monkeypatch):
    module, key = tmp_path / "_native.so", tmp_path / "_native.key"
    monkeypatch.setattr(build_mod, "NATIVE", str(module))
    monkeypatch.setattr(build_mod, "NATIVE_KEY", str(key))
    assert build_mod.native_needs_build()
    module.write_bytes(b"")
    assert build_mod.native_needs_build()                              # nobody says what it was built for
    key.write_text(build_mod.native_key())
    assert not build_mod.native_needs_build()
    key.write_text(build_mod.native_key().replace("torch ", "torch 1"))
    assert build_mod.native_needs_build()
    key.write_text(build_mod.native_key())
    os.utime(module, (1, 1))                                           # older than its source
    assert build_mod.native_needs_build()
