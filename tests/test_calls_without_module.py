"""The package where the CPython module of the per-token calls cannot be built: it builds, imports and runs through ctypes."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
WITHOUT = """import sys
sys.modules["paper_1609_07061_b200._qnn_calls"] = None       # an import of it raises ImportError
import pytest
from paper_1609_07061_b200 import binding
assert isinstance(binding._qnn_calls, type)                  # the stand-in
sys.exit(pytest.main(["-q", "-x", "-p", "no:cacheprovider"] + sys.argv[1:]))
"""


def run_without(*args):
    r = subprocess.run([sys.executable, "-c", WITHOUT, *args], cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]


def test_build_without_python_headers(monkeypatch, tmp_path, capfd):
    from paper_1609_07061_b200 import build
    build.build()
    target = tmp_path / "_qnn_calls.so"
    target.write_bytes(b"of another library")
    os.utime(target, (0, 0))
    monkeypatch.setattr(build, "CALLS", str(target))
    monkeypatch.setattr(build.sysconfig, "get_paths", lambda *a, **k: {"include": str(tmp_path)})
    assert build.build() == build.LIB
    assert not target.exists()                                # what does not match the library is not left to be loaded
    assert "ctypes" in capfd.readouterr().err


def test_module_is_tagged_with_its_interpreter():
    from paper_1609_07061_b200 import binding, build
    build.build()
    assert not os.path.exists(os.path.join(build.HERE, "_qnn_calls.so"))
    assert os.path.basename(build.CALLS) == "_qnn_calls" + build.sysconfig.get_config_var("EXT_SUFFIX")
    assert os.path.realpath(binding._qnn_calls.__file__) == os.path.realpath(build.CALLS)


def test_refusals_without_the_module():
    run_without("tests/test_int8_refusals.py", "tests/test_abi.py")


@pytest.mark.gpu
def test_calls_without_the_module():
    run_without("-m", "gpu", "tests/test_gpu_int8_chain.py")
