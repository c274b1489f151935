"""The package beside a torch without some of the 8-bit floating-point types: it imports, and the other calls work as before."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OLDER = """import sys
import torch
for name in sys.argv[2].split(","):
    delattr(torch, name)
if sys.argv[1] == "ctypes":
    sys.modules["paper_1609_07061_b200._qnn_calls"] = None       # an import of it raises ImportError
from paper_1609_07061_b200 import binding as q
assert isinstance(q._qnn_calls, type) == (sys.argv[1] == "ctypes")
x, i, s = torch.zeros(4, 64), torch.zeros(4, 64, dtype=torch.int8), torch.zeros(64, dtype=torch.uint8)
try:
    q.qnn_quantize_rows_i8(x, -1, 64, 64, i, 64, x[0])
    raise SystemExit("not refused")
except q.QnnError as e:
    assert e.status == q.QNN_ERR_INVALID_ARG, e
for codes in (i, x, *(torch.zeros(64, dtype=torch.uint8).view(getattr(torch, n)) for n in ("float8_e4m3fn", "float8_e5m2") if hasattr(torch, n))):
    try:
        q.qnn_quantize_blocks_f8(x, -1, 64, 64, codes, 64, s, 16)
        raise SystemExit("not refused")
    except q.QnnError as e:
        assert e.status == q.QNN_ERR_INVALID_ARG and codes is not i and codes is not x, e
    except TypeError as e:
        assert codes is i or codes is x, e
print("ok")
"""


@pytest.mark.parametrize("lacking", ["float8_e8m0fnu", "float8_e4m3fn,float8_e5m2,float8_e8m0fnu"])
@pytest.mark.parametrize("calls", ["module", "ctypes"])
def test_imports_without_the_types(calls, lacking):
    from paper_1609_07061_b200 import build
    build.build()
    r = subprocess.run([sys.executable, "-c", OLDER, calls, lacking], cwd=ROOT, capture_output=True, text=True, timeout=300,
                       env={**os.environ, "CUDA_VISIBLE_DEVICES": ""})
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout[-2000:] + r.stderr[-2000:]
