"""CPU: a plan that the HIP runtime does not let be created says why.  The condition is forced in a process that sees no device."""
import os
import subprocess
import sys

from paper_2210_17357_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
import ctypes as C
from paper_2210_17357_amd import binding as B
lib, table = B.lib(), B.layer_table([0, 10], [10, 5], [0, 0], [0, 0])
o = C.c_void_p(1)
assert lib.lgreco_optim_create(C.byref(o), C.addressof(table), 2, None, None) == B.EHIP and not o.value
text = lib.lgreco_optim_last_hip_error(None).decode()
assert "hipGetDevice" in text and "no ROCm-capable device" in text, text
import threading                                       # each thread has the text of its own calls
seen = []
t = threading.Thread(target=lambda: seen.append(lib.lgreco_optim_last_hip_error(None)))
t.start()
t.join()
assert seen == [b""]
assert lib.lgreco_optim_create(C.byref(o), C.addressof(table), 0, None, None) == B.EINVAL
assert lib.lgreco_optim_last_hip_error(None) == b""    # (of the last creation only)
import torch
torch.cuda.current_device = lambda: 0                  # so that the binding comes to the library
try:
    B.Optim(table)
except B.LgrecoError as e:
    assert e.status == B.EHIP and "no ROCm-capable device" in str(e), str(e)
else:
    raise AssertionError("no error")
print("done")
"""


def test_creation_without_a_device_says_so():
    if not os.path.exists(B.LIB_PATH):
        from paper_2210_17357_amd import build
        build.build()
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, env={**os.environ, "HIP_VISIBLE_DEVICES": "-1", "ROCR_VISIBLE_DEVICES": ""},
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.endswith("done\n"), r.stdout + r.stderr
