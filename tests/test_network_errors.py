"""Errors of the network operators that come from the HIP runtime, without a device."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# (the pointers are never followed: no device is visible to the process, so that every
# launch fails, which is made sure of first)
SCRIPT = """
import ctypes as C, sys
sys.path.insert(0, sys.argv[1])
from paper_1609_06119_amd._lib import lib
L = lib()
hip = C.CDLL("libamdhip64.so", mode=C.RTLD_GLOBAL)
hip.hipGetErrorString.restype = C.c_char_p
count = C.c_int(0)
status = hip.hipGetDeviceCount(C.byref(count))
assert status != 0 and count.value == 0, (status, count.value)
hip.hipGetLastError()
why = hip.hipGetErrorString(status)
A = 1 << 20
calls = {
    "fbdt_event_tokens": (A, 10, 3, 16, 16, A + 4096, None),
    "fbdt_embed": (A, 1, 48, 64, 64, A + 65536, 4, 10, 1.0, 2 * A, 64, None),
    "fbdt_packed_weight_grad": (A, 16, 4, 9, 2 * A, 256, 3 * A, 4, 200, 4 * A, 0, 200, None, 0, None),
}
for name, args in calls.items():
    assert getattr(L, name)(*args) == -6, name
    text = L.fbdt_last_error()
    assert text.startswith(name.encode()) and text.endswith(why), (name, text, why)
print("errors ok")
"""


def test_a_launch_that_fails_names_its_call_and_the_cause():
    env = dict(os.environ, HIP_VISIBLE_DEVICES="-1", ROCR_VISIBLE_DEVICES="-1")
    run = subprocess.run([sys.executable, "-c", SCRIPT, ROOT], capture_output=True, text=True, env=env,
                         timeout=120)
    assert run.returncode == 0, (run.stdout[-1000:], run.stderr[-3000:])
    assert "errors ok" in run.stdout
