"""A launch that fails is reported: the calls that launch without rows, on a machine without a device."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# (no device is visible to the process that runs this, so the address is touched by nobody)
CODE = """
import ctypes, sys
import torch
from paper_2104_08378_amd import sp24
assert torch.cuda.device_count() == 0
A = 0x10000000
L, f = sp24.lib(), ctypes.c_float
want = L.sp24_moe_route(A, None, 2 * A, 3 * A, None, 4 * A, 8, 64, 4, 1, 1, 2, 0, 1, f(1.0), 64, sp24.F32, None)
got = L.sp24_moe_route(None, None, None, None, None, 4 * A, 0, 64, 4, 1, 1, 2, 0, 1, f(1.0), 64, sp24.F32, None)
none = L.sp24_moe_route(None, None, None, None, None, None, 0, 64, 4, 1, 1, 2, 0, 1, f(1.0), 64, sp24.F32, None)
print(L.sp24_status_string(want).decode(), '/', L.sp24_status_string(got).decode(), '/', L.sp24_status_string(none).decode())
"""


def test_the_load_of_no_rows():
    env = dict(os.environ, HIP_VISIBLE_DEVICES="-1", ROCR_VISIBLE_DEVICES="-1", PYTHONPATH=ROOT)
    said = subprocess.run([sys.executable, "-c", CODE], env=env, cwd=ROOT, stdout=subprocess.PIPE, timeout=120, check=True).stdout.decode()
    some, empty, nothing = (s.strip() for s in said.strip().splitlines()[-1].split("/"))
    assert some == empty != nothing
