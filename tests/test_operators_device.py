"""The operators leave the caller's current device as it was (CPU: a HIP
runtime that notes launches instead of running them)."""

import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

HEAD = """
import ctypes, os, sys
sys.path.insert(0, {root!r})
hip = ctypes.CDLL({stub!r}, mode=ctypes.RTLD_GLOBAL)


class Launch(ctypes.Structure):
    _fields_ = [("grid", ctypes.c_uint32 * 3), ("block", ctypes.c_uint32 * 3), ("device", ctypes.c_int32),
                ("pad", ctypes.c_int32), ("arg", ctypes.c_uint64 * 6)]


now = ctypes.c_int.in_dll(hip, "current_device")
count = ctypes.c_int.in_dll(hip, "n_launches")
broken = ctypes.c_int.in_dll(hip, "launch_error")
noted = (Launch * 4096).in_dll(hip, "launches")
from paper_2606_07019_amd import pccl as P
assert "torch" not in sys.modules
M = 1 << 40          # addresses: nothing is read there
"""


def run_with_recorder(tmp_path, body):
    """Runs `body` in a process whose HIP runtime is tests/hip_recorder.c."""
    stub = os.path.join(str(tmp_path), "hip_recorder.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", stub, os.path.join(ROOT, "tests", "hip_recorder.c")], check=True, timeout=60)
    r = subprocess.run([sys.executable, "-c", HEAD.format(root=ROOT, stub=stub) + body], capture_output=True, text=True, timeout=120, cwd=ROOT)
    assert r.returncode == 0, r.stdout + r.stderr
    return r.stdout


BODY = """
h = P.pccl_create(1, 0)
now.value = 0
calls = [
    lambda m: P.pccl_mx_quantize(h, m, P.PCCL_BF16, 200, 300, 300, M, M, M, M),
    lambda m: P.pccl_mx_quantize(h, m, P.PCCL_BF16, 200, 300, 300, M, M),
    lambda m: P.pccl_mx_dequantize(h, m, M, 200, 300, M, P.PCCL_F32, 300),
    lambda m: P.pccl_mx_matmul(h, m, M, M, M, 7, 300, 300, M, P.PCCL_F32, 300),
    lambda m: P.pccl_mx_matmul(h, m, M, M, M, 700, 300, 300, M, P.PCCL_F32, 300),
    lambda m: P.pccl_moe_route(h, m, P.PCCL_F32, 20, 8, 8, 2, 1, None, M, M, M, M),
    lambda m: P.pccl_moe_route_backward(h, m, P.PCCL_F32, 20, 8, 8, 2, 0, None, M, M, M, M, 8),
    lambda m: P.pccl_moe_layer(h, m, P.PCCL_BF16, 64, 2, 4, 2, 64, 64, 1, None, M, M, None, M, None, M, 64, M, 1 << 30),
]
for i, call in enumerate(calls):
    for at in (0, 1):
        now.value, count.value = at, 0
        call(M)
        assert now.value == at, (i, at, "a call that succeeds")
        assert count.value and all(noted[j].device == 1 for j in range(count.value)), (i, at)
        for address, error in ((None, 0), (M, 98)):
            broken.value = error
            try:
                call(address)
            except P.PcclError as e:
                assert e.name == ("PCCL_EDEVICE" if error else "PCCL_EINVAL"), (i, e)
            else:
                raise AssertionError(i)
            assert now.value == at, (i, at, "a call that fails")
print("left alone")
"""


def test_calls_leave_the_current_device_alone(tmp_path):
    assert "left alone" in run_with_recorder(tmp_path, BODY)


def test_making_and_closing_a_context_leave_the_current_device_alone(monkeypatch):
    torch = pytest.importorskip("torch")
    from paper_2606_07019_amd import operators
    from paper_2606_07019_amd import pccl as P
    state = {"now": 0}

    class Guard:
        def __init__(self, device):
            self.device = torch.device(device).index

        def __enter__(self):
            self.before, state["now"] = state["now"], self.device

        def __exit__(self, *exc):
            state["now"] = self.before

    def create(device, seed):
        state["now"] = device
        return 7

    monkeypatch.setattr(torch.cuda, "device", Guard)
    monkeypatch.setattr(P, "load_library", lambda: None)
    monkeypatch.setattr(P, "pccl_create", create)
    monkeypatch.setattr(P, "pccl_destroy", lambda h: state.update(now=1, gone=h))
    ops = operators.Operators(1)
    assert state["now"] == 0
    ops.close()
    assert state == {"now": 0, "gone": 7} and ops.h is None
