"""Lists whose tables the host has no memory for: an error of the call, where an exception would end the caller's process (no GPU)."""
import subprocess
import sys

import pytest

_CHILD = """
import ctypes as C, resource, sys
from paper_2604_24708_b200 import binding as B
lib = B.raw_library()
cfg = B.hdet_config(n_replicas=2, n_groups=1, optimizer=B.HDET_OPT_SGD, grad_dtype=B.HDET_DTYPE_F32, sync_interval=1)
numel = 1 << 38                          # tables of a gigabyte
t = B.hdet_tensor(param=0x1000, grad=0x2000, numel=numel, param_stride=numel, grad_stride=numel)
used = int(open("/proc/self/statm").read().split()[0]) * resource.getpagesize()
resource.setrlimit(resource.RLIMIT_AS, (used + (256 << 20), resource.getrlimit(resource.RLIMIT_AS)[1]))
out, n = C.c_void_p(), C.c_int64(0)
if sys.argv[1] == "create":
    status = lib.hdet_create(C.byref(cfg), C.byref(t), 1, C.byref(out))
else:
    status = lib.hdet_plan_tiles(C.byref(cfg), C.byref(t), 1, None, None, 0, C.byref(n), None, None)
assert status == B.HDET_ERR_INVALID_ARG and not out.value, status
assert lib.hdet_last_error(None).endswith(b": out of host memory"), lib.hdet_last_error(None)
"""


@pytest.mark.parametrize("call", ["create", "plan"])
def test_tables_that_do_not_fit(call):
    res = subprocess.run([sys.executable, "-c", _CHILD, call], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, (res.returncode, res.stderr[-500:])
