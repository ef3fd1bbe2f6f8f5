"""How the operators that train a retrieval layer start their kernels, without a
GPU: a stand-in for HIP's launch calls records them."""
import os
import subprocess
import sys

from tests.test_operator_launches import stand_in  # noqa: F401

HERE = os.path.dirname(os.path.abspath(__file__))

HEADER = """
import ctypes, sys
hip = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
import paper_2402_01964_amd as nlb
from tests.test_training_refusals import *
lib = nlb.load_library()

def sizes():
    out = []
    for i in range(hip.launched()):
        v = (ctypes.c_uint64 * 6)()
        hip.launch_sizes(i, v)
        out.append(list(v))
    hip.forget()
    return out

def rows_by_id(c):
    return lib.nlb_lookup(c, P, 64, P, 64, None)

def whole(c):
    return lib.nlb_lookup_backward(c, P, 64, P, 64, None, None, P, BIG, None)

def listed(c):
    return lib.nlb_lookup_backward(c, P, 64, P, 64, P, P, P, BIG, None)

def turned(c):
    return lib.nlb_norm_rotate(c, ROWS, ROWS, None)
"""


def run(stand_in, body):  # noqa: F811
    got = subprocess.run([sys.executable, "-c", HEADER + body, stand_in], cwd=os.path.dirname(HERE),
                         capture_output=True, text=True, timeout=300)
    assert got.returncode == 0, got.stdout + got.stderr


def test_no_launch_passes_a_grid_dimension(stand_in):  # noqa: F811
    """A launch holds fewer than 2^32 work items a dimension, and 2^16 workgroups
    in the second."""
    run(stand_in, """
most = 2**31 - 1
calls = []
for dtype in (nlb.DTYPE_BF16, nlb.DTYPE_F32):
    for n, width in ((1, 1), (most, 1), (most, 65536), (1000, 65536), (most, 9000)):
        c = lookup(n=n, rows=most, width=width, dtype=dtype)
        calls += [(rows_by_id, c), (whole, c), (listed, c)]
    for q, k, heads, dim in ((1, 1, 1, 1), (most, most, 256, 128), (most, 1, 1, 1), (1, most, 256, 3)):
        c = rotate(q_rows=q, k_rows=k, heads=heads, kv_heads=heads, dim=dim, freqs=0, dtype=dtype)
        calls += [(turned, c), (lambda c: rotate_backward(lib, c), c)]
    for rows, batch, width in ((1, 1, 1), (2147480000, 1, 1), (2147480000, 2**31 - 2, 65536), (1, 7, 65536), (70000, 3, 8)):
        c = scan(rows=rows, batch=batch, width=width, dtype=dtype, h0=None)
        calls += [(lambda c: scan_forward(lib, c, last=None), c), (lambda c: scan_backward(lib, c, dh0=None), c)]
for call, c in calls:
    assert call(c) == nlb.NLB_OK
    got = sizes()
    assert got
    for v in got:
        assert all(v[i] * v[i + 3] < 2**32 for i in range(3)) and v[1] < 2**16 and v[2] == 1, v
        assert all(v), v
""")


def test_calls_without_work_start_nothing(stand_in):  # noqa: F811
    run(stand_in, """
assert rows_by_id(lookup(n=0, ids=None)) == nlb.NLB_OK and not sizes()
assert turned(rotate(q_rows=0, k_rows=0)) == nlb.NLB_OK and not sizes()
assert whole(lookup(n=0, ids=None)) == nlb.NLB_OK and len(sizes()) == 1     # zeros
assert listed(lookup(n=0, ids=None)) == nlb.NLB_OK and len(sizes()) == 1    # the number of rows
assert rotate_backward(lib, rotate(q_rows=0, k_rows=0)) == nlb.NLB_OK and len(sizes()) == 1
assert scan_forward(lib, scan(rows=0)) == nlb.NLB_OK and len(sizes()) == 1  # states go through
""")


def test_nothing_follows_a_launch_that_fails(stand_in):  # noqa: F811
    """A call whose first, second, ... launch is refused returns NLB_EDEVICE and
    starts none after it; an error that an earlier call left is not this call's."""
    run(stand_in, """
at = ctypes.c_int.in_dll(hip, "fail_at")
big, small = lookup(n=3_000_000, rows=2**25, width=128), lookup()
calls = [lambda: rows_by_id(small), lambda: whole(small), lambda: listed(small), lambda: whole(big), lambda: listed(big),
         lambda: turned(rotate()), lambda: rotate_backward(lib, rotate()), lambda: scan_forward(lib, scan()),
         lambda: scan_backward(lib, scan()), lambda: scan_forward(lib, scan(rows=100)),
         lambda: scan_forward(lib, scan(rows=100_000)), lambda: scan_backward(lib, scan(rows=100_000))]
for k, call in enumerate(calls):
    hip.leave_error(1)
    assert call() == nlb.NLB_OK, k
    n = hip.launched()
    assert n > 0
    hip.forget()
    for at.value in range(n):
        assert call() == nlb.NLB_EDEVICE, (k, at.value)
        assert hip.launched() == at.value + 1, (k, at.value, hip.launched())
        hip.forget()
    at.value = -1
""")
