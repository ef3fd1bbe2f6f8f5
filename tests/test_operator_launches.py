"""How the operators without a table start their kernels, without a GPU: a
stand-in for HIP's launch calls records them.  Each test runs in a process of
its own, in which the stand-in is loaded before the library."""
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))

HEADER = """
import ctypes, sys
hip = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
import paper_2402_01964_amd as nlb
from tests.test_operator_refusals import P, ROWS, _backward, _call, _norm
lib = nlb.load_library()

def sizes():
    out = []
    for i in range(hip.launched()):
        v = (ctypes.c_uint64 * 6)()
        hip.launch_sizes(i, v)
        out.append(list(v))
    hip.forget()
    return out

def forward(c, work=P, size=1 << 50):
    return lib.nlb_attention(c, ROWS, P, work, size, None)

def backward(c, **kw):
    return _backward(lib, c, work=P, size=1 << 50, **kw)
"""


@pytest.fixture(scope="module")
def stand_in(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("hip") / "stand_in.so")
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-o", out, os.path.join(HERE, "hip_stand_in.cpp")], check=True)
    return out


def run(stand_in, body):
    got = subprocess.run([sys.executable, "-c", HEADER + body, stand_in], cwd=os.path.dirname(HERE),
                         capture_output=True, text=True, timeout=120)
    assert got.returncode == 0, got.stdout + got.stderr


def test_no_launch_passes_a_grid_dimension(stand_in):
    """A launch holds fewer than 2^32 work items a dimension; calls that need
    more take several launches."""
    run(stand_in, """
def check(what, least):
    got = sizes()
    assert got, what
    for v in got:
        assert all(v[i] * v[i + 3] < 2**32 for i in range(3)), (what, v)
    assert sum(v[0] for v in got) >= least, (what, got)
    return got

assert forward(_call()) == nlb.NLB_OK and len(sizes()) == 1
# 1 050 000 sequences of 4 rows, 16 heads: 18.9 million narrow workgroups
n = 1_050_000
c = _call(heads=16, kv_heads=4, batch=n, q_rows=4 * n, k_rows=4 * n, q_start=P, k_start=P)
assert forward(c) == nlb.NLB_OK
check("forward", (n + n // 8) * 16)
assert backward(c) == nlb.NLB_OK
check("backward", (n + n // 8) * (16 + 4))
c = _call(heads=16, kv_heads=16, batch=n, q_rows=4 * n, k_rows=4 * n, q_start=P, k_start=P)
assert backward(c) == nlb.NLB_OK
check("backward over keys", (n + n // 8) * 32)
# wide workgroups of long sequences: 2^24 and one more
for dtype in (nlb.DTYPE_BF16, nlb.DTYPE_F32):
    c = _call(dtype=dtype, dim=128, heads=64, kv_heads=64, batch=1, q_rows=128 * 2**18, k_rows=256)
    assert forward(c) == nlb.NLB_OK
    check("forward, wide", (2**18 + 1) * 64)
    assert backward(c) == nlb.NLB_OK
    check("backward, wide", (2**18 + 1) * 64)
# 300 000 lists of 10 slots, 64 heads in 8 groups
c = _call(heads=64, kv_heads=8, batch=300_000, q_rows=300_000, k_rows=3_000_000)
assert forward(c) == nlb.NLB_OK
check("lists", 1)
assert backward(c) == nlb.NLB_OK
check("lists, backward", 300_000 * 64)
# single rows over ragged histories: the joining launch
c = _call(heads=256, kv_heads=1, batch=66_000, q_rows=66_000, k_rows=100 * 66_000, k_start=P)
assert forward(c) == nlb.NLB_OK
got = check("join", 66_000 * 256)
# the largest batch
c = _call(heads=256, kv_heads=1, batch=2**23 - 1, q_rows=2**23 - 1, k_rows=2**31 - 1024, k_start=P)
assert forward(c) == nlb.NLB_OK
check("join", (2**23 - 1) * 256)
""")


def test_nothing_follows_a_launch_that_fails(stand_in):
    """A call whose first, second, ... launch is refused returns NLB_EDEVICE
    and starts none after it: those would read what the missing one leaves.
    An error that an earlier call of the program left is not this call's."""
    run(stand_in, """
at = ctypes.c_int.in_dll(hip, "fail_at")
bias = dict(buckets=4, bias=P, bounds=P)
million = dict(heads=16, batch=1_050_000, q_rows=4_200_000, k_rows=4_200_000, q_start=P, k_start=P)
calls = {
    "tiles": (lambda: forward(_call()), 1),
    "tiles in pieces": (lambda: forward(_call(**million)), 2),
    "lists": (lambda: forward(_call(batch=9000, q_rows=9000, k_rows=90_000)), 1),
    "chunks": (lambda: forward(_call(q_rows=2, k_rows=2000)), 2),
    "backward": (lambda: backward(_call()), 3),               # rows, keys, the sum of a group's heads
    "backward, wide rows": (lambda: backward(_call(dim=128)), 4),
    "backward, pieces": (lambda: backward(_call(**million)), 3),
    "backward, bias": (lambda: backward(_call(**bias), dbias=P), 4),
    "backward, bias of many": (lambda: backward(_call(q_rows=600_000, **bias), dbias=P), 5),
    "backward, lists": (lambda: backward(_call(q_rows=2, k_rows=20, **bias), dbias=P), 2),
    "norm": (lambda: lib.nlb_layer_norm(_norm(), None, 1e-5, P, 100, None), 1),
    "norm, backward": (lambda: lib.nlb_layer_norm_backward(_norm(), P, 100, P, 100, P, P, P, 1 << 40, None), 2),
}
for what, (call, n) in calls.items():
    hip.leave_error(1)
    assert call() == nlb.NLB_OK, what
    assert hip.launched() == n, (what, hip.launched())
    hip.forget()
    for at.value in range(n):
        assert call() == nlb.NLB_EDEVICE, (what, at.value)
        assert hip.launched() == at.value + 1, (what, at.value, hip.launched())
        hip.forget()
    at.value = -1
""")
