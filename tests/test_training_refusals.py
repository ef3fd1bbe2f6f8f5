"""What the operators that train a retrieval layer (rows by id, norm and
rotation, gated recurrence) refuse, on the host, before any device work: no GPU
is needed, and nothing here would launch a kernel."""
import ctypes

import pytest

import paper_2402_01964_amd as nlb

P = 4096                                                      # a stand-in pointer, never followed
BIG = 1 << 50


def _set(c, kw):
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def ids(b):
    return ",".join(f"{k}={v}" for k, v in b.items())


# ---------------------------------------------------------------- rows by id
def lookup(**kw):
    return _set(nlb._LookupCall(-1, nlb.DTYPE_BF16, 100, 50, 64, 2.0, P), kw)


BAD_LOOKUPS = [dict(dtype=2), dict(n=2**31), dict(rows=0), dict(rows=2**31), dict(width=0), dict(width=-1),
               dict(width=65537), dict(scale=float("nan")), dict(scale=float("inf")), dict(ids=None), dict(ids=P + 2)]


@pytest.mark.parametrize("bad", BAD_LOOKUPS, ids=ids)
def test_lookup_refuses(bad):
    lib, n, c = nlb.load_library(), ctypes.c_size_t(7), lookup(**bad)
    assert lib.nlb_lookup(c, P, 64, P, 64, None) == nlb.NLB_EINVAL
    assert lib.nlb_lookup_work(c, 0, n) == nlb.NLB_EINVAL and n.value == 7
    assert lib.nlb_lookup_backward(c, P, 64, P, 64, None, None, P, BIG, None) == nlb.NLB_EINVAL
    assert lib.nlb_lookup_backward(c, P, 64, P, 64, P, P, P, BIG, None) == nlb.NLB_EINVAL


def test_lookup_refuses_its_own_arguments():
    lib, n, c = nlb.load_library(), ctypes.c_size_t(), lookup()
    assert lib.nlb_lookup(None, P, 64, P, 64, None) == nlb.NLB_EINVAL
    assert lib.nlb_lookup_work(None, 0, n) == nlb.NLB_EINVAL
    assert lib.nlb_lookup_work(c, 0, None) == nlb.NLB_EINVAL
    for t, ts, o, os_ in ((None, 64, P, 64), (P + 1, 64, P, 64), (P, -1, P, 64), (P, 2**31, P, 64), (P, 64, None, 64),
                          (P, 64, P + 1, 64), (P, 64, P, -64), (P, 64, P, 2**31)):
        assert lib.nlb_lookup(c, t, ts, o, os_, None) == nlb.NLB_EINVAL
        assert lib.nlb_lookup_backward(c, t, ts, o, os_, None, None, P, BIG, None) == nlb.NLB_EINVAL
    for row_ids, count, work in ((P, None, P), (None, P, P), (P + 2, P, P), (P, P + 1, P), (P, P, P + 8)):
        assert lib.nlb_lookup_backward(c, P, 64, P, 64, row_ids, count, work, BIG, None) == nlb.NLB_EINVAL
    # a gradient of no ids is still the whole table's
    assert lib.nlb_lookup_backward(lookup(n=0), P, 64, None, 64, None, None, P, BIG, None) == nlb.NLB_EINVAL


@pytest.mark.parametrize("listed", [0, 1])
@pytest.mark.parametrize("n", [0, 1, 100, 5_000_000, 2**31 - 1])
def test_lookup_work_is_checked(n, listed):
    lib, size, c = nlb.load_library(), ctypes.c_size_t(), lookup(n=n)
    assert lib.nlb_lookup_work(c, listed, size) == nlb.NLB_OK and size.value > 16 * n
    args = (P, P) if listed else (None, None)
    for work, have in ((P, size.value - 1), (None, size.value), (None, 0)):
        assert lib.nlb_lookup_backward(c, P, 64, P, 64, *args, work, have, None) == nlb.NLB_ESCRATCH


# ---------------------------------------------------------------- norm and rotation
def rotate(**kw):
    c = nlb._RotateCall()
    for k, v in dict(device=-1, dtype=nlb.DTYPE_BF16, dim=64, freqs=32, heads=4, kv_heads=2, q_rows=10, k_rows=12,
                     eps=1e-5, freq=P, q_pos=P, k_pos=P, wq=P, wk=P, q=P, q_row=256, q_head=64, k=P, k_row=128,
                     k_head=64).items():
        setattr(c, k, v)
    return _set(c, kw)


BAD_ROTATIONS = [dict(dtype=2), dict(dim=0), dict(dim=129), dict(freqs=-1), dict(freqs=33), dict(heads=0),
                 dict(heads=257), dict(kv_heads=0), dict(kv_heads=-1), dict(kv_heads=257), dict(q_rows=2**31),
                 dict(k_rows=2**31), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(freq=None),
                 dict(freq=P + 2), dict(q_pos=None), dict(k_pos=None), dict(q_pos=P + 1), dict(k_pos=P + 2),
                 dict(wq=P + 2), dict(wk=P + 1), dict(q=None), dict(k=None), dict(q=P + 1), dict(q_row=-1),
                 dict(k_row=2**31), dict(k_head=-64), dict(q_head=2**31)]
ROWS = nlb._AttRows(P, 256, 64)


def rotate_backward(lib, c, gq=ROWS, gk=ROWS, dq=ROWS, dk=ROWS, dwq=P, dwk=P, work=P, size=BIG):
    return lib.nlb_norm_rotate_backward(c, gq, gk, dq, dk, dwq, dwk, work, size, None)


@pytest.mark.parametrize("bad", BAD_ROTATIONS, ids=ids)
def test_norm_rotate_refuses(bad):
    lib, n, c = nlb.load_library(), ctypes.c_size_t(7), rotate(**bad)
    assert lib.nlb_norm_rotate(c, ROWS, ROWS, None) == nlb.NLB_EINVAL
    assert lib.nlb_norm_rotate_work(c, n) == nlb.NLB_EINVAL and n.value == 7
    assert rotate_backward(lib, c) == nlb.NLB_EINVAL


BAD_ROWS = [None, nlb._AttRows(None, 256, 64), nlb._AttRows(P + 1, 256, 64), nlb._AttRows(P, -1, 64),
            nlb._AttRows(P, 256, 2**31)]


def test_norm_rotate_refuses_its_own_arguments():
    lib, n, c = nlb.load_library(), ctypes.c_size_t(), rotate()
    assert lib.nlb_norm_rotate(None, ROWS, ROWS, None) == nlb.NLB_EINVAL
    assert lib.nlb_norm_rotate_work(None, n) == nlb.NLB_EINVAL
    assert lib.nlb_norm_rotate_work(c, None) == nlb.NLB_EINVAL
    for bad in BAD_ROWS:
        assert lib.nlb_norm_rotate(c, bad, ROWS, None) == nlb.NLB_EINVAL
        assert lib.nlb_norm_rotate(c, ROWS, bad, None) == nlb.NLB_EINVAL
        for name in ("gq", "gk", "dq", "dk"):
            assert rotate_backward(lib, c, **{name: bad}) == nlb.NLB_EINVAL
    for kw in (dict(dwq=P + 2), dict(dwk=P + 1), dict(work=P + 4)):
        assert rotate_backward(lib, c, **kw) == nlb.NLB_EINVAL
    assert lib.nlb_norm_rotate_work(c, n) == nlb.NLB_OK and n.value > 0
    for kw in (dict(work=None), dict(size=n.value - 1), dict(size=n.value - 1, dwq=None), dict(work=None, dwk=None)):
        assert rotate_backward(lib, c, **kw) == nlb.NLB_ESCRATCH


# ---------------------------------------------------------------- gated recurrence
def scan(**kw):
    c = nlb._ScanCall()
    for k, v in dict(device=-1, dtype=nlb.DTYPE_BF16, rows=3000, batch=3, width=64, start=P, h0=P, x=P, x_row=64, g=P,
                     g_row=64).items():
        setattr(c, k, v)
    return _set(c, kw)


BAD_SCANS = [dict(dtype=2), dict(width=0), dict(width=65537), dict(rows=2147480001), dict(batch=0), dict(batch=2**31),
             dict(batch=7, start=None), dict(x=None), dict(g=None), dict(x=P + 1), dict(g=P + 1), dict(x_row=-1),
             dict(g_row=2**31), dict(start=P + 2), dict(h0=P + 1)]
SROWS = nlb._ScanRows(P, 64)


def scan_forward(lib, c, h=SROWS, last=1 << 30, states=P, work=P, size=BIG):
    return lib.nlb_gated_scan(c, h, last, states, work, size, None)


def scan_backward(lib, c, states=P, dh=SROWS, dlast=P, dx=SROWS, dg=SROWS, dh0=1 << 30, work=P, size=BIG):
    return lib.nlb_gated_scan_backward(c, states, dh, dlast, dx, dg, dh0, work, size, None)


@pytest.mark.parametrize("bad", BAD_SCANS, ids=ids)
def test_gated_scan_refuses(bad):
    lib, n, c = nlb.load_library(), ctypes.c_size_t(7), scan(**bad)
    assert scan_forward(lib, c) == nlb.NLB_EINVAL
    assert lib.nlb_gated_scan_work(c, n) == nlb.NLB_EINVAL and n.value == 7
    assert scan_backward(lib, c) == nlb.NLB_EINVAL


def test_gated_scan_refuses_its_own_arguments():
    lib, n, c = nlb.load_library(), ctypes.c_size_t(), scan()
    assert scan_forward(lib, None) == nlb.NLB_EINVAL and scan_backward(lib, None) == nlb.NLB_EINVAL
    assert lib.nlb_gated_scan_work(None, n) == nlb.NLB_EINVAL
    assert lib.nlb_gated_scan_work(c, None) == nlb.NLB_EINVAL
    for bad in (None, nlb._ScanRows(None, 64), nlb._ScanRows(P + 1, 64), nlb._ScanRows(P, -1), nlb._ScanRows(P, 2**31)):
        assert scan_forward(lib, c, h=bad) == nlb.NLB_EINVAL
        for name in ("dh", "dx", "dg"):
            assert scan_backward(lib, c, **{name: bad}) == nlb.NLB_EINVAL
    for kw in (dict(last=P + 2), dict(states=P + 1), dict(work=P + 8)):
        assert scan_forward(lib, c, **kw) == nlb.NLB_EINVAL
    for kw in (dict(states=None), dict(states=P + 2), dict(dlast=P + 1), dict(dh0=P + 2), dict(work=P + 8)):
        assert scan_backward(lib, c, **kw) == nlb.NLB_EINVAL
    assert lib.nlb_gated_scan_work(c, n) == nlb.NLB_OK and n.value > 0
    for call in (scan_forward, scan_backward):
        for kw in (dict(work=None), dict(size=n.value - 1)):
            assert call(lib, c, **kw) == nlb.NLB_ESCRATCH


def test_gated_scan_refuses_states_that_overlap():
    """A sequence's last state would be written while its first is read."""
    lib = nlb.load_library()
    size = 3 * 64 * 4
    for at in (0, 4, size - 4, 4 - size):
        assert scan_forward(lib, scan(h0=P), last=P + at) == nlb.NLB_EINVAL
        assert scan_forward(lib, scan(h0=P, start=None), last=P + at) == nlb.NLB_EINVAL
        assert scan_backward(lib, scan(h0=P), dlast=1 << 30, dh0=P + at) == nlb.NLB_EINVAL
        assert scan_backward(lib, scan(h0=1 << 40), dlast=P, dh0=P + at) == nlb.NLB_EINVAL
        if at:                                                # single rows: the same array or another one
            assert scan_forward(lib, scan(h0=P, start=None, rows=3), last=P + at) == nlb.NLB_EINVAL
