"""What the operators without a table refuse, on the host, before any device
work: no GPU is needed, and nothing here would launch a kernel."""
import ctypes

import pytest

import paper_2402_01964_amd as nlb

P = 4096                                                      # a stand-in pointer, never followed


def _call(**kw):
    c = nlb._AttCall()
    c.device, c.dtype, c.heads, c.kv_heads, c.dim, c.scale = -1, nlb.DTYPE_BF16, 4, 2, 64, 0.125
    c.batch, c.q_rows, c.k_rows = 2, 10, 10
    for k in ("q", "k", "v"):
        setattr(c, k, P)
        setattr(c, k + "_row", 256)
        setattr(c, k + "_head", 64)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


ROWS = nlb._AttRows(P, 256, 64)
BAD_CALLS = [
    dict(dtype=2), dict(heads=0), dict(heads=257, kv_heads=257), dict(kv_heads=0), dict(kv_heads=3), dict(dim=0),
    dict(dim=129), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=2.0**21), dict(scale=2.0**-21), dict(causal=2), dict(batch=0), dict(batch=2**31),
    dict(q_rows=2**31), dict(k_rows=2**31), dict(q_rows=2**31 - 1023, q_start=P), dict(k_rows=2**31 - 1023, k_start=P), dict(q_rows=11), dict(k_rows=11), dict(buckets=-1), dict(buckets=65, bias=P,
                                                                                                     bounds=P),
    dict(buckets=4), dict(bias=P), dict(buckets=4, bias=P), dict(buckets=4, bias=P, bounds=P + 2),
    dict(buckets=4, bias=P + 1, bounds=P), dict(q_pos=P), dict(q_start=P + 1), dict(k_start=P + 2), dict(k_pos=P + 1),
    dict(buckets=4, bias=P, bounds=P, k_pos=P), dict(q=None), dict(k=None),
    dict(v=P + 1), dict(q_row=-1), dict(k_row=2**31), dict(v_head=-64),
]


@pytest.mark.parametrize("bad", BAD_CALLS, ids=lambda b: ",".join(b))
def test_attention_refuses(bad):
    lib, n = nlb.load_library(), ctypes.c_size_t(7)
    c = _call(**bad)
    assert lib.nlb_attention_work(ctypes.byref(c), 0, ctypes.byref(n)) == nlb.NLB_EINVAL
    assert n.value == 7
    assert lib.nlb_attention(ctypes.byref(c), ctypes.byref(ROWS), None, None, 0, None) == nlb.NLB_EINVAL


def test_attention_refuses_null_and_misaligned():
    lib, n = nlb.load_library(), ctypes.c_size_t()
    c = _call()
    assert lib.nlb_attention_work(None, 0, ctypes.byref(n)) == nlb.NLB_EINVAL
    assert lib.nlb_attention_work(ctypes.byref(c), 0, None) == nlb.NLB_EINVAL
    for o, lse, work in ((None, None, None), (nlb._AttRows(None, 256, 64), None, None),
                         (nlb._AttRows(P, 2**31, 64), None, None), (ROWS, P + 2, None), (ROWS, None, P + 8)):
        assert lib.nlb_attention(ctypes.byref(c), o, lse, work, 0, None) == nlb.NLB_EINVAL


def test_attention_work_is_checked():
    """Single rows over long sequences work in chunks; too little memory for
    them is refused."""
    lib, n = nlb.load_library(), ctypes.c_size_t()
    for c, some in ((_call(), False), (_call(q_rows=2, k_rows=2000), True), (_call(q_rows=2, k_rows=20), False),
                    (_call(q_rows=2, k_rows=2001, k_start=P), True), (_call(q_rows=20, k_rows=2000), False)):
        assert lib.nlb_attention_work(ctypes.byref(c), 0, ctypes.byref(n)) == nlb.NLB_OK
        assert (n.value > 0) == some
        if some:
            for work, size in ((P, n.value - 1), (None, n.value), (None, 0)):
                assert lib.nlb_attention(ctypes.byref(c), ROWS, None, work, size, None) == nlb.NLB_ESCRATCH


def test_attention_grid_limit():
    lib = nlb.load_library()
    c = _call(heads=256, kv_heads=256, q_rows=2**31 - 1024, q_start=P)
    assert lib.nlb_attention(ctypes.byref(c), ROWS, None, None, 0, None) == nlb.NLB_EINVAL


def _backward(lib, c, o=ROWS, lse=P, dout=ROWS, dq=ROWS, dk=ROWS, dv=ROWS, dbias=None, work=None, size=0):
    return lib.nlb_attention_backward(ctypes.byref(c), o, lse, dout, dq, dk, dv, dbias, work, size, None)


@pytest.mark.parametrize("bad", BAD_CALLS, ids=lambda b: ",".join(b))
def test_attention_backward_refuses(bad):
    lib, n = nlb.load_library(), ctypes.c_size_t(7)
    c = _call(**bad)
    assert lib.nlb_attention_work(ctypes.byref(c), 1, ctypes.byref(n)) == nlb.NLB_EINVAL
    assert n.value == 7
    assert _backward(lib, c, work=P, size=1 << 40) == nlb.NLB_EINVAL


@pytest.mark.parametrize("bad", [
    dict(o=None), dict(dout=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(lse=None), dict(lse=P + 2),
    dict(o=nlb._AttRows(None, 256, 64)), dict(dout=nlb._AttRows(P + 1, 256, 64)), dict(dq=nlb._AttRows(P, -1, 0)),
    dict(dk=nlb._AttRows(None, 0, 0)), dict(dv=nlb._AttRows(P, 0, 2**31)), dict(dbias=P), dict(work=P + 4)],
    ids=lambda b: ",".join(b))
def test_attention_backward_refuses_its_own_arguments(bad):
    lib = nlb.load_library()
    assert _backward(lib, _call(), **{"work": P, "size": 1 << 40, **bad}) == nlb.NLB_EINVAL
    c = _call(buckets=4, bias=P, bounds=P)
    assert _backward(lib, c, dbias=P + 1, work=P, size=1 << 40) == nlb.NLB_EINVAL


def test_attention_backward_work_is_checked():
    lib, n = nlb.load_library(), ctypes.c_size_t()
    for c in (_call(), _call(buckets=4, bias=P, bounds=P), _call(q_rows=2, buckets=4, bias=P, bounds=P)):
        assert lib.nlb_attention_work(ctypes.byref(c), 1, ctypes.byref(n)) == nlb.NLB_OK
        assert n.value > 0
        for work, size in ((P, n.value - 1), (None, n.value), (None, 0)):
            assert _backward(lib, c, work=work, size=size) == nlb.NLB_ESCRATCH
    c = _call(heads=256, kv_heads=256, k_rows=2**31 - 1024, k_start=P)
    assert _backward(lib, c, work=P, size=1 << 50) == nlb.NLB_EINVAL      # more workgroups than a grid has


def _norm(**kw):
    c = nlb._NormCall()
    c.device, c.dtype, c.rows, c.width, c.x, c.x_stride, c.mean, c.rstd = -1, nlb.DTYPE_BF16, 10, 100, P, 100, P, P
    for k, v in kw.items():
        setattr(c, k, v)
    return c


BAD_NORMS = [dict(dtype=2), dict(rows=2**31), dict(width=0), dict(width=8193), dict(x=None), dict(x=P + 1), dict(w=P + 2),
             dict(mean=P + 2), dict(rstd=P + 1), dict(x_stride=-1), dict(x_stride=2**31)]


@pytest.mark.parametrize("bad", BAD_NORMS, ids=lambda b: ",".join(b))
def test_layer_norm_refuses(bad):
    lib, n = nlb.load_library(), ctypes.c_size_t(7)
    c = _norm(**bad)
    assert lib.nlb_layer_norm(ctypes.byref(c), None, 1e-5, P, 100, None) == nlb.NLB_EINVAL
    assert lib.nlb_layer_norm_work(ctypes.byref(c), ctypes.byref(n)) == nlb.NLB_EINVAL and n.value == 7
    assert lib.nlb_layer_norm_backward(ctypes.byref(c), P, 100, P, 100, P, P, P, 1 << 40, None) == nlb.NLB_EINVAL


def test_layer_norm_refuses_its_own_arguments():
    lib, n = nlb.load_library(), ctypes.c_size_t()
    c = _norm()
    for b, eps, y, stride in ((P + 2, 1e-5, P, 100), (None, -1.0, P, 100), (None, float("nan"), P, 100),
                              (None, float("inf"), P, 100), (None, 1e-5, None, 100), (None, 1e-5, P + 1, 100),
                              (None, 1e-5, P, -1), (None, 1e-5, P, 2**31)):
        assert lib.nlb_layer_norm(ctypes.byref(c), b, eps, y, stride, None) == nlb.NLB_EINVAL
    assert lib.nlb_layer_norm(None, None, 1e-5, P, 100, None) == nlb.NLB_EINVAL
    assert lib.nlb_layer_norm_work(ctypes.byref(c), None) == nlb.NLB_EINVAL
    assert lib.nlb_layer_norm_work(ctypes.byref(c), ctypes.byref(n)) == nlb.NLB_OK and n.value > 0
    back = lib.nlb_layer_norm_backward
    for dy, dys, dx, dxs, dw, db, work in ((None, 100, P, 100, P, P, P), (P, -1, P, 100, P, P, P),
                                           (P, 100, None, 100, P, P, P), (P, 100, P, 2**31, P, P, P),
                                           (P, 100, P, 100, P + 2, P, P), (P, 100, P, 100, P, P + 1, P),
                                           (P, 100, P, 100, P, P, P + 8)):
        assert back(ctypes.byref(c), dy, dys, dx, dxs, dw, db, work, 1 << 40, None) == nlb.NLB_EINVAL
    for bad in (dict(mean=None), dict(rstd=None)):
        assert back(ctypes.byref(_norm(**bad)), P, 100, P, 100, P, P, P, 1 << 40, None) == nlb.NLB_EINVAL
    for work, size in ((None, 1 << 40), (P, n.value - 1)):
        assert back(ctypes.byref(c), P, 100, P, 100, P, None, work, size, None) == nlb.NLB_ESCRATCH


def test_binding_checks_its_tensors():
    import torch
    x = torch.zeros(4, 2, 8)
    with pytest.raises(TypeError):
        nlb.attention(x, x, x)
    with pytest.raises(TypeError):
        nlb.layer_norm(x)
