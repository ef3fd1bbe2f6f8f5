"""Rows whose places pass 32 bits: the same call on rows that lie far apart and on
a compact copy of them gives the same bits (strides do not set the order of
sums)."""
import pytest

pytestmark = pytest.mark.gpu


def far(rows, width, dtype, seed):
    """[rows, width] within 5 GB, its last row behind 2^32 bytes; and a copy."""
    import torch
    gap = 5_000_000_000 // (rows * torch.finfo(dtype).bits // 8)
    big = torch.empty(rows, gap, dtype=dtype, device="cuda")
    x = big[:, gap - width - 1:gap - 1]
    torch.manual_seed(seed)
    x.copy_(torch.randn(rows, width, device="cuda"))
    assert x.stride(0) * rows * x.element_size() > 2**32
    return x, x.contiguous()


@pytest.mark.parametrize("name", ["bfloat16", "float32"])
def test_rows_by_id(name):
    import torch
    import paper_2402_01964_amd as nlb
    dtype = getattr(torch, name)
    x, near = far(3000, 100, dtype, 0)
    ids = torch.randint(-1, 3000, (4000,), dtype=torch.int32, device="cuda")
    assert torch.equal(nlb.lookup(x, ids, 3.0), nlb.lookup(near, ids, 3.0))
    ids = torch.randint(-1, 50, (3000,), dtype=torch.int32, device="cuda")
    want = nlb.lookup_backward(near, ids, 50, 3.0)
    assert torch.equal(nlb.lookup_backward(x, ids, 50, 3.0), want)
    ids = ids * 20_000_000                                     # into a table of 10^9 rows
    grads, row_ids, count = nlb.lookup_backward_listed(x, ids, 10**9, 3.0)
    n = int(count)
    assert torch.equal(row_ids[:n] // 20_000_000, want.abs().sum(1).nonzero()[:, 0].int())
    assert torch.equal(grads[:n], want[(row_ids[:n] // 20_000_000).long()])
    out, _ = far(3000, 100, dtype, 1)
    nlb.lookup_backward(near, ids // 20_000_000, 3000, 3.0, dtable=out)
    assert torch.equal(out[:50], want) and not out[50:].any()


@pytest.mark.parametrize("name", ["bfloat16", "float32"])
def test_recurrence(name):
    import torch
    import paper_2402_01964_amd as nlb
    dtype = getattr(torch, name)
    rows = [far(2500, 130, dtype, s) for s in range(3)]
    (x, nx), (g, ng), (d, nd) = rows
    start = torch.tensor([0, 900, 901, 2500], dtype=torch.int32, device="cuda")
    want, near_last, states = nlb.gated_scan(nx, ng, start=start)
    grads = nlb.gated_scan_backward(nd, nx, ng, states, start=start)
    h, last, states = nlb.gated_scan(x, g, start=start, out=x.clone(memory_format=torch.preserve_format))
    assert torch.equal(h, want) and torch.equal(last, near_last)
    dx, dg, _ = nlb.gated_scan_backward(d, x, g, states, start=start, dx=d)
    assert dx is d and torch.equal(dx, grads[0]) and torch.equal(dg, grads[1])
    nlb.gated_scan(x, g, start=start, out=x)
    assert torch.equal(x, want)


@pytest.mark.parametrize("name", ["bfloat16", "float32"])
def test_norm_and_rotation(name):
    import torch
    import paper_2402_01964_amd as nlb
    dtype = getattr(torch, name)
    (q, nq), (d, nd) = (far(2000, 3 * 50, dtype, s) for s in range(2))
    q, nq, d, nd = (t.unflatten(1, (3, 50)) for t in (q, nq, d, nd))
    pos = torch.randint(0, 2**30, (2000,), dtype=torch.int32, device="cuda")
    freq = torch.rand(20, device="cuda")
    w = torch.rand(50, device="cuda")
    want, _ = nlb.norm_rotate(nq, None, freq, pos, None, w)
    grads = nlb.norm_rotate_backward(nd, None, nq, None, freq, pos, None, w)
    got = nlb.norm_rotate_backward(d, None, q, None, freq, pos, None, w, dq=d)
    assert torch.equal(got[0], grads[0]) and torch.equal(got[2], grads[2])
    nlb.norm_rotate(q, None, freq, pos, None, w, q_out=q)
    assert torch.equal(q, want)
