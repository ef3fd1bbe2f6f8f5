"""Rows by id and the table's gradient on the GPU (nlb_lookup) against 64 bits.

Bounds, with w = 2^-24 and u half a step of the rows' type (2^-8 bf16, w fp32):
a row is its table's times the scale, rounded in fp32 and to its type: (w + u) of
itself.  A gradient sums the k places of its id in fp32 in some order: (k - 1) w
of the sum of their magnitudes, and then as a row.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

W = 2.0 ** -24
HALF_STEP = {"bf16": 2.0 ** -8, "f32": W}
SENTINEL = 77.0
DTYPES = pytest.mark.parametrize("dtype", ["bf16", "f32"])


def rand(dtype, n, width, gap, seed):
    import torch
    gen = torch.Generator().manual_seed(seed)
    return torch.randn(n, width + gap, generator=gen).to(
        {"bf16": torch.bfloat16, "f32": torch.float32}[dtype])[:, :width]


def cuda(t):
    import torch
    out = torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda")
    return out.copy_(t)


def f64(t):
    return t.double().cpu().numpy()


def check_rows(dtype, ids, rows, width, scale=1.0, gap=0, seed=0):
    import torch
    import paper_2402_01964_amd as nlb
    table = rand(dtype, rows, width, gap, seed)
    got = f64(nlb.lookup(cuda(table), torch.from_numpy(ids).cuda(), scale))
    there = (ids >= 0) & (ids < rows)
    want = np.where(there[:, None], f64(table)[np.where(there, ids, 0)], 0) * scale
    assert (np.abs(got - want) <= (W + HALF_STEP[dtype]) * np.abs(want)).all()


def check_gradient(dtype, ids, rows, width, scale=1.0, gap=0, seed=0, listed=(False, True)):
    import torch
    import paper_2402_01964_amd as nlb
    n = len(ids)
    dout = rand(dtype, n, width, gap, seed)
    there = (ids >= 0) & (ids < rows)
    found, inverse, many = np.unique(ids[there], return_inverse=True, return_counts=True)
    want, size = np.zeros((len(found), width)), np.zeros((len(found), width))
    np.add.at(want, inverse, f64(dout)[there])
    np.add.at(size, inverse, np.abs(f64(dout)[there]))
    want, size = want * scale, size * abs(scale)
    far = (many[:, None] - 1) * W * size
    far += (W + HALF_STEP[dtype]) * (np.abs(want) + far)
    d, i = cuda(dout), torch.from_numpy(ids).cuda()
    if False in listed:
        dtable = torch.full((rows, width + gap), SENTINEL, dtype=dout.dtype, device="cuda")
        out = nlb.lookup_backward(d, i, rows, scale, dtable=dtable[:, :width])
        got = f64(out)
        assert (f64(dtable)[:, width:] == SENTINEL).all()
        off = np.abs(got[found] - want) - far
        assert off.size == 0 or (off <= 0).all(), (n, rows, width, float(off.max()))
        rest = np.ones(rows, bool)
        rest[found] = False
        assert not got[rest].any()
    if True in listed:
        grads = torch.full((n, width), SENTINEL, dtype=dout.dtype, device="cuda")
        out, row_ids, count = nlb.lookup_backward_listed(d, i, rows, scale, grads=grads)
        assert out is grads and count.tolist() == [len(found)]
        row_ids, got = row_ids.cpu().numpy(), f64(grads)
        assert (row_ids[:len(found)] == found).all() and (row_ids[len(found):] == -1).all()
        off = np.abs(got[:len(found)] - want) - far
        assert off.size == 0 or (off <= 0).all(), (n, rows, width, float(off.max()))
        assert (got[len(found):] == SENTINEL).all()


def some_ids(n, rows, seed=0, fill=0.8, popular=False):
    rng = np.random.default_rng(seed)
    ids = rng.integers(0, rows, n)
    if popular:
        ids = (rows ** rng.random(n)).astype(np.int64) % rows
    wrong = rng.integers(0, 4, n)
    ids = np.where(rng.random(n) < fill, ids,
                   np.select([wrong == 0, wrong == 1, wrong == 2], [-1, rows, -2**31], 2**31 - 1))
    return ids.astype(np.int32)


WIDTHS = [1, 2, 3, 4, 5, 7, 8, 9, 16, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 172, 256, 300, 512, 513, 1030]


@DTYPES
@pytest.mark.parametrize("width", WIDTHS)
def test_rows(dtype, width):
    for n in (1, 5, 700):
        check_rows(dtype, some_ids(n, 50, width), 50, width, scale=width ** 0.5, seed=width)


@DTYPES
@pytest.mark.parametrize("width", WIDTHS)
def test_gradient_widths(dtype, width):
    check_gradient(dtype, some_ids(700, 50, width), 50, width, scale=width ** 0.5, seed=width)
    check_gradient(dtype, some_ids(90, 1000, width), 1000, width, seed=width)


@DTYPES
@pytest.mark.parametrize("gap", [1, 3, 8])
def test_strides(dtype, gap):
    for width in (5, 64, 130):
        check_rows(dtype, some_ids(300, 40), 40, width, gap=gap)
        check_gradient(dtype, some_ids(300, 40), 40, width, gap=gap)


@DTYPES
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 49, 64, 255, 256, 257, 1000, 4095, 4096, 4097, 9000])
def test_one_row_takes_all_and_two_share(dtype, n):
    check_gradient(dtype, np.zeros(n, np.int32), 1, 20)
    check_gradient(dtype, np.full(n, 2**31 - 2, np.int32), 2**31 - 1, 3, listed=(True,))
    ids = np.full(n, 5, np.int32)
    ids[: n // 3] = 2
    check_gradient(dtype, ids, 7, 20)


@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 30, 31, 32, 33, 34, 47, 48, 49, 50, 63, 64, 65, 100])
def test_rows_over_the_edges_of_runs(length):
    """Rows of a given number of places at every offset from the runs of 16."""
    for before in range(18):
        many = [1] * before + [length, 3, length, 1, 40]
        ids = np.repeat(np.arange(len(many)), many).astype(np.int32)
        check_gradient("f32", np.random.default_rng(before).permutation(ids), len(many) + 2, 4, seed=before)


@DTYPES
@pytest.mark.parametrize("rows", [1, 2, 255, 256, 257, 511, 512, 513, 17_000, 262_144, 262_145, 1_000_000])
def test_tables_of_all_sizes(dtype, rows):
    for popular in (False, True):
        check_gradient(dtype, some_ids(10_000, rows, rows, popular=popular), rows, 8)


@DTYPES
def test_large_calls(dtype):
    check_gradient(dtype, some_ids(300_000, 3000, 1, popular=True), 3000, 12)
    check_gradient(dtype, some_ids(1_000_003, 900_000, 2, fill=0.5), 900_000, 5)
    check_gradient(dtype, some_ids(70_000, 2**31 - 1, 3), 2**31 - 1, 100, listed=(True,))
    check_rows(dtype, some_ids(200_001, 70_000, 4), 70_000, 100)
    check_rows(dtype, some_ids(40, 30, 4), 30, 20_000)
    check_gradient(dtype, some_ids(300, 30, 4), 30, 9000)


@DTYPES
def test_no_ids_and_none_that_is_a_row(dtype):
    check_gradient(dtype, np.zeros(0, np.int32), 9, 16)
    check_gradient(dtype, np.full(5000, -1, np.int32), 9, 16)
    check_gradient(dtype, np.full(3, 9, np.int32), 9, 16)
    check_rows(dtype, np.zeros(0, np.int32), 9, 16)
    check_rows(dtype, np.full(70, -1, np.int32), 9, 16)


def test_more_dimensions():
    """A retrieved list's neighbours, [queries, slots], as sample returns them."""
    import torch
    import paper_2402_01964_amd as nlb
    table = torch.randn(30, 24, device="cuda")
    ids = torch.from_numpy(some_ids(12, 30, 5)).cuda().view(4, 3)
    out = nlb.lookup(table, ids, 2.0)
    assert out.shape == (4, 3, 24) and torch.equal(out.view(12, 24), nlb.lookup(table, ids.view(12), 2.0))
    dout = torch.randn_like(out)
    assert torch.equal(nlb.lookup_backward(dout, ids, 30, 2.0), nlb.lookup_backward(dout.view(12, 24), ids.view(12), 30, 2.0))
    one = nlb.lookup(table, torch.tensor(3, dtype=torch.int32, device="cuda"))
    assert one.shape == (24,) and torch.equal(one, table[3])


def test_what_no_row_takes_goes_nowhere():
    import torch
    import paper_2402_01964_amd as nlb
    ids = some_ids(3000, 100, 6)
    dout = torch.randn(3000, 33, device="cuda")
    i = torch.from_numpy(ids).cuda()
    clean = nlb.lookup_backward(dout, i, 100)
    dout[(i < 0) | (i >= 100)] = float("nan")
    assert torch.equal(clean, nlb.lookup_backward(dout, i, 100))
    # a row's own values stay its own (the ids are the same: they set the order of the sums)
    i[0] = 3
    dout[0] = 1.0
    clean = nlb.lookup_backward(dout, i, 100)
    dout[0] = float("inf")
    got = nlb.lookup_backward(dout, i, 100)
    rest = [r for r in range(100) if r != 3]
    assert torch.equal(got[rest], clean[rest]) and got[3].isinf().all()


def test_gradient_against_differences():
    """Linear in the table: differences are exact up to their roundings (24
    terms of magnitude below 5, a step of one half)."""
    import torch
    import paper_2402_01964_amd as nlb
    torch.manual_seed(0)
    table, ids = torch.randn(6, 4, device="cuda"), torch.from_numpy(some_ids(24, 6, 7)).cuda()
    dout = torch.randn(24, 4, device="cuda")
    grad = nlb.lookup_backward(dout, ids, 6, 3.0)

    def loss(t):
        return float((nlb.lookup(t, ids, 3.0).double() * dout.double()).sum())
    for at in [(0, 0), (3, 2), (5, 3)]:
        both = []
        for s in (0.5, -0.5):
            t = table.clone()
            t[at] += s
            both.append(loss(t))
        assert abs(both[0] - both[1] - float(grad[at])) < 24 * 24 * 5 * 3 * W


def test_same_bits_streams_and_work():
    import torch
    import paper_2402_01964_amd as nlb
    ids = torch.from_numpy(some_ids(50_000, 400, 8, popular=True)).cuda()
    dout = torch.randn(50_000, 60, device="cuda", dtype=torch.bfloat16)
    want = nlb.lookup_backward(dout, ids, 400), nlb.lookup_backward_listed(dout, ids, 400)
    n = [nlb.lookup_work(dout, ids, 400, listed=k) for k in (False, True)]
    assert 0 < n[0] <= n[1]
    work = torch.full((n[1] + 64,), 255, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        got = nlb.lookup_backward(dout, ids, 400, work=work)
        assert torch.equal(got, want[0])
        got, row_ids, count = nlb.lookup_backward_listed(dout, ids, 400, work=work)
        assert torch.equal(row_ids, want[1][1]) and torch.equal(count, want[1][2])
        assert torch.equal(got[:int(count)], want[1][0][:int(count)])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = nlb.lookup_backward(dout, ids, 400, stream=side)
    side.synchronize()
    assert torch.equal(got, want[0])


def test_captured_step():
    import torch
    import paper_2402_01964_amd as nlb
    turns = [torch.from_numpy(some_ids(30_000, 5000, s, fill=f, popular=p)).cuda()
             for s, f, p in ((9, 0.9, True), (10, 0.3, False))]
    table, dout = torch.randn(5000, 40, device="cuda"), torch.randn(30_000, 40, device="cuda")

    def step(ids):
        grads = torch.zeros_like(dout)
        return (nlb.lookup(table, ids), nlb.lookup_backward(dout, ids, 5000)) + nlb.lookup_backward_listed(
            dout, ids, 5000, grads=grads)
    want = [[t.clone() for t in step(i)] for i in turns]
    ids = turns[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step(ids)
    for turn in range(4):
        ids.copy_(turns[turn % 2])
        graph.replay()
        other = step(turns[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[turn % 2]))
        assert all(torch.equal(a, b) for a, b in zip(other, want[1]))
