"""Attention over packed sequences on the GPU (nlb_attention and its backward
pass) against 64 bits, within the bounds that attention_ref derives."""
import numpy as np
import pytest

from tests import attention_ref as ref

pytestmark = pytest.mark.gpu

BOUNDS = [-5, 0, 1, 2, 4, 9, 30, 100]
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def _dtype(name):
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def make(dtype, lq, lk, heads, kv_heads, dim, *, bias=False, times=False, closed=0.2, train=False, seed=0, gap=0,
         sharp=2.0):
    """Inputs on the CPU; gap: values between a row's end and the next row's
    head, so that nothing is contiguous or aligned."""
    import torch
    gen = torch.Generator().manual_seed(seed)
    dt = _dtype(dtype)

    def rows(n, h, scale=1.0):
        return (scale * torch.randn(n, h, dim + gap, generator=gen)).to(dt)[:, :, gap // 2:gap // 2 + dim]
    c = {"q": rows(sum(lq), heads, sharp), "k": rows(sum(lk), kv_heads), "v": rows(sum(lk), kv_heads), "bias": None,
         "bounds": None, "q_pos": None, "k_pos": None, "do": rows(sum(lq), heads) if train else None}
    if bias:
        c["bias"] = torch.randn(len(BOUNDS) + 1, heads, generator=gen).to(dt)
        c["bounds"] = torch.tensor(BOUNDS, dtype=torch.int32)
    if times:
        c["q_pos"] = torch.randint(0, 300, (sum(lq),), generator=gen, dtype=torch.int32)
        c["k_pos"] = torch.randint(0, 300, (sum(lk),), generator=gen, dtype=torch.int32)
        c["k_pos"][torch.rand(sum(lk), generator=gen) < closed] = -1
    return c


def _f64(t):
    return None if t is None else t.double().numpy()


def _u32(t):
    return None if t is None else t.numpy().view(np.uint32)


def _cuda(t):
    """On the GPU with the strides it has."""
    import torch
    if t is None or t.is_contiguous():
        return None if t is None else t.cuda()
    full = torch.empty(t.untyped_storage().nbytes() // t.element_size(), dtype=t.dtype, device="cuda")
    full = full.as_strided(t.size(), t.stride(), t.storage_offset())
    full.copy_(t)
    return full


def run(c, lq, lk, *, causal, one=False, scale=None, **more):
    """The library's outputs; one: single query rows without q_start."""
    import torch
    import paper_2402_01964_amd as nlb
    how = dict(batch=len(lq), causal=causal, scale=scale, **more)
    if not one:
        how["q_start"] = torch.from_numpy(ref.starts(lq)).cuda()
    if len(set(lk)) > 1:
        how["k_start"] = torch.from_numpy(ref.starts(lk)).cuda()
    for n in ("bias", "bounds", "q_pos", "k_pos"):
        how[n] = _cuda(c[n])
    q, k, v, do = (_cuda(c[n]) for n in ("q", "k", "v", "do"))
    o, lse = nlb.attention(q, k, v, **how)
    got = {"o": o, "lse": lse}
    if do is not None:
        got["dq"], got["dk"], got["dv"], dbias = nlb.attention_backward(do, q, k, v, o, lse, **how)
        if dbias is not None:
            got["dbias"] = dbias
    torch.cuda.synchronize()
    return got


def check(c, lq, lk, got, *, causal, dtype, scale=None, what=""):
    dim = c["q"].shape[2]
    want, far = ref.attention(_f64(c["q"]), _f64(c["k"]), _f64(c["v"]), lq, lk, u=HALF_STEP[dtype], causal=causal,
                              scale=dim ** -0.5 if scale is None else scale, bias=_f64(c["bias"]),
                              bounds=None if c["bounds"] is None else c["bounds"].numpy(), q_pos=_u32(c["q_pos"]),
                              k_pos=_u32(c["k_pos"]), do=_f64(c["do"]))
    for n, x in want.items():
        g = got[n].double().cpu().numpy()
        assert g.shape == x.shape, (what, n)
        fine = np.isfinite(x)
        assert np.array_equal(g[~fine], x[~fine]), (what, n, "infinities")
        off = np.abs(g[fine] - x[fine]) - far[n][fine]
        assert np.isfinite(g[fine]).all() and (off <= 0).all(), (
            what, n, f"{(off > 0).sum()} of {off.size} values too far, worst by {np.nanmax(off):.3g}")


LENGTHS = {
    "one": ([1], [1]),
    "odd": ([33, 1, 200, 0, 64], [40, 7, 200, 3, 20]),
    "no keys": ([5, 70, 3], [0, 70, 0]),
    "edges": ([127, 128, 129, 63, 64, 65], [127, 128, 129, 31, 300, 65]),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("mode", ["plain", "places", "times"])
@pytest.mark.parametrize("dim", [1, 8, 25, 32, 50, 64, 100, 128])
def test_packed_sequences(dtype, causal, mode, dim):
    for name, (lq, lk) in LENGTHS.items():
        heads, kv_heads = (4, 2) if dim != 25 else (3, 3)
        c = make(dtype, lq, lk, heads, kv_heads, dim, bias=mode != "plain", times=mode == "times", seed=dim)
        check(c, lq, lk, run(c, lq, lk, causal=causal), causal=causal, dtype=dtype, what=name)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mode", ["plain", "places", "times"])
@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 1), (4, 1, 25), (6, 2, 50), (7, 1, 64), (8, 8, 128), (2, 2, 33)])
def test_single_rows(dtype, mode, heads, kv_heads, dim):
    """Lists of one length (1, 10, 64, 700 slots) and of many, empty ones too."""
    for lk in ([1] * 3, [10] * 50, [64] * 5, [700] * 2, [2000, 0, 3, 255, 256, 257, 513], [0, 0]):
        lq = [1] * len(lk)
        c = make(dtype, lq, lk, heads, kv_heads, dim, bias=mode != "plain", times=mode == "times", seed=dim)
        for causal in (False, True):
            check(c, lq, lk, run(c, lq, lk, causal=causal, one=True), causal=causal, dtype=dtype, what=str(lk))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_fixed_lengths_without_starts(dtype):
    """q_start and k_start left out: every sequence has rows / batch rows."""
    import torch
    import paper_2402_01964_amd as nlb
    lq, lk = [50] * 6, [70] * 6
    c = make(dtype, lq, lk, 4, 4, 40, bias=True)
    o, lse = nlb.attention(c["q"].cuda(), c["k"].cuda(), c["v"].cuda(), batch=6, causal=True, bias=c["bias"].cuda(),
                           bounds=c["bounds"].cuda())
    torch.cuda.synchronize()
    check(c, lq, lk, {"o": o, "lse": lse}, causal=True, dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, -0.3, 1.7, 2.0 ** -20])
def test_scales(dtype, scale):
    """Zero, negative and other scales, with and without a bias."""
    for one, lq, lk in ((False, [40, 90], [50, 90]), (True, [1] * 9, [30] * 9), (True, [1], [700])):
        for mode in (False, True):
            c = make(dtype, lq, lk, 4, 2, 32, bias=mode, train=True, sharp=0.5)
            check(c, lq, lk, run(c, lq, lk, causal=True, one=one, scale=scale), causal=True, dtype=dtype, scale=scale)


def test_many_buckets():
    """64 buckets, so close that many share a cell of the search, and few."""
    import torch
    for bounds in (range(-20, 43), range(1000, 1063), [3 * i * i for i in range(63)], [0], []):
        for times in (False, True):
            for one, lq, lk in ((False, [150], [220]), (True, [1] * 4, [60] * 4)):
                c = make("f32", lq, lk, 2, 1, 16, bias=True, times=times, train=True)
                c["bounds"] = torch.tensor(list(bounds), dtype=torch.int32)
                c["bias"] = torch.randn(len(c["bounds"]) + 1, 2, generator=torch.Generator().manual_seed(1))
                if times:
                    c["k_pos"] = torch.where(c["k_pos"] >= 0, c["k_pos"] * 8, c["k_pos"])
                    c["q_pos"] = c["q_pos"] * 9
                check(c, lq, lk, run(c, lq, lk, causal=False, one=one), causal=False, dtype="f32", what=str(bounds))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gap", [3, 8])
def test_strided_rows(dtype, gap):
    for one, lq, lk in ((False, [40, 90], [50, 90]), (True, [1] * 9, [30] * 9)):
        c = make(dtype, lq, lk, 4, 2, 50, bias=True, times=True, gap=gap, train=True)
        assert not c["q"].is_contiguous()
        check(c, lq, lk, run(c, lq, lk, causal=False, one=one), causal=False, dtype=dtype)


def test_long_and_wide_groups():
    """Thousands of keys (many chunks, many tiles), sixteen heads on one."""
    for one, lq, lk in ((True, [1, 1], [9000, 40]), (False, [300], [5000])):
        c = make("bf16", lq, lk, 16, 1, 64, bias=True, train=True)
        check(c, lq, lk, run(c, lq, lk, causal=True, one=one), causal=True, dtype="bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("one", [False, True])
def test_closed_keys_may_hold_anything(dtype, one):
    """NaN and infinities in rows that no query may see leave no trace."""
    lq, lk = ([1] * 4, [100] * 4) if one else ([60, 5, 9], [60, 70, 80])
    c = make(dtype, lq, lk, 2, 2, 64, bias=True, times=True, closed=0.5, train=True)
    c["k_pos"][:lk[0]] = -1                                   # nothing open at all in the first
    shut = c["k_pos"] == -1
    clean = run(c, lq, lk, causal=False, one=one)
    for n, x in (("k", float("nan")), ("v", float("inf"))):
        c[n][shut] = x
    got = run(c, lq, lk, causal=False, one=one)
    for n in clean:
        assert (got[n] == clean[n]).all(), n
    assert (got["o"][:lq[0]] == 0).all() and (got["lse"][:lq[0]] == -float("inf")).all()
    check(c, lq, lk, got, causal=False, dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("one", [False, True])
@pytest.mark.parametrize("low", ["inf", "lowest"])
def test_bias_that_closes_a_bucket(dtype, one, low):
    """Minus infinity or the type's lowest value close a bucket, all of a
    row's keys too."""
    import torch
    lq, lk = ([1] * 3, [50, 9, 200]) if one else ([50, 9, 150], [50, 9, 200])
    for shut in ([0, 1], [5, 6, 7, 8], list(range(9))):
        c = make(dtype, lq, lk, 2, 1, 32, bias=True, train=True)
        c["bias"][shut] = -float("inf") if low == "inf" else torch.finfo(_dtype(dtype)).min
        check(c, lq, lk, run(c, lq, lk, causal=True, one=one), causal=True, dtype=dtype, what=str(shut))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mode", ["places", "times"])
@pytest.mark.parametrize("one", [False, True])
def test_bounds_that_do_not_increase(dtype, mode, one):
    """Equal bounds have empty buckets between them.  Falling ones leave open
    which bucket a gap is in, but it is one of them: with the same bias in all
    of them that is the one answer."""
    import torch
    lq, lk = ([1] * 5, [300, 1, 70, 0, 33]) if one else ([200, 33], [260, 70])
    c = make(dtype, lq, lk, 4, 2, 32, bias=True, times=mode == "times", train=True)
    c["bounds"] = torch.tensor([-5, 0, 0, 0, 4, 4, 30, 30], dtype=torch.int32)
    check(c, lq, lk, run(c, lq, lk, causal=False, one=one), causal=False, dtype=dtype, what="equal")
    c["bias"] = c["bias"][:1].expand(9, 4).contiguous()
    got = run(dict(c, bounds=torch.tensor([100, 30, 9, 4, 2, 1, 0, -5], dtype=torch.int32)), lq, lk, causal=False,
              one=one)
    assert torch.isfinite(got.pop("dbias")).all()
    want, far = ref.attention(*(_f64(c[n]) for n in "qkv"), lq, lk, u=HALF_STEP[dtype], causal=False,
                              scale=32 ** -0.5, bias=_f64(c["bias"]), bounds=BOUNDS, q_pos=_u32(c["q_pos"]),
                              k_pos=_u32(c["k_pos"]), do=_f64(c["do"]))
    for n, x in got.items():
        fine = np.isfinite(want[n])
        assert (np.abs(x.double().cpu().numpy()[fine] - want[n][fine]) <= far[n][fine]).all(), n


def test_gaps_of_unsigned_positions_are_clamped():
    """Positions over the whole unsigned range; gaps beyond int32."""
    import torch
    for one, lq, lk in ((True, [1] * 6, [6] * 6), (False, [6], [6])):
        c = make("f32", lq, lk, 2, 2, 16, bias=True, times=True, closed=0, train=True)
        at = torch.tensor([0, 1, 2**31 - 1, 2**31, 2**32 - 2, 2**32 - 3], dtype=torch.int64)
        c["q_pos"] = at.to(torch.uint32).view(torch.int32)
        c["k_pos"] = at.repeat(len(lk)).to(torch.uint32).view(torch.int32)
        c["bounds"] = torch.tensor([-2**31 + 1, -2**31 + 2, -3, 0, 1, 2, 2**31 - 2, 2**31 - 1], dtype=torch.int32)
        check(c, lq, lk, run(c, lq, lk, causal=False, one=one), causal=False, dtype="f32")


def test_rows_outside_the_sequences_stay():
    """Rows before the first and behind the last sequence are not written, and
    start values outside the rows are taken as the nearest end."""
    import torch
    import paper_2402_01964_amd as nlb
    c = make("bf16", [100], [100], 2, 2, 32)
    q, k, v = (c[n].cuda() for n in "qkv")
    o, lse = torch.full_like(q, 7.0), torch.full((100, 2), 7.0, device="cuda")
    st = torch.tensor([10, 40, 40, 90], dtype=torch.int32, device="cuda")
    nlb.attention(q, k, v, q_start=st, k_start=st, causal=True, out=o, lse=lse)
    torch.cuda.synchronize()
    for t in (o, lse):
        assert (t[:10] == 7).all() and (t[90:] == 7).all() and (t[10:90] != 7).any(-1).all()
    check({n: None if x is None else x[10:90] if n in "qkv" else x for n, x in c.items()}, [30, 0, 50], [30, 0, 50],
          {"o": o[10:90], "lse": lse[10:90]}, causal=True, dtype="bf16")
    wild = torch.tensor([-5, 40, 2**31 - 1, 50], dtype=torch.int32, device="cuda")
    o.fill_(7.0)
    nlb.attention(q, k, v, q_start=wild, k_start=wild, causal=True, out=o, lse=lse)
    torch.cuda.synchronize()
    check({n: None if x is None else x[:40] if n in "qkv" else x for n, x in c.items()}, [40], [40],
          {"o": o[:40], "lse": lse[:40]}, causal=True, dtype="bf16")


def test_graph_and_streams():
    """A captured call replayed with new inputs, on a stream of its own; two
    calls in flight on two streams, each with its working memory."""
    import torch
    import paper_2402_01964_amd as nlb
    lq, lk = [1, 1], [3000, 100]
    cs = [make("bf16", lq, lk, 4, 2, 64, bias=True, seed=s) for s in range(2)]
    st = torch.from_numpy(ref.starts(lk)).cuda()
    how = dict(batch=2, k_start=st, bounds=cs[0]["bounds"].cuda())
    ins = [[c[n].cuda() for n in ("q", "k", "v", "bias")] for c in cs]
    want = [nlb.attention(q, k, v, bias=b, **how)[0].clone() for q, k, v, b in ins]
    q, k, v, b = [x.clone() for x in ins[0]]
    work = torch.empty(nlb.attention_work(q, k, v, bias=b, **how), dtype=torch.uint8, device="cuda")
    assert work.numel() > 0
    o, lse = torch.empty_like(q), torch.empty((2, 4), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        nlb.attention(q, k, v, bias=b, out=o, lse=lse, work=work, **how)
    for turn in range(4):
        for x, y in zip((q, k, v, b), ins[turn % 2]):
            x.copy_(y)
        o.fill_(0)
        graph.replay()
        other = nlb.attention(*ins[1][:3], bias=ins[1][3], stream=side, **how)[0]
        torch.cuda.synchronize()
        assert torch.equal(o, want[turn % 2]) and torch.equal(other, want[1])


def test_same_bits_each_time():
    import torch
    for one, lq, lk in ((False, [300, 5], [400, 5]), (True, [1] * 300, [60] * 300)):
        c = make("bf16", lq, lk, 4, 2, 64, bias=True, times=True, train=True)
        a, b = (run(c, lq, lk, causal=True, one=one) for _ in range(2))
        for n in a:
            assert torch.equal(a[n], b[n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("mode", ["plain", "places", "times"])
@pytest.mark.parametrize("dim", [1, 8, 25, 32, 50, 64, 100, 128])
def test_gradients_of_packed_sequences(dtype, causal, mode, dim):
    for name, (lq, lk) in LENGTHS.items():
        heads, kv_heads = (4, 2) if dim != 25 else (3, 3)
        c = make(dtype, lq, lk, heads, kv_heads, dim, bias=mode != "plain", times=mode == "times", seed=dim,
                 train=True)
        check(c, lq, lk, run(c, lq, lk, causal=causal), causal=causal, dtype=dtype, what=name)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mode", ["plain", "places", "times"])
@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 1), (4, 1, 25), (6, 2, 50), (7, 1, 64), (8, 8, 128), (2, 2, 33)])
def test_gradients_of_single_rows(dtype, mode, heads, kv_heads, dim):
    """Lists that the single-row form takes, and lists too long for it."""
    for lk in ([1] * 3, [10] * 50, [64] * 5, [700] * 2, [600, 0, 3, 255, 256, 257, 1, 1, 1], [0, 0]):
        lq = [1] * len(lk)
        c = make(dtype, lq, lk, heads, kv_heads, dim, bias=mode != "plain", times=mode == "times", seed=dim,
                 train=True)
        check(c, lq, lk, run(c, lq, lk, causal=True, one=True), causal=True, dtype=dtype, what=str(lk))


def test_many_lists_keep_their_heads():
    """More lists than wavefronts in flight, an odd number of key/value heads."""
    for kv_heads, n in ((3, 5000), (5, 3000)):
        c = make("f32", [1] * n, [7] * n, kv_heads, kv_heads, 16, bias=True, times=True, train=True)
        check(c, [1] * n, [7] * n, run(c, [1] * n, [7] * n, causal=False, one=True), causal=False, dtype="f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv_heads", [1, 64, 256])
def test_most_heads_and_buckets(dtype, kv_heads):
    """256 heads, 64 buckets: the largest tables in LDS."""
    import torch
    for one, lq, lk in ((False, [40], [50]), (True, [1] * 3, [20] * 3), (True, [1], [600])):
        c = make(dtype, lq, lk, 256, kv_heads, 32 if dtype == "bf16" else 16, bias=True, times=True, train=True)
        c["bounds"] = torch.arange(-100, 215, 5, dtype=torch.int32)
        c["bias"] = torch.randn(64, 256, generator=torch.Generator().manual_seed(1)).to(_dtype(dtype))
        check(c, lq, lk, run(c, lq, lk, causal=False, one=one), causal=False, dtype=dtype, what=str(lk))


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 50)])
@pytest.mark.parametrize("mode", ["plain", "places", "times"])
def test_wide_and_narrow_workgroups(dtype, dim, mode):
    """Calls large enough for 128 rows a workgroup, ragged ends among them."""
    lq, lk = [300, 129, 1000, 1], [300, 700, 1000, 64]
    c = make(dtype, lq, lk, 16, 4, dim, bias=mode != "plain", times=mode == "times", train=True)
    for causal in (False, True):
        check(c, lq, lk, run(c, lq, lk, causal=causal), causal=causal, dtype=dtype)


def test_longer_and_shorter_than_a_tile_together():
    """Hundreds of sequences whose starts lie anywhere in the tiles' slots."""
    rng = np.random.default_rng(3)
    lq = [int(x) for x in rng.integers(0, 70, 300)]
    lk = [int(x) for x in rng.integers(0, 70, 300)]
    c = make("f32", lq, lk, 2, 2, 16, bias=True, train=True)
    check(c, lq, lk, run(c, lq, lk, causal=True), causal=True, dtype="f32")


def test_gradients_against_differences():
    """dq, dk, dv and dbias against differences of the forward pass itself."""
    import torch
    lq, lk = [5, 9], [8, 9]
    c = make("f32", lq, lk, 2, 1, 16, bias=True, train=True, sharp=1.0)
    got = run(c, lq, lk, causal=True)
    gen = torch.Generator().manual_seed(5)
    for n, grad in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("bias", "dbias")):
        step = torch.randn(c[n].shape, generator=gen)
        vals, h = [], 2.0 ** -7
        for sign in (1.0, -1.0):
            d = dict(c, do=None)
            d[n] = c[n] + sign * h * step
            vals.append((run(d, lq, lk, causal=True)["o"].cpu().double() * c["do"].double()).sum())
        slope = float(vals[0] - vals[1]) / (2 * h)
        want = float((got[grad].cpu().double() * step.double()).sum())
        # the forward pass is off by about 2^-24 of each of 448 terms of size 1 or so, over 2 h: 2^-24 448 64 = 2e-3;
        # the difference's own third-order term is h^2 times a third derivative of some tens: 6e-5 x 100
        assert abs(slope - want) <= 8e-3 + 1e-2 * abs(want) ** 0.5, (n, slope, want)


def test_gradients_into_a_joint_projection():
    """q, k, v as slices of one tensor, their gradients into slices of another."""
    import torch
    import paper_2402_01964_amd as nlb
    c = make("bf16", [70, 60], [70, 60], 4, 2, 64, bias=True, train=True)
    qkv = torch.cat([c["q"], c["k"], c["v"]], 1).cuda()
    grad = torch.full_like(qkv, 7.0)
    part = lambda t: (t[:, :4], t[:, 4:6], t[:, 6:])  # noqa: E731
    st = torch.from_numpy(ref.starts([70, 60])).cuda()
    how = dict(q_start=st, k_start=st, causal=True, bias=c["bias"].cuda(), bounds=c["bounds"].cuda())
    o, lse = nlb.attention(*part(qkv), **how)
    dq, dk, dv = part(grad)
    dbias = nlb.attention_backward(c["do"].cuda(), *part(qkv), o, lse, dq=dq, dk=dk, dv=dv, **how)[3]
    torch.cuda.synchronize()
    got = {"o": o, "lse": lse, "dq": grad[:, :4], "dk": grad[:, 4:6], "dv": grad[:, 6:], "dbias": dbias}
    check(c, [70, 60], [70, 60], got, causal=True, dtype="bf16")
    more = nlb.attention_backward(c["do"].cuda(), *part(qkv), o, lse, need_dbias=False, **how)
    torch.cuda.synchronize()
    assert more[3] is None
    check({**c}, [70, 60], [70, 60], {**got, "dq": more[0], "dk": more[1], "dv": more[2]}, causal=True, dtype="bf16")


def test_gradient_rows_outside_the_sequences_stay():
    import torch
    import paper_2402_01964_amd as nlb
    c = make("bf16", [100], [100], 2, 2, 32, train=True)
    q, k, v, do = (c[n].cuda() for n in ("q", "k", "v", "do"))
    st = torch.tensor([10, 40, 40, 90], dtype=torch.int32, device="cuda")
    kw = dict(q_start=st, k_start=st, causal=True)
    o, lse = nlb.attention(q, k, v, **kw)
    d = [torch.full_like(q, 7.0) for _ in range(3)]
    nlb.attention_backward(do, q, k, v, o, lse, dq=d[0], dk=d[1], dv=d[2], **kw)
    torch.cuda.synchronize()
    for t in d:
        assert (t[:10] == 7).all() and (t[90:] == 7).all() and (t[10:90] != 7).flatten(1).any(-1).all()


@pytest.mark.parametrize("one,dim", [(False, 64), (False, 128), (True, 64)])
def test_captured_training_step(one, dim):
    """Forward and backward captured with their working memory, replayed with
    new inputs, eager calls between (128 values: kernels with over 64 KiB of
    LDS)."""
    import torch
    import paper_2402_01964_amd as nlb
    lq, lk = ([1] * 40, [20] * 40) if one else ([100, 33], [100, 70]) if dim == 64 else ([700] * 6, [700] * 6)
    cs = [make("bf16", lq, lk, 4, 2, dim, bias=True, times=True, train=True, seed=s) for s in range(2)]
    how = dict(batch=len(lq), bounds=cs[0]["bounds"].cuda())
    if not one:
        how.update(q_start=torch.from_numpy(ref.starts(lq)).cuda(), k_start=torch.from_numpy(ref.starts(lk)).cuda())
    names = ("q", "k", "v", "do", "bias", "q_pos", "k_pos")

    def step(t):
        kw = dict(how, **{n: t[n] for n in names[4:]})
        o, lse = nlb.attention(t["q"], t["k"], t["v"], **kw)
        return (o, lse) + nlb.attention_backward(t["do"], t["q"], t["k"], t["v"], o, lse, **kw)
    ins = [{n: c[n].cuda() for n in names} for c in cs]
    want = [[x.clone() for x in step(t)] for t in ins]
    t = {n: x.clone() for n, x in ins[0].items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step(t)
    for turn in range(4):
        for n in names:
            t[n].copy_(ins[turn % 2][n])
        for x in got:
            x.fill_(0)
        graph.replay()
        other = step(ins[1])
        torch.cuda.synchronize()
        for a, b, x, y in zip(got, want[turn % 2], other, want[1]):
            assert torch.equal(a, b) and torch.equal(x, y)


def test_offsets_beyond_32_bits():
    """Rows so far apart that their byte offsets pass 2^32."""
    import torch
    import paper_2402_01964_amd as nlb
    n, far = 70, 50_000_000                                   # 70 rows x 100 MB
    c = make("bf16", [1, n - 1], [1, n - 1], 1, 1, 32)
    big = torch.empty(n * far + 64, dtype=torch.bfloat16, device="cuda")
    st = torch.tensor([0, 1, n], dtype=torch.int32, device="cuda")
    k = big.as_strided((n, 1, 32), (far, 32, 1), 0)
    k.copy_(c["k"])
    for q, starts in ((c["q"].cuda(), dict(q_start=st, k_start=st)), (c["q"][:1].cuda(), dict(batch=1))):
        o, lse = nlb.attention(q, k, k, **starts)
        torch.cuda.synchronize()
        lens = ([1, n - 1], [1, n - 1]) if len(q) > 1 else ([1], [n])
        check({**c, "q": q.cpu(), "v": c["k"]}, *lens, {"o": o, "lse": lse}, causal=False, dtype="bf16")
