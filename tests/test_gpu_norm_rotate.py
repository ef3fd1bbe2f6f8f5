"""Norm and rotation of queries and keys and their gradients on the GPU
(nlb_norm_rotate) against 64 bits.

Bounds, with w = 2^-24 and u half a step of the rows' type (2^-8 bf16, w fp32):
the sum of d squares is off by d w of itself, its reciprocal root by er = (d / 2
+ 4) w (the instruction's 2 w among them); a sine or cosine by es = 4 w + |a|
2^-51 absolutely (the angle's rounding to fp32 after its reduction, the series,
and 64-bit steps of |a|).  A rotated value is off by its two terms' (er + es + 4
w), a rotated gradient by its two's (es + 2 w); sums over d by d w of their
magnitudes; what is of the rows' type by u more.  dw sums up to 4096 rows' terms
in fp32 one after the other, then in fp64.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

W = 2.0 ** -24
HALF_STEP = {"bf16": 2.0 ** -8, "f32": W}


def want_of(x, pos, freq, w, eps, dy, u):
    """x, dy [rows, heads, dim] float64, pos int64 (uint32 values)."""
    n, h, d = x.shape
    m = len(freq)
    there = (pos != 0xFFFFFFFF)[:, None, None]
    x = np.where(there, x, 0.0)
    dy = np.where(there, dy, 0.0)
    w = np.ones(d) if w is None else w
    r = ((x * x).mean(2, keepdims=True) + eps) ** -0.5
    er = (d / 2 + 4) * W
    a = pos[:, None].astype(np.float64) * freq               # |a| 2^-53 off, within es
    es = np.zeros((n, 1, d))
    es[:, 0, :m] = es[:, 0, m:2 * m] = 4 * W + np.abs(a) * 2.0 ** -51
    cos, sin = np.cos(a)[:, None], np.sin(a)[:, None]

    def turn(v, sign):
        lo, hi = v[..., :m], v[..., m:2 * m]
        return np.concatenate([lo * cos - sign * hi * sin, hi * cos + sign * lo * sin, v[..., 2 * m:]], 2)

    def both(v):                                              # magnitudes of the two terms
        s = np.abs(v[..., :m]) + np.abs(v[..., m:2 * m])
        return np.concatenate([s, s, np.abs(v[..., 2 * m:])], 2)

    v = x * r * w
    y = turn(v, 1)
    out = {"y": (y, both(v) * (er + es + 4 * W) + u * np.abs(y))}
    du = turn(dy, -1)
    e_du = both(dy) * (es + 2 * W)
    xh = x * r
    terms = np.abs(du * xh)
    dw = (du * xh).sum((0, 1))
    out["dw"] = (dw, (e_du * np.abs(xh)).sum((0, 1)) + (er + 2 * W + min(n * h, 4096) * W) * terms.sum((0, 1))
                 + W * np.abs(dw))
    g, e_g = du * w, e_du * np.abs(w) + W * np.abs(du * w)
    s = (g * x).mean(2, keepdims=True) * r * r
    e_s = ((e_g * np.abs(x)).mean(2, keepdims=True) + (d + 4) * W * np.abs(g * x).mean(2, keepdims=True)) * r * r \
        + np.abs(s) * (2 * er + 4 * W)
    dx = r * (g - x * s)
    e_dx = r * (e_g + np.abs(x) * e_s + 2 * W * (np.abs(g) + np.abs(x * s))) + np.abs(dx) * (er + W)
    out["dx"] = (dx, e_dx + u * np.abs(dx))
    return out


def case(dtype, q_rows, k_rows, heads, kv_heads, dim, m, *, fill=1.0, weights=True, joint=False, gap=0, seed=0, top=2**28,
         scale=1.0):
    import torch
    t = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    gen = torch.Generator().manual_seed(seed)
    rand = lambda *s: (scale * torch.randn(*s, generator=gen)).to(t)  # noqa: E731

    def pair():
        if joint:
            both = rand(q_rows, heads + kv_heads + 1, dim + gap)[..., :dim]
            return both[:, :heads], both[:, heads:heads + kv_heads]
        return rand(q_rows, heads, dim + gap)[..., :dim], rand(k_rows, kv_heads, dim + gap)[..., :dim]

    q, k = pair()
    dq, dk = pair()
    freq = torch.from_numpy(10.0 ** (-9.0 * np.arange(m) / max(1, m - 1))).float()
    q_pos, k_pos = (torch.randint(0, top, (n,), generator=gen) for n in (q.shape[0], k.shape[0]))
    for p in (q_pos, k_pos):
        p[torch.rand(len(p), generator=gen) >= fill] = 0xFFFFFFFF
    wq, wk = (1 + 0.3 * torch.randn(dim, generator=gen) if weights else None for _ in range(2))
    return dict(dtype=dtype, q=q, k=k, dq=dq, dk=dk, freq=freq, q_pos=q_pos, k_pos=k_pos, wq=wq, wk=wk, eps=1e-5)


def cuda(t):
    import torch
    if t is None:
        return None
    if t.dtype == torch.int64:                                # positions as the words they are
        return torch.from_numpy(t.numpy().astype(np.uint32).view(np.int32)).cuda()
    out = torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda")
    return out.copy_(t)


def run(c, stream=None):
    import torch
    import paper_2402_01964_amd as nlb
    args = [cuda(c["q"]), cuda(c["k"]), cuda(c["freq"]) if len(c["freq"]) else None, cuda(c["q_pos"]), cuda(c["k_pos"]),
            cuda(c["wq"]), cuda(c["wk"]), c["eps"]]
    got = {}
    got["q"], got["k"] = nlb.norm_rotate(*args)
    got["dq"], got["dk"], got["dwq"], got["dwk"] = nlb.norm_rotate_backward(cuda(c["dq"]), cuda(c["dk"]), *args)
    torch.cuda.synchronize()
    return got


def check(c):
    got = run(c)
    f64 = lambda t: None if t is None else t.double().numpy()  # noqa: E731
    for side in "qk":
        want = want_of(f64(c[side]), c[side + "_pos"].numpy(), f64(c["freq"]), f64(c["w" + side]), c["eps"],
                       f64(c["d" + side]), HALF_STEP[c["dtype"]])
        for name, key in (("y", side), ("dx", "d" + side), ("dw", "dw" + side)):
            v, far = want[name]
            off = np.abs(got[key].double().cpu().numpy() - v) - far
            assert off.size == 0 or (np.isfinite(off).all() and (off <= 0).all()), (
                c["dtype"], c[side].shape, key, float(off.max()), np.argwhere(off == off.max())[0])


DTYPES = pytest.mark.parametrize("dtype", ["bf16", "f32"])


@DTYPES
@pytest.mark.parametrize("dim", [1, 2, 3, 4, 5, 8, 15, 16, 25, 31, 32, 33, 48, 50, 63, 64, 65, 96, 100, 127, 128])
def test_dims_and_parts_that_turn(dtype, dim):
    for m in sorted({0, dim // 4, dim // 2}):
        check(case(dtype, 9, 13, 3, 2, dim, m, seed=dim, fill=0.8))


@DTYPES
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (2, 1), (3, 3), (16, 4), (32, 8), (256, 1), (7, 256)])
def test_heads(dtype, heads, kv_heads):
    check(case(dtype, 5, 7, heads, kv_heads, 64, 32))
    check(case(dtype, 1, 1, heads, kv_heads, 50, 25))


@DTYPES
def test_many_rows(dtype):
    check(case(dtype, 3000, 9000, 4, 2, 64, 32, fill=0.7))
    check(case(dtype, 40_000, 1, 1, 1, 8, 4))
    check(case(dtype, 2, 30_000, 2, 2, 25, 12, fill=0.3))


@DTYPES
@pytest.mark.parametrize("gap", [0, 1, 3, 8])
def test_slices_of_a_projection(dtype, gap):
    for dim, m in ((64, 32), (64, 16), (50, 25), (128, 64)):
        check(case(dtype, 70, 70, 6, 2, dim, m, joint=True, gap=gap))


@DTYPES
def test_without_weights_small_and_large_values(dtype):
    check(case(dtype, 33, 20, 2, 2, 100, 50, weights=False))
    check(case(dtype, 33, 20, 2, 2, 64, 32, scale=1e-4))
    check(case(dtype, 33, 20, 2, 2, 64, 32, scale=1e8))


@DTYPES
def test_positions_of_all_sizes(dtype):
    for top in (1, 2, 1000, 2**32 - 1):
        check(case(dtype, 64, 64, 2, 1, 32, 16, top=top))


def test_a_row_of_zeros():
    import torch
    import paper_2402_01964_amd as nlb
    q = torch.zeros(3, 2, 16, device="cuda")
    pos = torch.arange(3, dtype=torch.int32, device="cuda")
    freq = torch.ones(8, device="cuda")
    y, none = nlb.norm_rotate(q, None, freq, pos, None)
    assert none is None and not y.any()
    dq, dk, dwq, dwk = nlb.norm_rotate_backward(torch.ones_like(q), None, q, None, freq, pos, None)
    assert dk is None and dwk is None and not dwq.any() and dq.isfinite().all()


@DTYPES
def test_what_empty_slots_hold_goes_nowhere(dtype):
    import torch
    c = case(dtype, 50, 80, 2, 2, 64, 32, fill=0.5)
    clean = run(c)
    for side in "qk":
        empty = c[side + "_pos"] == 0xFFFFFFFF
        assert empty.any()
        c[side][empty], c["d" + side][empty] = float("nan"), float("inf")
    got = run(c)
    assert all(torch.equal(clean[k], got[k]) for k in clean)
    assert not got["k"][(c["k_pos"] == 0xFFFFFFFF).cuda()].any()


def test_scores_depend_on_gaps_alone():
    """Queries and keys moved on by the same time: the same products.  Values of
    norm sqrt(64): a product of 64 terms, each off by some 2 (er + es) 2 = 150 w
    and |a| 2^-50 (|a| below 2^20 here): below 64 * 4 * 150 w = 2.3e-3."""
    import torch
    import paper_2402_01964_amd as nlb
    torch.manual_seed(0)
    q, k = torch.randn(40, 1, 64, device="cuda"), torch.randn(40, 1, 64, device="cuda")
    freq = 10.0 ** (-9.0 * torch.arange(32, device="cuda", dtype=torch.float64) / 31)
    freq = (freq.float() * 2**12).round() / 2**12             # exact multiples: the same angles in 64 bits
    pos = torch.randint(0, 2**19, (40,), dtype=torch.int32, device="cuda")

    def scores(by):
        a, b = nlb.norm_rotate(q, k, freq, pos + by, pos.flip(0) + by)
        return a[:, 0] @ b[:, 0].T
    assert (scores(0) - scores(2**18 + 77)).abs().max() < 2.3e-3


def test_against_differences():
    """As the formulas', against central differences of the forward pass: a step
    of 2^-7 leaves some 2^-14 of third derivatives of order 10, and a rounding
    of 2^-24 * 50 / 2^-7."""
    import torch
    import paper_2402_01964_amd as nlb
    c = case("f32", 4, 3, 2, 1, 10, 4)
    q, k, freq, q_pos, k_pos, wq, wk = (cuda(c[n]) for n in ("q", "k", "freq", "q_pos", "k_pos", "wq", "wk"))
    dq, dk = cuda(c["dq"]), cuda(c["dk"])

    def loss(q, k, wq, wk):
        a, b = nlb.norm_rotate(q, k, freq, q_pos, k_pos, wq, wk)
        return float((a.double() * dq.double()).sum() + (b.double() * dk.double()).sum())
    grads = nlb.norm_rotate_backward(dq, dk, q, k, freq, q_pos, k_pos, wq, wk)
    step = 2.0 ** -7
    for n, d in enumerate(grads):
        t = (q, k, wq, wk)[n]
        for at in {(0,) * t.dim(), tuple(s - 1 for s in t.shape)}:
            args, both = [q, k, wq, wk], []
            for s in (step, -step):
                args[n] = t.clone()
                args[n][at] += s
                both.append(loss(*args))
            assert abs((both[0] - both[1]) / (2 * step) - float(d[at])) < 2e-3, (n, at)


def test_in_place_streams_and_no_rows():
    import torch
    import paper_2402_01964_amd as nlb
    c = case("bf16", 300, 200, 4, 2, 128, 64, joint=False)
    want, again = run(c), run(c)
    assert all(torch.equal(want[k], again[k]) for k in want)
    args = [cuda(c[n]) for n in ("q", "k", "freq", "q_pos", "k_pos", "wq", "wk")]
    dq, dk = cuda(c["dq"]), cuda(c["dk"])
    got = nlb.norm_rotate_backward(dq, dk, *args, dq=dq, dk=dk)
    assert got[0] is dq and all(torch.equal(a, want[k]) for a, k in zip(got, ("dq", "dk", "dwq", "dwk")))
    got = nlb.norm_rotate_backward(cuda(c["dq"]), cuda(c["dk"]), *args, need_dw=False)
    assert got[2] is None and got[3] is None and torch.equal(got[0], want["dq"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    q, k = nlb.norm_rotate(*args, q_out=args[0], k_out=args[1], stream=side)
    side.synchronize()
    assert q is args[0] and torch.equal(q, want["q"]) and torch.equal(k, want["k"])
    e, p = torch.empty(0, 2, 16, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    freq = torch.ones(8, device="cuda")
    q, k = nlb.norm_rotate(e, e, freq, p, p)
    assert q.shape == k.shape == e.shape
    dq, dk, dwq, dwk = nlb.norm_rotate_backward(e, e, e, e, freq, p, p)
    assert not dwq.any() and not dwk.any()


def test_captured_step():
    import torch
    import paper_2402_01964_amd as nlb
    c = case("f32", 500, 700, 2, 2, 50, 25, fill=0.8)
    args = [cuda(c[n]) for n in ("q", "k", "freq", "q_pos", "k_pos", "wq", "wk")]
    dq, dk = cuda(c["dq"]), cuda(c["dk"])
    turns = [args[4].clone(), args[4].flip(0).clone()]

    def step(k_pos):
        a = args[:4] + [k_pos] + args[5:]
        return nlb.norm_rotate(*a) + nlb.norm_rotate_backward(dq, dk, *a)
    want = [[t.clone() for t in step(p)] for p in turns]
    k_pos = turns[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step(k_pos)
    for turn in range(4):
        k_pos.copy_(turns[turn % 2])
        for t in got:
            t.fill_(0)
        graph.replay()
        other = step(turns[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[turn % 2]))
        assert all(torch.equal(a, b) for a, b in zip(other, want[1]))
