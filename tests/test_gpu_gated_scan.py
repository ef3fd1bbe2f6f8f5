"""The gated linear recurrence and its gradients on the GPU (nlb_gated_scan)
against 64 bits.

Bounds, with w = 2^-24 and u half a step of the rows' type (2^-8 bf16, w fp32):
a gate and its complement are off by 12 w of themselves (the exponential's two
words, its 2 w, the sum, the reciprocal and a product).  One step takes 13 w of
what it adds and 16 w of what it carries; with H the same recurrence of
magnitudes, H_t = z H_{t-1} + (1 - z) |x|, a state is off by
  E_t = z E_{t-1} + 16 w H_t,  and by 64 w H_t more
where maps of rows are joined (up to 32 joins, each 2 w of its terms).  So for
d (F, from D), and dx = y d is off by y F + 14 w |dx|, dg = z y d (h' - x) by
z y (F |h' - x| + D (E' + w |h' - x|)) + 30 w |dg|; results of the rows' type
are rounded once more, by u.  Below the smallest normal number, 2^-126, steps
are absolute: bf16's are 2^-133 there, and a rounding is off by half of one.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

W = 2.0 ** -24
HALF_STEP = {"bf16": 2.0 ** -8, "f32": W}
SENTINEL = 12345.0


def chain(z, b, first, into):
    """h_t = z_t h_{t-1} + b_t within sequences, from `into`."""
    h = np.empty_like(b)
    for lo, hi, h0 in zip(first[:-1], first[1:], into):
        for t in range(lo, hi):
            h0 = z[t] * h0 + b[t]
            h[t] = h0
    return h


def shifted(x, first, into, by=1):
    """x of the row before (by = -1: behind), `into` at the sequences' edges."""
    out = np.empty_like(x)
    for lo, hi, v in zip(first[:-1], first[1:], into):
        if lo == hi:
            continue
        if by == 1:
            out[lo], out[lo + 1:hi] = v, x[lo:hi - 1]
        else:
            out[hi - 1], out[lo:hi - 1] = v, x[lo + 1:hi]
    return out


def want_of(x, g, first, h0, dh, dlast, u):
    """Results and bounds; rows are those of the sequences, from row 0 on."""
    g = np.clip(g, -80, 80)       # gates beyond 80 count as 80, by the definition (a difference of e^-80 = 1.8e-35)
    with np.errstate(over="ignore"):
        z, y = 1 / (1 + np.exp(-g)), 1 / (1 + np.exp(g))
    n = len(first) - 1
    zero = np.zeros((n, x.shape[1]))
    h0 = zero if h0 is None else h0
    dlast = zero if dlast is None else dlast
    flip = [first[-1] - f for f in first[::-1]]

    def back(b, into):            # d_t = b_t + z_{t+1} d_{t+1}
        zn = shifted(z, first, zero, -1)
        b = b.copy()
        for lo, hi, v in zip(first[:-1], first[1:], into):
            if lo < hi:
                b[hi - 1] += v
        return chain(zn[::-1], b[::-1], flip, zero)[::-1]

    h = chain(z, y * x, first, h0)
    big = chain(z, y * np.abs(x), first, np.abs(h0))
    e = chain(z, 16 * W * big, first, zero)
    far = e + 64 * W * big
    d = back(dh, dlast)
    dbig = back(np.abs(dh), np.abs(dlast))
    f = back(16 * W * dbig, zero) + 64 * W * dbig
    hp, ep = shifted(h, first, h0), shifted(far, first, zero)
    dx, gap = y * d, hp - x
    dg = z * y * d * gap
    # the gap's own rounding of its two terms is within 2 w of their magnitudes
    out = {"h": (h, far + u * np.abs(h)),
           "dx": (dx, y * f + 14 * W * np.abs(dx) + u * np.abs(dx)),
           "dg": (dg, z * y * (f * np.abs(gap) + dbig * (ep + W * np.abs(gap))) + 30 * W * np.abs(dg)
                  + u * np.abs(dg))}
    last, lfar, dh0, dfar = h0.copy(), zero.copy(), dlast.copy(), zero.copy()
    for b, (lo, hi) in enumerate(zip(first[:-1], first[1:])):
        if lo < hi:
            last[b], lfar[b] = h[hi - 1], far[hi - 1]
            dh0[b], dfar[b] = z[lo] * d[lo], z[lo] * f[lo] + 14 * W * z[lo] * dbig[lo]
    out["last"], out["dh0"] = (last, lfar), (dh0, dfar)
    return out


def case(dtype, lengths, width, *, before=0, behind=0, starts=True, first=True, dlast=True, gap=0, seed=0, bias=1.0,
         spread=2.0):
    import torch
    t = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    gen = torch.Generator().manual_seed(seed)
    rows, n = before + sum(lengths) + behind, len(lengths)

    def rand(scale=1.0, shift=0.0):
        return (scale * torch.randn(rows, width + gap, generator=gen) + shift).to(t)[:, :width]

    x, g, dh = rand(), rand(spread, bias), rand()
    start = torch.tensor(np.cumsum([before] + list(lengths)), dtype=torch.int32) if starts else None
    h0 = torch.randn(n, width, generator=gen) if first else None
    dl = torch.randn(n, width, generator=gen) if dlast else None
    return dict(dtype=dtype, lengths=lengths, before=before, x=x, g=g, dh=dh, start=start, h0=h0, dlast=dl, n=n)


def cuda(t, gap=0):
    """A copy on the GPU with the same strides."""
    import torch
    if t is None:
        return None
    out = torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda")
    out.copy_(t)
    return out


def run(c, **more):
    import torch
    import paper_2402_01964_amd as nlb
    x, g, dh = cuda(c["x"]), cuda(c["g"]), cuda(c["dh"])
    how = dict(batch=c["n"], start=cuda(c["start"]), h0=cuda(c["h0"]))
    new = lambda: torch.full_like(x, SENTINEL)  # noqa: E731
    h, last, states = nlb.gated_scan(x, g, out=new(), **how, **more)
    dx, dg, dh0 = nlb.gated_scan_backward(dh, x, g, states, dlast=cuda(c["dlast"]), dx=new(), dg=new(), **how, **more)
    torch.cuda.synchronize()
    return {"h": h, "last": last, "dx": dx, "dg": dg, "dh0": dh0}


def check(c):
    got = run(c)
    lo, hi = c["before"], c["before"] + sum(c["lengths"])
    f64 = lambda t: None if t is None else t.double().numpy()  # noqa: E731
    first = [0] + list(np.cumsum(c["lengths"]))
    want = want_of(f64(c["x"])[lo:hi], f64(c["g"])[lo:hi], first, f64(c["h0"]), f64(c["dh"])[lo:hi], f64(c["dlast"]),
                   HALF_STEP[c["dtype"]])
    for name, (v, far) in want.items():
        if got[name] is None:
            assert name == "dh0" and c["h0"] is None
            continue
        have = got[name].double().cpu().numpy()
        if name in ("h", "dx", "dg"):
            assert (have[:lo] == np.float64(got[name].new_tensor(SENTINEL).item())).all()
            assert (have[hi:] == np.float64(got[name].new_tensor(SENTINEL).item())).all()
            have = have[lo:hi]
        off = np.abs(have - v) - (far + 2.0 ** -134)
        assert np.isfinite(off).all() and (off <= 0).all(), (
            c["dtype"], have.shape, name, float(off.max()), np.argwhere(off == off.max())[0])


DTYPES = pytest.mark.parametrize("dtype", ["bf16", "f32"])


@DTYPES
@pytest.mark.parametrize("width", [1, 2, 7, 8, 9, 15, 16, 17, 31, 33, 63, 64, 65, 100, 127, 128, 129, 200, 257])
def test_widths(dtype, width):
    check(case(dtype, [5, 1, 40, 0, 130, 3], width, before=3, behind=2, seed=width))


@DTYPES
@pytest.mark.parametrize("lengths", [[1], [2], [15], [16], [17], [63], [64], [65], [127], [128], [129], [1000], [2500],
                                     [1] * 300, [0, 0, 7, 0], [0], [0, 0], [128, 128, 1], [64, 0, 0, 64, 63, 65],
                                     [300, 700, 0, 5, 1500]], ids=lambda v: f"{len(v)}x{max(v)}")
@pytest.mark.parametrize("width", [100, 10])
def test_lengths(dtype, lengths, width):
    check(case(dtype, lengths, width, seed=len(lengths)))


@DTYPES
@pytest.mark.parametrize("length", [1, 2, 3, 16, 50, 64, 128, 333])
@pytest.mark.parametrize("width", [24, 130])
def test_equal_lengths_without_starts(dtype, length, width):
    check(case(dtype, [length] * 9, width, starts=False, seed=length))


@DTYPES
def test_without_first_and_last_states(dtype):
    check(case(dtype, [40, 300, 0, 2], 70, first=False, dlast=False))
    check(case(dtype, [40, 300, 0, 2], 70, first=True, dlast=False))
    check(case(dtype, [40, 300, 0, 2], 70, first=False, dlast=True))


@DTYPES
@pytest.mark.parametrize("gap", [1, 2, 3, 8])
def test_strides(dtype, gap):
    for width in (5, 64, 131):
        check(case(dtype, [70, 9, 200], width, gap=gap))


@DTYPES
@pytest.mark.parametrize("lengths", [[3000], [900, 2100], [1] * 1500 + [1500]], ids=lambda v: f"{len(v)}x{max(v)}")
def test_chunks_of_several_tiles(dtype, lengths):
    """So wide that a workgroup's chunk is more than one tile."""
    check(case(dtype, lengths, 16_384 if dtype == "bf16" else 8192))


@DTYPES
def test_many_chunks(dtype):
    """More tiles than workgroups, and narrow rows."""
    check(case(dtype, [50_000, 1, 149_999], 3, behind=7))
    check(case(dtype, [9000, 200, 40_000] + [13] * 300, 65))


@DTYPES
def test_many_empty_sequences_and_single_rows(dtype):
    check(case(dtype, [0] * 700 + [5] + [0] * 1300 + [200] + [0] * 70 + [1] * 200, 20))


@DTYPES
def test_gates_of_all_sizes(dtype):
    check(case(dtype, [400], 64, spread=30.0, bias=0.0))
    check(case(dtype, [2000], 64, spread=1.0, bias=9.0))       # long memories
    check(case(dtype, [400], 64, spread=1.0, bias=-9.0))


def test_gates_beyond_the_exponential():
    """Infinite and huge gates: held and replaced states."""
    import torch
    import paper_2402_01964_amd as nlb
    g = torch.tensor([[float("inf")], [-float("inf")], [3e38], [-3e38], [90.0]], device="cuda")
    x = torch.tensor([[1.0], [2.0], [3.0], [4.0], [5.0]], device="cuda")
    h0 = torch.tensor([[7.0]], device="cuda")
    h, last, _ = nlb.gated_scan(x, g, h0=h0)
    assert h[:, 0].tolist() == [7.0, 2.0, 2.0, 4.0, 4.0] and last.item() == 4.0


def test_a_sequence_keeps_its_nan():
    import torch
    import paper_2402_01964_amd as nlb
    lengths = [100, 300, 1, 50, 700]
    c = case("f32", lengths, 40)
    clean = run(c)
    edges = np.cumsum([0] + lengths)
    for bad in (1, 3):
        c["x"][edges[bad] + 2, 5], c["x"][edges[bad] + 3, 7] = float("nan"), float("inf")
        c["dh"][edges[bad + 1] - 1, 9] = float("nan")
        c["g"][edges[bad] + 1, 11] = float("nan")
    got = run(c)
    for b in (0, 2, 4):
        rows = slice(int(edges[b]), int(edges[b + 1]))
        for name in ("h", "dx", "dg"):
            assert torch.equal(got[name][rows], clean[name][rows]), (b, name)
        assert torch.equal(got["last"][b], clean["last"][b]) and torch.equal(got["dh0"][b], clean["dh0"][b])
    assert got["h"][edges[1] + 2:edges[2], 5].isnan().all()


def test_against_differences():
    """Gradients against central differences of the forward pass (fp32; a step
    of 2^-6 leaves a truncation of some 2^-12 / 6 of third derivatives below
    one and a rounding of 2^-24 |sum| / 2^-6)."""
    import torch
    import paper_2402_01964_amd as nlb
    c = case("f32", [3, 0, 20, 9], 6, bias=0.0, spread=1.0)
    x, g, dh, h0, dl = (cuda(c[k]) for k in ("x", "g", "dh", "h0", "dlast"))
    how = dict(start=cuda(c["start"]))

    def loss(x, g, h0):
        h, last, _ = nlb.gated_scan(x, g, h0=h0, **how)
        return float((h.double() * dh.double()).sum() + (last.double() * dl.double()).sum())
    _, _, states = nlb.gated_scan(x, g, h0=h0, **how)
    grads = nlb.gated_scan_backward(dh, x, g, states, dlast=dl, h0=h0, **how)
    step = 2.0 ** -6
    for k, (t, d) in enumerate(zip((x, g, h0), grads)):
        for at in [(0, 0), (1, 3), (t.shape[0] - 1, 5)]:
            args = [x, g, h0]
            both = []
            for s in (step, -step):
                args[k] = t.clone()
                args[k][at] += s
                both.append(loss(*args))
            assert abs((both[0] - both[1]) / (2 * step) - float(d[at])) < 1e-3, (k, at)


def test_one_event_at_a_time_is_the_scan():
    """States moved on in place, one row a sequence, as the whole scan has them."""
    import torch
    import paper_2402_01964_amd as nlb
    torch.manual_seed(0)
    n, steps, width = 37, 12, 100
    x, g = torch.randn(n, steps, width, device="cuda"), torch.randn(n, steps, width, device="cuda")
    state = torch.randn(n, width, device="cuda")
    whole, last, _ = nlb.gated_scan(x.view(-1, width), g.view(-1, width), batch=n, h0=state)
    for t in range(steps):
        h, now, states = nlb.gated_scan(x[:, t], g[:, t], batch=n, h0=state, last=state, need_states=False)
        assert now is state and states is None
        # each step's roundings, carried on: 12 steps of at most 8 roundings of values below 8
        assert (h - whole.view(n, steps, width)[:, t]).abs().max() < 12 * 8 * 8 * W
    assert (state - last).abs().max() < 12 * 8 * 8 * W


def test_in_place_streams_and_same_bits():
    import torch
    import paper_2402_01964_amd as nlb
    c = case("bf16", [400, 0, 3000, 17], 200)
    a, b = run(c), run(c)
    assert all(torch.equal(a[k], b[k]) for k in a)
    x, g, dh = (cuda(c[k]) for k in ("x", "g", "dh"))
    how = dict(start=cuda(c["start"]), h0=cuda(c["h0"]))
    n = nlb.gated_scan_work(x, g, **how)
    assert n > 0
    work = torch.empty(n + 16, dtype=torch.uint8, device="cuda")
    _, _, states = nlb.gated_scan(x, g, work=work, **how)
    dx, dg, dh0 = nlb.gated_scan_backward(dh, x, g, states, dlast=cuda(c["dlast"]), dx=dh, work=work, **how)
    assert dx is dh and torch.equal(dx, a["dx"]) and torch.equal(dg, a["dg"]) and torch.equal(dh0, a["dh0"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    h, last, _ = nlb.gated_scan(x, g, out=x, stream=side, **how)
    side.synchronize()
    assert h is x and torch.equal(h, a["h"]) and torch.equal(last, a["last"])


def test_captured_step():
    """Captured with lengths that change between replays, and eager calls
    between them."""
    import torch
    import paper_2402_01964_amd as nlb
    width, rows = 130, 1500
    torch.manual_seed(1)
    x, g, dh = (torch.randn(rows, width, device="cuda", dtype=torch.bfloat16) for _ in range(3))
    h0, dl = torch.randn(4, width, device="cuda"), torch.randn(4, width, device="cuda")
    starts = [torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, 10, 600, 600, 1500], [5, 700, 701, 900, 902])]

    def step(start):
        out = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(x)
        h, last, states = nlb.gated_scan(x, g, start=start, h0=h0, out=out[0])
        return (h, last) + nlb.gated_scan_backward(dh, x, g, states, dlast=dl, start=start, h0=h0, dx=out[1], dg=out[2])
    want = [[t.clone() for t in step(s)] for s in starts]
    start = starts[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step(start)
    for turn in range(4):
        start.copy_(starts[turn % 2])
        graph.replay()
        other = step(starts[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[turn % 2]))
        assert all(torch.equal(a, b) for a, b in zip(other, want[1]))


def test_starts_outside_the_rows():
    """They count as the nearest end: nothing is read or written there."""
    import torch
    import paper_2402_01964_amd as nlb
    torch.manual_seed(2)
    x, g = torch.randn(200, 33, device="cuda"), torch.randn(200, 33, device="cuda")
    ok = torch.tensor([0, 0, 150, 200, 200], dtype=torch.int32, device="cuda")
    far = torch.tensor([-2**31, -5, 150, 10_000, 2**31 - 1], dtype=torch.int32, device="cuda")
    a, b = nlb.gated_scan(x, g, start=ok), nlb.gated_scan(x, g, start=far)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_no_rows():
    import torch
    import paper_2402_01964_amd as nlb
    x = torch.empty(0, 12, device="cuda")
    h0, dl = torch.randn(5, 12, device="cuda"), torch.randn(5, 12, device="cuda")
    for start in (None, torch.zeros(6, dtype=torch.int32, device="cuda")):
        h, last, states = nlb.gated_scan(x, x, batch=5, start=start, h0=h0)
        assert h.shape == (0, 12) and torch.equal(last, h0)
        dx, dg, dh0 = nlb.gated_scan_backward(x, x, x, states, dlast=dl, batch=5, start=start, h0=h0)
        assert torch.equal(dh0, dl)
