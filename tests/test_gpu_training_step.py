"""A training step through a table's answers and the nodes' own histories:
neighbours' rows looked up by nlb_sample's ids, queries and keys normed and
rotated by its times, attention over the lists, a gated recurrence over each
node's answers in time, and back to the gradient of the whole table of rows;
against the same in 64 bits with torch's automatic gradients."""
import dataclasses

import numpy as np
import pytest

import synth
from tests.gpu_helpers import make_gpu_table, to_dev

pytestmark = pytest.mark.gpu

HEADS, WIDTH, EPS = 4, 64, 1e-5
SCALE = 8.0


def _turn64(x, pos, freq, w):
    import torch
    u = x * (x.square().mean(-1, keepdim=True) + EPS) ** -0.5 * w
    m = len(freq)
    a = (pos.double()[..., None] * freq)[..., None, :]
    lo, hi = u[..., :m], u[..., m:2 * m]
    return torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin(), u[..., 2 * m:]], -1)


def _step64(rows, w, nbr, node, ts, tq, lengths):
    import torch
    n, s = nbr.shape
    x = torch.where((nbr >= 0)[..., None], rows[nbr.clamp(min=0)] * SCALE, torch.zeros(()))
    own = rows[node] * SCALE
    v = x.view(n, s, HEADS, -1)
    q = _turn64(own.view(n, HEADS, -1), tq, w["freq"], w["wq"])
    k = _turn64(v, ts, w["freq"], w["wk"])
    t = (q[:, None] * k).sum(3) * (WIDTH // HEADS) ** -0.5
    open_ = ts != 0xFFFFFFFF
    t = torch.where(open_[..., None], t, torch.full_like(t, -1e300))
    p = torch.softmax(t, 1) * open_.any(1)[:, None, None]
    o = (p[..., None] * v).sum(1).reshape(n, WIDTH)
    z, out, at = torch.sigmoid(own + 1.0), [], 0
    for b, m in enumerate(lengths):
        h = w["h0"][b]
        for i in range(at, at + m):
            h = z[i] * h + (1 - z[i]) * o[i]
            out.append(h)
        at += m
    return torch.stack(out)


def test_rows_norm_rotation_attention_recurrence_and_back():
    import torch
    import paper_2402_01964_amd as nlb
    w = dataclasses.replace(synth.scaled(synth.workload(5), 3 * 2000, num_nodes=400), batch=2000)
    src, dst, t, neg = synth.host_links(w)
    table = make_gpu_table(w)
    table.insert(*(to_dev(x[:4000]) for x in (src, dst, t)))
    nodes = np.concatenate([src, dst, neg])[4000:4300].astype(np.int32)
    node, tq = to_dev(nodes), to_dev(np.full(300, int(t[4000]), np.uint32))
    got = table.sample(node, tq, want=("nbr", "ts"))
    n, s = got["nbr"].shape
    lengths = [100, 0, 150, 1, 49]
    start = torch.tensor(np.cumsum([0] + lengths), dtype=torch.int32, device="cuda")
    gen = torch.Generator().manual_seed(1)
    m = WIDTH // HEADS // 2
    p = {"rows": torch.randn(w.num_nodes, WIDTH, generator=gen) / SCALE,
         "wq": 1 + 0.1 * torch.randn(2 * m, generator=gen), "wk": 1 + 0.1 * torch.randn(2 * m, generator=gen),
         "h0": torch.randn(len(lengths), WIDTH, generator=gen)}
    freq = torch.from_numpy(10.0 ** (-9.0 * np.arange(m) / (m - 1))).float()
    dh = torch.randn(n, WIDTH, generator=gen)
    dev = {k: v.cuda() for k, v in p.items()}

    x = nlb.lookup(dev["rows"], got["nbr"], SCALE)
    own = nlb.lookup(dev["rows"], node, SCALE)
    v = x.view(n * s, HEADS, -1)
    turn = (own.view(n, HEADS, -1), v, freq.cuda(), tq, got["ts"].view(-1), dev["wq"], dev["wk"], EPS)
    q, k = nlb.norm_rotate(*turn)
    how = dict(batch=n, k_pos=got["ts"])
    o, lse = nlb.attention(q, k, v, **how)
    gate = own + 1.0
    h, last, states = nlb.gated_scan(o.view(n, WIDTH), gate, start=start, h0=dev["h0"])
    do, dgate, dh0 = nlb.gated_scan_backward(dh.cuda(), o.view(n, WIDTH), gate, states, start=start, h0=dev["h0"])
    dq, dk, dv, _ = nlb.attention_backward(do.view(n, HEADS, -1), q, k, v, o, lse, **how)
    down, dx, dwq, dwk = nlb.norm_rotate_backward(dq, dk, *turn)
    drows = nlb.lookup_backward((dx + dv).view(n, s, WIDTH), got["nbr"], w.num_nodes, SCALE) \
        + nlb.lookup_backward(down.view(n, WIDTH) + dgate, node, w.num_nodes, SCALE)
    torch.cuda.synchronize()
    assert table.status() == 0

    ts = torch.from_numpy(got["ts"].cpu().numpy().view(np.uint32).astype(np.int64))
    some = (ts != 0xFFFFFFFF).any(1)
    assert some.any() and not some.all() and not o[~some.cuda()].any()
    leaf = {name: v.double().requires_grad_() for name, v in p.items()}
    want = _step64(leaf["rows"], {**leaf, "freq": freq.double()}, got["nbr"].cpu().long(), torch.from_numpy(nodes).long(),
                   ts, torch.from_numpy(tq.cpu().numpy().view(np.uint32).astype(np.int64)), lengths)
    (want * dh.double()).sum().backward()
    # Each step is off by some 2^-24 of the magnitudes that it sums: 64 values of a row, 10 slots, up to 150 rows of a
    # history that forgets by a factor of 0.7 a row, 3300 places' gradients of 400 rows; angles of up to 2^28 by their
    # 2^-24.  Together below 300 steps of 2^-24: 2e-5 of the largest value of each result.
    for name, a, b in (("h", h, want), ("drows", drows, leaf["rows"].grad), ("dwq", dwq, leaf["wq"].grad),
                       ("dwk", dwk, leaf["wk"].grad), ("dh0", dh0, leaf["h0"].grad)):
        a, b = a.double().cpu(), b.detach()
        assert a.shape == b.shape and (a - b).abs().max() <= 2e-5 * b.abs().max(), (
            name, float((a - b).abs().max() / b.abs().max()))
