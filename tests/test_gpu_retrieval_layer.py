"""An attention layer over a table's own answers, forward and backward: what
nlb_sample returns goes in as it is (neighbours' rows as keys and values, ts
and tq as positions, empty slots as closed keys), layer norm before and after,
against the same in 64 bits with torch's automatic gradients."""
import dataclasses

import numpy as np
import pytest

import synth
from tests.gpu_helpers import feat_to_dev, make_gpu_table, to_dev

pytestmark = pytest.mark.gpu

BOUNDS = [1, 10, 100, 1000, 10_000]
HEADS, WIDTH = 4, 128


def _layer64(x_self, x_nbr, ts, tq, w, heads):
    """The layer in 64 bits; leaves require gradients."""
    import torch
    n, s, d = x_nbr.shape
    norm = lambda x, g, b: torch.nn.functional.layer_norm(x, (d,), g, b, 1e-5)  # noqa: E731
    a = norm(x_nbr, w["g1"], w["b1"])
    q = norm(x_self, w["g1"], w["b1"]).view(n, heads, d // heads)
    k = a.view(n, s, heads, d // heads)
    t = (q[:, None] * k).sum(3) * (d // heads) ** -0.5
    gap = tq[:, None] - ts
    bucket = (gap[..., None] >= torch.tensor(BOUNDS)).sum(2)
    t = t + w["bias"][bucket]
    open_ = ts != 0xFFFFFFFF
    t = torch.where(open_[..., None], t, torch.full_like(t, -1e300))
    p = torch.softmax(t, 1) * open_.any(1)[:, None, None]
    o = (p[..., None] * k).sum(1).reshape(n, d)
    return norm(o, w["g2"], w["b2"])


def test_sample_norm_attention_norm_and_back():
    import torch
    import paper_2402_01964_amd as nlb
    base = synth.workload(5)
    w = dataclasses.replace(synth.scaled(base, 3 * 2000, num_nodes=400), batch=2000)
    src, dst, t, neg = synth.host_links(w)
    rng = np.random.default_rng(0)
    rows = rng.standard_normal((w.num_nodes, WIDTH)).astype(np.float32)
    table = make_gpu_table(w, None, feat_to_dev(rows, "f32"))
    table.insert(*(to_dev(x[:4000]) for x in (src, dst, t)))
    node, tq = to_dev(np.concatenate([src, dst, neg])[4000:4300].astype(np.int32)), to_dev(
        np.full(300, int(t[4000]), np.uint32))
    out = table.sample(node, tq, want=("ts", "nfeat", "self"))
    n, s, d = out["nfeat"].shape
    gen = torch.Generator().manual_seed(1)
    p = {"g1": 1 + 0.1 * torch.randn(d, generator=gen), "b1": 0.1 * torch.randn(d, generator=gen),
         "g2": 1 + 0.1 * torch.randn(d, generator=gen), "b2": 0.1 * torch.randn(d, generator=gen),
         "bias": torch.randn(len(BOUNDS) + 1, HEADS, generator=gen)}
    dev = {k: v.cuda() for k, v in p.items()}
    dy = torch.randn(n, d, generator=gen)

    # the library's: keys are values, so their gradients add up
    xn, xs = out["nfeat"].view(n * s, d), out["self"]
    kn, m1, r1 = nlb.layer_norm(xn, dev["g1"], dev["b1"])
    qn, m2, r2 = nlb.layer_norm(xs, dev["g1"], dev["b1"])
    q, k = qn.view(n, HEADS, -1), kn.view(n * s, HEADS, -1)
    how = dict(batch=n, bias=dev["bias"], bounds=torch.tensor(BOUNDS, dtype=torch.int32, device="cuda"), q_pos=tq,
               k_pos=out["ts"])
    o, lse = nlb.attention(q, k, k, **how)
    y, m3, r3 = nlb.layer_norm(o.view(n, d), dev["g2"], dev["b2"])
    do, dg2, db2 = nlb.layer_norm_backward(dy.cuda(), o.view(n, d), dev["g2"], m3, r3)
    dq, dk, dv, dbias = nlb.attention_backward(do.view(n, HEADS, -1), q, k, k, o, lse, **how)
    dxn, dg1, db1 = nlb.layer_norm_backward((dk + dv).view(n * s, d), xn, dev["g1"], m1, r1)
    dxs, dg1s, db1s = nlb.layer_norm_backward(dq.view(n, d), xs, dev["g1"], m2, r2)
    torch.cuda.synchronize()
    assert table.status() == 0

    ts = out["ts"].cpu().numpy().view(np.uint32).astype(np.int64)
    some = (ts != 0xFFFFFFFF).any(1)
    assert some.any() and not some.all()                      # queries without neighbours among them: o = 0
    assert not o[torch.from_numpy(~some).cuda()].any()
    leaf = {name: v.double().requires_grad_() for name, v in p.items()}
    a, b = (x.cpu().double().view(shape).requires_grad_() for x, shape in ((xs, (n, d)), (xn, (n, s, d))))
    want = _layer64(a, b, torch.from_numpy(ts), torch.from_numpy(tq.cpu().numpy().view(np.uint32).astype(np.int64)),
                    leaf, HEADS)
    (want * dy.double()).sum().backward()
    # Each step is off by some 2^-24 of the magnitudes that it sums (128 values, 10 slots, 300 rows); the norm's
    # division by a small spread of o takes up to 1 / std(o) = 10 of it: 128 2^-24 10 = 8e-5 of the largest value.
    pairs = {"y": (y, want), "d self": (dxs, a.grad), "d neighbours": (dxn.view(n, s, d), b.grad),
             "dg2": (dg2, leaf["g2"].grad), "db2": (db2, leaf["b2"].grad), "dg1": (dg1 + dg1s, leaf["g1"].grad),
             "db1": (db1 + db1s, leaf["b1"].grad), "dbias": (dbias, leaf["bias"].grad)}
    for name, (x, ref) in pairs.items():
        x, ref = x.double().cpu(), ref.detach()
        assert x.shape == ref.shape and (x - ref).abs().max() <= 8e-5 * ref.abs().max(), (
            name, float((x - ref).abs().max() / ref.abs().max()))
