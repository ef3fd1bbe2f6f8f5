"""Attention calls of more workgroups than one launch holds (2^24 - 1), on the
GPU: bit for bit what the same sequences give in calls of their own, some of
them against 64 bits."""
import numpy as np
import pytest

from tests import attention_ref as ref
from tests.test_gpu_attention import check

pytestmark = pytest.mark.gpu


def _against_64_bits(t, got, lens, picks, dtype, scale):
    """Sequences `picks` of t's lens = (query rows, keys) each."""
    lq, lk = lens
    for b in picks:
        rows, keys = slice(b * lq, (b + 1) * lq), slice(b * lk, (b + 1) * lk)
        c = {n: t[n][rows if n in ("q", "do") else keys].cpu() for n in ("q", "k", "v", "do")}
        c.update(bias=None, bounds=None, q_pos=None, k_pos=None)
        check(c, [lq], [lk], {n: x[keys if n in ("dk", "dv") else rows] for n, x in got.items()}, causal=False,
              dtype=dtype, scale=scale, what=f"sequence {b}")


@pytest.mark.parametrize("dtype,batch,lq,lk,heads,kv_heads,dim", [
    ("f32", 66_000, 2, 3, 256, 256, 4),                       # tiles forward and backward
    ("bf16", 300_000, 1, 10, 64, 8, 8),                       # lists forward, tiles backward
])
def test_more_workgroups_than_a_launch_holds(dtype, batch, lq, lk, heads, kv_heads, dim):
    import torch
    import paper_2402_01964_amd as nlb
    gen = torch.Generator(device="cuda").manual_seed(1)
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    t = {n: torch.randn(batch * m, h, dim, device="cuda", generator=gen, dtype=dt)
         for n, m, h in (("q", lq, heads), ("k", lk, kv_heads), ("v", lk, kv_heads), ("do", lq, heads))}

    def step(lo, hi):
        q, do, k, v = (t[n][lo * m:hi * m] for n, m in (("q", lq), ("do", lq), ("k", lk), ("v", lk)))
        o, lse = nlb.attention(q, k, v, batch=hi - lo, scale=0.4)
        return (o, lse) + nlb.attention_backward(do, q, k, v, o, lse, batch=hi - lo, scale=0.4)[:3]
    whole = step(0, batch)
    part = (batch + 3) // 4
    for lo in range(0, batch, part):
        hi = min(batch, lo + part)
        for n, x, y in zip(("o", "lse", "dq", "dk", "dv"), whole, step(lo, hi)):
            m = lk if n in ("dk", "dv") else lq
            assert torch.equal(x[lo * m:hi * m], y), (n, lo)
    torch.cuda.synchronize()
    _against_64_bits(t, dict(zip(("o", "lse", "dq", "dk", "dv"), whole)), (lq, lk), [0, 1, batch // 2, batch - 1],
                     dtype, 0.4)


def test_more_joined_rows_than_a_launch_holds():
    """Single rows over ragged histories, most of one chunk, a few of several."""
    import torch
    import paper_2402_01964_amd as nlb
    batch, heads, dim = 66_000, 256, 4
    lk = np.full(batch, 99)
    long = [0, 5, batch // 2, batch - 2, batch - 1]
    lk[long] = 5000
    starts = ref.starts(lk)
    gen = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn(batch, heads, dim, device="cuda", generator=gen)
    k, v = (torch.randn(int(starts[-1]), 1, dim, device="cuda", generator=gen) for _ in range(2))
    o, lse = nlb.attention(q, k, v, batch=batch, k_start=torch.from_numpy(starts).cuda(),
                           out=torch.full_like(q, float("nan")))
    torch.cuda.synchronize()
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()
    for b in long + [1, 33_001, batch - 3]:
        keys = slice(int(starts[b]), int(starts[b + 1]))
        c = {"q": q[b:b + 1].cpu(), "k": k[keys].cpu(), "v": v[keys].cpu(), "do": None, "bias": None, "bounds": None,
             "q_pos": None, "k_pos": None}
        check(c, [1], [int(lk[b])], {"o": o[b:b + 1], "lse": lse[b:b + 1]}, causal=False, dtype="f32",
              what=f"sequence {b}")
