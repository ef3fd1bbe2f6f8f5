"""Many retrieved lists with a query row each (GPU): the forms that give a list
to a group of lanes, forward and backward, with lists of every length among
them.  A sample of the lists is held against 64 bits; the gradients of the
others' results are zero, so that the bias gradient is the sample's.

The bounds are attention_ref's with softmax weights and ds in fp32 (nothing
but the outputs is rounded to the rows' type), and what the gradients' form
adds: it takes d_j = dp_j - dp_f from the list's first open key f on, so where
attention_ref has |dp_j| and the row's a = sum p |do||v| there is F = |dp_f|
beside them.  With w = 2^-24, m keys and weights off by e (as there):
  ds_j: p_j ((m + 8) w + max e) (|dp_j| + a + 2 F), in dk and the bias gradient
  dq: the same, times |k_j| scale, summed"""
import numpy as np
import pytest

from tests import attention_ref as ref
from tests.test_gpu_attention import BOUNDS, HALF_STEP, _f64, _u32, make, run

pytestmark = pytest.mark.gpu


def extra(c, lq, lk, want, scale):
    """What the list form adds to the bounds of dq, dk and dbias, from the reference's lse."""
    q, k, v, do = (_f64(c[n]) for n in ("q", "k", "v", "do"))
    h, g, dim = q.shape[1], q.shape[1] // k.shape[1], q.shape[2]
    far = {n: np.zeros_like(want[n]) for n in ("dq", "dk", "dbias") if n in want}
    ks = ref.starts(lk)
    bias, kp, qp = _f64(c["bias"]), _u32(c["k_pos"]), _u32(c["q_pos"])
    for b, m in enumerate(lk):
        keys = slice(ks[b], ks[b] + m)
        opened = np.ones(m, bool) if kp is None else kp[keys] != ref.NO_KEY
        if not opened.any():
            continue
        gap = m - 1 - np.arange(m) if qp is None else int(qp[b]) - kp[keys].astype(np.int64)
        bk = ref.bucket_of(gap, BOUNDS)
        for j in range(h):
            kk, vv = (np.where(opened[:, None], x[keys, j // g], 0) for x in (k, v))
            add = np.where(opened, bias[bk, j], 0) if bias is not None else np.zeros(m)
            s = kk @ q[b, j] * scale + add
            lse = want["lse"][b, j]
            p = np.where(opened, np.exp(s - lse), 0)
            ab = np.abs(kk) @ np.abs(q[b, j]) * abs(scale) + np.abs(add)
            e = ref.W * ((dim + 8) * ab.max() + 4 * (abs(lse) + np.abs(s[opened]).max()) + m + 16)
            dp, dab = vv @ do[b, j], np.abs(vv) @ np.abs(do[b, j])
            x = p * ((m + 8) * ref.W + e) * (np.abs(dp) + (p * dab).sum() + 2 * abs(dp[np.argmax(opened)]))
            far["dq"][b, j] = x @ np.abs(kk) * abs(scale)
            far["dk"][keys, j // g] += x[:, None] * np.abs(q[b, j]) * abs(scale)
            if bias is not None:
                np.add.at(far["dbias"][:, j], bk, x)
    return far


def lists(lk, dtype, heads, kv_heads, dim, mode, *, gap=0, sample=60, lists_backward=True):
    """A call of one query row each over lists of lk keys, checked."""
    import torch
    n = len(lk)
    rng = np.random.default_rng(dim)
    c = make(dtype, [1] * n, lk, heads, kv_heads, dim, bias=mode != "plain", times=mode == "times", train=True, gap=gap,
             seed=dim)
    special = [int(np.flatnonzero(np.asarray(lk) == m)[0]) for m in sorted(set(lk))]
    picks = np.unique([0, 1, n - 2, n - 1, *special[:80], *rng.integers(0, n, sample)])
    zero = np.ones(n, bool)
    zero[picks] = False
    c["do"][torch.from_numpy(zero)] = 0
    if mode == "times":                                       # closed keys may hold anything
        shut = c["k_pos"] == -1
        c["k"][shut], c["v"][shut] = float("nan"), float("inf")
    got = run(c, [1] * n, lk, causal=False, one=True)
    for x in got.values():
        assert not torch.isnan(x).any()
    starts = ref.starts(lk)
    keys = np.concatenate([np.arange(starts[b], starts[b + 1]) for b in picks])
    at = {"q": picks, "do": picks, "q_pos": picks, "k": keys, "v": keys, "k_pos": keys}
    few = {m: x[torch.from_numpy(at[m])] if m in at and x is not None else x for m, x in c.items()}
    lens, scale = [lk[b] for b in picks], dim ** -0.5
    half = HALF_STEP[dtype]
    want, far = ref.attention(*(_f64(few[m]) for m in "qkv"), [1] * len(lens), lens, u=ref.W, causal=False, scale=scale,
                              bias=_f64(few["bias"]), bounds=BOUNDS, q_pos=_u32(few["q_pos"]),
                              k_pos=_u32(few["k_pos"]), do=_f64(few["do"]))
    if lists_backward:
        for m, x in extra(few, [1] * len(lens), lens, want, scale).items():
            far[m] += x
    else:                                                     # tiles: p and ds as bf16
        far.update({m: x for m, x in ref.attention(
            *(_f64(few[m]) for m in "qkv"), [1] * len(lens), lens, u=half, causal=False, scale=scale,
            bias=_f64(few["bias"]), bounds=BOUNDS, q_pos=_u32(few["q_pos"]), k_pos=_u32(few["k_pos"]),
            do=_f64(few["do"]))[1].items() if m not in ("o", "lse")})
    for m, x in want.items():
        y = got[m]
        if m != "dbias":
            y = y[torch.from_numpy(keys if m in ("dk", "dv") else picks).cuda()]
        y = y.double().cpu().numpy()
        fine = np.isfinite(x)
        assert np.array_equal(y[~fine], x[~fine]), m
        off = np.abs(y[fine] - x[fine]) - far[m][fine] - (half * np.abs(x[fine]) if m != "lse" else 0)
        assert (off <= 0).all(), (m, f"{(off > 0).sum()} of {off.size} values too far, worst by {off.max():.3g}")


SHAPES = [(4, 1, 64), (2, 2, 25), (2, 3, 50), (4, 4, 128), (2, 7, 64), (3, 1, 33), (2, 2, 128)]   # kv heads, group, dim


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mode", ["plain", "places", "times"])
@pytest.mark.parametrize("kv_heads,group,dim", SHAPES)
def test_many_lists_of_every_length(dtype, mode, kv_heads, group, dim):
    """8192 lists times key/value heads, 64 keys on average at most: empty
    lists, one key, lists around each turn of 16, 32 and 64 keys, and long ones."""
    rng = np.random.default_rng(1)
    n = 8192 // kv_heads + 5
    lk = rng.integers(0, 30, n)
    lk[7:7 + 17 * 16:17] = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 200]
    lk[n - 2], lk[n // 2] = 300, 1000
    assert lk.sum() // 64 <= n
    lists([int(x) for x in lk], dtype, kv_heads * group, kv_heads, dim, mode, gap=3 if dim == 50 else 0,
          lists_backward=group <= 4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mode", ["plain", "places", "times"])
@pytest.mark.parametrize("kv_heads,group,dim", [(8, 1, 32), (4, 2, 64), (8, 3, 25), (4, 4, 128)])
def test_many_longer_lists(dtype, mode, kv_heads, group, dim):
    """More than 64 keys on average: chunks forward, a group of lanes a list
    backward, which reads what lies behind a list's first 64 keys again."""
    rng = np.random.default_rng(2)
    n = 8192 // kv_heads + 3
    lk = rng.integers(60, 100, n)
    lk[3:3 + 19 * 8:19] = [0, 1, 64, 65, 128, 129, 192, 513]
    lk[n - 1] = 1500
    assert lk.sum() // 64 > n
    lists([int(x) for x in lk], dtype, kv_heads * group, kv_heads, dim, mode, sample=30)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [1, 2, 3, 4])
def test_few_lists_are_not_rounded_within(dtype, group):
    """Lists of one length without starts, few of them: weights and ds stay fp32."""
    for n, m in ((40, 20), (300, 64), (3, 1)):
        lists([m] * n, dtype, 2 * group, 2, 64, "times", sample=20)
