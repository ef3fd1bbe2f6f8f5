"""Position biases of any size (GPU): beyond 2^20 in magnitude they count as
2^20, up to the type's largest value; at or below -2^100 they close their
bucket.  Against 64 bits, within the bounds that attention_ref derives (wide
ones where a row has nothing but such biases: fp32 holds 2^20 in steps of 1/8)."""
import pytest

from tests.test_gpu_attention import _dtype, check, make, run

pytestmark = pytest.mark.gpu

FORMS = {
    "tiles": (False, [150, 9, 40], [200, 9, 300]),
    "wide tiles": (False, [700, 500, 1000], [700, 500, 1100]),
    "lists": (True, [1] * 6, [50, 9, 64, 1, 0, 33]),
    "chunks": (True, [1, 1], [1500, 40]),
}


def _counted(bias):
    """The bias as it counts."""
    import torch
    x = bias.double()
    return torch.where(x > -2.0 ** 100, x.clamp(-2.0 ** 20, 2.0 ** 20), x)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form,value", [
    (form, value) for form in FORMS
    for value in (["largest", 1e30, 1e9, 2.0 ** 20, 3000.0, -3000.0, -1e5, -1e9, -1e30] if form != "wide tiles"
                  else ["largest", -1e9])])                   # (7 s each on the CPU)
def test_biases_of_any_size(dtype, form, value):
    """In some buckets, in the far ones, and in all (rows with nothing else)."""
    import torch
    one, lq, lk = FORMS[form]
    heads = 16 if form == "wide tiles" else 2
    for times in (False, True):
        for which in ([0, 1], [5, 6, 7, 8], list(range(9))):
            c = make(dtype, lq, lk, heads, 2, 8, bias=True, times=times, train=True)
            c["bias"][which] = torch.finfo(_dtype(dtype)).max if value == "largest" else value
            got = run(c, lq, lk, causal=True, one=one)
            check(dict(c, bias=_counted(c["bias"])), lq, lk, got, causal=True, dtype=dtype, what=(times, which))


@pytest.mark.parametrize("value", ["largest", -1e30])
@pytest.mark.parametrize("form", list(FORMS))
def test_with_the_smallest_scale(form, value):
    import torch
    one, lq, lk = FORMS[form]
    heads = 16 if form == "wide tiles" else 2
    for scale in (2.0 ** -20, -2.0 ** -20, 0.0):
        c = make("f32", lq, lk, heads, 2, 8, bias=True, train=True)
        c["bias"][3:7] = torch.finfo(torch.float32).max if value == "largest" else value
        got = run(c, lq, lk, causal=True, one=one, scale=scale)
        check(dict(c, bias=_counted(c["bias"])), lq, lk, got, causal=True, dtype="f32", scale=scale, what=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("one", [False, True])
def test_padding_by_a_large_negative_bias(dtype, one):
    """A mask of -1e9: bit for bit as if it closed its bucket, but for rows
    that see nothing else, which take the softmax of their scores."""
    import torch
    lq, lk = ([1] * 6, [40] * 6) if one else ([70] * 3, [70] * 3)
    for mode in ("places", "times"):
        c = make(dtype, lq, lk, 2, 2, 16, bias=True, times=mode == "times", closed=0, train=True, seed=3)
        if mode == "times":
            c["q_pos"][:] = 500
            c["k_pos"] = torch.where(c["k_pos"] < 150, 1000, 0).to(torch.int32)
            c["k_pos"][:lk[0]] = 1000                         # nothing but masked keys in the first sequence
            c["bounds"] = torch.tensor([0], dtype=torch.int32)
        else:
            c["bounds"] = torch.tensor([30], dtype=torch.int32)
        closed = dict(c, bias=torch.zeros(2, 2, dtype=_dtype(dtype)))
        closed["bias"][0] = -float("inf")
        c["bias"] = torch.zeros(2, 2, dtype=_dtype(dtype))
        c["bias"][0] = -1e9
        got, want = run(c, lq, lk, causal=True, one=one), run(closed, lq, lk, causal=True, one=one)
        check(dict(c, bias=_counted(c["bias"])), lq, lk, got, causal=True, dtype=dtype, what=mode)
        if mode == "places":
            continue
        # rows that see an open key, and keys that only such rows see: those from a sequence's first open key on
        # (all of them where rows see all keys, a list's one row among them)
        for b in range(1, len(lk)):
            rows, keys = slice(sum(lq[:b]), sum(lq[:b + 1])), slice(sum(lk[:b]), sum(lk[:b + 1]))
            first = int((c["k_pos"][keys] == 0).nonzero()[0])
            assert first < 20
            for n, x in got.items():
                if n != "dbias":
                    part = keys if n in ("dk", "dv") else rows
                    skip = 0 if one else first
                    assert torch.equal(x[part][skip:], want[n][part][skip:]), (n, b)
        for n in ("o", "dk", "dv"):
            assert (got[n][:lk[0] if n != "o" else lq[0]] != 0).any(), n
