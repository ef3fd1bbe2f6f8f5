"""The operators of an attention layer over retrieved lists and histories, as
cases to be timed: what they compute in plain torch, and the library's calls.

The kinds of work:

  attend        attention over packed sequences of different lengths
  attend_train  the same, and its backward pass
  lists         one query per sequence: a query's retrieved list (a fixed number
                of slots, empty ones marked by their timestamp), or a single
                token over a long history
  lists_train   the same, and its backward pass
  norm          layer norm of rows
  norm_train    the same, and its backward pass

    s[i][j] = scale q_i . k_j + bias[bucket(pos_i - pos_j)][h]
    o_i     = sum_j softmax_j(s[i])  v_j       over the keys open to row i
    bucket(x) = the number of bounds <= x

Positions are places in the sequence (the last query row stands at the last
key row) or timestamps.  A key whose timestamp is 0xFFFFFFFF is closed; under
`causal` a row sees the keys up to its own place.  A row without an open key
gives zeros (and minus infinity as its log of the sum).
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
NO_KEY = -1          # an empty slot's timestamp, 0xFFFFFFFF as int32
EPS = 1e-5


def _attend(name, kind, dtype, batch, q_lo, q_hi, heads, kv_heads, dim, **more):
    """batch sequences of q_lo to q_hi query rows, each after up to `context`
    rows that are keys only.  buckets: rows of the bias (0: none); top: the
    distance at which its last bucket begins.  times: positions are
    timestamps.  slots: keys of every sequence (0: its rows).  fill: the share
    of keys that are open.  mix: seed of the lengths."""
    c = {"kind": kind, "dtype": dtype, "batch": batch, "q_lo": q_lo, "q_hi": q_hi, "heads": heads,
         "kv_heads": kv_heads, "dim": dim, "context": 0, "causal": True, "buckets": 0, "top": 128, "times": False,
         "slots": 0, "fill": 1.0, "mix": 1}
    c.update(more)
    return {"name": name, **c} if name else c


def _norm(name, kind, dtype, rows, width, gap=0):
    """gap: values between a row's end and the next row."""
    c = {"kind": kind, "dtype": dtype, "rows": rows, "width": width, "gap": gap}
    return {"name": name, **c} if name else c


def listed():
    return [
        # The smallest call: one short history of 33 rows, where the launch is
        # what counts.
        _attend("attend-tiny", "attend", "bf16", 1, 33, 33, 4, 2, 32),
        # A batch of histories of very different lengths, grouped heads, q, k
        # and v as slices of one projection's output.
        _attend("attend-packed", "attend", "bf16", 24, 16, 2048, 16, 4, 128),
        # One long history, with the bias by places.
        _attend("attend-long", "attend", "bf16", 1, 8000, 8000, 16, 2, 128, buckets=32),
        # fp32 rows of an odd width (100-wide statuses in two heads), not
        # causal, rows after a context, bias by timestamps, some rows closed.
        _attend("attend-times-f32", "attend", "f32", 37, 1, 700, 2, 2, 50, context=300, causal=False, buckets=17,
                top=1 << 20, times=True, fill=0.95),
        # A training step over packed histories with the bias and its gradient.
        _attend("train-packed", "attend_train", "bf16", 8, 128, 2048, 8, 2, 64, buckets=32),
        # A training step over long histories, no bias.
        _attend("train-long", "attend_train", "bf16", 2, 3500, 4096, 16, 4, 128),
        # A training step over many short fp32 lists of different lengths,
        # all rows seeing all rows, bias by timestamps.
        _attend("train-short-f32", "attend_train", "f32", 200, 3, 100, 4, 4, 25, causal=False, buckets=16,
                top=1 << 20, times=True, fill=0.9),
        # The retrieved lists of a large sparse batch: 300 000 queries, 10 slots.
        _attend("lists-large", "lists", "bf16", 300_000, 1, 1, 2, 2, 64, causal=False, slots=10, buckets=16,
                top=1 << 20, times=True, fill=0.6),
        # A training step over the retrieved lists of a batch: 12 000 queries
        # of 20 slots, fp32 statuses of width 100 in two heads.
        _attend("lists-train-f32", "lists_train", "f32", 12_000, 1, 1, 2, 2, 50, causal=False, slots=20, buckets=16,
                top=1 << 20, times=True, fill=0.7),
        # One new token each for 16 sequences over their long caches.
        _attend("token-long", "lists", "bf16", 16, 1, 1, 32, 8, 128, context=65_535),
        # A training step's norm over the rows of a large batch.
        _norm("norm-train-large", "norm_train", "bf16", 131_072, 1024),
        # The norm of the statuses of a small batch's queries.
        _norm("norm-small", "norm", "f32", 600, 100),
    ]


def draw(rng):
    """A case of the same ranges: 1 to 500 sequences of 1 to 4000 rows, 1 to
    16 heads of 8 to 128 values in 1 to 16 groups; lists of 1 to 100 slots for
    100 to 200 000 queries, caches of up to 60 000 keys; norms of 1 to 100 000
    rows of 2 to 8192 values."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["attend", "attend", "attend_train", "attend_train", "lists", "lists", "lists_train", "norm",
                       "norm_train"])
    dtype = rng.choice(["bf16", "f32"])
    if kind.startswith("norm"):
        rows = log(1, 100_000)
        return _norm("", kind, dtype, rows, log(2, max(2, min(8192, 100_000_000 // rows))), rng.choice([0, 0, 8, 3]))
    kv_heads = rng.choice([1, 2, 4])
    heads = kv_heads * rng.choice([1, 1, 2, 4])
    dim = rng.choice([25, 32, 50, 64, 64, 128, 128, rng.randint(8, 128)])
    more = dict(mix=rng.randint(1, 1 << 20), times=rng.random() < 0.5)
    if rng.random() < 0.7:
        more.update(buckets=rng.randint(2, 32), top=1 << 20 if more["times"] else log(32, 1000))
    if more["times"]:
        more.update(fill=rng.uniform(0.5, 1.0))
    if kind.startswith("lists"):
        if rng.random() < 0.3:
            return _attend("", kind, dtype, log(1, 32), 1, 1, heads, kv_heads, dim, context=log(100, 60_000), **more)
        slots = log(1, 100)
        more.update(slots=slots, times=True, causal=False, fill=rng.uniform(0.2, 1.0))
        if "buckets" in more:
            more.update(top=1 << 20)
        return _attend("", kind, dtype, log(100, min(200_000, 300_000_000 // (slots * heads * dim))), 1, 1, heads,
                       kv_heads, dim, **more)
    hi = log(16, 4000 if kind == "attend" else 2000)
    lo = rng.choice([1, max(1, hi // 8), hi])
    context = rng.choice([0, 0, 1, hi // 2])
    most = 250_000_000 if kind == "attend" else 60_000_000   # scores of the whole call
    batch = log(1, max(1, min(500, most // ((hi + context) * hi * heads))))
    return _attend("", kind, dtype, batch, lo, hi, heads, kv_heads, dim, context=context,
                   causal=rng.random() < 0.6, **more)


# ------------------------------------------------------------------ inputs
def _lengths(c):
    """Query rows and keys of each sequence."""
    r = random.Random(c["mix"])
    lo, hi = c["q_lo"], c["q_hi"]
    lq = [int(round(math.exp(r.uniform(math.log(lo), math.log(hi))))) for _ in range(c["batch"])]
    lq[0] = hi
    if c["slots"]:
        return lq, [c["slots"]] * c["batch"]
    lk = [n + (r.randint(0, c["context"]) if c["context"] else 0) for n in lq]
    lk[0] = hi + c["context"]
    return lq, lk


def _bounds(c):
    """buckets - 1 bounds, one apart near zero, then in equal ratios up to
    `top`; to both sides of zero where keys may lie ahead."""
    n = c["buckets"] - 1
    two_sided = not c["causal"] and not c["times"]
    m = n - n // 2 if two_sided else n
    near = (m + 1) // 2
    got = []
    for i in range(m):
        b = i + 1 if i < near else int(near * (c["top"] / near) ** ((i + 1 - near) / (m - near)))
        got.append(max(b, got[-1] + 1 if got else b))
    if two_sided:
        got = [1 - b for b in reversed(got[:n // 2])] + got
    return got


def _starts(lengths):
    t = torch.zeros(len(lengths) + 1, dtype=torch.int64)
    t[1:] = torch.cumsum(torch.tensor(lengths, dtype=torch.int64), 0)
    return t.to(torch.int32).cuda()


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)
    dtype = DTYPES[c["dtype"]]

    def randn(*shape, scale=1.0):
        x = torch.randn(shape, device="cuda", generator=gen, dtype=dtype)
        return x if scale == 1.0 else x.mul_(scale)

    if c["kind"].startswith("norm"):
        n, d = c["rows"], c["width"]
        x = randn(n, d + c["gap"]).mul_(2.0).add_(0.5)[:, :d]
        st = {"case": c, "x": x, "w": 1.0 + 0.1 * torch.randn(d, device="cuda", generator=gen),
              "b": 0.1 * torch.randn(d, device="cuda", generator=gen)}
        if c["kind"] == "norm_train":
            st["dy"] = randn(n, d + c["gap"])[:, :d]
        return st

    lq, lk = _lengths(c)
    tq, tk, h, hk, d = sum(lq), sum(lk), c["heads"], c["kv_heads"], c["dim"]
    if not c["context"] and not c["slots"]:     # one projection's output
        qkv = randn(tq, h + 2 * hk, d)
        q, k, v = qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:]
        q.mul_(2.0)
    else:
        q, k, v = randn(tq, h, d, scale=2.0), randn(tk, hk, d), randn(tk, hk, d)
    st = {"case": c, "q": q, "k": k, "v": v, "scale": d ** -0.5, "max_q": max(lq), "max_k": max(lk),
          "q_start": _starts(lq) if max(lq) > 1 else None, "k_start": None if c["slots"] else _starts(lk),
          "bias": None, "bounds": None, "q_pos": None, "k_pos": None}
    if c["buckets"]:
        st["bias"] = randn(c["buckets"], h)
        st["bounds"] = torch.tensor(_bounds(c), dtype=torch.int32, device="cuda")
    if c["times"]:
        def gaps(n):
            return torch.pow(2.0, torch.rand(n, device="cuda", generator=gen, dtype=torch.float64) * 16).long()
        if c["slots"]:                          # stored before the query, in no order
            q_pos = torch.randint(1 << 20, 1 << 28, (tq,), device="cuda", generator=gen)
            k_pos = q_pos.repeat_interleave(c["slots"]) - gaps(tk)
        else:                                   # a history in time order; its last rows are the queries
            k_pos = torch.cumsum(torch.pow(2.0, torch.rand(tk, device="cuda", generator=gen, dtype=torch.float64)
                                           * 10).long(), 0)
            ends = torch.cumsum(torch.tensor(lk), 0).cuda()
            n = torch.tensor(lq).cuda()
            first = (ends - n).repeat_interleave(n)
            row = torch.arange(tq, device="cuda") - (torch.cumsum(n, 0) - n).repeat_interleave(n)
            q_pos = k_pos[first + row]
        closed = torch.rand(tk, device="cuda", generator=gen) >= c["fill"]
        st["q_pos"] = q_pos.to(torch.int32)
        st["k_pos"] = k_pos.to(torch.int32).masked_fill_(closed, NO_KEY)
    if c["kind"].endswith("_train"):
        st["do"] = randn(tq, h, d)
    return st


# ------------------------------------------------------------------ the plain form
def _padded(x, start, batch, longest):
    """Rows [T, ...] as fp32 [batch, longest, ...], zeros behind a sequence's
    end, and which of them are rows."""
    if start is None:
        x = x.view(batch, longest, *x.shape[1:])
        return x.float(), torch.ones((batch, longest), dtype=torch.bool, device=x.device)
    at = start[:-1, None].long() + torch.arange(longest, device=x.device)
    there = at < start[1:, None]
    x = x[at.clamp(max=x.shape[0] - 1)].float()
    return x.masked_fill_(~there.view(*there.shape, *[1] * (x.dim() - 2)), 0), there


def _rows(x, there):
    """The rows of _padded() again, packed."""
    return x[there] if x.shape[1] > 1 else x.flatten(0, 1)


def _plain_attention(st):
    c = st["case"]
    batch, h, hk, d, nq, nk = c["batch"], c["heads"], c["kv_heads"], c["dim"], st["max_q"], st["max_k"]
    g = h // hk
    q, q_there = _padded(st["q"], st["q_start"], batch, nq)
    k, k_there = _padded(st["k"], st["k_start"], batch, nk)
    v, _ = _padded(st["v"], st["k_start"], batch, nk)

    def by_group(x):       # [batch, rows, h, d] -> [batch, hk, g * rows, d]
        return x.view(batch, nq, hk, g, d).permute(0, 2, 3, 1, 4).reshape(batch, hk, g * nq, d)

    def by_row(x):
        return x.view(batch, hk, g, nq, d).permute(0, 3, 1, 2, 4).reshape(batch, nq, h, d)

    q = by_group(q)
    k, v = k.permute(0, 2, 1, 3).contiguous(), v.permute(0, 2, 1, 3).contiguous()      # [batch, hk, nk, d]
    s = (q @ k.transpose(2, 3).contiguous()).mul_(st["scale"]).view(batch, h, nq, nk)
    # the last query row stands at the last key row
    place = torch.arange(nq, device=q.device) + (k_there.sum(1) - q_there.sum(1))[:, None]
    key = torch.arange(nk, device=q.device)
    if st["bias"] is not None:
        if c["times"]:
            i = _padded_ints(st["q_pos"], st["q_start"], batch, nq)
            j = _padded_ints(st["k_pos"], st["k_start"], batch, nk)
            gap = i[:, :, None] - j[:, None, :]
        else:
            gap = place[:, :, None] - key
        bucket = torch.bucketize(gap, st["bounds"].long(), right=True)
        s += st["bias"].float()[bucket].permute(0, 3, 1, 2)
    opened = k_there[:, None, :].expand(batch, nq, nk)
    if c["times"]:
        opened = opened & (_padded_ints(st["k_pos"], st["k_start"], batch, nk) != 0xFFFFFFFF)[:, None, :]
    if c["causal"]:
        opened = opened & (key <= place[:, :, None])
    s.masked_fill_(~opened[:, None], -math.inf)
    top = s.amax(3, keepdim=True)
    top.masked_fill_(top == -math.inf, 0)
    p = s.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    lse = (total.log() + top).view(batch, h, nq).transpose(1, 2)
    p = p.div_(total.masked_fill_(total == 0, 1)).view(batch, hk, g * nq, nk)
    o = by_row(p @ v)
    dtype = st["q"].dtype
    out = {"o": _rows(o, q_there).to(dtype), "lse": _rows(lse, q_there)}
    if "do" not in st:
        return out
    do = by_group(_padded(st["do"], st["q_start"], batch, nq)[0])
    dv = p.transpose(2, 3).contiguous() @ do
    ds = do @ v.transpose(2, 3).contiguous()
    ds.sub_((ds * p).sum(3, keepdim=True)).mul_(p)
    dq = by_row(ds @ k).mul_(st["scale"])
    dk = (ds.transpose(2, 3).contiguous() @ q).mul_(st["scale"])
    out.update(dq=_rows(dq, q_there).to(dtype), dk=_rows(dk.transpose(1, 2), k_there).to(dtype),
               dv=_rows(dv.transpose(1, 2), k_there).to(dtype))
    if st["bias"] is not None:
        n = c["buckets"]
        one = (bucket[:, :, None, :] == torch.arange(n, device=q.device)[:, None]).float().view(batch * nq, n, nk)
        ds = ds.view(batch, h, nq, nk).permute(0, 2, 3, 1).reshape(batch * nq, nk, h)
        out["dbias"] = (one @ ds).sum(0, dtype=torch.float64).to(dtype)
    return out


def _padded_ints(x, start, batch, longest):
    """Positions [T] as [batch, longest]."""
    x = x.long() & 0xFFFFFFFF
    if start is None:
        return x.view(batch, longest)
    at = start[:-1, None].long() + torch.arange(longest, device=x.device)
    return x[at.clamp(max=x.shape[0] - 1)]


def _plain_norm(st):
    x, w = st["x"].float(), st["w"]
    mean = x.mean(1, keepdim=True)
    x = x - mean
    rstd = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    x *= rstd
    out = {"y": (x * w + st["b"]).to(st["x"].dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if "dy" not in st:
        return out
    dy = st["dy"].float()
    g = dy * w
    dx = (g - g.mean(1, keepdim=True) - x * (g * x).mean(1, keepdim=True)) * rstd
    out.update(dx=dx.to(st["x"].dtype), dw=(dy * x).sum(0, dtype=torch.float64).float(),
               db=dy.sum(0, dtype=torch.float64).float())
    return out


# ------------------------------------------------------------------ one pass
def run(state):
    c = state["case"]
    if not own:
        return _plain_norm(state) if c["kind"].startswith("norm") else _plain_attention(state)
    import paper_2402_01964_amd as nlb
    if c["kind"].startswith("norm"):
        y, mean, rstd = nlb.layer_norm(state["x"], state["w"], state["b"], EPS)
        out = {"y": y, "mean": mean, "rstd": rstd}
        if "dy" in state:
            out["dx"], out["dw"], out["db"] = nlb.layer_norm_backward(state["dy"], state["x"], state["w"], mean, rstd)
        return out
    q, k, v = state["q"], state["k"], state["v"]
    how = dict(batch=c["batch"], q_start=state["q_start"], k_start=state["k_start"], causal=c["causal"],
               scale=state["scale"], bias=state["bias"], bounds=state["bounds"], q_pos=state["q_pos"],
               k_pos=state["k_pos"])
    o, lse = nlb.attention(q, k, v, **how)
    out = {"o": o, "lse": lse}
    if "do" in state:
        out["dq"], out["dk"], out["dv"], dbias = nlb.attention_backward(state["do"], q, k, v, o, lse, **how)
        if dbias is not None:
            out["dbias"] = dbias
    return out


# ------------------------------------------------------------------ in 64 bits
def _exact_sequence(q, k, v, do, bias, bucket, opened, scale, buckets):
    """One sequence and one kv head in fp64: q, do [g, nq, d]; k, v [nk, d];
    bias [buckets, g]; bucket, opened [nq, nk]."""
    s = torch.matmul(q, k.T.contiguous()) * scale
    if bias is not None:
        s = s + bias.T[:, bucket]
    s = torch.where(opened, s, torch.full_like(s, -math.inf))
    lse = torch.logsumexp(s, 2)
    p = torch.where(opened, torch.exp(s - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[..., None]),
                    torch.zeros_like(s))
    o = torch.matmul(p, v)
    if do is None:
        return o, lse, None
    dp = torch.matmul(do, v.T.contiguous())
    ds = p * (dp - (do * o).sum(2, keepdim=True))
    dbias = None
    if bias is not None:
        dbias = torch.stack([torch.where(bucket == b, ds, torch.zeros_like(ds)).sum((1, 2)) for b in range(buckets)])
    g, nq, nk = ds.shape
    return o, lse, (torch.matmul(ds, k) * scale,
                    torch.matmul(ds.reshape(g * nq, nk).T.contiguous(), q.reshape(g * nq, -1)) * scale,
                    torch.matmul(p.reshape(g * nq, nk).T.contiguous(), do.reshape(g * nq, -1)), dbias)


def _exact_lists(c, st):
    """One query and a fixed number of keys per sequence, in fp64."""
    n, slots, h, hk, d = c["batch"], c["slots"], c["heads"], c["kv_heads"], c["dim"]
    q = st["q"].double()
    k = st["k"].double().view(n, slots, hk, 1, d).expand(n, slots, hk, h // hk, d).reshape(n, slots, h, d)
    s = (q[:, None] * k).sum(3) * st["scale"]
    kp = st["k_pos"].long().view(n, slots) & 0xFFFFFFFF
    if st["bias"] is not None:
        gap = (st["q_pos"].long() & 0xFFFFFFFF)[:, None] - kp
        bucket = (gap[..., None] >= st["bounds"].long()).sum(2)
        s = s + st["bias"].double()[bucket]
    s = torch.where((kp != 0xFFFFFFFF)[..., None], s, torch.full_like(s, -math.inf))
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[:, None])
    v = st["v"].double().view(n, slots, hk, 1, d).expand(n, slots, hk, h // hk, d).reshape(n, slots, h, d)
    o = (p[..., None] * v).sum(1)
    out = {"o": o, "lse": lse}
    if "do" in st:
        do = st["do"].double()
        ds = p * ((do[:, None] * v).sum(3) - (do * o).sum(2)[:, None])
        out["dq"] = (ds[..., None] * k).sum(1) * st["scale"]
        out["dk"] = (ds[..., None] * q[:, None]).view(n * slots, hk, h // hk, d).sum(2) * st["scale"]
        out["dv"] = (p[..., None] * do[:, None]).view(n * slots, hk, h // hk, d).sum(2)
        if st["bias"] is not None:
            out["dbias"] = torch.stack([torch.where((bucket == b)[..., None], ds, torch.zeros_like(ds)).sum((0, 1))
                                        for b in range(c["buckets"])])
    return out


def exact(case, seed):
    c, st = case, prepare(case, seed)
    if c["kind"].startswith("norm"):
        x, w = st["x"].double(), st["w"].double()
        mean = x.mean(1)
        rstd = 1.0 / torch.sqrt(x.var(1, unbiased=False) + EPS)
        x = (x - mean[:, None]) * rstd[:, None]
        out = {"y": x * w + st["b"].double(), "mean": mean, "rstd": rstd}
        if "dy" in st:
            dy = st["dy"].double()
            g = dy * w
            out["dx"] = rstd[:, None] * (g - g.mean(1)[:, None] - x * (g * x).mean(1)[:, None])
            out["dw"], out["db"] = (dy * x).sum(0), dy.sum(0)
        return out
    if c["slots"]:
        return _exact_lists(c, st)
    lq, lk = _lengths(c)
    h, hk = c["heads"], c["kv_heads"]
    g = h // hk
    f64 = dict(dtype=torch.float64, device="cuda")
    out = {"o": torch.zeros(st["q"].shape, **f64), "lse": torch.zeros(st["q"].shape[:2], **f64)}
    if "do" in st:
        out.update(dq=torch.zeros(st["q"].shape, **f64), dk=torch.zeros(st["k"].shape, **f64),
                   dv=torch.zeros(st["v"].shape, **f64))
        if st["bias"] is not None:
            out["dbias"] = torch.zeros((c["buckets"], h), **f64)
    a = e = 0
    for n, m in zip(lq, lk):
        rows, keys = slice(a, a + n), slice(e, e + m)
        a, e = a + n, e + m
        place = torch.arange(m - n, m, device="cuda")
        key = torch.arange(m, device="cuda")
        opened = torch.ones((n, m), dtype=torch.bool, device="cuda")
        pi, pj = place, key
        if c["times"]:
            pi, pj = st["q_pos"][rows].long() & 0xFFFFFFFF, st["k_pos"][keys].long() & 0xFFFFFFFF
            opened &= (pj != 0xFFFFFFFF)
        if c["causal"]:
            opened &= key <= place[:, None]
        bucket = None
        if st["bias"] is not None:
            bucket = torch.zeros((n, m), dtype=torch.int64, device="cuda")
            for b in _bounds(c):
                bucket += (pi[:, None] - pj) >= b
        for j in range(hk):
            heads = slice(j * g, j * g + g)
            do = st["do"][rows, heads].double().transpose(0, 1).contiguous() if "do" in st else None
            o, lse, grads = _exact_sequence(
                st["q"][rows, heads].double().transpose(0, 1).contiguous(), st["k"][keys, j].double().contiguous(),
                st["v"][keys, j].double().contiguous(), do,
                st["bias"][:, heads].double() if bucket is not None else None, bucket, opened, st["scale"],
                c["buckets"])
            out["o"][rows, heads], out["lse"][rows, heads] = o.transpose(0, 1), lse.T
            if grads:
                out["dq"][rows, heads], out["dk"][keys, j], out["dv"][keys, j] = grads[0].transpose(0, 1), *grads[1:3]
                if bucket is not None:
                    out["dbias"][:, heads] += grads[3]
    return out


# ------------------------------------------------------------------ what it cannot do without
def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    train = c["kind"].endswith("_train")
    if c["kind"].startswith("norm"):
        n, d = c["rows"], c["width"]
        size, flops = 2 * e * n * d + 8 * n + 8 * d, 8 * n * d
        if train:
            size, flops = size + 3 * e * n * d + 8 * n + 12 * d, flops + 14 * n * d
        return {"bytes": float(size), "flops": float(flops)}
    lq, lk = _lengths(c)
    tq, tk, h, hk, d = sum(lq), sum(lk), c["heads"], c["kv_heads"], c["dim"]
    # (a list's keys past its last open slot are not known before they are read)
    pairs = sum(n * m - n * (n - 1) // 2 if c["causal"] else n * m for n, m in zip(lq, lk)) * c["fill"]
    keys = tk * c["fill"]
    size = e * d * (2 * h * tq + 2 * hk * keys) + 4 * h * tq + (4 * (tq + tk) if c["times"] else 0)
    flops = 4.0 * d * h * pairs
    if train:
        size += e * d * (3 * h * tq + 2 * hk * keys) + 4 * h * tq + e * d * (h * tq + 2 * hk * tk)
        flops += 10.0 * d * h * pairs
    return {"bytes": float(size + 2 * e * c["buckets"] * h), "flops": float(flops)}
