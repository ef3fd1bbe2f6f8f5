"""Attention over packed sequences with a bucketed position bias, and its
gradients, in 64 bits on the CPU: one sequence and one head at a time, from the
formulas; with each output, how far a kernel may be off it.

The bounds.  u is half a step of the rows' type relative to the value (2^-8
bf16, 2^-24 fp32), w = 2^-24.  Every output is rounded once: u |x|.
  A score sums dim products in fp32, takes the scale and the bias and goes
through an exponential against the row's maximum or lse, whose sum has up to lk
terms: a probability is off by at most
  e = w ((dim + 8) (|q||k| scale + |bias|) + 4 (|lse| + max |s|) + lk + 16)
relative to itself.  Where probabilities and ds enter a product they are
rounded to the rows' type (u more), and the product's sum of n terms is off by
n w times the sum of its terms' magnitudes.  With a = |do| . (sum_j p_j |v_j|):
  dp is off by dim w |do||v|; D, the row's sum of p dp, by the e and w terms
(fp32 rows without a bias take it as do . o: by 2 u a more).
"""
import numpy as np

NO_KEY = 0xFFFFFFFF
W = 2.0 ** -24


def starts(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def bucket_of(gap, bounds):
    return np.searchsorted(np.asarray(bounds, np.int64), np.clip(gap, -2**31, 2**31 - 1), side="right")


def attention(q, k, v, lq, lk, *, u, causal, scale, bias=None, bounds=None, q_pos=None, k_pos=None, do=None):
    """q, do: [q_rows, heads, dim]; k, v: [k_rows, kv_heads, dim], float64.
    Returns a dict of o, lse and, with do, dq, dk, dv, dbias, and a dict of
    the same with their bounds (lse's is absolute too)."""
    h, hk, dim = q.shape[1], k.shape[1], q.shape[2]
    g = h // hk
    out = {"o": np.zeros_like(q), "lse": np.full(q.shape[:2], -np.inf)}
    if do is not None:
        out.update(dq=np.zeros_like(q), dk=np.zeros_like(k), dv=np.zeros_like(v))
        if bias is not None:
            out["dbias"] = np.zeros_like(bias)
    far = {n: np.zeros_like(x) for n, x in out.items()}
    qs, ks = starts(lq), starts(lk)
    for b, (n, m) in enumerate(zip(lq, lk)):
        if n == 0 or m == 0:
            continue
        rows, keys = slice(qs[b], qs[b] + n), slice(ks[b], ks[b] + m)
        place, key = np.arange(n)[:, None] + (m - n), np.arange(m)[None]
        opened = np.broadcast_to(key <= place, (n, m)).copy() if causal else np.ones((n, m), bool)
        gap = place - key
        if k_pos is not None:
            kp = k_pos[keys].astype(np.int64)
            opened &= (kp != NO_KEY)[None]
            if q_pos is not None:
                gap = q_pos[rows].astype(np.int64)[:, None] - kp[None]
        for j in range(h):
            op, add = opened, np.zeros((n, m))
            if bias is not None:
                bk = bucket_of(gap, bounds)
                add = bias[bk, j]
                op = opened & (add > -2.0**100)
                add = np.where(op, add, 0)
            qq = q[rows, j]
            kk, vv = (np.where(op.any(0)[:, None], x[keys, j // g], 0) for x in (k, v))
            s = np.where(op, qq @ kk.T * scale + add, -np.inf)
            top = s.max(1, keepdims=True)
            top = np.where(np.isinf(top), 0, top)
            p = np.where(op, np.exp(s - top), 0)
            total = p.sum(1, keepdims=True)
            with np.errstate(divide="ignore"):
                lse = np.log(total) + top
            p = p / np.where(total == 0, 1, total)
            ab = np.abs(qq) @ np.abs(kk).T * abs(scale) + np.abs(add)
            e = W * ((dim + 8) * ab + 4 * (np.abs(np.where(total == 0, 0, lse)) + np.abs(top)) + m + 16)
            out["lse"][rows, j] = lse[:, 0]
            far["lse"][rows, j] = np.where(op, e, 0).max(1)
            o, pe = p @ vv, p * (e + u + m * W)
            out["o"][rows, j] = o
            far["o"][rows, j] = u * np.abs(o) + pe @ np.abs(vv)
            if do is None:
                continue
            d = do[rows, j]
            dp = d @ vv.T
            dd = (p * dp).sum(1, keepdims=True)
            ds = p * (dp - dd)
            dab = np.abs(d) @ np.abs(vv).T
            a = (p * dab).sum(1, keepdims=True)
            e_d = (p * (e + (dim + m) * W) * dab).sum(1, keepdims=True) + (2 * W * a if u == W else 0)
            e_ds = np.abs(ds) * (u + e) + p * (dim * W * dab + e_d + 2 * W * (np.abs(dp) + np.abs(dd)))
            gs = n * g
            out["dq"][rows, j] = ds @ kk * scale
            far["dq"][rows, j] = (e_ds + m * W * np.abs(ds)) @ np.abs(kk) * abs(scale)
            out["dk"][keys, j // g] += ds.T @ qq * scale
            far["dk"][keys, j // g] += (e_ds + gs * W * np.abs(ds)).T @ np.abs(qq) * abs(scale)
            out["dv"][keys, j // g] += p.T @ d
            far["dv"][keys, j // g] += (pe + gs * W * p).T @ np.abs(d)
            if bias is not None:
                # ds unrounded
                e_ds = np.abs(ds) * e + p * (dim * W * dab + e_d + 2 * W * (np.abs(dp) + np.abs(dd)))
                np.add.at(out["dbias"][:, j], bk.reshape(-1), ds.reshape(-1))
                np.add.at(far["dbias"][:, j], bk.reshape(-1), (e_ds + 256 * W * np.abs(ds)).reshape(-1))
    for name in ("dq", "dk", "dv", "dbias"):
        if name in out:
            far[name] += u * np.abs(out[name])
    return out, far
