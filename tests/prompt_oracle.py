"""Plain implementations, in 64 bits on the CPU, of the operators of scoring and prefilling prompts."""
import numpy as np

import tree_oracle


def norm(x, gain, bias, layer, eps):
    """x [rows, heads, hd]; gain and bias (or None) [hd] or [heads, hd] -> (y, the normalised x)"""
    x = np.asarray(x, dtype=np.float64)
    d = x - x.mean(axis=-1, keepdims=True) if layer else x
    z = d / np.sqrt((d * d).mean(axis=-1, keepdims=True) + eps)
    return z * gain + (0.0 if bias is None else bias), z


def attention(q, k, v, scale):
    """q [n, H, hd], k and v [T, Hkv, hd]: query i sees keys 0 .. i + T - n -> (out, sum of p |v|, largest sum of |q k| scale).  All finite."""
    n, H, hd = q.shape
    T, group = len(k), H // k.shape[1]
    out, size, dot = np.zeros((n, H, hd)), np.zeros((n, H, hd)), 0.0
    sees = np.arange(T)[None] <= np.arange(n)[:, None] + T - n
    some = sees.any(axis=1)
    for h in range(H if T and some.any() else 0):
        kk, vv = k[:, h // group], v[:, h // group]
        s = np.where(sees[some], q[some, h] @ kk.T * scale, -np.inf)
        w = np.exp(s - s.max(axis=1, keepdims=True))
        w /= w.sum(axis=1, keepdims=True)
        out[some, h], size[some, h] = w @ vv, w @ np.abs(vv)
        dot = max(dot, float((np.abs(q[:, h]) @ np.abs(kk).T).max()) * scale)
    return out, size, dot


def attention_wild(q, k, v, scale):
    """The same row by row, for keys and values that are infinite or NaN: what a query does not see is not touched."""
    n, T = len(q), len(k)
    return tree_oracle.attention(q, k, v, np.arange(T)[None] <= np.arange(n)[:, None] + T - n, scale)


def logprobs(z, tokens, n_top):
    """z [rows, V] -> dict of logprob, rank, entropy, ids, top; ln_s (log of the sum about the maximum), dist (sum p |z - max|)"""
    z = np.asarray(z, dtype=np.float64)
    rows, V = z.shape
    r = dict(logprob=np.full(rows, -np.inf), rank=np.full(rows, -1), entropy=np.zeros(rows), ids=np.full((rows, n_top), -1), top=np.full((rows, n_top), -np.inf),
             ln_s=np.zeros(rows), dist=np.zeros(rows), best=np.zeros(rows))
    for i in range(rows):
        known = 0 <= tokens[i] < V
        x = z[i]
        if known:
            r["rank"][i] = (x > x[tokens[i]]).sum() + (x[:tokens[i]] == x[tokens[i]]).sum()
        if np.isnan(x).any() or (x == np.inf).any():
            for n in ("logprob", "entropy", "top"):
                r[n][i] = np.nan
            continue
        m = x.max()
        if m == -np.inf:
            continue
        d = x - m
        e = np.exp(d)
        ln_s, far = np.log(e.sum()), np.where(e > 0, e * np.where(e > 0, d, 0.0), 0.0).sum() / e.sum()
        r["ln_s"][i], r["dist"][i], r["best"][i] = ln_s, -far, m
        r["entropy"][i] = ln_s - far
        if known:
            r["logprob"][i] = d[tokens[i]] - ln_s
        order = np.argsort(-x, kind="stable")[:n_top]
        order = order[x[order] > -np.inf]
        r["ids"][i, :len(order)], r["top"][i, :len(order)] = order, d[order] - ln_s
    return r
