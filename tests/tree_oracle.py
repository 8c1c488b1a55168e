"""Plain implementations, in 64 bits on the CPU, of the operators of a step of tree speculation."""
import math

import numpy as np


def fp8_store(x):
    """What an fp8 cache holds for rows x (float, last dimension = one head): codes times a power of two.  NaN for what is not finite."""
    x = np.asarray(x, dtype=np.float64)
    finite = np.isfinite(x)
    top = np.where(finite, np.abs(x), 0.0).max(axis=-1, keepdims=True)
    m, e = np.frexp(top)
    e = np.where(top > 0, np.clip(np.where(m <= 0.875, e - 9, e - 8), -100, 119), -100)
    y = np.clip(np.where(finite, x, 0.0) * np.ldexp(1.0, -e), -448.0, 448.0)
    step = np.ldexp(1.0, np.maximum(np.frexp(y)[1] - 1, -6) - 3)       # three bits behind the leading one; 2^-9 for the smallest
    code = np.rint(y / step) * step
    return np.where(finite, np.ldexp(code, e), np.nan)


def bf16_store(x):
    import torch
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).bfloat16().double().numpy()


def store(kind, x):
    return fp8_store(x) if kind == "fp8" else bf16_store(x) if kind == "bf16" else np.asarray(x, dtype=np.float64)


def frequencies(r, theta=10000.0, scaling="none", factor=1.0, trained=0.0, low=1.0, high=32.0):
    if scaling == "base":
        theta = theta * factor ** (r / (r - 2))
    f = [theta ** (-2.0 * i / r) for i in range(r // 2)]
    if scaling == "linear":
        f = [x / factor for x in f]
    if scaling == "parts":
        out = []
        for x in f:
            g = min(max((trained * x / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
            out.append(x * (g + (1 - g) / factor))
        f = out
    return np.array(f)


def rotary(x, positions, f, interleaved, magnitude=1.0):
    """x [rows, heads, hd] float64 -> (turned, |a| + |b| of every element's pair: what roundings scale with)."""
    x = np.asarray(x, dtype=np.float64)
    r = 2 * len(f)
    a, b = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    angle = np.asarray(positions, dtype=np.float64)[:, None, None] * f
    y, size = x.copy(), np.zeros_like(x)
    y[..., a] = magnitude * (x[..., a] * np.cos(angle) - x[..., b] * np.sin(angle))
    y[..., b] = magnitude * (x[..., b] * np.cos(angle) + x[..., a] * np.sin(angle))
    size[..., a] = size[..., b] = magnitude * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y, size


def attention(q, k, v, sees, scale):
    """q [n, H, hd], k and v [T, Hkv, hd], sees [n, T] -> (out, sum of p |v|, largest sum of |q k| scale).  What a row does not see is not
    touched; a row that sees nothing is 0."""
    n, H, hd = q.shape
    group = H // k.shape[1]
    out, size, dot = np.zeros((n, H, hd)), np.zeros((n, H, hd)), 0.0
    for i in range(n):
        t = np.flatnonzero(sees[i])
        if not len(t):
            continue
        for h in range(H):
            kk, vv = k[t, h // group], v[t, h // group]
            s = kk @ q[i, h] * scale
            w = np.exp(s - s.max())
            w /= w.sum()
            # a probability is never 0: exp(-800) underflows even in 64 bits, and 0 * inf would be NaN where the formula's p * inf is inf
            w = np.maximum(w, 5e-324)
            with np.errstate(invalid="ignore"):
                out[i, h] = w @ vv
            size[i, h] = w @ np.abs(np.where(np.isfinite(vv), vv, 0.0))
            dot = max(dot, float((np.abs(kk) @ np.abs(q[i, h])).max()) * scale)
    return out, size, dot


def ancestors(parents):
    n = len(parents)
    m = np.zeros((n, n), dtype=bool)
    for i in range(n):
        j = i
        while j >= 0:
            m[i, j] = True
            j = parents[j]
    return m


def pack_mask(sees, words):
    """bool [n, nodes] -> uint32 [n, words]"""
    n, m = sees.shape
    out = np.zeros((n, words), dtype=np.uint32)
    for i in range(n):
        for j in np.flatnonzero(sees[i]):
            if j < 32 * words:
                out[i, j // 32] |= np.uint32(1 << (j % 32))
    return out


def random_tree(rng, n, branch=3):
    parents, children = [-1], [0]
    while len(parents) < n:
        j = int(rng.choice([i for i in range(len(parents)) if children[i] < branch]))
        children[j] += 1
        parents.append(j)
        children.append(0)
    return parents[:n]


def _weights(rho):
    return np.trunc(np.minimum(rho, 1.0) * 2.0 ** 44)


def verify(tokens, parents, p, q, words, draw, max_path):
    """One sequence -> (path, next token): Python floats and integers, in the order of the definition."""
    n, V = len(tokens), p.shape[1]
    if n == 0:
        return [], -1
    path = [0]
    while True:
        at = path[-1]
        base = np.where(p[at].astype(np.float64) > 0, p[at].astype(np.float64), 0.0)
        rho, mass, step = base.copy(), 1.0, None
        for i in [j for j in range(at + 1, n) if parents[j] == at] if len(path) < max_path else []:
            x = int(tokens[i])
            r = (float(int(words[i]) & 0xFFFFFFFF) + 0.5) * 2.0 ** -32
            inside = 0 <= x < V
            if inside and r * (float(q[at, x]) if q is not None else 1.0) * mass < rho[x]:
                step = i
                break
            if q is not None:
                rho = rho - mass * q[at].astype(np.float64)
                rho = np.where(rho > 0, rho, 0.0)
            elif inside:
                rho[x] = 0.0
            mass = float(sum(int(w) for w in _weights(rho))) * 2.0 ** -44
        if step is None:
            break
        path.append(step)
    w = [int(y) for y in _weights(rho)]
    if sum(w) == 0:
        w = [int(y) for y in _weights(base)]
    if sum(w) == 0:
        return path, -1
    t = ((int(draw) & 0xFFFFFFFFFFFFFFFF) * sum(w)) >> 64
    c = 0
    for i, y in enumerate(w):
        c += y
        if c > t:
            return path, i
