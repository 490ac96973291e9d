"""Attention over windows with sinks and over trees, from the definitions, in numpy and 64 bits (no code of the library)."""
import math

import numpy as np


def ancestors(parents, i):
    """Row i and the rows above it, nearest first."""
    path = [i]
    while 0 <= parents[path[-1]] < path[-1]:
        path.append(int(parents[path[-1]]))
    return path


def depths(parents):
    return np.array([len(ancestors(parents, i)) - 1 for i in range(len(parents))], dtype=np.int64)


def sees_chain(t, n, window, sinks):
    """[n][t + n] truth values: step t + i sees key j."""
    j, p = np.arange(t + n), t + np.arange(n)[:, None]
    seen = j <= p
    return seen & ((j > p - window) | (j < sinks)) if window else seen


def sees_tree(t, parents, window, sinks):
    n, d = len(parents), depths(parents)
    seen = np.zeros((n, t + n), dtype=bool)
    for i in range(n):
        p = t + d[i]
        j = np.arange(t)
        seen[i, :t] = (j > p - window) | (j < sinks) if window else True
        for a in ancestors(parents, i):
            seen[i, t + a] = not window or d[i] - d[a] < window or t + d[a] < sinks
    return seen


def attention(q, K, V, seen, scale=None):
    """q [n][Hq][D], K, V [T][Hkv][D], seen [n][T]: (answers [n][Hq][D], sum p |v| / sum p).  Rows that nobody sees may hold anything."""
    n, Hq, D = q.shape
    Hkv = K.shape[1]
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    some = seen.any(0)
    K, V, seen = K[some], V[some], seen[:, some]
    out, size = np.zeros((n, Hq, D)), np.zeros((n, Hq, D))
    G = Hq // Hkv
    for h in range(Hkv):
        x = np.einsum("ngd,td->ngt", q[:, h * G:(h + 1) * G], K[:, h]) * scale
        x = np.where(seen[:, None], x, -np.inf)
        w = np.exp(x - x.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        out[:, h * G:(h + 1) * G], size[:, h * G:(h + 1) * G] = w @ V[:, h], w @ np.abs(V[:, h])
    return out, size


def within(got, out, size):
    """Rounding the weights to bf16 moves the numerator by at most 2^-8 size and the sum by 2^-8 of itself, rounding the answer is
    2^-8 |out| more; 3% of it for sums and exponentials in fp32."""
    bound = 1.03 * 2.0 ** -8 * (size + 2 * np.abs(out)) + 1e-30
    worst = np.max(np.abs(got - out) / bound) if out.size else 0.0
    assert not np.isnan(got).any() and worst <= 1.0, f"{worst:.3f} of the bound at {np.unravel_index(np.argmax(np.abs(got - out) / bound), out.shape)}"


def within_fp32(got, out, size, q, K, turns=0):
    """A logit of D products: D + 4 roundings of at most sum |q k| <= |q| |k| each, scale and log2 e among them; its weight is off by as much,
    and by 4 steps more for the power of two and the running maximum.  Sums over T keys: T/4 + 64 additions of four products, and a product by
    a power of two for each group of 32 keys.  Rows that were turned in fp32 (turns: of queries 1, of keys too 2): a product and a fused
    multiply-add of a pair, against one rounding: 3 roundings of at most sqrt(2) of it.  Numerator and sum are each off by that part of themselves; one division."""
    T, D = K.shape[0], K.shape[-1]
    norms = np.sqrt((q ** 2).sum(-1)).max() * np.sqrt(np.nanmax((K ** 2).sum(-1))) / math.sqrt(D)
    part = 2.0 ** -24 * ((D + 4 + 4.3 * turns) * norms + 8 + T / 4 + 64 + T / 8)
    bound = 1.03 * (part * (size + np.abs(out)) + 2.0 ** -24 * np.abs(out)) + 1e-37
    assert not np.isnan(got).any() and (np.abs(got - out) <= bound).all(), f"{np.max(np.abs(got - out) / bound):.3f} of the bound"


def turned(x, cos, sin):
    """Rows x [..., D], cosines and sines [..., D/2]."""
    half = x.shape[-1] // 2
    lo, hi = x[..., :half], x[..., half:]
    return np.concatenate([lo * cos - hi * sin, hi * cos + lo * sin], axis=-1)
