"""Oracle of the 8-bit token cache (float64, numpy): append, attention, eviction of one item.

A cache item is a dict of k, v [n_kv, capacity, hd] (the codes' own values, before the scale),
k_scale, v_scale [n_kv, capacity / 64] and weight [n_kv, capacity].  Rows are plain rows here;
the library's value layout (columns of a block) is undone by the tests.
"""
from __future__ import annotations

import numpy as np

BLOCK = 64
TOP = 448.0
LOW_EXP = -100


def e4m3(x: np.ndarray) -> np.ndarray:
    """The e4m3 number nearest to x (ties to the even mantissa); beyond 448 it is 448 (also
    for an infinity), a NaN stays one."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(x), TOP)                       # NaN passes
    _, e = np.frexp(np.where(a > 0, a, 1.0))             # a = m 2^e, m in [1/2, 1)
    step = np.exp2(np.maximum(e - 1, -6) - 3.0)          # 3 mantissa bits; subnormals below 2^-6
    return np.copysign(np.rint(a / step) * step, x)


def block_scale(amax: float) -> float:
    """Smallest power of two s >= 2^-100 with amax <= 448 s."""
    e = LOW_EXP
    if amax > 0:
        e = max(LOW_EXP, int(np.floor(np.log2(amax / TOP))) - 1)
        while TOP * 2.0 ** e < amax:
            e += 1
    return 2.0 ** e


def finite_amax(x: np.ndarray) -> float:
    a = np.abs(x[np.isfinite(x)])
    return float(a.max()) if a.size else 0.0


def rotate(x: np.ndarray, pos: np.ndarray, section, theta: float) -> np.ndarray:
    """Rotary positions of rows x [n, heads, hd]; pos [axes, n]."""
    hd = x.shape[-1]
    half = hd // 2
    axis = np.repeat(np.arange(3), section) if any(section) else np.zeros(half, np.int64)
    ang = np.asarray(pos, np.float64)[axis].T * theta ** (-2.0 * np.arange(half) / hd)
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = x[..., :half].astype(np.float64), x[..., half:].astype(np.float64)
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def dequant(cache: dict, name: str) -> np.ndarray:
    return cache[name] * np.repeat(cache[name + "_scale"], BLOCK, -1)[..., None]


def append(cache: dict, k: np.ndarray, v: np.ndarray, held: int) -> dict:
    """The cache after rows k (rotated), v [m, n_kv, hd] behind the `held` ones."""
    out = {n: t.copy() for n, t in cache.items()}
    cap = cache["k"].shape[1]
    m = min(k.shape[0], cap - held)
    for h in range(cache["k"].shape[0]):
        for name, x in (("k", k), ("v", v)):
            code, scale = out[name][h], out[name + "_scale"][h]
            for b in range(held // BLOCK, -(-(held + m) // BLOCK)):
                lo, hi = max(held, b * BLOCK), min(held + m, (b + 1) * BLOCK)
                if hi <= lo:
                    continue
                new = x[lo - held:hi - held, h]
                s = block_scale(finite_amax(new))
                if lo > b * BLOCK:
                    s = max(s, scale[b])
                    if s > scale[b]:
                        code[b * BLOCK:lo] = e4m3(code[b * BLOCK:lo] * (scale[b] / s))
                code[lo:hi] = e4m3(new / s)
                scale[b] = s
        out["weight"][h, held:held + m] = 0
    return out


def attention(k: np.ndarray, v: np.ndarray, q: np.ndarray, held: int, scale: float, mask=None):
    """k, v [n_kv, rows, hd] (dequantised), q [m, n_heads, hd]: the outputs [m, n_heads, hd], the
    probabilities [m, n_heads, rows], and for each output sum_j P_ij |v_j| and for each row
    max_j |scale| sum_d |q_d k_d| (what bounds the rounding errors)."""
    n_kv, rows, hd = k.shape
    m, H = q.shape[:2]
    G = H // n_kv
    out, prob = np.zeros((m, H, hd)), np.zeros((m, H, rows))
    absv, mass = np.zeros((m, H, hd)), np.zeros((m, H))
    for i in range(m):
        see = np.arange(rows) <= held + i
        if mask is not None:
            see &= np.asarray(mask[:rows]) != 0
        j = np.flatnonzero(see)
        if j.size == 0:
            continue
        for h in range(H):
            kk, vv, qq = k[h // G, j], v[h // G, j], q[i, h].astype(np.float64)
            s = kk @ qq * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            prob[i, h, j] = p
            out[i, h] = p @ vv
            absv[i, h] = p @ np.abs(vv)
            mass[i, h] = abs(scale) * float((np.abs(kk) @ np.abs(qq)).max())
    return out, prob, absv, mass


def group_weight(prob: np.ndarray, n_kv: int) -> np.ndarray:
    """Probabilities [m, H, rows] added up over tokens and each group's heads: [n_kv, rows]."""
    m, H, rows = prob.shape
    return prob.reshape(m, n_kv, H // n_kv, rows).sum((0, 2))


def kept_rows(w: np.ndarray, n: int, keep: int, sink: int, recent: int) -> np.ndarray:
    """Rows of one head that stay, ascending (equal weights: the lower row)."""
    if n <= keep:
        return np.arange(n)
    low = np.finfo(np.float32).min
    x = np.array([v if v >= low else low for v in w[:n].astype(np.float64)])
    mid = sorted(range(sink, n - recent), key=lambda j: (-x[j], j))[:keep - sink - recent]
    return np.array(sorted(list(range(sink)) + mid + list(range(n - recent, n))), np.int64)


def evict(cache: dict, dst: dict, n: int, keep: int, sink: int, recent: int):
    """(dst with the kept rows, kept rows [n_kv, left])."""
    out = {x: t.copy() for x, t in dst.items()}
    kept = []
    for h in range(cache["k"].shape[0]):
        rows = kept_rows(cache["weight"][h], n, keep, sink, recent)
        kept.append(rows)
        for name in ("k", "v"):
            val = cache[name][h, rows] * cache[name + "_scale"][h, rows // BLOCK][:, None]
            for b in range(-(-rows.size // BLOCK)):
                x = val[b * BLOCK:(b + 1) * BLOCK]
                s = block_scale(finite_amax(x))
                out[name][h, b * BLOCK:b * BLOCK + len(x)] = e4m3(x / s)
                out[name + "_scale"][h, b] = s
        out["weight"][h, :rows.size] = cache["weight"][h, rows]
    return out, np.array(kept)
