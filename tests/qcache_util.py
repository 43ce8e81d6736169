"""Between the library's 8-bit token cache and the oracle's: conversion and comparison.

Tolerances.  A rounding is off by at most half a step: 2^-8 of a bfloat16 number, 2^-4 of an e4m3
one (2^-10 of its block's scale among the subnormals), 2^-24 of a float32 one.
  * A rotated element a cos t - b sin t: the angle is reduced in 64 bits, its remainder of at most
    half a turn rounded to float32 (2^-25 turns: 2e-7 rad) and its cosine is good to a few 2^-24,
    so it is within (|a| + |b|) 2^-21.
  * A probability: the float32 sum of hd products is within hd 2^-24 sum|q k|, which the exponent
    turns into a relative error; the same for the largest exponent and for the sum of the
    probabilities, so 4 (hd + 4) 2^-24 max_j scale sum|q_d k_d| covers them, plus 2^-22 for the
    exponential, its argument's rounding and the quotient, plus 2^-24 for each of the rows that a
    sum runs over.
  * An output: that of its probabilities on sum P|v|, another 2^-8 there (P is rounded to bfloat16
    before the product with V), and 2^-8 of itself.
"""
from __future__ import annotations

import numpy as np
import torch

from oracle import qcache as oq

EMPTY = dict(k=0x11, v=0x22)     # codes that unwritten rows hold in the tests


def make(fc, B, kv, hd, cap, weight=True):
    c = fc.QCache.alloc(B, kv, hd, cap, weight=weight)
    c.k.fill_(EMPTY["k"])
    c.v.fill_(EMPTY["v"])
    c.k_scale.fill_(3.0)
    c.v_scale.fill_(5.0)
    if weight:
        c.weight.fill_(7.0)
    return c


def values(codes: torch.Tensor) -> np.ndarray:
    return codes.cpu().view(torch.float8_e4m3fn).float().numpy().astype(np.float64)


def to_oracle(c, b: int) -> dict:
    """Item b as the oracle holds it (code values in rows)."""
    kv, cap, hd = c.k.shape[1:]
    out = dict(k=values(c.k[b]), v=values(c.v[b]).transpose(0, 1, 3, 2).reshape(kv, cap, hd),
               k_scale=c.k_scale[b].cpu().numpy().astype(np.float64), v_scale=c.v_scale[b].cpu().numpy().astype(np.float64))
    if c.weight is not None:
        out["weight"] = c.weight[b].cpu().numpy().astype(np.float64)
    else:
        out["weight"] = np.zeros((kv, cap))
    return out


def same(a: np.ndarray, b: np.ndarray, what: str):
    np.testing.assert_array_equal(np.asarray(a, np.float64), np.asarray(b, np.float64), err_msg=what)


def check_appended(got: dict, before: dict, k_rows, k_slack, v_rows, held: int, m: int):
    """The cache after an append of rows k_rows [m, kv, hd] (rotated, in 64 bits; k_slack: how far
    float32 may have them off) and v_rows."""
    want = oq.append(before, k_rows, v_rows, held)
    m = min(m, before["k"].shape[1] - held)
    same(got["v"], want["v"], "value codes")
    same(got["v_scale"], want["v_scale"], "value scales")
    same(got["k_scale"], want["k_scale"], "key scales")
    same(got["weight"], want["weight"], "weights")
    new = slice(held, held + m)
    s = np.repeat(got["k_scale"], oq.BLOCK, -1)[:, new, None]
    x = np.asarray(k_rows[:m], np.float64).transpose(1, 0, 2)
    slack = np.asarray(k_slack[:m]).transpose(1, 0, 2)
    g = got["k"][:, new]
    fin = np.isfinite(x)
    off = np.abs(g * s - x)[fin]
    half = np.maximum(np.abs(x) * 2.0 ** -4, s * 2.0 ** -10) + slack
    assert (off <= half[fin]).all(), f"new keys off by {np.max(off - half[fin])}"
    same(np.isnan(g), np.isnan(x), "NaN keys")
    same(np.where(np.isinf(x), g, 0), np.where(np.isinf(x), np.copysign(448, x), 0), "infinite keys")
    rest = np.ones(g.shape[1] and got["k"].shape[1], bool)
    rest[new] = False
    same(got["k"][:, rest], want["k"][:, rest], "key codes of other rows")


def rotated(x: torch.Tensor, pos: np.ndarray, section, theta):
    """Rows [n, heads, hd] of bfloat16 rotated in 64 bits, and how far float32 may have them off."""
    y = x.float().cpu().numpy().astype(np.float64)
    half = y.shape[-1] // 2
    with np.errstate(invalid="ignore"):
        r = oq.rotate(y, pos, section, theta)
        pair = np.abs(y[..., :half]) + np.abs(y[..., half:])
    return r, np.concatenate([pair, pair], -1) * 2.0 ** -21


def check_attention(cache: dict, q: torch.Tensor, out: torch.Tensor, held: int, m: int, scale: float, mask=None,
                    before=None, after=None):
    """out [n, H, hd] of one item; before, after: its weights around an accumulating call."""
    k, v = oq.dequant(cache, "k")[:, :held + m], oq.dequant(cache, "v")[:, :held + m]
    qq = q[:m].float().cpu().numpy().astype(np.float64)
    hd = qq.shape[-1]
    with np.errstate(invalid="ignore"):
        want, prob, absv, mass = oq.attention(k, v, qq, held, scale, mask)
    rel = 4 * (hd + 4) * 2.0 ** -24 * mass + 2.0 ** -22 + (held + m) * 2.0 ** -24
    got = out[:m].float().cpu().numpy().astype(np.float64)
    same(np.isnan(got), np.isnan(want), "NaN outputs")
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + rel)[..., None] * absv
    fin = ~np.isnan(want)
    bad = (np.abs(got - want) > tol) & fin
    assert not bad.any(), f"{int(bad.sum())} outputs off, worst {np.max((np.abs(got - want) - tol)[fin])}"
    if after is not None:
        kv = k.shape[0]
        add = oq.group_weight(prob, kv)
        most = float(np.nanmax(rel, initial=0)) + m * (q.shape[1] // kv) * 2.0 ** -24
        same(after[:, held + m:], before[:, held + m:], "weights behind the last row")
        w, a = before[:, :held + m] + add, after[:, :held + m]
        same(np.isnan(a), np.isnan(w), "NaN weights")
        fin = ~np.isnan(w)
        assert (np.abs(a - w) <= most * add + 2.0 ** -24 * np.abs(w) + 1e-30)[fin].all(), "weights"
