"""Oracle of the paged token cache (numpy): the pages' plan, item by item and page by page, and attention
over an item's rows in 64 bits.

A pool is [n_pages, n_kv, page_rows, hd] with plain rows, for keys and values alike; a table is a list of
lists of pages (None: no page) of the items' rows.
"""
from __future__ import annotations

import numpy as np

from oracle.qcache import rotate  # noqa: F401  (the rotary positions are the 8-bit cache's)

TILE = 8


def pages_of(rows: int, page_rows: int) -> int:
    return -(-rows // page_rows)


class Pages:
    """Table and holders of the items, and the rows that a plan copies or moves."""

    def __init__(self, table, n_pages: int, page_rows: int, max_pages: int):
        self.table = [[p if p is not None and 0 <= p < n_pages else None for p in row] for row in table]
        self.P, self.R, self.M = n_pages, page_rows, max_pages

    def holders(self) -> list:
        n = [0] * self.P
        for row in self.table:
            for p in row:
                if p is not None:
                    n[p] += 1
        return n

    def step(self, src, lens, new, n: int):
        """(granted, [(from, to, rows)])."""
        R, cap, B = self.R, self.M * self.R, len(lens)
        lens = [min(max(x, 0), cap) for x in lens]
        src = list(range(B)) if src is None else src
        lens = [h if 0 <= s < B else 0 for s, h in zip(src, lens)]
        new = [min(n if new is None else min(max(new[b], 0), n), cap - lens[b]) for b in range(B)]
        old = [row + [None] * (self.M - len(row)) for row in self.table]
        self.table = [old[s][:pages_of(h, R)] if h else [] for s, h in zip(src, lens)]
        held = self.holders()
        free = [p for p in range(self.P) if held[p] == 0]
        granted, copies = [0] * B, []
        for b, (h, m) in enumerate(zip(lens, new)):
            row, into = self.table[b], h % R > 0 and m > 0
            if into and row[-1] is None:
                continue
            if into and held[row[-1]] > 1:
                if not free:
                    continue
                to = free.pop(0)
                held[row[-1]] -= 1
                held[to] += 1
                copies.append((row[-1], to, pages_of(h % R, TILE) * TILE))
                row[-1] = to
            while len(row) < pages_of(h + m, R) and free:
                held[free[0]] += 1
                row.append(free.pop(0))
            granted[b] = min(m, len(row) * R - h)
        return granted, copies

    def compact(self):
        """(live pages, [(from, to, rows)])."""
        held = self.holders()
        live = [p for p in range(self.P) if held[p]]
        L = len(live)
        moves = dict(zip([p for p in live if p >= L], [p for p in range(L) if not held[p]]))
        self.table = [[moves.get(p, p) for p in row] for row in self.table]
        return L, [(a, z, self.R) for a, z in moves.items()]


def attention(k, v, q, held: int, scale: float, shown):
    """k, v [n_kv, rows, hd], q [m, n_heads, hd], shown [rows] (mask and pages): outputs [m, n_heads, hd],
    and for each output sum_j P_ij |v_j| and for each row max_j |scale| sum_d |q_d k_d|."""
    n_kv, rows, hd = k.shape
    m, H = q.shape[:2]
    G = H // n_kv
    out, absv, mass = np.zeros((m, H, hd)), np.zeros((m, H, hd)), np.zeros((m, H))
    for h in range(H):
        kk, vv, qq = k[h // G], v[h // G], q[:, h]
        see = (np.arange(rows) <= held + np.arange(m)[:, None]) & (np.asarray(shown) != 0)
        s = np.where(see, qq @ np.where(see.any(0)[:, None], kk, 0).T * scale, -np.inf)
        top = s.max(-1, keepdims=True, initial=-np.inf)
        p = np.where(see, np.exp(s - np.where(np.isfinite(top), top, 0)), 0)
        p /= np.maximum(p.sum(-1, keepdims=True), 1e-300)
        vv = np.where(see.any(0)[:, None], vv, 0)
        out[:, h], absv[:, h] = p @ vv, p @ np.abs(vv)
        kq = np.where(see, np.abs(qq) @ np.where(see.any(0)[:, None], np.abs(kk), 0).T, 0)
        mass[:, h] = abs(scale) * kq.max(-1, initial=0)
    return out, absv, mass
