"""The paged token cache's oracle: its plan against rules that any plan has to keep, its attention against
torch's."""
import numpy as np
import pytest
import torch

from oracle import pcache as op


def held_rows(pages, lens):
    return [[(row[j // pages.R], j % pages.R) for j in range(n)] for row, n in zip(pages.table, lens)]


@pytest.mark.parametrize("seed", range(30))
def test_steps_keep_what_items_hold(seed):
    """Rows written by one item are read back by it and by who goes on from it, and by no other."""
    rng = np.random.default_rng(seed)
    B, R, M = int(rng.integers(1, 9)), int(rng.choice([8, 16])), int(rng.integers(1, 6))
    P = int(rng.integers(1, B * M + 3))
    pages, mem, lens, text = op.Pages([[] for _ in range(B)], P, R, M), {}, [0] * B, [[] for _ in range(B)]
    for turn in range(20):
        src = [int(x) for x in rng.integers(0, B, B)] if turn % 2 else None
        frm = src or list(range(B))
        keep = [int(rng.integers(0, lens[s] + 1)) if rng.random() < 0.5 else lens[s] for s in frm]
        n = int(rng.integers(0, 2 * R))
        granted, copies = pages.step(src, keep, None if turn % 5 == 0 else [int(x) for x in rng.integers(0, n + 1, B)], n)
        for a, z, rows in copies:
            for r in range(rows):
                mem[z, r] = mem.get((a, r))
        text = [text[s][:h] for s, h in zip(frm, keep)]
        for b in range(B):
            for i in range(granted[b]):
                j = keep[b] + i
                mem[pages.table[b][j // R], j % R] = (turn, b, i)
                text[b].append((turn, b, i))
        lens = [h + m for h, m in zip(keep, granted)]
        if turn % 3 == 2:
            L, moves = pages.compact()
            for a, z, rows in moves:
                for r in range(rows):
                    mem[z, r] = mem.get((a, r))
            assert sorted({p for row in pages.table for p in row}) == list(range(L))
        for b in range(B):
            assert [mem[x] for x in held_rows(pages, lens)[b]] == text[b]


def test_last_writer_keeps_the_page():
    p = op.Pages([[0, 1], [], []], 6, 8, 4)
    granted, copies = p.step([0, 0, 0], [11, 11, 11], [1, 1, 1], 1)
    assert granted == [1, 1, 1] and copies == [(1, 2, 8), (1, 3, 8)] and p.table == [[0, 2], [0, 3], [0, 1]]
    # not where an item that writes nothing holds it too
    p = op.Pages([[0, 1], [], []], 6, 8, 4)
    _, copies = p.step([0, 0, 0], [11, 11, 11], [1, 0, 1], 1)
    assert copies == [(1, 2, 8), (1, 3, 8)] and p.table == [[0, 2], [0, 1], [0, 3]]
    # nor where there is no page to copy to
    p = op.Pages([[0, 1], [], []], 3, 8, 4)
    granted, copies = p.step([0, 0, 0], [11, 11, 11], [9, 9, 9], 9)
    assert granted == [5, 0, 0] and copies == [(1, 2, 8)] and p.table == [[0, 2], [0, 1], [0, 1]]


@pytest.mark.parametrize("H,kv,masked", [(4, 2, False), (6, 2, True), (3, 3, True)])
def test_attention_is_torchs(H, kv, masked):
    g = torch.Generator().manual_seed(H)
    held, m, hd = 13, 5, 16
    k, v = (torch.randn(kv, held + m, hd, generator=g, dtype=torch.float64) for _ in range(2))
    q = torch.randn(m, H, hd, generator=g, dtype=torch.float64)
    shown = torch.rand(held + m, generator=g) > 0.3 if masked else torch.ones(held + m, dtype=torch.bool)
    shown[0] = True
    see = (torch.arange(held + m) <= held + torch.arange(m)[:, None]) & shown
    want = torch.nn.functional.scaled_dot_product_attention(q.transpose(0, 1), k.repeat_interleave(H // kv, 0), v.repeat_interleave(H // kv, 0), see, scale=0.3)
    got, absv, mass = op.attention(k.numpy(), v.numpy(), q.numpy(), held, 0.3, shown.numpy())
    np.testing.assert_allclose(got, want.transpose(0, 1).numpy(), rtol=0, atol=1e-13)
    assert (absv >= np.abs(got) - 1e-12).all() and (mass > 0).all()


def test_attention_without_a_visible_row_is_zero():
    x = np.full((1, 4, 8), np.nan)
    got, _, _ = op.attention(x, x, np.ones((2, 2, 8)), 2, 1.0, np.zeros(4))
    assert (got == 0).all()
