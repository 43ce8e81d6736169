"""The paged token cache at the ends of its ranges: tables that were written by hand, the smallest and the
largest numbers."""
import numpy as np
import pytest
import torch

from oracle import pcache as op
from tests.test_gpu_pcache import (HEADS, as_lists, ctx, f64, fc, fill_table, ints, item_rows, moved, plain, pool, randn,  # noqa: F401
                                   run_step)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------ pages
def compact(fc, ctx, caches):  # noqa: F811
    """A compaction against the oracle; entries that are no page stay as they are."""
    state, R = caches[0].pages, caches[0].k.shape[2]
    pages, table = op.Pages(as_lists(state), state.n_pages, R, state.max_pages), state.table.tolist()
    before = [plain(c) for c in caches]
    live = torch.full((1,), -5, dtype=torch.int32, device="cuda")
    fc.fc_pcache_compact(ctx, caches, live)
    torch.cuda.synchronize()
    L, moves = pages.compact()
    assert live.item() == L
    assert state.table.tolist() == [[x if p is None else p for p, x in zip(*rows)] for rows in zip(pages.table, table)]
    assert state.holders.tolist() == pages.holders()
    for c, (k, v) in zip(caches, before):
        k2, v2 = plain(c)
        assert torch.equal(k2, moved(k, moves, R)) and torch.equal(v2, moved(v, moves, R)), "rows moved"
    return len(moves)


@pytest.mark.parametrize("B,M,P", [(3, 5, 40), (2, 4, 7200)])
def test_compaction_of_a_table_written_by_hand(fc, ctx, B, M, P):  # noqa: F811
    """Entries that no step has counted are held all the same, whatever the holders' counts say: a page that the
    table names is not written over, and one that it does not name is free.  A pool whose counts a
    workgroup holds in LDS, and a larger one."""
    g = torch.Generator().manual_seed(P)
    R, kv, hd = 16, 1, 64
    state = fc.PageState.alloc(B, M, P)
    caches = [pool(g, state, kv, hd, R, fc) for _ in range(2)]
    run_step(fc, ctx, caches, None, [0] * B, [R * 3] * B, R * 3)
    # pages named by hand, some of them twice, and entries that are no page
    state.table[0, 0], state.table[0, 3], state.table[1, 3], state.table[1, 0] = P - 1, P - 3, P - 3, P
    state.table[B - 1, 1] = -9
    assert compact(fc, ctx, caches) > 0
    state.holders.copy_(torch.arange(P, dtype=torch.int32, device="cuda") % 3 - 1)
    state.table[0, 1] = P // 2
    assert compact(fc, ctx, caches) == 1
    state.table.fill_(-1)
    assert compact(fc, ctx, caches) == 0


# ------------------------------------------------------------------------------ numbers
FORMS = [("qwen", 1), ("one", 20), ("one", 40), ("three", 60)]    # few rows in one and in two tiles; many, in two waves and in four


@pytest.mark.parametrize("heads,n", FORMS)
@pytest.mark.parametrize("L", [0, 30, 700])
def test_small_values(fc, ctx, heads, n, L):  # noqa: F811
    """Values towards bfloat16's smallest.  A held probability is at least 2^-25 of the token's largest in one place, and
    what leaves float32 at its lower end is below 2^-126 for each row that is seen: 2^-101 of an output, and
    as much again where parts are joined."""
    H, kv, hd, _ = HEADS[heads]
    g = torch.Generator().manual_seed(n + L)
    R, rows = 64, L + n
    state = fc.PageState.alloc(1, op.pages_of(rows, R), 40)
    fill_table(state, [rows], R, g)
    cache = pool(g, state, kv, hd, R, fc)
    q = randn(g, 1, n, H, hd)
    out = torch.zeros_like(q)
    v = cache.v.clone()
    for e in (60, 80, 95, 105, 126, 130):
        cache.v.copy_((v.double() * 2.0 ** -e).to(torch.bfloat16))
        fc.fc_pcache_attention(ctx, cache, q, ints([L]), None, out)
        torch.cuda.synchronize()
        kk, vv, there = item_rows(cache, 0)
        want, absv, mass = op.attention(kk[:, :rows], vv[:, :rows], f64(q[0]), L, hd ** -0.5, there[:rows])
        rel = 4 * (hd + 4) * 2.0 ** -24 * mass + 2.0 ** -22 + rows * 2.0 ** -24
        # the sum of rounded probabilities (many rows) errs by up to 2^-8 of the output besides
        tol = 2 * 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + rel)[..., None] * absv + rows * 2.0 ** -100
        assert (np.abs(f64(out[0]) - want) <= tol).all(), e


@pytest.mark.parametrize("heads,n", FORMS)
@pytest.mark.parametrize("L", [0, 30, 700, 5000])
def test_mean_of_equal_values(fc, ctx, heads, n, L):  # noqa: F811
    """With more than 32 rows of a head the probabilities are added up as they enter the product, so that the mean of
    equal numbers is that number: both sums err by less than (rows + 64) 2^-23, far from half a step of 2^-9.
    With fewer the sum is of unrounded ones, and rounding them shows: 2^-8, and that of the output."""
    H, kv, hd, _ = HEADS[heads]
    g = torch.Generator().manual_seed(n + L)
    R = 64
    state = fc.PageState.alloc(1, op.pages_of(L + n, R), 100)
    fill_table(state, [L + n], R, g)
    cache = pool(g, state, kv, hd, R, fc)
    q, mean = randn(g, 1, n, H, hd), randn(g, kv, hd)
    cache.v.copy_(mean[:, None, :, None].expand_as(cache.v[0]))
    out = torch.zeros_like(q)
    fc.fc_pcache_attention(ctx, cache, q, ints([L]), None, out)
    torch.cuda.synchronize()
    want = mean.repeat_interleave(H // kv, 0).expand_as(out[0])
    if n * H // kv > 32:
        assert torch.equal(out[0], want)
    else:
        np.testing.assert_allclose(f64(out[0]), f64(want), rtol=2.01 * 2.0 ** -8)


@pytest.mark.parametrize("heads,n", FORMS[1:])
def test_scores_beyond_float32(fc, ctx, heads, n):  # noqa: F811
    """One token's scores leave float32: its outputs are not finite, the others' the same bytes as ever."""
    H, kv, hd, _ = HEADS[heads]
    g = torch.Generator().manual_seed(n)
    R, L = 64, 200
    state = fc.PageState.alloc(1, op.pages_of(L + n, R), 8)
    table = fill_table(state, [L + n], R, g)
    cache = pool(g, state, kv, hd, R, fc)
    q = randn(g, 1, n, H, hd)
    q[0, 3, :H // kv] = (cache.k[table[0][1], 0, 5].sign() * 3e38).bfloat16()      # the first key-value head's
    bad = torch.zeros(n, H, dtype=torch.bool, device="cuda")
    bad[3, :H // kv] = True
    want, got = torch.zeros_like(q), torch.zeros_like(q)
    fc.fc_pcache_attention(ctx, cache, q, ints([L]), None, got)
    fc.fc_pcache_attention(ctx, cache, torch.where(bad[None, :, :, None], 1.0, q), ints([L]), None, want)
    torch.cuda.synchronize()
    assert not torch.isfinite(got[0][bad]).any()
    assert torch.isfinite(want).all() and torch.equal(got[0][~bad], want[0][~bad])
