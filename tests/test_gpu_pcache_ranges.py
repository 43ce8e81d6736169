"""The paged token cache at the ends of its ranges: tables that were written by hand, the smallest values,
and the forms of the kernels that wide tables, other numbers of heads, larger batches or more layers
reach.  Tolerances are those of tests/test_gpu_pcache.py unless a test says otherwise."""
import numpy as np
import pytest
import torch

from oracle import pcache as op
from tests.test_gpu_pcache import (HEADS, as_lists, check, ctx, f64, fc, fill_table, ints, item_rows, moved, plain,  # noqa: F401
                                   pool, randn, run_attention, run_step)

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


def test_steps_over_more_layers_than_one_launch_takes(fc, ctx):  # noqa: F811
    """Copies and moves in 70 layers: two launches, of which the second has fewer layers."""
    g = torch.Generator().manual_seed(70)
    state = fc.PageState.alloc(2, 2, 6)
    caches = [pool(g, state, 1, 64, 16, fc) for _ in range(70)]
    run_step(fc, ctx, caches, None, [0, 0], [21, 16], 32)
    run_step(fc, ctx, caches, [0, 0], [21, 19], [2, 1], 2)                  # both write the last page: one copy
    run_step(fc, ctx, caches, None, [23, 0], [0, 0], 0)                      # the lower of the two second pages is free
    assert compact(fc, ctx, caches) > 0


def test_a_state_whose_memory_has_moved(fc, ctx):  # noqa: F811
    """Calls over all layers after calls on one of them, and the rows of a table with entries that are no page."""
    g = torch.Generator().manual_seed(4)
    state = fc.PageState.alloc(2, 4, 9)
    caches = [pool(g, state, 2, 64, 16, fc) for _ in range(3)]
    for one in (0, 2):
        state.state.set_(state.state.clone())
        fc.fc_pcache_init(ctx, caches[one])
        assert run_step(fc, ctx, caches, None, [0, 0], [30, 20], 64) == [30, 20]
        run_step(fc, ctx, caches, [0, 0], [30, 30], [5, 5], 5)
        compact(fc, ctx, caches)
    state.table[0, 1], state.table[1, 0], state.table[1, 3] = 9, 2 ** 31 - 1, -2 ** 31
    for b in range(2):
        k, v, there = item_rows(caches[1], b)
        assert not there.all()
        for x, values in ((k, False), (v, True)):
            np.testing.assert_array_equal(f64(caches[1].rows(b, values)), np.where(there[:, None], x, 0))


# ------------------------------------------------------------------------------ few rows
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("heads,n", [("qwen", 1), ("qwen", 2), ("toy", 1), ("toy", 4)])
def test_short_items_in_a_wide_table(fc, ctx, heads, n, masked):  # noqa: F811
    """Table and pool beyond 384 MiB of rows, of which a few pages are held: the loads that pass the caches.  What
    is in no item's rows is NaN."""
    H, kv, hd, _ = HEADS[heads]
    g = torch.Generator().manual_seed(n + hd)
    R, held = 32, [4000, 130, 0]
    B = len(held)
    M, P = ((384 << 20) // (x * kv * hd * 4 * R) + 5 for x in (B, 1))
    state = fc.PageState.alloc(B, M, P)
    fill_table(state, [h + n for h in held], R, g, holes=[(0, 7), (0, 8)])
    cache = fc.PCache.alloc(state, kv, hd, R)
    cache.k.fill_(float("nan"))
    cache.v.fill_(float("nan"))
    table = state.table.tolist()
    for b in range(B):
        for j in range(0, held[b] + n, R):
            p, rows = table[b][j // R], min(R, held[b] + n - j)
            if 0 <= p < P:
                cache.k[p, :, :rows] = randn(g, kv, rows, hd)
                v = cache.v[p].transpose(-1, -2).reshape(kv, R, hd)
                v[:, :rows] = randn(g, kv, rows, hd)
                cache.v[p] = v.view(kv, R // 8, 8, hd).transpose(-1, -2)
    q = randn(g, B, n, H, hd)
    out = torch.full_like(q, 9.0)
    mask = (torch.rand(B, M * R, generator=g) > 0.3).cuda() if masked else None
    fc.fc_pcache_attention(ctx, cache, q, ints(held), None, out, key_mask=mask)
    torch.cuda.synchronize()
    for b in range(B):
        check(cache, b, q[b], out[b], held[b], n, hd ** -0.5, None if mask is None else mask[b].cpu().numpy())


OTHER = {"kv3": (6, 3, 128), "kv5": (15, 5, 64), "kv16": (16, 16, 64), "kv12": (24, 12, 128), "kv300": (300, 300, 64)}


@pytest.mark.parametrize("heads", list(OTHER))
@pytest.mark.parametrize("n,R,held,new,mask", [(1, 16, [900, 77, 0], None, None), (1, 64, [3000, 10, 1], [1, 0, 1], 0.3), (8, 32, [300, 31, 0], [8, 8, 3], None),
                                               (40, 32, [300, 31, 0], [40, 8, 0], 0.3), (90, 64, [500, 0, 63], None, None)])
def test_other_numbers_of_heads(fc, ctx, monkeypatch, heads, n, R, held, new, mask):  # noqa: F811
    """Key-value heads whose number does not divide the XCDs, or exceeds the CUs."""
    if heads == "kv300":
        held = [h // 8 for h in held]
    monkeypatch.setitem(HEADS, heads, (*OTHER[heads], (0, 0, 0)))
    run_attention(fc, ctx, torch.Generator().manual_seed(n), heads, n, R, held, new, mask=mask, holes=[(0, 1)], extra=1)


@pytest.mark.parametrize("heads,B,n", [("one", 130, 1), ("group2", 70, 2), ("one", 65, 20), ("group2", 128, 1)])
def test_few_rows_of_more_items_than_a_wave_has_lanes(fc, ctx, heads, B, n):  # noqa: F811
    """More items than one look at the lengths takes, and more workgroups than items: dealt by their lengths, which
    are far apart; some items bring nothing."""
    held = [(b * 997) % 3000 if b % 5 else 0 for b in range(B)]
    new = [0 if b % 7 == 3 else n - b % n for b in range(B)]
    run_attention(fc, ctx, torch.Generator().manual_seed(B), heads, n, 64, held, new)


# ------------------------------------------------------------------------------ many rows
@pytest.mark.parametrize("heads,n,B", [("qwen", 300, 20), ("toy", 500, 100)])
def test_many_rounds_with_mask_holes_and_odd_values(fc, ctx, heads, n, B):  # noqa: F811
    """Ragged batches whose pieces come from queues, with rows hidden by a mask, rows without a page, hidden rows and
    unheld pages of NaN and infinities, and at last one row that is not finite and that later tokens see."""
    H, kv, hd, _ = HEADS[heads]
    g = torch.Generator().manual_seed(n)
    R, M = 64, 14
    held, new = [(53 * b) % 390 for b in range(B)], [n - (b * 37) % n if b % 6 else 0 for b in range(B)]
    held[1], new[1] = 200, n
    state = fc.PageState.alloc(B, M, B * M)
    table = fill_table(state, [h + m for h, m in zip(held, new)], R, g, holes=[(b, 1) for b in range(0, B, 3)])
    cache = pool(g, state, kv, hd, R, fc)
    mask = torch.rand(B, M * R, generator=g) > 0.2
    mask[4, :300] = False                              # blocks that nobody sees
    q = randn(g, B, n, H, hd)
    lens, news, shown = ints(held), ints(new), mask.cuda()
    want, got = torch.full_like(q, 9.0), torch.full_like(q, 9.0)
    fc.fc_pcache_attention(ctx, cache, q, lens, news, want, key_mask=shown)
    torch.cuda.synchronize()
    for b in (1, 3, 4, 6, B - 1):
        check(cache, b, q[b], want[b], held[b], new[b], hd ** -0.5, mask[b].numpy())
    for b in range(B):
        assert (want[b, new[b]:] == 9).all() and torch.isfinite(want[b].float()).all()
    # what is hidden
    odd = torch.tensor([float("nan"), float("inf"), -float("inf")], dtype=torch.bfloat16, device="cuda")
    seen = torch.zeros(state.n_pages, R, dtype=torch.bool)
    for b in range(B):
        for i, p in enumerate(table[b]):
            if 0 <= p < state.n_pages:
                j = torch.arange(i * R, i * R + R)
                seen[p] = mask[b, j] & (j < held[b] + new[b])
    hidden = ~seen.cuda()
    kind = odd[torch.arange(R, device="cuda") % 3]
    cache.k.copy_(torch.where(hidden[:, None, :, None], kind[:, None], cache.k))
    by_rows = cache.v.transpose(-1, -2).reshape(cache.k.shape)
    by_rows = torch.where(hidden[:, None, :, None], kind.roll(1)[:, None], by_rows)
    cache.v.copy_(by_rows.view(-1, kv, R // 8, 8, hd).transpose(-1, -2))
    fc.fc_pcache_attention(ctx, cache, q, lens, news, got, key_mask=shown)
    torch.cuda.synchronize()
    assert torch.equal(got, want), "hidden bytes"
    # a row of item 1 that its tokens from the 90th on see: in its columns they alone are not finite
    j = held[1] + 90
    shown[1, j] = True
    p, r = table[1][j // R], j % R
    cache.k[p, :, r] = 0.1
    cache.v[p, :, r // 8, :, r % 8] = 0.5
    fc.fc_pcache_attention(ctx, cache, q, lens, news, want, key_mask=shown)
    cols = [0, 5, hd - 1]
    for d, x in zip(cols, odd):
        cache.v[p, :, r // 8, d, r % 8] = x
    fc.fc_pcache_attention(ctx, cache, q, lens, news, got, key_mask=shown)
    torch.cuda.synchronize()
    rest = [d for d in range(hd) if d not in cols]
    assert torch.equal(got[:1], want[:1]) and torch.equal(got[2:], want[2:]) and torch.equal(got[1, :90], want[1, :90])
    assert torch.equal(got[1, 90:, :, rest], want[1, 90:, :, rest])
    assert torch.isnan(got[1, 90:, :, 0]).all() and not torch.isfinite(got[1, 90:][..., cols]).any()


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
