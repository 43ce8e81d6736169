"""The paged token cache on the GPU against its oracle in 64 bits: appends, attention, the pages' plans,
the calls chained as a program runs them, refusals, and what the calls must leave alone.

Tolerances.  A rounding is off by at most half a step: 2^-8 of a bfloat16 number, 2^-24 of a float32 one.
  * A rotated element a cos t - b sin t: its angle is reduced in 64 bits and rounded to float32 as a
    part of a turn, so it is within (|a| + |b|) 2^-21 before its rounding to bfloat16.
  * A probability: the float32 sum of hd products is within hd 2^-24 sum|q k|, which the exponent turns into
    a relative error; the same for the largest exponent and for the sum of the probabilities, so
    4 (hd + 4) 2^-24 max_j scale sum|q_d k_d| covers them, plus 2^-22 for the exponential, its argument's
    rounding and the quotient, plus 2^-24 for each of the rows that a sum runs over.
  * An output: that of its probabilities on sum P|v|, another 2^-8 there (P is rounded to bfloat16
    before the product with V), and 2^-8 of itself.
"""
import numpy as np
import pytest
import torch

from oracle import pcache as op

pytestmark = pytest.mark.gpu

HEADS = {"qwen": (28, 4, 128, (16, 24, 24)), "toy": (4, 4, 64, (8, 8, 16)), "one": (1, 1, 128, (0, 0, 0)),
         "group2": (4, 2, 64, (0, 0, 0)), "wide": (40, 2, 64, (32, 0, 0)), "three": (6, 2, 128, (0, 40, 24))}
SMALL = dict(max_batch=4, max_height=224, max_width=224, max_tokens=256, max_seq=288, max_d_model=256, max_ffn=1024, max_qkv=768)


@pytest.fixture(scope="module")
def fc():
    import paper_2604_24391_amd as fc
    fc.lib()
    return fc


@pytest.fixture(scope="module")
def ctx(fc):
    with fc.Context(fc.Caps(**SMALL)) as c:
        yield c


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def randn(g, *shape):
    return torch.randn(*shape, generator=g, dtype=torch.float32).cuda().bfloat16()


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def pool(g, pages, kv, hd, R, fc):
    c = fc.PCache.alloc(pages, kv, hd, R)
    for t in (c.k, c.v):
        t.copy_(randn(g, *t.shape))
    return c


def fill_table(state, rows, R, g, spare=3, holes=()):
    """Pages in no order for `rows` of each item; (item, place) in holes gets none.  Rows of places beyond the
    items' stay without."""
    order = torch.randperm(state.n_pages, generator=g).tolist()
    table = [[-1] * state.max_pages for _ in rows]
    for b, n in enumerate(rows):
        for i in range(op.pages_of(n, R)):
            table[b][i] = order.pop()
    for b, i in holes:
        table[b][i] = [-1, -7, state.n_pages, 2 ** 31 - 1][(b + i) % 4]
    state.table.copy_(ints(table))
    count = np.zeros(state.n_pages, np.int64)
    for row in table:
        for p in row:
            if 0 <= p < state.n_pages:
                count[p] += 1
    state.holders.copy_(ints(count.tolist()))
    return table


def item_rows(c, b):
    """An item's rows by its table, [n_kv, capacity, hd] in 64 bits, and which have a page."""
    t = c.pages.table[b].cpu().numpy()
    R = c.k.shape[2]
    there = np.repeat((t >= 0) & (t < c.pages.n_pages), R)
    t = torch.from_numpy(np.where((t >= 0) & (t < c.pages.n_pages), t, 0)).cuda()
    k = f64(c.k[t].transpose(0, 1).flatten(1, 2))
    v = f64(c.v[t].transpose(-1, -2).flatten(2, 3).transpose(0, 1).flatten(1, 2))
    return k, v, there


# ------------------------------------------------------------------------------ append
@pytest.mark.parametrize("heads", list(HEADS))
@pytest.mark.parametrize("n,R,held,new", [
    (1, 16, [0, 1, 15], None), (1, 64, [63, 64, 7], None), (5, 16, [14, 12, 11], [5, 5, 0]), (8, 32, [0, 8, 31], None),
    (64, 64, [0, 32, 64], None), (130, 32, [0, 3, 61], [130, 129, 1]), (300, 1024, [1, 0, 900], [300, 63, 64]), (37, 128, [250, 256, 0], [37, -4, 99])])
def test_append(fc, ctx, heads, n, R, held, new):
    g = torch.Generator().manual_seed(n)
    H, kv, hd, sec = HEADS[heads]
    B, M = 3, max(2, op.pages_of(300, R))
    state = fc.PageState.alloc(B, M, B * M + 2)
    fill_table(state, [M * R] * B, R, g, holes=[(1, 0)] if n == 130 else [])
    cache = pool(g, state, kv, hd, R, fc)
    rope = fc.RopeAxes(1e6, sec)
    before_k, before_v = f64(cache.k), f64(cache.v)
    q, k, v = (randn(g, B, n, H + 2 * kv, hd) * 3).split([H, kv, kv], 2)
    pos = torch.randint(0, 40000, (rope.axes, B, n), generator=g, dtype=torch.int32).cuda()
    q_out = torch.full((B, n, H, hd), 9.0, dtype=torch.bfloat16, device="cuda")
    fc.fc_pcache_append(ctx, cache, rope, q, k, v, pos, ints(held), None if new is None else ints(new), q_out)
    torch.cuda.synchronize()
    want_k, want_v, slack_k = before_k.copy(), before_v.copy(), np.zeros_like(before_k)
    table = state.table.cpu().tolist()
    for b in range(B):
        m = min(n if new is None else min(max(new[b], 0), n), M * R - held[b])
        p = pos[:, b].cpu().numpy()

        def turned(x):
            x = f64(x)
            pair = np.abs(x[..., :hd // 2]) + np.abs(x[..., hd // 2:])
            return op.rotate(x, p, sec, 1e6), np.concatenate([pair, pair], -1) * 2.0 ** -21
        qr, qs = turned(q[b])
        got = f64(q_out[b])
        assert (np.abs(got[:m] - qr[:m]) <= 2.0 ** -8 * np.abs(qr[:m]) + qs[:m]).all(), "queries"
        assert (got[m:] == 9).all(), "queries of tokens that do not count"
        kr, ks = turned(k[b])
        vr = f64(v[b])
        for i in range(m):
            page, r = table[b][(held[b] + i) // R], (held[b] + i) % R
            if not 0 <= page < state.n_pages:
                continue
            want_k[page, :, r], slack_k[page, :, r] = kr[i], ks[i]
            want_v[page, :, r // 8, :, r % 8] = vr[i]
    np.testing.assert_array_equal(f64(cache.v), want_v)
    moved = slack_k > 0
    got = f64(cache.k)
    np.testing.assert_array_equal(got[~moved], want_k[~moved])
    assert (np.abs(got - want_k) <= 2.0 ** -8 * np.abs(want_k) + slack_k).all(), "keys"


# ------------------------------------------------------------------------------ attention
def run_attention(fc, ctx, g, heads, n, R, held, new, mask=None, holes=(), scale=None, cache=None, q=None, extra=0):
    H, kv, hd, _ = HEADS[heads]
    B = len(held)
    ms = [n if new is None else min(max(new[b], 0), n) for b in range(B)]
    M = op.pages_of(max(h + m for h, m in zip(held, ms)), R) + extra
    need = sum(op.pages_of(h + m, R) for h, m in zip(held, ms))
    state = fc.PageState.alloc(B, M, need + 3)
    fill_table(state, [h + m for h, m in zip(held, ms)], R, g, holes=holes)
    cache = pool(g, state, kv, hd, R, fc)
    q = randn(g, B, n, H, hd) * 2
    out = torch.full_like(q, 9.0)
    km = None
    if mask is not None:
        km = (torch.rand(B, M * R, generator=g) > mask).cuda()
        km[0, :min(2 * R, M * R)] = False            # pages that nobody sees
    fc.fc_pcache_attention(ctx, cache, q, ints(held), None if new is None else ints(new), out, key_mask=km, scale=scale)
    torch.cuda.synchronize()
    for b in range(B):
        check(cache, b, q[b], out[b], held[b], ms[b], hd ** -0.5 if scale is None else scale, None if km is None else km[b].cpu().numpy())
    return cache, q, out, km


def check(cache, b, q, out, held, m, scale, mask=None):
    k, v, there = item_rows(cache, b)
    L, hd = held + m, q.shape[-1]
    shown = there[:L] if mask is None else there[:L] & (mask[:L] != 0)
    want, absv, mass = op.attention(k[:, :L], v[:, :L], f64(q[:m]), held, scale, shown)
    rel = 4 * (hd + 4) * 2.0 ** -24 * mass + 2.0 ** -22 + L * 2.0 ** -24
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + rel)[..., None] * absv
    got = f64(out)
    assert (got[m:] == 9).all(), "outputs of tokens that do not count"
    off = np.abs(got[:m] - want) - tol
    assert (off <= 0).all(), f"item {b}: {int((off > 0).sum())} outputs off, worst by {off.max()}"


@pytest.mark.parametrize("heads", list(HEADS))
@pytest.mark.parametrize("n,R,held,new", [
    (1, 16, [0, 1, 200], None), (1, 64, [63, 64, 500], [1, 0, 1]), (1, 1024, [2176, 10, 0], None), (3, 32, [100, 33, 31], [3, 2, 1]),
    (8, 16, [0, 300, 70], [8, 8, 0]), (17, 64, [40, 0, 257], None), (64, 128, [0, 65, 300], [64, 1, 33]), (200, 32, [0, 17, 100], [200, 199, 5])])
def test_attention(fc, ctx, heads, n, R, held, new):
    run_attention(fc, ctx, torch.Generator().manual_seed(7 * n + R), heads, n, R, held, new, extra=2)


@pytest.mark.parametrize("heads", ["qwen", "toy", "wide"])
@pytest.mark.parametrize("n,R", [(1, 16), (1, 64), (2, 128), (9, 32), (40, 16), (90, 64)])
def test_attention_masked_and_missing_pages(fc, ctx, heads, n, R):
    g = torch.Generator().manual_seed(n)
    run_attention(fc, ctx, g, heads, n, R, [150, 600, 3, 0], [n, n, n, n], mask=0.3, holes=[(1, 0), (1, 2), (0, 1)])


@pytest.mark.parametrize("heads,n,B", [("qwen", 1, 1), ("qwen", 1, 9), ("toy", 1, 3), ("qwen", 4, 2), ("wide", 5, 2), ("qwen", 16, 1), ("qwen", 300, 1)])
def test_attention_long_histories(fc, ctx, heads, n, B):
    """Work split over the keys: items of very unlike length."""
    g = torch.Generator().manual_seed(B)
    run_attention(fc, ctx, g, heads, n, 64, [5000 // (b * b + 1) for b in range(B)], None)


@pytest.mark.parametrize("heads,n,B", [("toy", 64, 1), ("one", 40, 2), ("wide", 10, 1), ("three", 100, 1)])
def test_attention_in_many_parts(fc, heads, n, B):
    """Histories that many rows are split over: tens of parts to a row."""
    with fc.Context(fc.Caps(max_batch=4, max_height=448, max_width=448, max_tokens=1024, max_seq=4096, max_d_model=2048, max_ffn=8192, max_qkv=4096)) as ctx:
        run_attention(fc, ctx, torch.Generator().manual_seed(n), heads, n, 64, [9000 // (b + 1) for b in range(B)], None)


@pytest.mark.parametrize("heads,n,B,new", [("qwen", 1316, 1, False), ("toy", 40, 160, True), ("group2", 1700, 8, False)])
def test_attention_up_to_two_workgroups_a_cu(fc, ctx, heads, n, B, new):
    """Numbers of pieces whose shortest go beside the longest, in one group of pairs and in several."""
    g = torch.Generator().manual_seed(n)
    held = [(5 * b) % 90 for b in range(B)]
    run_attention(fc, ctx, g, heads, n, 64, held, [n - b % 30 for b in range(B)] if new else None)


@pytest.mark.parametrize("heads,n", [("qwen", 1), ("toy", 1), ("qwen", 4), ("qwen", 9), ("wide", 30), ("three", 150)])
def test_hidden_bytes_have_no_effect(fc, ctx, heads, n):
    """NaN and infinities in masked rows, in pages that nobody holds, behind the last row, in the buffers'
    tokens that do not count; later rows too, for the tokens before them."""
    H, kv, hd, _ = HEADS[heads]
    g = torch.Generator().manual_seed(n)
    B, R, M, held, new = 3, 32, 12, [200, 77, 0], [n, max(1, n // 2), n]
    state = fc.PageState.alloc(B, M, B * M + 1)
    table = fill_table(state, [h + m for h, m in zip(held, new)], R, g, holes=[(0, 3)])
    cache = pool(g, state, kv, hd, R, fc)
    q = randn(g, B, n, H, hd)
    mask = (torch.rand(B, M * R, generator=g) > 0.2).cuda()
    mask[0, 10] = True
    lens, news = ints(held), ints(new)
    want = [torch.zeros_like(q) for _ in range(2)]
    for w, m in zip(want, (mask, None)):
        fc.fc_pcache_attention(ctx, cache, q, lens, news, w, key_mask=m)
    odd = torch.tensor([float("nan"), float("inf"), -float("inf"), -float("nan")], dtype=torch.bfloat16, device="cuda")
    free = sorted(set(range(state.n_pages)) - {p for row in table for p in row})
    for p in free:
        cache.k[p], cache.v[p] = odd[0], odd[1]
    q2 = q.clone()
    for b in range(B):
        q2[b, new[b]:] = odd[0]

        def put(j, x):
            p, r = table[b][j // R], j % R
            if 0 <= p < state.n_pages:
                cache.k[p, :, r], cache.v[p, :, r // 8, :, r % 8] = odd[x % 4], odd[(x + b) % 4]
        for j in range(held[b] + new[b], op.pages_of(held[b] + new[b], R) * R):
            put(j, j)
    got = torch.zeros_like(q)
    fc.fc_pcache_attention(ctx, cache, q2, lens, news, got)
    torch.cuda.synchronize()
    assert torch.equal(got, want[1]), "rows behind the last one"
    for b in range(B):
        for j in range(held[b] + new[b]):
            if not mask[b, j]:
                p, r = table[b][j // R], j % R
                if 0 <= p < state.n_pages:
                    cache.k[p, :, r], cache.v[p, :, r // 8, :, r % 8] = odd[j % 4], odd[(j // 4) % 4]
    fc.fc_pcache_attention(ctx, cache, q2, lens, news, got, key_mask=mask)
    torch.cuda.synchronize()
    assert torch.equal(got, want[0]), "masked rows"
    # a value that the tokens from the second one on see: they alone are not finite there, in its columns
    if n > 1:
        j = held[0] + 1
        mask[0, j] = True
        p, r = table[0][j // R], j % R
        cache.k[p, :, r] = 0.1
        cache.v[p, :, r // 8, :, r % 8] = 0.5
        fc.fc_pcache_attention(ctx, cache, q2, lens, news, want[0], key_mask=mask)
        cols = torch.tensor([0, 5, hd - 1], device="cuda")
        for x, val in enumerate((float("nan"), float("inf"), -float("inf"))):
            cache.v[p, :, r // 8, cols[x], r % 8] = val
        fc.fc_pcache_attention(ctx, cache, q2, lens, news, got, key_mask=mask)
        torch.cuda.synchronize()
        assert torch.equal(got[0, 0], want[0][0, 0]) and torch.equal(got[1:], want[0][1:])
        rest = torch.ones(hd, dtype=torch.bool, device="cuda")
        rest[cols] = False
        assert torch.equal(got[0, 1:, :, rest], want[0][0, 1:, :, rest])
        assert torch.isnan(got[0, 1:new[0], :, 0]).all() and not torch.isfinite(got[0, 1:new[0]][..., cols]).any()


@pytest.mark.parametrize("heads,n", [("qwen", 4), ("qwen", 9), ("qwen", 16), ("toy", 50), ("wide", 20)])
def test_later_tokens_do_not_change_how_earlier_ones_are_rounded(fc, ctx, heads, n):
    """Scores that rise from step to step, and keys of the second half of the tokens that are far larger, or
    not: the first half's outputs are the same bytes, though they share tiles with rows that see those."""
    H, kv, hd, _ = HEADS[heads]
    g = torch.Generator().manual_seed(n)
    R, held = 32, 100
    state = fc.PageState.alloc(1, 8, 8)
    table = fill_table(state, [held + n], R, g)
    cache = pool(g, state, kv, hd, R, fc)
    for j in range(held + n):
        cache.k[table[0][j // R], :, j % R] *= 0.02 * 1.02 ** min(j, 64) if j < 80 else 2.0
    q = randn(g, 1, n, H, hd)
    outs = []
    for large in (1, 40):
        for j in range(held + n // 2, held + n):
            cache.k[table[0][j // R], :, j % R] *= large
        outs.append(torch.zeros_like(q))
        fc.fc_pcache_attention(ctx, cache, q, ints([held]), None, outs[-1])
    torch.cuda.synchronize()
    assert torch.equal(outs[0][:, :n // 2], outs[1][:, :n // 2])
    assert not torch.equal(outs[0][:, n // 2:], outs[1][:, n // 2:])


@pytest.mark.parametrize("n", [1, 3, 9])
def test_attention_extreme_numbers(fc, ctx, n):
    """Scores of many orders, and values whose sum leaves float32 where their mean does not."""
    H, kv, hd, _ = HEADS["one"]
    g = torch.Generator().manual_seed(n)
    R, M, L = 64, 10, 600
    state = fc.PageState.alloc(1, M, M)
    table = fill_table(state, [L + n], R, g)
    cache = pool(g, state, kv, hd, R, fc)
    q = randn(g, 1, n, H, hd)
    cache.v.fill_(3e38)
    out = torch.zeros_like(q)
    fc.fc_pcache_attention(ctx, cache, q, ints([L]), None, out)
    torch.cuda.synchronize()
    # a mean of equal numbers: probabilities rounded by 2^-8 each, their sum by less, the output by 2^-8
    np.testing.assert_allclose(f64(out), f64(cache.v[0, 0, 0, 0, 0]), rtol=3 * 2.0 ** -8)
    # one score far above all others, early and late; all scores equal and huge
    cache.v.copy_(randn(g, *cache.v.shape))
    for j in (0, 300, L):
        cache.k.copy_(randn(g, *cache.k.shape))
        cache.k[table[0][j // R], 0, j % R] = (q[0, 0, 0].float() * 40).bfloat16()
        fc.fc_pcache_attention(ctx, cache, q, ints([L]), None, out)
        torch.cuda.synchronize()
        check(cache, 0, q[0], out[0], L, n, hd ** -0.5)
    for scale in (0.0, -0.7, 30.0):
        fc.fc_pcache_attention(ctx, cache, q, ints([L]), None, out, scale=scale)
        torch.cuda.synchronize()
        check(cache, 0, q[0], out[0], L, n, scale)


@pytest.mark.parametrize("heads,n,B", [("qwen", 300, 48), ("toy", 700, 70)])
def test_attention_many_rounds_of_workgroups(fc, ctx, heads, n, B):
    """Ragged batches of four rounds of workgroups and more."""
    g = torch.Generator().manual_seed(n)
    H, kv, hd, _ = HEADS[heads]
    R, M = 64, 18
    held, new = [(7 * b) % 400 for b in range(B)], [n - (b * 37) % n if b % 6 else 0 for b in range(B)]
    state = fc.PageState.alloc(B, M, B * M)
    fill_table(state, [h + m for h, m in zip(held, new)], R, g)
    cache = pool(g, state, kv, hd, R, fc)
    q = randn(g, B, n, H, hd)
    out = torch.full_like(q, 9.0)
    fc.fc_pcache_attention(ctx, cache, q, ints(held), ints(new), out)
    torch.cuda.synchronize()
    for b in range(0, B, 7):
        check(cache, b, q[b], out[b], held[b], new[b], hd ** -0.5)
    for b in range(B):
        assert (out[b, new[b]:] == 9).all() and torch.isfinite(out[b].float()).all()


def test_attention_in_a_small_workspace(fc):
    """No room for parts: one workgroup an item."""
    g = torch.Generator().manual_seed(3)
    with fc.Context(fc.Caps(max_batch=1, max_height=28, max_width=28, max_tokens=1, max_seq=8, max_d_model=64, max_ffn=64, max_qkv=64)) as small:
        for heads, n in (("qwen", 1), ("wide", 5)):
            run_attention(fc, small, g, heads, n, 64, [900, 70], None)


def test_attention_offsets_past_32_bits(fc, ctx):
    """Pages whose first byte lies beyond 2^32 (a pool of 5 GiB each of keys and values)."""
    H, kv, hd, sec = HEADS["three"]
    g = torch.Generator().manual_seed(5)
    R, M = 1024, 3
    P = 5 * 2 ** 30 // (R * kv * hd * 2)
    state = fc.PageState.alloc(2, M, P)
    state.table.copy_(ints([[P - 1, 0, P - 2], [P // 2 + 1, P - 3, 1]]))
    cache = fc.PCache.alloc(state, kv, hd, R)
    n, held = 90, [2500, 1100]
    for p in state.table.flatten().tolist():
        cache.k[p], cache.v[p] = randn(g, kv, R, hd), randn(g, kv, R // 8, hd, 8)
    k, v, q = randn(g, 2, n, kv, hd), randn(g, 2, n, kv, hd), randn(g, 2, n, H, hd)
    pos = torch.zeros(3, 2, n, dtype=torch.int32, device="cuda")      # nothing turned
    q_out = torch.zeros_like(q)
    fc.fc_pcache_append(ctx, cache, fc.RopeAxes(1e6, sec), q, k, v, pos, ints(held), None, q_out)
    assert torch.equal(q_out, q)
    for b in range(2):
        kr, vr, _ = item_rows(cache, b)
        np.testing.assert_array_equal(kr[:, held[b]:held[b] + n], f64(k[b]).transpose(1, 0, 2))
        np.testing.assert_array_equal(vr[:, held[b]:held[b] + n], f64(v[b]).transpose(1, 0, 2))
    for rows in (n, 1):
        out = torch.zeros(2, rows, H, hd, dtype=torch.bfloat16, device="cuda")
        fc.fc_pcache_attention(ctx, cache, q[:, :rows].contiguous(), ints(held), None, out)
        torch.cuda.synchronize()
        for b in range(2):
            check(cache, b, q[b, :rows], out[b], held[b], rows, hd ** -0.5)


# ------------------------------------------------------------------------------ pages
def as_lists(state):
    return [[p if 0 <= p < state.n_pages else None for p in row] for row in state.table.cpu().tolist()]


def moved(before, moves, R):
    """Pools [P, kv, R, hd] (plain rows) after rows have been copied."""
    out = before.clone()
    for a, z, rows in moves:
        out[z, :, :rows] = before[a, :, :rows]
    return out


def plain(c):
    return c.k.clone(), c.v.transpose(-1, -2).reshape(c.k.shape).clone()


def run_step(fc, ctx, caches, src, lens, new, n):
    """One step against the oracle; returns what was granted."""
    state, R = caches[0].pages, caches[0].k.shape[2]
    pages = op.Pages(as_lists(state), state.n_pages, R, state.max_pages)
    before = [plain(c) for c in caches]
    granted = torch.full((state.B,), -5, dtype=torch.int32, device="cuda")
    fc.fc_pcache_step(ctx, caches, ints(lens), None if new is None else ints(new), n, granted, src=None if src is None else ints(src))
    torch.cuda.synchronize()
    want, copies = pages.step(src, lens, new, n)
    assert granted.tolist() == want
    same_state(state, pages)
    for c, (k, v) in zip(caches, before):
        k2, v2 = plain(c)
        assert torch.equal(k2, moved(k, copies, R)) and torch.equal(v2, moved(v, copies, R)), "rows copied"
    return want


def same_state(state, pages):
    table = [[-1 if p is None else p for p in row] + [-1] * (state.max_pages - len(row)) for row in pages.table]
    assert state.table.tolist() == table
    assert state.holders.tolist() == pages.holders()


def run_compact(fc, ctx, caches):
    state, R = caches[0].pages, caches[0].k.shape[2]
    pages = op.Pages(as_lists(state), state.n_pages, R, state.max_pages)
    before = [plain(c) for c in caches]
    live = torch.full((1,), -5, dtype=torch.int32, device="cuda")
    fc.fc_pcache_compact(ctx, caches, live)
    torch.cuda.synchronize()
    L, moves = pages.compact()
    assert live.item() == L
    same_state(state, pages)
    for c, (k, v) in zip(caches, before):
        k2, v2 = plain(c)
        assert torch.equal(k2, moved(k, moves, R)) and torch.equal(v2, moved(v, moves, R)), "rows moved"


@pytest.mark.parametrize("seed", range(12))
def test_steps_and_compactions(fc, ctx, seed):
    """Random plans, one after the other: items fork, grow, shrink, end and begin, also where pages run out."""
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    B, R, M = int(rng.integers(1, 20)), int(rng.choice([16, 32, 64])), int(rng.integers(1, 9))
    P, layers, (_, kv, hd, _) = int(rng.integers(1, B * M + 2)), int(rng.integers(1, 4)), HEADS["group2" if seed % 2 else "three"]
    state = fc.PageState.alloc(B, M, P)
    caches = [pool(g, state, kv, hd, R, fc) for _ in range(layers)]
    lens = [0] * B
    for turn in range(12):
        src = None if turn % 3 == 0 else [int(s) for s in rng.integers(-1, B + 1, B)] if turn % 3 == 1 else [int(rng.integers(0, B))] * B
        base = lens if src is None else [lens[s] if 0 <= s < B else 0 for s in src]
        keep = [int(rng.integers(0, h + 1)) if rng.random() < 0.3 else h for h in base]
        n = int(rng.integers(0, 3 * R))
        new = None if turn % 4 == 3 else [int(x) for x in rng.integers(-2, n + 3, B)]
        got = run_step(fc, ctx, caches, src, keep, new, n)
        lens = [h + m for h, m in zip(keep, got)]
        if turn % 4 == 2:
            run_compact(fc, ctx, caches)


def test_step_edges(fc, ctx):
    g = torch.Generator().manual_seed(1)
    _, kv, hd, _ = HEADS["toy"]
    R, M = 16, 4
    state = fc.PageState.alloc(5, M, 9)
    caches = [pool(g, state, kv, hd, R, fc)]
    run_compact(fc, ctx, caches)                                             # nothing is held
    assert run_step(fc, ctx, caches, None, [0, 0, 0, 0, 0], [20, 0, 64, 1, 64], 64) == [20, 0, 64, 1, 32]
    # a row count beyond the capacity, negative counts, a source that is none
    assert run_step(fc, ctx, caches, [0, 1, 2, 3, -1], [20, -3, 999, 1, 32], [5, 5, 5, -1, 7], 5) == [5, 5, 0, 0, 5]
    # an entry that names no page in the place of the last kept row: nothing can be written there
    state.table[0, 1] = 77
    assert run_step(fc, ctx, caches, None, [20, 0, 16, 0, 0], [2, 0, 0, 0, 0], 2) == [0, 0, 0, 0, 0]
    # all of one item: the last writer keeps the page, the others copy it
    assert run_step(fc, ctx, caches, None, [0, 3, 0, 0, 0], [0, 2, 0, 0, 0], 4) == [0, 0, 0, 0, 0]   # (it holds none)
    run_step(fc, ctx, caches, None, [0] * 5, [0, 7, 0, 0, 0], 7)
    assert run_step(fc, ctx, caches, [1] * 5, [7] * 5, [1, 1, 0, 1, 1], 1) == [1, 1, 0, 1, 1]
    run_compact(fc, ctx, caches)
    # fewer free pages than copies
    run_step(fc, ctx, caches, None, [0] * 5, [16 * 4, 16 * 2, 9, 0, 0], 64)
    assert run_step(fc, ctx, caches, [0, 1, 2, 2, 2], [64, 32, 9, 9, 9], [0, 0, 2, 2, 2], 2) == [0, 0, 2, 2, 2]
    run_step(fc, ctx, caches, None, [0] * 5, [64, 64, 9, 0, 0], 64)
    assert run_step(fc, ctx, caches, [0, 1, 2, 2, 2], [64, 64, 9, 9, 9], [0, 0, 2, 2, 2], 2) == [0, 0, 0, 0, 0]


def test_step_many_items_and_pages(fc, ctx):
    """More items than a workgroup has threads, more pages than it holds counts of."""
    g = torch.Generator().manual_seed(2)
    for B, M, P, kv, hd in ((1500, 3, 5000, 1, 64), (40, 200, 9001, 2, 64), (3, 3000, 9000, 1, 64)):
        R = 16
        state = fc.PageState.alloc(B, M, P)
        caches = [pool(g, state, kv, hd, R, fc)]
        rng = np.random.default_rng(B)
        lens = run_step(fc, ctx, caches, None, [0] * B, [int(x) for x in rng.integers(0, M * R + 1, B)], M * R)
        src = [int(x) for x in rng.integers(0, B, B)]
        keep = [int(lens[s] * rng.random()) for s in src]
        run_step(fc, ctx, caches, src, keep, [int(x) for x in rng.integers(0, 40, B)], 40)
        run_compact(fc, ctx, caches)


def test_init(fc, ctx):
    state = fc.PageState(torch.full((103,), 5, dtype=torch.int32, device="cuda"), 3, 7, 75)      # 21 entries, 3 zeros, 75 holders, the rest not its own
    cache = fc.PCache.alloc(state, 1, 64, 16)
    fc.fc_pcache_init(ctx, cache)
    assert state.state.tolist() == [-1] * 21 + [0] * 78 + [5] * 4


# ------------------------------------------------------------------------------ as a program runs them
@pytest.mark.parametrize("heads,R", [("qwen", 64), ("toy", 16), ("three", 32)])
def test_answers_from_one_history(fc, ctx, heads, R):
    """A prompt, answers that go on from it and from each other, items that end and begin, a compaction: at
    every step the attention is that over the rows which each item's own text has brought."""
    g = torch.Generator().manual_seed(9)
    H, kv, hd, sec = HEADS[heads]
    B, M, layers = 4, op.pages_of(150, R) + 1, 2
    state = fc.PageState.alloc(B, M, B * M)
    caches = [fc.PCache.alloc(state, kv, hd, R) for _ in range(layers)]
    rope = fc.RopeAxes(1e6, sec)
    none = torch.zeros(0, kv, hd, dtype=torch.float64)
    rows = [[(none, none)] * B for _ in range(layers)]      # what each item has brought, per layer: keys rotated in 64 bits, values
    lens = [0] * B
    plan = [(None, [77, 0, 0, 0]), ([0, 0, 0, -1], [1, 1, 1, 0]), (None, [1, 1, 1, 1]), ([1, 1, 2, 1], [5, 5, 5, 0]), (None, [1, 0, 2, 1]),
            ([3, 2, 2, 0], [40, 1, 1, 1])]
    for turn, (src, new) in enumerate(plan):
        base = [(lens[s] if 0 <= s < B else 0) for s in (src or range(B))]
        if turn == 4:
            base[2] = 60                                     # rows given up
        n = max(new)
        granted = torch.zeros(B, dtype=torch.int32, device="cuda")
        fc.fc_pcache_step(ctx, caches, ints(base), ints(new), n, granted, src=None if src is None else ints(src))
        if turn == 3:
            fc.fc_pcache_compact(ctx, caches)
        assert granted.tolist() == new
        for layer, c in enumerate(caches):
            q, k, v = randn(g, B, n, H + 2 * kv, hd).split([H, kv, kv], 2)
            pos = torch.randint(0, 3000, (rope.axes, B, n), generator=g, dtype=torch.int32).cuda()
            qo, out = torch.zeros(B, n, H, hd, dtype=torch.bfloat16, device="cuda"), torch.full((B, n, H, hd), 9.0, dtype=torch.bfloat16, device="cuda")
            fc.fc_pcache_append(ctx, c, rope, q, k, v, pos, ints(base), granted, qo)
            fc.fc_pcache_attention(ctx, c, qo, ints(base), granted, out)
            torch.cuda.synchronize()
            old = [rows[layer][s] if 0 <= s < B else (none, none) for s in (src or range(B))]
            for b in range(B):
                kr = torch.from_numpy(op.rotate(f64(k[b]), pos[:, b].cpu().numpy(), sec, 1e6))
                kk = torch.cat([old[b][0][:base[b]], kr[:new[b]]])
                vv = torch.cat([old[b][1][:base[b]], torch.from_numpy(f64(v[b]))[:new[b]]])
                rows[layer][b] = (kk, vv)
                m, L = new[b], base[b] + new[b]
                want, absv, mass = op.attention(kk.numpy().transpose(1, 0, 2), vv.numpy().transpose(1, 0, 2), f64(qo[b, :m]), base[b], hd ** -0.5, np.ones(L))
                # keys are rounded to bfloat16 when they are appended: 2^-8 of sum |q k|, twice in a quotient of exponentials
                rel = (4 * (hd + 4) * 2.0 ** -24 + 2 * 1.01 * 2.0 ** -8) * mass + 2.0 ** -22 + L * 2.0 ** -24
                rel = np.expm1(rel)
                off = np.abs(f64(out[b, :m]) - want) - 2.0 ** -8 * np.abs(want) - (2.0 ** -8 + rel)[..., None] * absv
                assert (off <= 0).all() and (out[b, m:] == 9).all(), f"turn {turn}, layer {layer}, item {b}: {off.max()}"
                # and exactly what the cache holds
                check(c, b, qo[b], out[b], base[b], m, hd ** -0.5)
        lens = [h + m for h, m in zip(base, new)]


def test_captured_step_replays_match_eager(fc, ctx):
    """Pages granted, rows appended, attention, the lengths' advance and a compaction captured into one graph,
    replayed with other inputs and with eager calls between; each replay equals the eager calls."""
    g = torch.Generator().manual_seed(14)
    H, kv, hd, sec = HEADS["qwen"]
    B, n, R, M, P = 3, 3, 32, 8, 20
    rope = fc.RopeAxes(1e6, sec)

    def make():
        state = fc.PageState.alloc(B, M, P)
        return dict(pages=state, c=[fc.PCache.alloc(state, kv, hd, R) for _ in range(2)], src=ints([0] * B), lens=ints([0] * B), new=ints([0] * B),
                    granted=ints([0] * B), live=ints([0]), x=torch.zeros(B, n, H + 2 * kv, hd, dtype=torch.bfloat16, device="cuda"), pos=ints([[[0] * n] * B] * 3),
                    q=torch.zeros(B, n, H, hd, dtype=torch.bfloat16, device="cuda"), out=torch.zeros(B, n, H, hd, dtype=torch.bfloat16, device="cuda"))

    def step(s):
        fc.fc_pcache_step(ctx, s["c"], s["lens"], s["new"], n, s["granted"], src=s["src"])
        fc.fc_pcache_compact(ctx, s["c"], s["live"])
        q, k, v = s["x"].split([H, kv, kv], 2)
        for c in s["c"]:
            fc.fc_pcache_append(ctx, c, rope, q, k, v, s["pos"], s["lens"], s["granted"], s["q"])
            fc.fc_pcache_attention(ctx, c, s["q"], s["lens"], s["granted"], s["out"])
        s["lens"].add_(s["granted"])

    def tensors(s):
        return [c.k for c in s["c"]] + [c.v for c in s["c"]] + [s["pages"].state] + [s[x] for x in ("lens", "granted", "live", "q", "out")]

    init = make()
    fill_table(init["pages"], [200, 40, 0], R, g)
    for c in init["c"]:
        c.k.copy_(randn(g, *c.k.shape))
        c.v.copy_(randn(g, *c.v.shape))
    a, e = make(), make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(a)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a)
    for rep, (src, held, new) in enumerate([([0, 1, 2], [200, 40, 0], [3, 1, 2]), ([0, 0, 0], [199, 130, 65], [3, 3, 3]), ([1, 1, 0], [39, 40, 5], [0, 2, 3]),
                                            ([0, 1, 1], [200, 33, 33], [3, 1, 1])]):
        x = randn(g, B, n, H + 2 * kv, hd)
        pos = torch.randint(0, 999, (3, B, n), generator=g, dtype=torch.int32).cuda()
        for s in (a, e):
            for c, d in zip(s["c"], init["c"]):
                c.k.copy_(d.k)
                c.v.copy_(d.v)
            s["pages"].state.copy_(init["pages"].state)
            for name, t in (("x", x), ("pos", pos), ("src", ints(src)), ("lens", ints(held)), ("new", ints(new))):
                s[name].copy_(t)
            s["q"].zero_()
            s["out"].zero_()
        step(e)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (u, w) in enumerate(zip(tensors(a), tensors(e))):
            assert torch.equal(u.view(torch.uint8), w.view(torch.uint8)), f"replay {rep}, tensor {i}"


def test_two_streams_two_contexts(fc, ctx):
    """Calls at once on two streams, each with its own context, give what they give alone."""
    g = torch.Generator().manual_seed(15)
    H, kv, hd, _ = HEADS["qwen"]
    B, R, M, lens = 2, 64, 33, [2000, 1500]
    caches, q = [], [randn(g, B, n, H, hd) for n in (1, 40)]
    for _ in range(2):
        state = fc.PageState.alloc(B, M, B * M)
        fill_table(state, [h + 40 for h in lens], R, g)
        caches.append(pool(g, state, kv, hd, R, fc))
    out, want = [torch.zeros_like(x) for x in q], [torch.zeros_like(x) for x in q]
    for i in range(2):
        fc.fc_pcache_attention(ctx, caches[i], q[i], ints(lens), None, want[i])
    torch.cuda.synchronize()
    t = ints(lens)
    with fc.Context(fc.Caps(**SMALL)) as other:
        streams = [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(20):
            for i, (s, c) in enumerate(zip(streams, (ctx, other))):
                with torch.cuda.stream(s):
                    fc.fc_pcache_attention(c, caches[i], q[i], t, None, out[i])
        torch.cuda.synchronize()
        for i in range(2):                                   # a stream by name
            out[i].zero_()
        torch.cuda.synchronize()
        fc.fc_pcache_attention(other, caches[1], q[1], t, None, out[1], stream=streams[0])
        streams[0].synchronize()
        assert torch.equal(out[1], want[1])
        fc.fc_pcache_attention(other, caches[0], q[0], t, None, out[0], stream=streams[1])
        torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(out[i], want[i])


@pytest.mark.parametrize("heads,n", [("qwen", 1), ("wide", 37), ("qwen", 300)])
def test_same_inputs_same_bytes(fc, ctx, heads, n):
    """And an item's rows do not depend on what else is in its batch's pages, nor on which pages hold them."""
    g = torch.Generator().manual_seed(16)
    H, kv, hd, _ = HEADS[heads]
    B, R, M, lens = 3, 32, 60, [900, 500, 0]
    k, v, q = randn(g, B, kv, M * R, hd), randn(g, B, kv, M * R, hd), randn(g, B, n, H, hd)
    got = []
    for turn in range(3):
        state = fc.PageState.alloc(B, M, B * M + 5)
        table = fill_table(state, [h + n for h in lens], R, g)
        cache = pool(g, state, kv, hd, R, fc)
        for b in range(B):
            for i, p in enumerate(table[b]):
                if p >= 0:
                    cache.k[p] = k[b, :, i * R:(i + 1) * R]
                    cache.v[p] = v[b, :, i * R:(i + 1) * R].reshape(kv, R // 8, 8, hd).transpose(-1, -2)
        for _ in range(2):
            out = torch.zeros_like(q)
            fc.fc_pcache_attention(ctx, cache, q, ints(lens), None, out)
            got.append(out)
    for o in got[1:]:
        assert torch.equal(o, got[0])


def test_guards(fc, ctx):
    """Every buffer inside a larger allocation whose bytes around it stay as they are."""
    from tests.test_gpu_guards import Guarded
    g = torch.Generator().manual_seed(17)
    H, kv, hd, sec = HEADS["qwen"]
    B, n, R, M, P = 3, 70, 32, 7, 17
    gd = Guarded()

    def buf(shape, dtype, fill):
        return gd.new(shape, dtype, fill if isinstance(fill, torch.Tensor) else torch.full((1,), fill, dtype=dtype, device="cuda"))
    bf, i32 = torch.bfloat16, torch.int32
    state = fc.PageState(buf((24 + P,), i32, -1), B, M, P)
    caches = [fc.PCache(buf((P, kv, R, hd), bf, float("nan")), buf((P, kv, R // 8, hd, 8), bf, float("nan")), state) for _ in range(2)]
    fc.fc_pcache_init(ctx, caches[0])
    x = buf((B, n, H + 2 * kv, hd), bf, randn(g, B, n, H + 2 * kv, hd))
    q, out = buf((B, n, H, hd), bf, 0), buf((B, n, H, hd), bf, 0)
    pos, lens, new = buf((3, B, n), i32, 5), buf((B,), i32, ints([0, 0, 0])), buf((B,), i32, ints([70, 64, 3]))
    granted, live, src = buf((B,), i32, 0), buf((1,), i32, 0), buf((B,), i32, ints([2, 0, 0]))
    mask = buf((B, M * R), torch.uint8, 1)
    for turn in range(4):
        fc.fc_pcache_step(ctx, caches, lens, new, n, granted, src=src if turn == 1 else None)
        fc.fc_pcache_compact(ctx, caches, live)
        a, b, c = x.split([H, kv, kv], 2)
        for cache in caches:
            fc.fc_pcache_append(ctx, cache, fc.RopeAxes(1e6, sec), a, b, c, pos, lens, granted, q)
            fc.fc_pcache_attention(ctx, cache, q, lens, granted, out, key_mask=mask)
        lens.copy_(ints([3, 40, 70]) if turn == 0 else lens + granted)
    gd.check()
    assert not out.isnan().any()


def test_debug_mode_and_kernel_times(fc, ctx):
    """The calls run under the debug mode, and their kernels appear in the context's timing."""
    g = torch.Generator().manual_seed(18)
    prev = fc.fc_debug(True)
    fc.fc_profile_enable(ctx, True)
    try:
        fc.fc_profile_read(ctx, None, reset=True)
        test_append(fc, ctx, "toy", 5, 16, [14, 12, 11], [5, 5, 0])
        run_attention(fc, ctx, g, "toy", 1, 16, [700], None)
        run_attention(fc, ctx, g, "toy", 60, 16, [700], None)
        test_step_edges(fc, ctx)
        test_init(fc, ctx)
        for name in ("fc_pappend", "fc_pattn", "fc_pattn_rows", "fc_pattn_join", "fc_pstep", "fc_pstep_copy", "fc_pcompact", "fc_pcompact_move", "fc_pinit"):
            assert fc.fc_profile_read(ctx, name)[1] >= 1, name
    finally:
        fc.fc_profile_enable(ctx, False)
        fc.fc_profile_read(ctx, None, reset=True)
        fc.fc_debug(prev)


def test_binding_refusals(fc, ctx):
    """What the binding and the library refuse, with nothing written."""
    H, kv, hd, sec = HEADS["toy"]
    state, other = fc.PageState.alloc(2, 4, 9), fc.PageState.alloc(2, 4, 9)
    c, d = fc.PCache.alloc(state, kv, hd, 32), fc.PCache.alloc(other, kv, hd, 32)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    x = torch.ones(2, 3, H + 2 * kv, hd, **bf)
    q, k, v = x.split([H, kv, kv], 2)
    pos, lens, rope = ints([[[0] * 3] * 2] * 3), ints([0, 0]), fc.RopeAxes(1e6, sec)
    qo, granted, live = torch.ones(2, 3, H, hd, **bf), ints([7, 7]), ints([7])
    state.table.fill_(3)
    kept = [c.k, c.v, state.state, qo, granted, live]
    before = [t.clone() for t in kept]
    bad = [
        lambda: fc.fc_pcache_append(ctx, c, rope, q, k, v, pos[0], lens, None, qo),                      # one axis for three
        lambda: fc.fc_pcache_append(ctx, c, rope, q, k, v, pos, lens, None, None),
        lambda: fc.fc_pcache_append(ctx, c, rope, q, k[:1], v, pos, lens, None, qo),
        lambda: fc.fc_pcache_append(ctx, c, rope, q, k.float(), v, pos, lens, None, qo),
        lambda: fc.fc_pcache_append(ctx, c, rope, q, k, v, pos, lens.long(), None, qo),
        lambda: fc.fc_pcache_append(ctx, c, rope, q, k, v, pos, lens, ints([1]), qo),
        lambda: fc.fc_pcache_append(ctx, c, rope, q, k, v, pos.cpu(), lens, None, qo),
        lambda: fc.fc_pcache_attention(ctx, c, qo[..., :32].contiguous(), lens, None, qo),
        lambda: fc.fc_pcache_attention(ctx, c, qo[:1], lens, None, qo),
        lambda: fc.fc_pcache_attention(ctx, c, qo[0], lens, None, qo),
        lambda: fc.fc_pcache_attention(ctx, c, qo, lens, None, torch.ones(2, 3, H, hd, device="cuda")),
        lambda: fc.fc_pcache_attention(ctx, c, qo, lens, None, torch.ones_like(qo), key_mask=torch.ones(2, 127, dtype=torch.uint8, device="cuda")),
        lambda: fc.fc_pcache_step(ctx, [], lens, None, 3, granted),
        lambda: fc.fc_pcache_step(ctx, [c, d], lens, None, 3, granted),
        lambda: fc.fc_pcache_step(ctx, [c], lens[:1], None, 3, granted),
        lambda: fc.fc_pcache_step(ctx, [c], lens, None, 3, granted.long()),
        lambda: fc.fc_pcache_step(ctx, [c], lens, None, 3, granted, src=lens.cpu()),
        lambda: fc.fc_pcache_compact(ctx, [d, c], live),
        lambda: fc.PCache(c.k[:8], c.v[:8], state),
        lambda: fc.PCache(c.k, c.v.view(9, kv, 4, 8, hd), state),
        lambda: fc.PCache(c.k.float(), c.v, state),
        lambda: fc.PageState(state.state[:16], 2, 4, 9),
        lambda: fc.PageState(state.state.long(), 2, 4, 9),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {i} went through")
    status = [
        (1, lambda: fc.fc_pcache_append(ctx, c, fc.RopeAxes(1e6, (8, 8, 8)), q, k, v, pos, lens, None, qo)),
        (2, lambda: fc.fc_pcache_append(ctx, c, rope, q[:, :, :3], k, v, pos, lens, None, qo)),
        (1, lambda: fc.fc_pcache_append(ctx, c, rope, q, k, v, pos, lens, None, x.view(-1)[:2 * 3 * H * hd].view(2, 3, H, hd))),
        (1, lambda: fc.fc_pcache_attention(ctx, c, qo, lens, None, qo)),
        (1, lambda: fc.fc_pcache_attention(ctx, c, qo, lens, None, torch.ones_like(qo), scale=float("nan"))),
        (2, lambda: fc.fc_pcache_attention(ctx, c, torch.ones(2, 129, H, hd, **bf), lens, None, torch.ones(2, 129, H, hd, **bf))),
        (1, lambda: fc.fc_pcache_step(ctx, [c, c], lens, None, 3, granted)),
        (2, lambda: fc.fc_pcache_step(ctx, [c], lens, None, -1, granted)),
        (1, lambda: fc.fc_pcache_step(ctx, [c], granted, None, 3, granted)),
        (1, lambda: fc.fc_pcache_compact(ctx, [c], state.holders)),
        (2, lambda: fc.fc_pcache_step(ctx, [c, fc.PCache.alloc(state, kv, 128, 32)], lens, None, 3, granted)),
        (6, lambda: fc.fc_pcache_attention(ctx, fc.PCache.alloc(state, kv, 32, 32), torch.ones(2, 1, H, 32, **bf), lens, None, torch.ones(2, 1, H, 32, **bf))),
        (2, lambda: fc.fc_pcache_init(ctx, fc.PCache.alloc(state, kv, hd, 8))),
    ]
    for i, (want, f) in enumerate(status):
        with pytest.raises(fc.FcError) as e:
            f()
            pytest.fail(f"call {i} went through")
        assert e.value.status == want, (i, str(e.value))
    torch.cuda.synchronize()
    for t, u in zip(before, kept):
        assert torch.equal(t.view(torch.uint8), u.view(torch.uint8))


def test_a_cache_whose_memory_has_moved(fc, ctx):
    """The layers' descriptors follow their tensors."""
    g = torch.Generator().manual_seed(19)
    _, kv, hd, _ = HEADS["toy"]
    state = fc.PageState.alloc(2, 4, 9)
    caches = [pool(g, state, kv, hd, 16, fc) for _ in range(2)]
    run_step(fc, ctx, caches, None, [0, 0], [30, 20], 64)
    old = caches[1].k.clone()
    caches[1].k.set_(old)
    run_step(fc, ctx, caches, [0, 0], [30, 30], [5, 5], 5)
    caches[0].v.set_(caches[0].v[:8].clone())
    with pytest.raises(ValueError, match="elements"):
        fc.fc_pcache_step(ctx, caches, ints([0, 0]), None, 64, ints([0, 0]))
