"""The 8-bit token cache on the GPU against its oracle in 64 bits (tests/qcache_util.py derives the
tolerances): appends, attention, evictions, the three chained as an episode runs them, refusals,
and what the calls must leave alone."""
import numpy as np
import pytest
import torch

from oracle import qcache as oq
from tests import qcache_util as qu

pytestmark = pytest.mark.gpu

HEADS = {"qwen": (28, 4, 128, (16, 24, 24)), "toy": (4, 4, 64, (8, 8, 16)), "one": (1, 1, 128, (0, 0, 0)),
         "group2": (4, 2, 64, (0, 0, 0)), "wide": (40, 2, 64, (32, 0, 0)), "three": (6, 2, 128, (0, 40, 24))}


@pytest.fixture(scope="module")
def fc():
    import paper_2604_24391_amd as fc
    fc.lib()
    return fc


@pytest.fixture(scope="module")
def ctx(fc):
    with fc.Context(fc.Caps(max_batch=4, max_height=224, max_width=224, max_tokens=256, max_seq=288, max_d_model=256, max_ffn=1024,
                            max_qkv=768)) as c:
        yield c


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def randn(g, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=g, dtype=torch.float32).cuda().to(dtype)


def filled(fc, g, B, kv, hd, cap, weight=True):
    """A cache whose every row is held: random codes (no NaN) and scales, random weights."""
    c = fc.QCache.alloc(B, kv, hd, cap, weight=weight)
    for t in (c.k, c.v):
        x = torch.randn(t.shape, generator=g) * 20
        t.copy_(x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).cuda())
    for t in (c.k_scale, c.v_scale):
        t.copy_(torch.exp2(torch.randint(-7, -3, t.shape, generator=g).float()).cuda())
    if weight:
        c.weight.copy_(torch.rand(c.weight.shape, generator=g).cuda())
    return c


# ------------------------------------------------------------------------------ append
def run_append(fc, ctx, g, heads, B, n, cap, held, new, rows=None, theta=1e6, pos=None):
    H, kv, hd, sec = HEADS[heads]
    cache = qu.make(fc, B, kv, hd, cap)
    rope = fc.RopeAxes(theta, sec)
    # what is held came through the call too
    if max(held) > 0:
        k, v = randn(g, B, max(held), kv, hd), randn(g, B, max(held), kv, hd)
        p = torch.randint(0, 300, (rope.axes, B, max(held)), generator=g, dtype=torch.int32).cuda()
        fc.fc_qcache_append(ctx, cache, rope, None, k, v, p, ints([0] * B), ints(held), None)
        cache.weight.fill_(7.0)
    before = [qu.to_oracle(cache, b) for b in range(B)]
    x = randn(g, B, n, (H + 2 * kv) * hd) * 3 if rows is None else rows
    q, k, v = x.view(B, n, H + 2 * kv, hd).split([H, kv, kv], 2)
    if pos is None:
        pos = torch.randint(0, 40000, (rope.axes, B, n), generator=g, dtype=torch.int32).cuda()
    q_out = torch.full((B, n, H, hd), 9.0, dtype=torch.bfloat16, device="cuda")
    fc.fc_qcache_append(ctx, cache, rope, q, k, v, pos, ints(held), None if new is None else ints(new), q_out)
    torch.cuda.synchronize()
    for b in range(B):
        m = n if new is None else min(max(new[b], 0), n)
        m = min(m, cap - held[b])
        p = pos.view(rope.axes, B, n)[:, b, :].cpu().numpy()
        kr, slack = qu.rotated(k[b], p, sec, theta)
        qu.check_appended(qu.to_oracle(cache, b), before[b], kr[:m], slack[:m], v[b, :m].float().cpu().numpy().astype(np.float64), held[b], m)
        qr, slack = qu.rotated(q[b], p, sec, theta)
        got = q_out[b].float().cpu().numpy()
        fin = np.isfinite(qr[:m])
        assert (np.abs(got[:m] - qr[:m])[fin] <= (2.0 ** -8 * np.abs(qr[:m]) + slack[:m])[fin]).all(), "rotated queries"
        qu.same(got[m:], np.full_like(got[m:], 9.0), "queries of tokens that do not count")
    return cache, q_out


@pytest.mark.parametrize("heads", list(HEADS))
@pytest.mark.parametrize("n,held,new", [
    (1, [0, 1, 63], None), (1, [64, 65, 127], None), (5, [62, 60, 59], [5, 5, 0]), (64, [0, 32, 64], None), (130, [0, 3, 61], [130, 129, 1]),
    (200, [1, 0, 7], [200, 63, 64])])
def test_append(fc, ctx, heads, n, held, new):
    g = torch.Generator().manual_seed(n)
    run_append(fc, ctx, g, heads, 3, n, 256, held, new)


def test_append_drops_rows_past_the_capacity_and_clamps_counts(fc, ctx):
    g = torch.Generator().manual_seed(1)
    run_append(fc, ctx, g, "toy", 3, 40, 128, [100, 128, 127], [40, 99, -3])


def test_append_far_positions(fc, ctx):
    """Positions of tens of millions, of both signs: float32 angles would be off by radians (and 64-bit
    ones are good to 2^-26 there, so that the oracle can still tell)."""
    g = torch.Generator().manual_seed(2)
    pos = torch.randint(-2 ** 26, 2 ** 26, (3, 2, 9), generator=g).to(torch.int32).cuda()
    run_append(fc, ctx, g, "qwen", 2, 9, 128, [3, 60], None, pos=pos, theta=1e4)


def test_append_extreme_numbers(fc, ctx):
    """Zeros, bfloat16's largest and smallest, infinities and NaN among the values and keys."""
    g = torch.Generator().manual_seed(3)
    H, kv, hd, _ = HEADS["toy"]
    x = randn(g, 2, 70, (H + 2 * kv) * hd)
    v = x.view(2, 70, H + 2 * kv, hd)
    v[0, :, H + kv:] = 0                                       # a zero block of values
    v[1, 3, H + kv + 1, 5], v[1, 4, H + kv + 2, 6], v[1, 5, H + kv + 3, 7] = float("inf"), float("-inf"), float("nan")
    v[1, 6, H + kv + 1] = 1e-38
    v[1, 66, H + kv, 0] = 3e38
    v[0, 7, H, :] = 0
    v[0, 8, H + 1, 3] = float("nan")
    v[0, :3, H + 2] = 1e30
    run_append(fc, ctx, g, "toy", 2, 70, 128, [5, 0], None, rows=x, pos=torch.randint(0, 99, (3, 2, 70), generator=g, dtype=torch.int32).cuda())


def test_append_from_a_frame_cache_and_in_place(fc, ctx):
    """Keys and values of a layer's bf16 cache (raw keys, rows of another stride, a run of its rows)
    and queries rotated in place."""
    g = torch.Generator().manual_seed(4)
    H, kv, hd, sec = HEADS["qwen"]
    k, v = randn(g, 2, 100, kv, hd), randn(g, 2, 100, kv, hd)   # [B, S, n_kv, hd]
    cache, rope = qu.make(fc, 2, kv, hd, 64), fc.RopeAxes(1e6, sec)
    pos = torch.randint(0, 99, (3, 2, 40), generator=g, dtype=torch.int32).cuda()
    before = [qu.to_oracle(cache, b) for b in range(2)]
    q = randn(g, 2, 40, H, hd)
    want = torch.empty_like(q)
    fc.fc_qcache_append(ctx, cache, rope, q, k[:, 30:70], v[:, 30:70], pos, ints([0, 0]), None, want)
    fc.fc_qcache_append(ctx, cache, rope, q, k[:, 30:70], v[:, 30:70], pos, ints([0, 0]), None, q)
    assert torch.equal(q.view(torch.int16), want.view(torch.int16))
    for b in range(2):
        kr, slack = qu.rotated(k[b, 30:70], pos[:, b].cpu().numpy(), sec, 1e6)
        qu.check_appended(qu.to_oracle(cache, b), before[b], kr, slack, v[b, 30:70].float().cpu().numpy().astype(np.float64), 0, 40)
    # one item's rows for both (stride 0)
    other = qu.make(fc, 2, kv, hd, 64)
    fc.fc_qcache_append(ctx, other, rope, None, k[:1, 30:70].expand(2, -1, -1, -1), v[:1, 30:70].expand(2, -1, -1, -1), pos[:, :1].expand(-1, 2, -1).contiguous(),
                        ints([0, 0]), None, None)
    assert torch.equal(other.k[0], other.k[1]) and torch.equal(other.k[0], cache.k[0]) and torch.equal(other.v[1], cache.v[0])


# ------------------------------------------------------------------------------ attention
def run_attention(fc, ctx, g, heads, B, n, cap, held, new, mask=None, weight=True, scale=None, poison=True, cache=None, q=None):
    H, kv, hd, _ = HEADS[heads]
    if cache is None:
        cache = filled(fc, g, B, kv, hd, cap, weight)
    q = randn(g, B, n, H, hd) if q is None else q
    tot = [h + (n if new is None else min(max(new[b], 0), n)) for b, h in enumerate(held)]
    if poison:                       # NaN in every row behind the last one
        for b in range(B):
            cache.k[b, :, tot[b]:] = 0x7F
            full = torch.arange(cap, device="cuda") >= tot[b]
            cache.v[b].copy_(torch.where(full.view(1, -1, 1, 64), torch.tensor(0xFF, dtype=torch.uint8, device="cuda"), cache.v[b]))
    before = cache.weight.clone() if weight else None
    out = torch.full((B, n, H, hd), 9.0, dtype=torch.bfloat16, device="cuda")
    fc.fc_qcache_attention(ctx, cache, q, ints(held), None if new is None else ints(new), out, key_mask=mask, scale=scale, accumulate=weight)
    torch.cuda.synchronize()
    for b in range(B):
        m = tot[b] - held[b]
        qu.check_attention(qu.to_oracle(cache, b), q[b], out[b], held[b], m, hd ** -0.5 if scale is None else scale,
                           None if mask is None else mask[b].cpu().numpy(),
                           before[b].cpu().numpy().astype(np.float64) if weight else None,
                           cache.weight[b].cpu().numpy().astype(np.float64) if weight else None)
        qu.same(out[b, m:].float().cpu(), np.full(out[b, m:].shape, 9.0), "outputs of tokens that do not count")
    return cache, out


@pytest.mark.parametrize("heads", list(HEADS))
@pytest.mark.parametrize("n,held,new", [
    (1, [0, 5, 63], None), (1, [64, 190, 255], None), (2, [0, 62, 100], [2, 1, 0]), (7, [0, 58, 200], None), (19, [3, 0, 50], [19, 5, 1]),
    (70, [0, 1, 130], [70, 33, 69])])
def test_attention(fc, ctx, heads, n, held, new):
    g = torch.Generator().manual_seed(n)
    run_attention(fc, ctx, g, heads, 3, n, 256, held, new)


@pytest.mark.parametrize("heads,n,held", [("qwen", 1, [1000, 3]), ("toy", 1, [1500, 2047]), ("wide", 3, [1900, 64]), ("three", 40, [700, 1200])])
def test_attention_split_over_a_longer_cache(fc, ctx, heads, n, held):
    g = torch.Generator().manual_seed(5)
    run_attention(fc, ctx, g, heads, 2, n, 2048, held, None)
    run_attention(fc, ctx, g, heads, 2, n, 2048, held, None, weight=False)


@pytest.mark.parametrize("heads", ["qwen", "toy", "wide"])
@pytest.mark.parametrize("n", [1, 6, 66])
def test_attention_masked_keys(fc, ctx, heads, n):
    """Keys hidden one by one, in whole blocks and all of an item's (its tokens then see nothing and
    give 0), with NaN and infinities in the hidden rows."""
    g = torch.Generator().manual_seed(6)
    H, kv, hd, _ = HEADS[heads]
    B, cap, held = 4, 384, [200, 317, 100, 0]
    cache = filled(fc, g, B, kv, hd, cap)
    mask = torch.rand(B, cap, generator=g) > 0.4
    mask[1, 64:256] = False
    mask[2] = False
    mask[3, 0] = False           # the first token's only key
    mask = mask.cuda()
    hidden = ~mask
    cache.k.copy_(torch.where(hidden[:, None, :, None], torch.tensor(0xFF, dtype=torch.uint8, device="cuda"), cache.k))
    cache.v.copy_(torch.where(hidden.view(B, 1, -1, 1, 64), torch.tensor(0x7F, dtype=torch.uint8, device="cuda"), cache.v))
    _, out = run_attention(fc, ctx, g, heads, B, n, cap, held, None, mask=mask.to(torch.uint8) * 3, cache=cache)
    assert not out[2].any() and not out[3, 0].any()


@pytest.mark.parametrize("heads,n", [("qwen", 5), ("toy", 70), ("one", 20), ("three", 33)])
def test_attention_nan_reaches_who_sees_it(fc, ctx, heads, n):
    """A NaN among a new row's key or value reaches that token and the later ones, no earlier one; one
    in a long-held row reaches all."""
    g = torch.Generator().manual_seed(7)
    H, kv, hd, _ = HEADS[heads]
    cap, held = 256, [70, 100, 128]
    cache = filled(fc, g, 3, kv, hd, cap)

    def put(b, h, j, d, value):
        if value:
            cache.v[b, h, j // 64, d, j % 64] = 0x7F
        else:
            cache.k[b, h, j, d] = 0xFF
    put(0, 0, held[0] + n // 2, 3, True)
    put(1, kv - 1, held[1] + n - 1, 60, True)
    put(1, kv - 1, held[1] + n // 3, 7, False)
    put(2, 0, 5, 0, True)
    _, out = run_attention(fc, ctx, g, heads, 3, n, cap, held, None, cache=cache)
    nan = out.isnan().any(-1)
    assert nan[0, n // 2:, 0].all() and not nan[0, :n // 2].any() and nan[2, :, 0].all()


def test_attention_extreme_scores(fc, ctx):
    """Scores of hundreds (one key takes all), equal scores, and a scale of 0."""
    g = torch.Generator().manual_seed(8)
    H, kv, hd, _ = HEADS["qwen"]
    cache = filled(fc, g, 1, kv, hd, 256)
    run_attention(fc, ctx, g, "qwen", 1, 3, 256, [180], None, scale=4.0, cache=cache)
    run_attention(fc, ctx, g, "qwen", 1, 3, 256, [180], None, scale=0.0, cache=cache)
    q = torch.zeros(1, 3, H, hd, dtype=torch.bfloat16, device="cuda")
    run_attention(fc, ctx, g, "qwen", 1, 3, 256, [180], None, cache=cache, q=q)
    # scales at both ends: keys that vanish and values that are huge
    cache.k_scale[:, :, 0], cache.v_scale[:, :, 1] = 2.0 ** -100, 2.0 ** 100
    run_attention(fc, ctx, g, "qwen", 1, 3, 256, [180], None, cache=cache)


@pytest.mark.parametrize("heads,n", [("toy", 1), ("qwen", 3), ("three", 9), ("toy", 66)])
def test_attention_many_ragged_items(fc, ctx, heads, n):
    """More items than a wave has lanes, of lengths from nothing to the whole cache, some without new
    rows, the long ones at the end and in the middle."""
    g = torch.Generator().manual_seed(20 + n)
    B, cap = 133, 512
    held = [(37 * b * b) % 200 for b in range(B)]
    new = [(b * 7) % (n + 1) for b in range(B)]
    held[3] = held[64] = held[129] = 0
    new[3] = new[64] = n
    held[63], held[130], new[130] = cap - n, cap - n, n
    held[70] = cap                                      # full: its tokens are dropped
    tail = slice(100, 110)
    new[tail] = [0] * 10
    run_attention(fc, ctx, g, heads, B, n, cap, held, [min(x, cap - h) for x, h in zip(new, held)])


@pytest.mark.parametrize("heads,n,B,cap", [("qwen", 20, 300, 192), ("wide", 26, 400, 128)])
def test_attention_many_rounds_of_workgroups(fc, ctx, heads, n, B, cap):
    """Ragged batches of several times the workgroups that run at once: every item against products in
    64 bits (the tolerance of check_attention), tokens that do not count left alone, replays equal."""
    g = torch.Generator().manual_seed(50)
    H, kv, hd, _ = HEADS[heads]
    cache = filled(fc, g, B, kv, hd, cap)
    q = randn(g, B, n, H, hd)
    new = [(b * 5) % (n + 1) for b in range(B)]
    held = [0 if b % 50 == 7 else (b * b * 3) % (cap - n) for b in range(B)]
    before, k, v = cache.weight.clone(), cache.rows().double(), cache.rows(values=True).double()
    lens, m_new, out = ints(held), ints(new), torch.full_like(q, 9.0)
    call = lambda: fc.fc_qcache_attention(ctx, cache, q, lens, m_new, out, accumulate=True)  # noqa: E731
    call()
    first, weight = out.clone(), cache.weight.clone()
    for b in range(B):
        m, rows, G = new[b], held[b] + new[b], H // kv
        assert bool((out[b, m:] == 9.0).all())
        if m == 0:
            assert torch.equal(weight[b], before[b])
            continue
        kk, vv = k[b, :, :rows].repeat_interleave(G, 0), v[b, :, :rows].repeat_interleave(G, 0)
        qq = q[b, :m].double().transpose(0, 1).contiguous()
        hide = torch.arange(rows, device="cuda")[None] > held[b] + torch.arange(m, device="cuda")[:, None]
        p = (torch.matmul(qq, kk.transpose(1, 2).contiguous()) * hd ** -0.5).masked_fill(hide, float("-inf")).softmax(-1)
        mass = float((torch.matmul(qq.abs(), kk.abs().transpose(1, 2).contiguous()) * hd ** -0.5).max())
        rel = 4 * (hd + 4) * 2.0 ** -24 * mass + 2.0 ** -22 + rows * 2.0 ** -24
        want, absv = torch.matmul(p, vv).transpose(0, 1), torch.matmul(p, vv.abs()).transpose(0, 1)
        assert bool(((out[b, :m].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + rel) * absv).all()), b
        add = p.sum(1).view(kv, G, rows).sum(1)
        w = before[b, :, :rows].double() + add
        assert bool(((weight[b, :, :rows].double() - w).abs() <= (rel + m * G * 2.0 ** -24) * add + 2.0 ** -24 * w.abs() + 1e-30).all()), b
        assert torch.equal(weight[b, :, rows:], before[b, :, rows:])
    for _ in range(3):
        cache.weight.copy_(before)
        call()
        assert torch.equal(out, first) and torch.equal(cache.weight, weight)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        cache.weight.copy_(before)
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first) and torch.equal(cache.weight, weight)


@pytest.mark.parametrize("heads,n", [("qwen", 1), ("three", 7), ("qwen", 9), ("three", 50), ("toy", 90)])
def test_attention_masked_and_split(fc, ctx, heads, n):
    """Hidden keys (NaN in their rows) and a NaN that some tokens see, over cache lengths that splits share."""
    g = torch.Generator().manual_seed(30 + n)
    H, kv, hd, _ = HEADS[heads]
    B, cap, held = 3, 2048, [1900, 700, 64]
    cache = filled(fc, g, B, kv, hd, cap)
    mask = torch.rand(B, cap, generator=g) > 0.3
    mask[0, 300:1200] = False
    mask[2] = False
    mask = mask.cuda()
    cache.k.copy_(torch.where(~mask[:, None, :, None], torch.tensor(0x7F, dtype=torch.uint8, device="cuda"), cache.k))
    cache.v.copy_(torch.where(~mask.view(B, 1, -1, 1, 64), torch.tensor(0xFF, dtype=torch.uint8, device="cuda"), cache.v))
    j = held[0] + n // 2
    mask[0, j] = True
    cache.k[0, :, j] = 0x11
    cache.v[0, :, j // 64, :, j % 64] = 0x22
    cache.v[0, 0, j // 64, 5, j % 64] = 0x7F
    _, out = run_attention(fc, ctx, g, heads, B, n, cap, held, [n, n, max(1, n - 1)], mask=mask.to(torch.uint8), cache=cache)
    assert not out[2, :max(1, n - 1)].any()
    assert out[0, n // 2:, 0].isnan().any(-1).all() and not out[0, :n // 2].isnan().any()


@pytest.mark.parametrize("heads,n", [("qwen", 1), ("three", 9), ("qwen", 30)])
def test_attention_other_scales(fc, ctx, heads, n):
    """A negative scale turns the order of the keys; one that is huge leaves scores of 0 at 0."""
    g = torch.Generator().manual_seed(40 + n)
    H, kv, hd, _ = HEADS[heads]
    run_attention(fc, ctx, g, heads, 2, n, 1024, [900, 70], None, scale=-0.2)
    q = torch.zeros(2, n, H, hd, dtype=torch.bfloat16, device="cuda")
    run_attention(fc, ctx, g, heads, 2, n, 1024, [900, 70], None, scale=3e38, q=q)


def test_attention_few_heads_in_a_small_workspace(fc):
    """A context whose workspace holds no split's parts: one split, the same results."""
    g = torch.Generator().manual_seed(9)
    with fc.Context(fc.Caps(max_batch=1, max_height=28, max_width=28, max_tokens=4, max_seq=8, max_d_model=64, max_ffn=64, max_qkv=192)) as small:
        run_attention(fc, small, g, "toy", 1, 1, 2048, [1500], None)
        run_attention(fc, small, g, "toy", 1, 300, 512, [100], None, weight=False)
        run_attention(fc, small, g, "qwen", 1, 300, 512, [100], None)      # the rows' sums fit
        with pytest.raises(fc.FcError) as e:
            run_attention(fc, small, g, "qwen", 1, 600, 1024, [100], None)   # 16800 of them do not
        assert e.value.status == 3


def test_attention_offsets_past_32_bits(fc, ctx):
    """A cache of more than 2^32 bytes in one head, all but a few rows hidden: rows on both sides of
    the 4 GiB line count."""
    cap = 2 ** 25 + 4096
    cache = fc.QCache.alloc(1, 1, 128, cap)
    g = torch.Generator().manual_seed(10)
    mask = torch.zeros(1, cap, dtype=torch.uint8, device="cuda")
    rows = [0, 77, 2 ** 24 - 1, 2 ** 24, 2 ** 25 - 1, 2 ** 25, 2 ** 25 + 1000, 2 ** 25 + 2001]
    mask[0, rows] = 1
    cache.k_scale.fill_(2.0 ** -5)
    cache.v_scale.fill_(2.0 ** -5)
    code = lambda *s: (torch.randn(*s, generator=g) * 20).to(torch.float8_e4m3fn).view(torch.uint8).cuda()  # noqa: E731
    kc, vc = code(len(rows), 128), code(len(rows), 128)
    for i, r in enumerate(rows):
        cache.k[0, 0, r] = kc[i]
        cache.v[0, 0, r // 64, :, r % 64] = vc[i]
    q = randn(g, 1, 1, 1, 128)
    out = torch.empty_like(q)
    fc.fc_qcache_attention(ctx, cache, q, ints([2 ** 25 + 2001]), None, out, key_mask=mask, accumulate=True)
    k, v = (qu.values(x)[None] * 2.0 ** -5 for x in (kc, vc))
    want, prob, absv, _ = oq.attention(k, v, q[0].float().cpu().numpy(), len(rows), 128 ** -0.5)
    assert (np.abs(out[0].float().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -7 * absv).all()
    np.testing.assert_allclose(cache.weight[0, 0, rows].cpu().numpy(), prob[0, 0], rtol=1e-4)
    assert int((cache.weight != 0).sum()) == len(rows)
    # and an append there
    x = randn(g, 1, 2, 1, 128)
    fc.fc_qcache_append(ctx, cache, fc.RopeAxes(), None, x, x, ints([[0, 0]]), ints([2 ** 25 + 2002]), None, None)
    got = qu.values(cache.k[0, 0, 2 ** 25 + 2002:2 ** 25 + 2004]) * float(cache.k_scale[0, 0, (2 ** 25 + 2002) // 64])
    ref = x[0, :, 0].float().cpu().numpy()
    assert (np.abs(got - ref) <= np.maximum(2.0 ** -4 * np.abs(ref), 2.0 ** -15)).all()


# ------------------------------------------------------------------------------ evict
def run_evict(fc, ctx, g, heads, B, cap, held, keep, sink, recent, cache=None, cap2=None, weight2=True):
    H, kv, hd, _ = HEADS[heads]
    cache = filled(fc, g, B, kv, hd, cap) if cache is None else cache
    dst = qu.make(fc, B, kv, hd, cap2 or -(-keep // 64) * 64, weight2)
    before = [qu.to_oracle(dst, b) for b in range(B)]
    src = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.weight)]
    kept = torch.full((B, kv, keep), 77, dtype=torch.int32, device="cuda")
    left = torch.full((B,), -5, dtype=torch.int32, device="cuda")
    fc.fc_qcache_evict(ctx, cache, dst, ints(held), keep, sink, recent, kept, left)
    torch.cuda.synchronize()
    for t, u in zip(src, (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.weight)):
        assert torch.equal(t.view(torch.uint8), u.view(torch.uint8)), "the source changed"
    for b in range(B):
        n = min(max(held[b], 0), cap)
        with np.errstate(invalid="ignore"):
            want, rows = oq.evict(qu.to_oracle(cache, b), before[b], n, keep, sink, recent)
        m = min(n, keep)
        qu.same(kept[b].cpu(), np.pad(rows.reshape(kv, m), ((0, 0), (0, keep - m)), constant_values=-1), "kept rows")
        assert int(left[b]) == m
        got = qu.to_oracle(dst, b)
        for name in ("k", "v", "k_scale", "v_scale") + (("weight",) if weight2 else ()):
            qu.same(got[name], want[name], name)
    return dst


@pytest.mark.parametrize("heads", ["qwen", "toy", "one"])
@pytest.mark.parametrize("held,keep,sink,recent", [
    ([300, 0, 64], 100, 4, 20), ([320, 129, 63], 64, 0, 64), ([200, 201, 319], 200, 200, 0), ([320, 65, 1], 1, 0, 0), ([310, 250, 199], 199, 0, 0),
    ([66, 130, 5], 128, 0, 1)])
def test_evict(fc, ctx, heads, held, keep, sink, recent):
    g = torch.Generator().manual_seed(keep)
    run_evict(fc, ctx, g, heads, 3, 320, held, keep, sink, recent)
    run_evict(fc, ctx, g, heads, 3, 320, held, keep, sink, recent, cap2=512, weight2=False)


@pytest.mark.parametrize("cap,held,keep,sink,recent", [
    (4160, [4160, 4097, 1000], 2100, 4, 128), (16384, [16384, 9000, 3001], 3000, 0, 700), (16448, [16448, 16385, 64], 1500, 64, 0),
    (40000, [40000, 33333, 17000], 16900, 5, 77)])
def test_evict_long_caches(fc, ctx, cap, held, keep, sink, recent):
    """Caches of thousands of rows, with weights of few exponents and, for one item, few values."""
    g = torch.Generator().manual_seed(cap)
    B = len(held)
    cache = filled(fc, g, B, 2, 64, cap)
    cache.weight[1].copy_(torch.randint(0, 50, cache.weight[1].shape, generator=g).float().cuda() / 64)
    run_evict(fc, ctx, g, "group2", B, cap, held, keep, sink, recent, cache=cache)


def test_evict_long_cache_in_a_small_workspace(fc):
    """A context without room for the counts of several workgroups selects by one a head."""
    g = torch.Generator().manual_seed(60)
    with fc.Context(fc.Caps(max_batch=1, max_height=28, max_width=28, max_tokens=4, max_seq=8, max_d_model=64, max_ffn=64, max_qkv=192)) as small:
        run_evict(fc, small, g, "group2", 2, 16448, [16448, 16000], 4000, 9, 100)


def test_evict_ties_and_odd_weights(fc, ctx):
    """Few distinct weights (ties to the lower row), zeros of both signs, NaN, infinities, negative and
    subnormal weights."""
    g = torch.Generator().manual_seed(11)
    cache = filled(fc, g, 4, 2, 64, 1280)
    cache.weight.copy_(torch.randint(0, 3, cache.weight.shape, generator=g).float().cuda())
    odd = torch.tensor([0.0, -0.0, float("nan"), float("inf"), float("-inf"), -1.0, 1e-40, 2e-40, -1e-40, 3e38, -3.4028235e38])
    cache.weight[1] = odd[torch.randint(0, len(odd), (2, 1280), generator=g)].cuda()
    cache.weight[2] = 1.0
    for keep, sink, recent in ((700, 3, 5), (100, 0, 0), (1279, 0, 0)):
        run_evict(fc, ctx, g, "group2", 4, 1280, [1280, 1100, 1280, 900], keep, sink, recent, cache=cache)


def test_evict_numbers_that_are_not_finite(fc, ctx):
    """NaN codes move as NaN and set no scale; scales at both ends."""
    g = torch.Generator().manual_seed(12)
    cache = filled(fc, g, 2, 4, 64, 256)
    cache.k[0, 0, 17, 3] = 0x7F
    cache.v[0, 1, 1, 9, 5] = 0xFF
    cache.k_scale[1, 0, 1], cache.v_scale[1, 2, 0], cache.v_scale[1, 3] = 2.0 ** -100, 2.0 ** 100, 2.0 ** -100
    cache.v[1, 1] = 0
    run_evict(fc, ctx, g, "toy", 2, 256, [256, 200], 150, 20, 30, cache=cache)


# ------------------------------------------------------------------------------ together
def test_episode(fc, ctx):
    """A prompt, frames and single tokens of two items of different lengths, two layers that share the
    lengths, evictions into a spare cache when the budget is passed; every call against the oracle
    on the state before it."""
    g = torch.Generator().manual_seed(13)
    heads, B, L, cap, keep = "qwen", 2, 2, 256, 150
    H, kv, hd, sec = HEADS[heads]
    rope = fc.RopeAxes(1e6, sec)
    caches = [qu.make(fc, B, kv, hd, cap) for _ in range(L)]
    spare = qu.make(fc, B, kv, hd, cap)
    lens, time = [0, 0], [0, 0]
    for n, new in ((70, [70, 33]), (36, [36, 36]), (1, [1, 1]), (1, [1, 0]), (36, [30, 36]), (20, [20, 20]), (1, [1, 1]), (50, [50, 50]), (1, [1, 1])):
        if max(lens) + n > 200:
            left = ints([0, 0])
            for i in range(L):
                src = caches[i]
                before = [qu.to_oracle(spare, b) for b in range(B)]
                kept = torch.empty(B, kv, keep, dtype=torch.int32, device="cuda")
                fc.fc_qcache_evict(ctx, src, spare, ints(lens), keep, 4, 40, kept, left)
                for b in range(B):
                    want, _ = oq.evict(qu.to_oracle(src, b), before[b], lens[b], keep, 4, 40)
                    got = qu.to_oracle(spare, b)
                    for name in want:
                        qu.same(got[name], want[name], f"evict {name}")
                caches[i], spare = spare, src
            assert left.tolist() == [min(x, keep) for x in lens]
            lens = left.tolist()
        pos = torch.tensor([[[time[b] + t // 6 * (a > 0) for t in range(n)] for b in range(B)] for a in range(3)], dtype=torch.int32).cuda()
        for cache in caches:
            x = randn(g, B, n, (H + 2 * kv) * hd)
            q, k, v = x.view(B, n, H + 2 * kv, hd).split([H, kv, kv], 2)
            before = [qu.to_oracle(cache, b) for b in range(B)]
            qr, out = torch.zeros(B, n, H, hd, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, n, H, hd, dtype=torch.bfloat16, device="cuda")
            fc.fc_qcache_append(ctx, cache, rope, q, k, v, pos, ints(lens), ints(new), qr)
            mid = [qu.to_oracle(cache, b) for b in range(B)]
            fc.fc_qcache_attention(ctx, cache, qr, ints(lens), ints(new), out, accumulate=True)
            for b in range(B):
                m = new[b]
                kr, slack = qu.rotated(k[b], pos[:, b].cpu().numpy(), sec, 1e6)
                qu.check_appended(mid[b], before[b], kr[:m], slack[:m], v[b, :m].float().cpu().numpy().astype(np.float64), lens[b], m)
                qu.check_attention(mid[b], qr[b], out[b], lens[b], m, hd ** -0.5, None, mid[b]["weight"], cache.weight[b].cpu().numpy().astype(np.float64))
        lens = [a + b for a, b in zip(lens, new)]
        time = [t + 1 for t in time]


def test_captured_step_replays_match_eager(fc, ctx):
    """Append, accumulating attention, the lengths' advance and an eviction captured into one graph,
    replayed with other inputs and with eager calls between; each replay equals the eager calls."""
    g = torch.Generator().manual_seed(14)
    H, kv, hd, sec = HEADS["qwen"]
    B, n, cap, keep = 2, 3, 192, 100
    rope = fc.RopeAxes(1e6, sec)

    def state():
        c, d = qu.make(fc, B, kv, hd, cap), qu.make(fc, B, kv, hd, 128)
        return dict(c=c, d=d, lens=ints([0, 0]), new=ints([0, 0]), left=ints([0, 0]), kept=ints([[[0] * keep] * kv] * B),
                    x=torch.zeros(B, n, H + 2 * kv, hd, dtype=torch.bfloat16, device="cuda"), pos=ints([[[0] * n] * B] * 3),
                    q=torch.zeros(B, n, H, hd, dtype=torch.bfloat16, device="cuda"), out=torch.zeros(B, n, H, hd, dtype=torch.bfloat16, device="cuda"))

    def step(s):
        q, k, v = s["x"].split([H, kv, kv], 2)
        fc.fc_qcache_append(ctx, s["c"], rope, q, k, v, s["pos"], s["lens"], s["new"], s["q"])
        fc.fc_qcache_attention(ctx, s["c"], s["q"], s["lens"], s["new"], s["out"], accumulate=True)
        s["lens"].add_(s["new"])
        fc.fc_qcache_evict(ctx, s["c"], s["d"], s["lens"], keep, 2, 10, s["kept"], s["left"])

    def tensors(s):
        return [s["c"].k, s["c"].v, s["c"].k_scale, s["c"].v_scale, s["c"].weight, s["d"].k, s["d"].v, s["d"].k_scale, s["d"].v_scale,
                s["d"].weight, s["lens"], s["left"], s["kept"], s["q"], s["out"]]

    init = filled(fc, g, B, kv, hd, cap)
    a, e = state(), state()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(a)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a)
    for rep, (held, new) in enumerate([([0, 0], [3, 1]), ([60, 150], [3, 3]), ([62, 10], [0, 2]), ([189, 128], [3, 1])]):
        x = randn(g, B, n, H + 2 * kv, hd)
        pos = torch.randint(0, 999, (3, B, n), generator=g, dtype=torch.int32).cuda()
        for s in (a, e):
            for name in ("k", "v", "k_scale", "v_scale", "weight"):
                getattr(s["c"], name).copy_(getattr(init, name))
                getattr(s["d"], name).zero_()
            for name, t in (("x", x), ("pos", pos), ("lens", ints(held)), ("new", ints(new)), ("kept", torch.zeros_like(s["kept"]))):
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
    caches = [filled(fc, g, 2, kv, hd, 2048) for _ in range(2)]
    q = [randn(g, 2, 9, H, hd) for _ in range(2)]
    w0 = [c.weight.clone() for c in caches]
    want, out = [torch.zeros_like(x) for x in q], [torch.zeros_like(x) for x in q]
    lens = ints([2000, 1500])
    for i in range(2):
        fc.fc_qcache_attention(ctx, caches[i], q[i], lens, None, want[i], accumulate=True)
    torch.cuda.synchronize()
    w1 = [c.weight.clone() for c in caches]
    with fc.Context(fc.Caps(max_batch=4, max_height=224, max_width=224, max_tokens=256, max_seq=288, max_d_model=256, max_ffn=1024, max_qkv=768)) as other:
        for c, w in zip(caches, w0):
            c.weight.copy_(w)
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        for _ in range(3):
            for i, (s, c) in enumerate(zip(streams, (ctx, other))):
                with torch.cuda.stream(s):
                    caches[i].weight.copy_(w0[i])
                    fc.fc_qcache_attention(c, caches[i], q[i], lens, None, out[i], accumulate=True)
        torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(out[i], want[i]) and torch.equal(caches[i].weight, w1[i])


def test_same_inputs_same_bytes(fc, ctx):
    g = torch.Generator().manual_seed(16)
    H, kv, hd, _ = HEADS["wide"]
    cache = filled(fc, g, 3, kv, hd, 1024)
    w, q, lens = cache.weight.clone(), randn(g, 3, 37, H, hd), ints([900, 500, 0])
    got = []
    for _ in range(3):
        cache.weight.copy_(w)
        out = torch.zeros_like(q)
        fc.fc_qcache_attention(ctx, cache, q, lens, ints([37, 20, 5]), out, accumulate=True)
        got.append((out, cache.weight.clone()))
    for o, x in got[1:]:
        assert torch.equal(o, got[0][0]) and torch.equal(x, got[0][1])


def test_written_buffers_share_no_memory(fc, ctx):
    H, kv, hd, sec = HEADS["toy"]
    c, lens = qu.make(fc, 1, kv, hd, 128), ints([0])
    x = torch.ones(1, 2, H, hd, dtype=torch.bfloat16, device="cuda")
    over = c.k.view(-1)[:x.numel() * 2].view(torch.bfloat16).view(x.shape)
    k = c.v.view(-1)[:2 * 2 * kv * hd].view(torch.bfloat16).view(1, 2, kv, hd)
    one = torch.ones(1, 2, kv, hd, dtype=torch.bfloat16, device="cuda")
    before = [c.k.clone(), c.v.clone()]
    for f in (lambda: fc.fc_qcache_attention(ctx, c, x, lens, None, over),
              lambda: fc.fc_qcache_append(ctx, c, fc.RopeAxes(1e6, sec), x, one, one, ints([[[0, 0]]] * 3), lens, None, over),
              lambda: fc.fc_qcache_append(ctx, c, fc.RopeAxes(1e6, sec), None, k, one, ints([[[0, 0]]] * 3), lens, None, None)):
        with pytest.raises(fc.FcError) as e:
            f()
        assert e.value.status == 1
    torch.cuda.synchronize()
    assert torch.equal(c.k, before[0]) and torch.equal(c.v, before[1])


def test_guards(fc, ctx):
    """Every buffer inside a larger allocation whose bytes around it stay as they are."""
    from tests.test_gpu_guards import Guarded
    g = torch.Generator().manual_seed(17)
    H, kv, hd, sec = HEADS["qwen"]
    B, n, cap, keep = 3, 70, 192, 100
    gd = Guarded()

    def buf(shape, dtype, fill):
        return gd.new(shape, dtype, fill if isinstance(fill, torch.Tensor) else torch.full((1,), fill, dtype=dtype, device="cuda"))

    def cache(c):
        nb = c // 64
        u8, f = torch.uint8, torch.float32
        return fc.QCache(buf((B, kv, c, hd), u8, 0x7F), buf((B, kv, nb, hd, 64), u8, 0x7F), buf((B, kv, nb), f, 1.0), buf((B, kv, nb), f, 1.0),
                         buf((B, kv, c), f, 1.0))
    src, dst = cache(cap), cache(128)
    bf = torch.bfloat16
    x = buf((B, n, H + 2 * kv, hd), bf, randn(g, B, n, H + 2 * kv, hd))
    q, out = buf((B, n, H, hd), bf, 0), buf((B, n, H, hd), bf, 0)
    i32 = torch.int32
    pos, lens, new = buf((3, B, n), i32, 5), buf((B,), i32, ints([0, 0, 0])), buf((B,), i32, ints([70, 64, 3]))
    kept, left = buf((B, kv, keep), i32, 0), buf((B,), i32, 0)
    mask = buf((B, cap), torch.uint8, 1)
    for _ in range(3):
        a, b, c = x.split([H, kv, kv], 2)
        fc.fc_qcache_append(ctx, src, fc.RopeAxes(1e6, sec), a, b, c, pos, lens, new, q)
        fc.fc_qcache_attention(ctx, src, q, lens, new, out, key_mask=mask, accumulate=True)
        lens.add_(new)
        fc.fc_qcache_evict(ctx, src, dst, lens, keep, 3, 20, kept, left)
    gd.check()
    assert not out.isnan().any()


def test_debug_mode_and_kernel_times(fc, ctx):
    """The calls run under the debug mode, and their kernels appear in the context's timing."""
    g = torch.Generator().manual_seed(18)
    prev = fc.fc_debug(True)
    fc.fc_profile_enable(ctx, True)
    try:
        fc.fc_profile_read(ctx, None, reset=True)
        run_append(fc, ctx, g, "toy", 1, 3, 128, [0], None)
        run_attention(fc, ctx, g, "toy", 1, 3, 128, [20], None)
        run_evict(fc, ctx, g, "toy", 1, 128, [128], 64, 1, 2)
        for name in ("fc_qappend", "fc_qattn", "fc_qevict_pick", "fc_qevict_move"):
            assert fc.fc_profile_read(ctx, name)[1] >= 1, name
    finally:
        fc.fc_profile_enable(ctx, False)
        fc.fc_profile_read(ctx, None, reset=True)
        fc.fc_debug(prev)


def test_binding_refusals(fc, ctx):
    """What the binding and the library refuse, with nothing written."""
    H, kv, hd, sec = HEADS["toy"]
    c, d = qu.make(fc, 2, kv, hd, 128), qu.make(fc, 2, kv, hd, 64)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    x = torch.ones(2, 3, H + 2 * kv, hd, **bf)
    q, k, v = x.split([H, kv, kv], 2)
    pos, lens, rope = ints([[[0] * 3] * 2] * 3), ints([0, 0]), fc.RopeAxes(1e6, sec)
    qo = torch.ones(2, 3, H, hd, **bf)
    kept = ints([[[0] * 64] * kv] * 2)
    state = [t.clone() for t in (c.k, c.v, c.weight, d.k, qo, kept)]
    bad = [
        lambda: fc.fc_qcache_append(ctx, c, rope, q, k, v, pos[0], lens, None, qo),                      # one axis for three
        lambda: fc.fc_qcache_append(ctx, c, rope, q, k, v, pos, lens, None, None),
        lambda: fc.fc_qcache_append(ctx, c, rope, q, k[:1], v, pos, lens, None, qo),
        lambda: fc.fc_qcache_append(ctx, c, rope, q, k.float(), v, pos, lens, None, qo),
        lambda: fc.fc_qcache_append(ctx, c, rope, q, k, v.transpose(2, 3).contiguous().transpose(2, 3), pos, lens, None, qo),
        lambda: fc.fc_qcache_append(ctx, c, rope, q, k, v, pos, lens.long(), None, qo),
        lambda: fc.fc_qcache_append(ctx, c, rope, q, k, v, pos, lens, ints([1]), qo),
        lambda: fc.fc_qcache_append(ctx, c, rope, q, k, v, pos.cpu(), lens, None, qo),
        lambda: fc.fc_qcache_attention(ctx, c, qo[..., :32].contiguous(), lens, None, qo),
        lambda: fc.fc_qcache_attention(ctx, c, qo[:1], lens, None, qo),
        lambda: fc.fc_qcache_attention(ctx, c, qo, lens, None, torch.ones(2, 3, H, hd, device="cuda")),
        lambda: fc.fc_qcache_attention(ctx, c, qo, lens, None, torch.ones_like(qo), key_mask=torch.ones(2, 64, dtype=torch.uint8, device="cuda")),
        lambda: fc.fc_qcache_evict(ctx, c, d, lens, 65, 0, 0, kept),
        lambda: fc.QCache(c.k, c.v, c.k_scale[..., :1], c.v_scale, c.weight),
        lambda: fc.QCache(c.k, c.v.view(torch.int8), c.k_scale, c.v_scale, c.weight),
        lambda: fc.QCache(c.k[..., :100, :], c.v, c.k_scale, c.v_scale),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {i} went through")
    status = [
        (1, lambda: fc.fc_qcache_append(ctx, c, fc.RopeAxes(1e6, (8, 8, 8)), q, k, v, pos, lens, None, qo)),
        (1, lambda: fc.fc_qcache_append(ctx, c, fc.RopeAxes(1.0, sec), q, k, v, pos, lens, None, qo)),
        (2, lambda: fc.fc_qcache_append(ctx, c, rope, q[:, :, :3], k, v, pos, lens, None, qo)),
        (1, lambda: fc.fc_qcache_append(ctx, c, rope, q, k, v, pos, lens, None, x.view(-1)[:2 * 3 * H * hd].view(2, 3, H, hd))),
        (1, lambda: fc.fc_qcache_attention(ctx, c, qo, lens, None, qo)),
        (1, lambda: fc.fc_qcache_attention(ctx, fc.QCache(c.k, c.v, c.k_scale, c.v_scale), qo, lens, None, torch.ones_like(qo), accumulate=True)),
        (1, lambda: fc.fc_qcache_attention(ctx, c, qo, lens, None, torch.ones_like(qo), scale=float("nan"))),
        (2, lambda: fc.fc_qcache_attention(ctx, d, torch.ones(2, 65, H, hd, **bf), lens, None, torch.ones(2, 65, H, hd, **bf))),
        (1, lambda: fc.fc_qcache_evict(ctx, c, d, lens, 64, 40, 30, kept)),
        (1, lambda: fc.fc_qcache_evict(ctx, c, c, lens, 64, 0, 0, kept)),
        (1, lambda: fc.fc_qcache_evict(ctx, c, d, lens, 64, 0, 0, kept, lens)),
        (2, lambda: fc.fc_qcache_evict(ctx, c, qu.make(fc, 2, kv, 128, 64), lens, 64, 0, 0, kept)),
        (2, lambda: fc.fc_qcache_evict(ctx, c, d, lens, 65, 0, 0, ints([[[0] * 65] * kv] * 2))),
        (6, lambda: fc.fc_qcache_attention(ctx, qu.make(fc, 2, kv, 32, 64), torch.ones(2, 1, H, 32, **bf), lens, None, torch.ones(2, 1, H, 32, **bf))),
    ]
    for i, (want, f) in enumerate(status):
        with pytest.raises(fc.FcError) as e:
            f()
            pytest.fail(f"call {i} went through")
        assert e.value.status == want, (i, str(e.value))
    torch.cuda.synchronize()
    for t, u in zip(state, (c.k, c.v, c.weight, d.k, qo, kept)):
        assert torch.equal(t.view(torch.uint8), u.view(torch.uint8))
