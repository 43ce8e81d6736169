"""The 8-bit token cache's attention at the ends of its ranges: the largest numbers, hidden and
seen, and the numbers of splits that only longer caches or larger batches reach.  Tolerances are
those of tests/qcache_util.py."""
import pytest
import torch

from tests import qcache_util as qu
from tests.test_gpu_qcache import HEADS, ctx, fc, filled, ints, randn, run_attention  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def wide_ctx(fc):  # noqa: F811
    """A context whose workspace holds the parts of large batches."""
    with fc.Context(fc.Caps(max_batch=64, max_height=224, max_width=224, max_tokens=256, max_seq=288, max_d_model=256, max_ffn=1024,
                            max_qkv=768)) as c:
        yield c


def codes(x):
    return x.to(torch.float8_e4m3fn).view(torch.uint8)


def check_on_device(cache, before, q, out, held, new, mask=None):
    """Every item against products in 64 bits on the GPU, with the tolerance of check_attention.  before:
    the weights before the call.  NaN among the values reaches who sees it."""
    B, n, H, hd = q.shape
    kv = cache.k.shape[1]
    G = H // kv
    for b in range(B):
        m, rows = new[b], held[b] + new[b]
        assert bool((out[b, m:] == 9.0).all()), b
        if m == 0:
            assert torch.equal(cache.weight[b], before[b]), b
            continue
        nb = -(-rows // 64)
        item = lambda t, s, by_columns: ((t.transpose(-1, -2) if by_columns else t.view(kv, -1, 64, hd))[:, :nb].contiguous()  # noqa: E731
                                         .view(torch.float8_e4m3fn).double() * s[:, :nb, None, None].double()).reshape(kv, -1, hd)[:, :rows]
        k, v = item(cache.k[b], cache.k_scale[b], False), item(cache.v[b], cache.v_scale[b], True)
        hide = torch.arange(rows, device="cuda")[None] > held[b] + torch.arange(m, device="cuda")[:, None]
        if mask is not None:
            hide = hide | (mask[b, :rows] == 0)
        add = torch.zeros(kv, rows, dtype=torch.float64, device="cuda")
        worst = 0.0
        for h in range(H):
            kk, vv, qq = k[h // G], v[h // G], q[b, :m, h].double()
            s = (qq @ kk.t().contiguous() * hd ** -0.5).masked_fill(hide, float("-inf"))
            p = s.softmax(-1).nan_to_num(0.0)                     # no key seen: no weight
            mass = float((qq.abs() @ kk.abs().t().contiguous() * hd ** -0.5).masked_fill(hide, 0.0).max())
            rel = 4 * (hd + 4) * 2.0 ** -24 * mass + 2.0 ** -22 + rows * 2.0 ** -24
            worst = max(worst, rel)
            odd = ((~hide).double() @ vv.isnan().double()) > 0    # some NaN seen
            vv = vv.nan_to_num(0.0)
            want, absv = p @ vv, p @ vv.abs()
            got = out[b, :m, h].double()
            assert torch.equal(got.isnan(), odd), f"item {b}, head {h}: NaN"
            off = (got - want).abs().masked_fill(odd, 0.0)
            assert bool((off <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + rel) * absv).all()), f"item {b}, head {h}"
            add[h // G] += p.sum(0)
        w = before[b, :, :rows].double() + add
        err = (cache.weight[b, :, :rows].double() - w).abs()
        assert bool((err <= (worst + m * G * 2.0 ** -24) * add + 2.0 ** -24 * w.abs() + 1e-30).all()), f"weights of item {b}"
        assert torch.equal(cache.weight[b, :, rows:], before[b, :, rows:]), b


@pytest.mark.parametrize("heads,n,cap", [("qwen", 1, 256), ("toy", 5, 256), ("wide", 1, 256), ("qwen", 2, 2048), ("three", 30, 256), ("toy", 60, 256),
                                         ("three", 40, 2048)])
def test_hidden_rows_of_the_largest_numbers(fc, ctx, heads, n, cap):  # noqa: F811
    """In a block whose scale is 2^120 (as a value of bfloat16's lowest number gives it) codes of 256 and
    more lie beyond float32.  Hidden by the mask, behind the last row or in a later token's row, they
    have no effect on a token."""
    g = torch.Generator().manual_seed(70 + n)
    H, kv, hd, _ = HEADS[heads]
    cache = filled(fc, g, 2, kv, hd, cap)
    held = [cap - 64 - n, cap - 128 + 10]
    mask = torch.ones(2, cap, dtype=torch.uint8, device="cuda")
    for b in range(2):
        last = held[b] + n - 1
        for blk in {held[b] // 64, last // 64}:
            cache.v_scale[b, :, blk] = 2.0 ** 120
            cache.v[b, :, blk] = codes(torch.randn(kv, hd, 64, generator=g) * 0.1).cuda()
        j = held[b] - 3                                # a hidden row among them: lowest number and -infinity as they are held
        mask[b, j] = 0
        cache.v[b, :, j // 64, :, j % 64] = 0xF8
        cache.v[b, :, j // 64, 1, j % 64] = 0xFE
        cache.v[b, :, last // 64, 2, last % 64] = 0x78   # the last token's row
        tail = torch.arange(cap, device="cuda").view(-1, 64) > last
        cache.v[b] = torch.where(tail[None, :, None], 0x7E, cache.v[b])
        cache.k[b, :, last + 1:] = 0x7E
    _, out = run_attention(fc, ctx, g, heads, 2, n, cap, held, None, mask=mask, poison=False, cache=cache)
    assert not out.isnan().any() and (n == 1 or not out[:, :-1].isinf().any())
    if n > 1:                                          # the same without a mask: later tokens and the rows behind alone
        for b in range(2):
            j = held[b] - 3
            cache.v[b, :, j // 64, :, j % 64] = 0x08
        _, out = run_attention(fc, ctx, g, heads, 2, n, cap, held, None, poison=False, cache=cache)
        assert not out.isnan().any() and not out[:, :-1].isinf().any()


@pytest.mark.parametrize("heads,n,cap", [("qwen", 1, 512), ("toy", 3, 512), ("wide", 1, 512), ("three", 40, 512), ("toy", 70, 512), ("qwen", 20, 2048)])
def test_values_whose_sum_passes_float32(fc, ctx, heads, n, cap):  # noqa: F811
    """Values up to 448 2^119 (2.98e38), seen by equal shares and by ordinary ones: their mean is a finite
    number though their sum is none."""
    g = torch.Generator().manual_seed(80 + n)
    H, kv, hd, _ = HEADS[heads]
    cache = filled(fc, g, 2, kv, hd, cap)
    cache.v.copy_(codes(torch.rand(cache.v.shape, generator=g) * 400 + 40).cuda())
    cache.v_scale.fill_(2.0 ** 119)
    held = [400, 333]
    q = torch.zeros(2, n, H, hd, dtype=torch.bfloat16, device="cuda")
    for x in (q, randn(g, 2, n, H, hd)):
        _, out = run_attention(fc, ctx, g, heads, 2, n, cap, held, None, poison=False, cache=cache, q=x)
        assert bool(out.isfinite().all())


@pytest.mark.parametrize("heads,n", [("qwen", 1), ("toy", 6), ("three", 40), ("toy", 70)])
def test_least_values(fc, ctx, heads, n):  # noqa: F811
    """Values of the smallest scale, down to the least number 2^-109, keep their bits."""
    g = torch.Generator().manual_seed(85 + n)
    H, kv, hd, _ = HEADS[heads]
    cache = filled(fc, g, 2, kv, hd, 512)
    cache.v.copy_(codes(torch.randn(cache.v.shape, generator=g) * 0.03).cuda())
    cache.v_scale.fill_(2.0 ** -100)
    run_attention(fc, ctx, g, heads, 2, n, 512, [400, 3], None, poison=False, cache=cache)


@pytest.mark.parametrize("heads,B,n,cap,masked", [
    ("toy", 1, 40, 4096, False),        # 16 splits: the join takes two rounds of eight
    ("qwen", 1, 40, 16384, False),      # 32 splits of eight blocks at least
    ("wide", 1, 90, 8192, True),        # 16 of them
    ("toy", 60, 66, 2048, False),       # 2 splits of eight blocks at least
    ("three", 180, 30, 4608, False)])   # 4 splits, which fill a last round
def test_numbers_of_splits(fc, wide_ctx, heads, B, n, cap, masked):  # noqa: F811
    """Many rows in as many splits as long caches and batches of less than a round get, ragged, weighed,
    with items that fill some of the splits only; replays equal."""
    g = torch.Generator().manual_seed(90 + n)
    H, kv, hd, _ = HEADS[heads]
    cache = filled(fc, g, B, kv, hd, cap)
    q = randn(g, B, n, H, hd)
    new = [n - 3] if B == 1 else [(b * 7) % (n + 1) if b % 3 else n for b in range(B)]
    held = [cap - n - 200] if B == 1 else [cap - n - (b * b * 37) % (cap - n) if b % 4 else cap - n for b in range(B)]
    mask = (torch.rand(B, cap, generator=g) > 0.3).to(torch.uint8).cuda() if masked else None
    before, out = cache.weight.clone(), torch.full_like(q, 9.0)
    lens, m_new = ints(held), ints(new)
    call = lambda: fc.fc_qcache_attention(wide_ctx, cache, q, lens, m_new, out, key_mask=mask, accumulate=True)  # noqa: E731
    call()
    first, weight = out.clone(), cache.weight.clone()
    step = max(1, B // 24)
    some = list(range(0, B, step)) + [B - 1]
    part = fc.QCache(*(t[some].contiguous() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.weight)))
    check_on_device(part, before[some], q[some], out[some], [held[b] for b in some], [new[b] for b in some], None if mask is None else mask[some])
    for _ in range(2):
        cache.weight.copy_(before)
        out.fill_(9.0)
        call()
        assert torch.equal(out, first) and torch.equal(cache.weight, weight)


@pytest.mark.parametrize("heads,B,n,cap,masked", [("qwen", 2, 2, 131072, False), ("wide", 1, 1, 524288, True), ("three", 4, 10, 65536, False)])
def test_few_rows_whose_scores_do_not_fit(fc, ctx, heads, B, n, cap, masked):  # noqa: F811
    """Weighed calls of a few rows over caches so large that the workspace has no room for their scores:
    the weights compute them again."""
    g = torch.Generator().manual_seed(60 + n)
    H, kv, hd, _ = HEADS[heads]
    cache = filled(fc, g, B, kv, hd, cap)
    q = randn(g, B, n, H, hd)
    held = [cap - n - 1000 * b - 17 if b < 3 else 5 for b in range(B)]
    new = [max(1, n - b) for b in range(B)]
    mask = (torch.rand(B, cap, generator=g) > 0.3).to(torch.uint8).cuda() if masked else None
    before, out = cache.weight.clone(), torch.full_like(q, 9.0)
    fc.fc_qcache_attention(ctx, cache, q, ints(held), ints(new), out, key_mask=mask, accumulate=True)
    check_on_device(cache, before, q, out, held, new, mask)


@pytest.mark.parametrize("heads,B,n,cap", [("qwen", 300, 20, 192), ("wide", 400, 26, 128)])
@pytest.mark.parametrize("odd", [False, True])
def test_many_rounds_masked(fc, ctx, heads, B, n, cap, odd):  # noqa: F811
    """Batches of several rounds of workgroups with a key mask, NaN in the hidden rows and (odd) in some
    that tokens see; all of one length too."""
    g = torch.Generator().manual_seed(95)
    H, kv, hd, _ = HEADS[heads]
    cache = filled(fc, g, B, kv, hd, cap)
    q = randn(g, B, n, H, hd)
    mask = torch.rand(B, cap, generator=g) > 0.3
    mask[5] = False
    mask = mask.cuda()
    cache.k.copy_(torch.where(~mask[:, None, :, None], torch.tensor(0x7F, dtype=torch.uint8, device="cuda"), cache.k))
    cache.v.copy_(torch.where(~mask.view(B, 1, -1, 1, 64), torch.tensor(0xFF, dtype=torch.uint8, device="cuda"), cache.v))
    ragged = [(b * 5) % (n + 1) for b in range(B)], [0 if b % 50 == 7 else (b * b * 3) % (cap - n) for b in range(B)]
    for new, held in (ragged, ([n] * B, [cap - n - 5] * B)):
        if odd:
            for b in range(0, B, 9):
                j = min(held[b] + new[b] // 2, cap - 1)
                mask[b, j] = True
                cache.k[b, :, j] = 0x11
                cache.v[b, :, j // 64, :, j % 64] = 0x22
                cache.v[b, b % kv, j // 64, 5, j % 64] = 0x7F
        before, out = cache.weight.clone(), torch.full_like(q, 9.0)
        fc.fc_qcache_attention(ctx, cache, q, ints(held), ints(new), out, key_mask=mask.to(torch.uint8), accumulate=True)
        some = list(range(0, B, 9)) + [1, 5, B - 1]
        part = fc.QCache(*(t[some].contiguous() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.weight)))
        check_on_device(part, before[some], q[some], out[some], [held[b] for b in some], [new[b] for b in some], mask[some])


@pytest.mark.parametrize("heads,n,cap,held", [("qwen", 1, 256, [130, 60]), ("toy", 6, 256, [130, 60]), ("qwen", 5, 2048, [1900, 700]), ("three", 40, 256, [130, 60]),
                                              ("toy", 70, 256, [130, 60]), ("three", 40, 2048, [1900, 700]), ("qwen", 70, 512, [300, 64])])
@pytest.mark.parametrize("masked", [False, True])
def test_hidden_rows_leave_no_bit(fc, ctx, heads, n, cap, held, masked):  # noqa: F811
    """A token's output and the weights of what it sees keep every bit whatever stands in rows that are
    hidden from it: masked ones, those behind the last, and, for all but the last token, that one's
    own (its key far above all others for some queries)."""
    g = torch.Generator().manual_seed(100 + n)
    H, kv, hd, _ = HEADS[heads]
    cache = filled(fc, g, 2, kv, hd, cap)
    q = randn(g, 2, n, H, hd)
    mask = (torch.rand(2, cap, generator=g) > 0.3).to(torch.uint8).cuda() if masked else None
    lens, w0 = ints(held), cache.weight.clone()
    got = []
    for change in (False, True):
        for b in range(2) if change else ():
            last = held[b] + n - 1
            hide = torch.arange(cap, device="cuda") > last
            if masked:
                hide |= mask[b] == 0
            junk = codes((torch.randn(cache.k[b].shape, generator=g) * 200).clamp(-448, 448)).cuda()
            cache.k[b] = torch.where(hide[None, :, None], junk, cache.k[b])
            junk = codes((torch.randn(cache.v[b].shape, generator=g) * 200).clamp(-448, 448)).cuda()
            cache.v[b] = torch.where(hide.view(-1, 64)[None, :, None], junk, cache.v[b])
            if n > 1:
                cache.k[b, :, last] = codes((torch.randn(kv, hd, generator=g) * 400).clamp(-448, 448)).cuda()
                cache.v[b, :, last // 64, :, last % 64] = codes((torch.randn(kv, hd, generator=g) * 400).clamp(-448, 448)).cuda()
        cache.weight.copy_(w0)
        out = torch.full_like(q, 9.0)
        fc.fc_qcache_attention(ctx, cache, q, lens, None, out, key_mask=mask, accumulate=n == 1)
        got.append((out, cache.weight.clone()))
    seen = slice(0, n - 1) if n > 1 else slice(0, 1)
    a, c = got[0][0][:, seen], got[1][0][:, seen]
    assert torch.equal(a.view(torch.int16), c.view(torch.int16)), f"{int((a != c).sum())} outputs of {a.numel()} changed"
    assert torch.equal(got[0][1], got[1][1])


@pytest.mark.parametrize("heads,n,cap,held", [("qwen", 1, 512, [400, 300]), ("toy", 6, 512, [400, 300]), ("qwen", 2, 2048, [1900, 700]), ("three", 40, 512, [400, 300]),
                                              ("toy", 70, 512, [400, 300]), ("three", 40, 2048, [1900, 700])])
def test_hidden_blocks_of_any_scale(fc, ctx, heads, n, cap, held):  # noqa: F811
    """Whole blocks hidden by the mask (rows counted as held that nothing was written to): neither their
    codes nor their scales have an effect, whatever they hold."""
    g = torch.Generator().manual_seed(110 + n)
    H, kv, hd, _ = HEADS[heads]
    cache = filled(fc, g, 2, kv, hd, cap)
    q = randn(g, 2, n, H, hd)
    mask = torch.ones(2, cap, dtype=torch.uint8, device="cuda")
    mask[0, :128], mask[1, 64:256] = 0, 0
    w0, lens, got = cache.weight.clone(), ints(held), []
    odd = [float("nan"), float("inf"), float("-inf"), 0.0, -1.0, 3.4e38, 1e-44, 5.0, 2.0 ** -111, -2.0 ** -111]
    for junk in (None, *odd):
        if junk is not None:
            for b, blocks in ((0, (0, 1)), (1, (1, 2, 3))):
                for blk in blocks:
                    cache.k_scale[b, :, blk] = cache.v_scale[b, :, blk] = junk
                    cache.k[b, :, 64 * blk:64 * blk + 64] = codes((torch.randn(kv, 64, hd, generator=g) * 200).clamp(-448, 448)).cuda()
                    cache.v[b, :, blk] = codes((torch.randn(kv, hd, 64, generator=g) * 200).clamp(-448, 448)).cuda()
        cache.weight.copy_(w0)
        out = torch.full_like(q, 9.0)
        fc.fc_qcache_attention(ctx, cache, q, lens, None, out, key_mask=mask, accumulate=True)
        got.append((out.view(torch.int16), cache.weight.clone()))
    for junk, (o, w) in zip(odd, got[1:]):
        assert torch.equal(o, got[0][0]) and torch.equal(w, got[0][1]), f"scale {junk}"
