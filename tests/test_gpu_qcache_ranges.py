"""The 8-bit token cache's attention at the ends of its ranges: the largest numbers, hidden and
seen, and the least.  Tolerances are those of tests/qcache_util.py."""
import pytest
import torch

from tests import qcache_util as qu
from tests.test_gpu_qcache import HEADS, ctx, fc, filled, ints, randn, run_attention  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


def codes(x):
    return x.to(torch.float8_e4m3fn).view(torch.uint8)


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
