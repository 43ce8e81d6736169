"""Pins of the 8-bit token cache's oracle against things other than itself: torch's e4m3 type,
closed forms of the block scale, the layer oracle's rotary positions,
scaled_dot_product_attention in float64, and brute force over small evictions."""
import itertools

import numpy as np
import pytest
import torch
import torch.nn.functional as F

from oracle import layer as ol
from oracle import qcache as oq


def test_e4m3_is_torchs_type():
    """Every e4m3 number is itself; every bfloat16 number within 448 rounds as torch's cast does."""
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    fin = codes[np.isfinite(codes)]
    np.testing.assert_array_equal(oq.e4m3(fin), fin)
    x = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float()
    x = x[x.abs() <= 448]
    np.testing.assert_array_equal(oq.e4m3(x.numpy()), x.to(torch.float8_e4m3fn).float().numpy())


def test_e4m3_range():
    np.testing.assert_array_equal(oq.e4m3([449.0, 1e30, np.inf, -np.inf, -500.0]), [448, 448, 448, -448, -448])
    assert np.isnan(oq.e4m3(np.nan))
    np.testing.assert_array_equal(oq.e4m3([17.0, 19.0, 18.0, 2.0 ** -10, 3 * 2.0 ** -10]), [16, 20, 18, 0, 2.0 ** -8])


@pytest.mark.parametrize("amax,want", [(448.0, 1.0), (448.0001, 2.0), (224.0, 0.5), (1.0, 2.0 ** -8), (0.875, 2.0 ** -9),
                                       (0.0, 2.0 ** -100), (1e-38, 2.0 ** -100), (3.0e38, 2.0 ** 120)])
def test_block_scale(amax, want):
    assert oq.block_scale(amax) == want


def test_rotation_is_the_layers():
    """Sections and pairing are those of the decoder layer's multimodal positions, and one axis
    those of its plain ones (float32 cosines there)."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((7, 3, 128))
    pos = rng.integers(0, 5000, (3, 7))
    c, s = ol.mrope_cos_sin(pos.T, (16, 24, 24), 128, 1e6)
    np.testing.assert_allclose(oq.rotate(x, pos, (16, 24, 24), 1e6), ol.rope(x, c, s), atol=1e-5)
    c, s = ol.rope_cos_sin(pos[0], 128, 1e6)
    np.testing.assert_allclose(oq.rotate(x, pos[:1], (0, 0, 0), 1e6), ol.rope(x, c, s), atol=1e-5)


def test_rotation_is_relative():
    """q . k after rotation depends on the difference of the positions of each axis only."""
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 1, 64))
    for d in (0, 9, 100000):
        a = oq.rotate(q, np.array([[5 + d], [7 + d], [1 + d]]), (8, 8, 16), 1e4)
        b = oq.rotate(k, np.array([[2 + d], [9 + d], [0 + d]]), (8, 8, 16), 1e4)
        dot = float((a * b).sum())
        if d == 0:
            first = dot
        assert abs(dot - first) < 1e-8


def _empty(kv, cap, hd):
    z = np.zeros
    return dict(k=z((kv, cap, hd)), v=z((kv, cap, hd)), k_scale=z((kv, cap // 64)), v_scale=z((kv, cap // 64)), weight=np.ones((kv, cap)))


def test_append_in_parts_is_near_append_at_once():
    """Half a step of the block's final scale from the numbers, however the rows arrive; the scale is
    that of the largest number either way; rows beyond stay."""
    rng = np.random.default_rng(2)
    k, v = rng.standard_normal((2, 150, 2, 16)) * np.exp2(rng.integers(-3, 4, (2, 150, 1, 1)))
    whole = oq.append(_empty(2, 192, 16), k, v, 0)
    parts, at = _empty(2, 192, 16), 0
    for m in (1, 62, 1, 5, 60, 21):
        parts = oq.append(parts, k[at:at + m], v[at:at + m], at)
        at += m
    assert at == 150
    for name, x in (("k", k), ("v", v)):
        np.testing.assert_array_equal(whole[name + "_scale"], parts[name + "_scale"])
        for c in (whole, parts):
            got = oq.dequant(c, name)[:, :150].transpose(1, 0, 2)
            step = np.repeat(c[name + "_scale"], 64, -1)[:, :150].T[..., None] * 2.0 ** -10
            assert (np.abs(got - x) <= np.maximum(np.abs(x) * 2.0 ** -4, step) * 1.0001 + step * (c is parts)).all()
            assert (c[name][:, 150:] == 0).all()
    assert (whole["weight"][:, :150] == 0).all() and (whole["weight"][:, 150:] == 1).all()


def test_append_drops_rows_past_the_capacity():
    k = np.ones((10, 1, 16))
    c = oq.append(_empty(1, 64, 16), k, k, 60)
    assert (oq.dequant(c, "k")[0, 60:] == 1).all() and (c["weight"][0, :60] == 1).all()


@pytest.mark.parametrize("H,kv,masked", [(4, 4, False), (6, 2, True)])
def test_attention_is_torchs(H, kv, masked):
    rng = np.random.default_rng(3)
    m, rows, hd, held = 5, 23, 16, 18
    q, k, v = rng.standard_normal((m, H, hd)), rng.standard_normal((kv, rows, hd)), rng.standard_normal((kv, rows, hd))
    mask = (rng.random(rows) > 0.3).astype(np.uint8) if masked else None
    if masked:
        mask[0] = 1
    out, prob, _, _ = oq.attention(k, v, q, held, 0.25, mask)
    see = torch.arange(rows) <= held + torch.arange(m)[:, None]
    if masked:
        see &= torch.from_numpy(mask) != 0
    t = lambda x: torch.from_numpy(np.repeat(x, H // kv, 0))  # noqa: E731
    want = F.scaled_dot_product_attention(torch.from_numpy(q).transpose(0, 1), t(k), t(v), attn_mask=see, scale=0.25)
    np.testing.assert_allclose(out, want.transpose(0, 1).numpy(), atol=1e-12)
    np.testing.assert_allclose(prob.sum(-1), 1, atol=1e-12)
    np.testing.assert_allclose(oq.group_weight(prob, kv).sum(), m * H, atol=1e-10)


def test_attention_without_a_visible_row_is_zero():
    one = np.ones((1, 4, 16))
    out, prob, _, _ = oq.attention(one, one, np.ones((2, 1, 16)), 2, 1.0, np.zeros(4))
    assert not out.any() and not prob.any()


def test_kept_rows_brute_force():
    """Of all choices between sink and recent, the one with the largest weights, ties to lower rows."""
    rng = np.random.default_rng(4)
    for _ in range(60):
        n = int(rng.integers(1, 9))
        w = rng.integers(0, 3, n).astype(np.float32)
        keep = int(rng.integers(1, 9))
        sink = int(rng.integers(0, keep + 1))
        recent = int(rng.integers(0, keep - sink + 1))
        got = oq.kept_rows(w, n, keep, sink, recent)
        if n <= keep:
            np.testing.assert_array_equal(got, np.arange(n))
            continue
        ends = set(range(sink)) | set(range(n - recent, n))
        best = max((c for c in itertools.combinations(sorted(set(range(n)) - ends), keep - len(ends))),
                   key=lambda c: (sum(w[list(c)]), tuple(-x for x in c)), default=())
        assert set(got.tolist()) == ends | set(best)
    np.testing.assert_array_equal(oq.kept_rows(np.array([np.nan, -0.0, 0.0, -np.inf, -1.0], np.float32), 5, 3, 0, 0), [1, 2, 4])


def test_evict_keeps_numbers():
    """Kept rows stand for what they stood for, to half a step of the new block's scale, which is
    the smallest for them; everything stays when there is room."""
    rng = np.random.default_rng(5)
    c = oq.append(_empty(2, 256, 16), *rng.standard_normal((2, 200, 2, 16)) * np.exp2(rng.integers(-5, 5, (1, 200, 1, 1))), 0)
    c["weight"] = rng.random((2, 256))
    for keep in (70, 200):
        got, kept = oq.evict(c, _empty(2, 256, 16), 200, keep, 3, 9)
        assert kept.shape == (2, keep)
        for h in range(2):
            for name in ("k", "v"):
                a, b = oq.dequant(c, name)[h, kept[h]], oq.dequant(got, name)[h, :keep]
                s = np.repeat(got[name + "_scale"], 64, -1)[h, :keep, None]
                assert (np.abs(a - b) <= s * 2.0 ** -10).all()   # only subnormal codes lose bits
                assert (np.abs(a) <= 448 * s).all()
            np.testing.assert_array_equal(got["weight"][h, :keep], c["weight"][h, kept[h]])
