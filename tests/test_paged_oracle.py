"""The 8-bit cache's oracle against torch's own conversions, closed forms and plain definitions (CPU)."""
import numpy as np
import torch

from oracle import paged


def test_e4m3_is_torchs():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    got = paged.e4m3_decode(codes)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(got).sum() == 2
    np.testing.assert_array_equal(got[~np.isnan(got)], want[~np.isnan(want)])
    rng = np.random.default_rng(1)
    mids = (paged.POSITIVE[1:] + paged.POSITIVE[:-1]) / 2  # ties
    x = np.concatenate([rng.normal(size=20000) * 2.0 ** rng.integers(-12, 8, 20000), paged.POSITIVE, mids, -mids]).astype(np.float32)
    x = np.clip(x, -448, 448)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(paged.e4m3_encode(x), want)
    assert (paged.e4m3_encode(np.array([np.nan, np.inf, -np.inf])) == 127).all()


def test_scale_is_the_smallest_power():
    for a in (448.0, 448.0001, 447.9, 1.0, 3.5, 3.5000001, 2.0 ** -130, 0.0, 3e38):
        s = float(paged.scale_for(a))
        assert a <= 448 * s and s >= 2.0 ** -126 and np.log2(s) == np.round(np.log2(s))
        assert s == 2.0 ** -126 or a > 448 * s / 2
    assert float(paged.scale_for(448.0)) == 1.0 and float(paged.scale_for(448.0001)) == 2.0


def test_rotation_keeps_lengths_and_differences():
    rng = np.random.default_rng(2)
    x, freq = rng.normal(size=(5, 3, 128)), 10000.0 ** (-np.arange(0, 64, 2) / 64)
    for inter in (False, True):
        y = paged.rope(x, [0, 1, -7, 1000, 10 ** 6], freq, inter)
        np.testing.assert_array_equal(y[0], x[0])
        np.testing.assert_array_equal(y[..., 64:], x[..., 64:])
        np.testing.assert_allclose(np.linalg.norm(y, axis=-1), np.linalg.norm(x, axis=-1))
        q, k = np.repeat(x[:1], 2, 0), np.repeat(x[1:2], 2, 0)  # a logit depends on the distance of the positions alone
        a, b = paged.rope(q, [11, 1011], freq, inter), paged.rope(k, [4, 1004], freq, inter)
        np.testing.assert_allclose((a[0] * b[0]).sum(-1), (a[1] * b[1]).sum(-1))
        back = paged.rope(paged.rope(x, [3] * 5, freq, inter), [-3] * 5, freq, inter)
        np.testing.assert_allclose(back, x, atol=1e-12)


def test_growing_a_block_in_steps_is_near_filling_it_at_once():
    rng = np.random.default_rng(3)
    x = np.ldexp(rng.integers(-128, 129, (40, 2, 128)), -6).astype(np.float64) * (1 + np.arange(40)[:, None, None])
    table = np.array([2, 0, 1])
    one = [np.zeros((3, 2, 16, 128), np.uint8), np.zeros((3, 2, 1))]
    paged.append_quant(*one, x, 0, table)
    many = [np.full((3, 2, 16, 128), 127, np.uint8), np.full((3, 2, 1), np.nan)]
    for t in range(40):
        paged.append_quant(*many, x[t:t + 1], t, table)
    np.testing.assert_array_equal(one[1], many[1])
    a, b = paged.dequant(*one, table, 40), paged.dequant(*many, table, 40)
    scale = one[1][table[np.arange(40) // 16], :, 0][..., None]
    assert (np.abs(a - x) <= np.abs(x) * 2.0 ** -4 + scale * 2.0 ** -10).all()
    assert (np.abs(a - b) <= scale * 2.0 ** -9).all()  # only codes below the normal range are rounded again
    assert (one[0][1, :, 8:] == 0).all()               # rows behind the last token stay


def test_attention_of_equal_keys_is_the_mean():
    rng = np.random.default_rng(4)
    v = rng.normal(size=(7, 2, 128))
    out, bound = paged.attend(rng.normal(size=(4, 128)), np.ones((7, 2, 128)), v, 0.1)
    np.testing.assert_allclose(out[:2], np.repeat(v[:, 0].mean(0)[None], 2, 0))
    assert (bound > 0).all() and bound.max() < 1e-3
    assert not paged.attend(rng.normal(size=(4, 128)), np.ones((0, 2, 128)), v[:0], 0.1)[0].any()
