"""Pins of the key/value cache's oracle: the grid by brute force, the layout by hand, the
attention by closed forms."""
import numpy as np
import pytest

from oracle import kv as okv


@pytest.mark.parametrize("seed", range(6))
def test_codes_are_nearest_levels(seed):
    """No level of the grid is nearer to an element than the chosen one (beyond fp32 rounding)."""
    x = np.random.default_rng(seed).standard_normal(64).astype(np.float32) * 10.0 ** (seed - 3) + seed % 2
    n, bits, z = okv.quantize_group(x)
    s = float(bits.view(np.float32))
    levels = s * (np.arange(16) - z)
    got = np.abs(s * (n.astype(float) - z) - x)
    best = np.abs(levels[None, :] - x[:, None]).min(1)
    assert np.all(got <= best + 1e-5 * s)
    assert np.all(got <= s * (0.5 + 1e-5))


def test_grid_contains_zero_and_spans_the_group():
    for x in ([1.0, 2.0, 4.0], [-3.0, -1.0], [0.0, 0.0], [-1.0, 2.0], [1e-44, 0.0], [5e-324]):
        n, bits, z = okv.quantize_group(np.array(x, np.float32))
        assert 0 <= z <= 15 and n.min() >= 0 and n.max() <= 15
        assert int(bits) % 16 == 0 and bits.view(np.float32) >= np.float32(2.0 ** -126)
    n, bits, z = okv.quantize_group(np.array([0.0, 15.0], np.float32))
    assert (list(n), float(bits.view(np.float32)), z) == ([0, 15], 1.0, 0)
    n, bits, z = okv.quantize_group(np.array([-15.0, 0.0], np.float32))
    assert (list(n), z) == ([0, 15], 15)


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_non_finite_groups_read_as_nan(bad):
    _, bits, z = okv.quantize_group(np.array([1.0, bad, 2.0], np.float32))
    assert np.isnan(bits.view(np.float32)) and z == 0
    _, bits, _ = okv.quantize_group(np.array([3e38, -3e38], np.float32))
    assert np.isnan(bits.view(np.float32))


def test_record_layout_by_hand():
    """dim 64, group 32: two words a lane (NC = 2), two groups."""
    dp, ng, rec = okv.sizes(64, 32)
    assert (dp, ng, rec) == (64, 2, 2560)
    pages = np.zeros((1, 1, 1, rec), np.uint8)
    kc, vc = np.zeros(64, np.uint8), np.zeros(64, np.uint8)
    kc[41], vc[42] = 9, 7
    okv.put(pages, 3, 0, kc, np.array([0x3f800001, 0x40000002], np.uint32), vc,
            np.array([16, 32], np.uint32), 32)
    r = pages[0, 0, 0]
    # channel 41: octet 5 = 4 * 1 + 1 -> word j NC + c = 1 * 2 + 1 = 3 of row 3, byte 0, high nibble
    assert r[3 * 32 + 12] == 0x90
    assert r[1024 + 12:1024 + 16].tobytes() == b"\x01\x00\x80\x3f"
    assert r[1024 + 128 + 12:1024 + 128 + 16].tobytes() == b"\x02\x00\x00\x40"
    # value channel 42: unit 10, nibble 2 of token 3's half-word
    assert r[1280 + 64 * 10 + 2 * 3 + 1] == 7
    assert np.count_nonzero(r) == 2 + 3 + 2 + 2


def test_attention_closed_forms():
    k = np.zeros((5, 1, 8))
    v = np.random.default_rng(0).standard_normal((5, 1, 8))
    q = np.ones((2, 1, 8))
    out, lse, _ = okv.attention(q, k, v, [3, 4], 1.0)
    assert np.allclose(out[0, 0], v[:4, 0].mean(0)) and np.allclose(lse[:, 0], np.log([4, 5]))
    out, lse, _ = okv.attention(q, k, v, [-1, 2], 1.0, window=1)
    assert not out[0].any() and lse[0, 0] == -np.inf and np.allclose(out[1, 0], v[2, 0])
    # slopes: weights 2^-(distance)
    out, _, _ = okv.attention(q, k, v, [1, 4], 1.0, slopes=[np.log(2.0)])
    assert np.allclose(out[0, 0], (v[0, 0] / 2 + v[1, 0]) / 1.5)
