"""The oracle of the 8-bit caches: e4m3 against torch's own conversion, the scale by its definition, appending against quantising whole."""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as Q


def test_codes_are_e4m3():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(t, Q.VALUES)
    g = np.random.default_rng(0)
    x = np.concatenate([g.standard_normal(4000) * 2.0 ** g.integers(-12, 8, 4000), Q.VALUES[:127], (Q.VALUES[:126] + Q.VALUES[1:127]) / 2])
    x = np.concatenate([x, -x])
    x = x[np.abs(x) <= Q.TOP].astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(Q.encode(x), want)
    assert (Q.encode([np.inf, -np.inf, np.nan]) == 127).all()


@pytest.mark.parametrize("e", [-110, -100, -9, 0, 1, 60, 119])
def test_scale_is_the_smallest_that_fits(e):
    s = 2.0 ** e
    assert Q.scale_of(448 * s) == s
    assert Q.scale_of(np.nextafter(448 * s, np.inf)) == 2 * s
    assert Q.scale_of(0.0) == 2.0 ** -110 and Q.scale_of(3.4e38) == 2.0 ** 120


def test_values_that_were_read_back_are_quantised_without_loss():
    """Unless they become subnormal: a block's values within 2^14 of its largest."""
    g = np.random.default_rng(1)
    x = g.standard_normal((70, 16))
    x = np.where(np.abs(x) < 0.01, 0.01, x)
    c, s = Q.quantize(x)
    v = Q.values(c, s)
    c2, s2 = Q.quantize(v)
    np.testing.assert_array_equal(Q.values(c2, s2), v)
    g2, t2 = Q.quantize(np.roll(v, 13, axis=0))            # other neighbours, other scales
    np.testing.assert_array_equal(Q.values(g2, t2), np.roll(v, 13, axis=0))


@pytest.mark.parametrize("n,m", [(0, 1), (0, 64), (1, 1), (31, 1), (32, 1), (33, 100), (40, 20)])
def test_appending(n, m):
    g = np.random.default_rng(n * 100 + m)
    x = g.standard_normal((n + m, 8)) * np.where(np.arange(n + m) < n, 1.0, 50.0)[:, None]
    c, s = Q.append(*Q.quantize(x[:n]), x[n:])
    whole = Q.quantize(x)
    np.testing.assert_array_equal(s, whole[1])             # scales as if quantised whole
    err = np.abs(Q.values(c, s) - x)
    scale = np.repeat(s, Q.BLOCK)[:n + m, None]
    # each rounding is off by at most 2^-4 of the value or half a subnormal step (2^-10 of the scale); old rows are rounded twice
    once = np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * scale)
    assert (err <= np.where(np.arange(n + m)[:, None] < n, once + 2.0 ** -10 * scale, once)).all()
    np.testing.assert_array_equal(c[n:], whole[0][n:])
