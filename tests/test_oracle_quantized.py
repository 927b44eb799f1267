"""Pins of the fp64 definitions of 8-bit rows and of the rotation over several axes."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as qo


def test_e4m3_table_is_the_type():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(qo.E4M3, want, equal_nan=True)


def test_rounding_is_to_nearest_even():
    mid = (qo.E4M3[1:127] + qo.E4M3[:126]) / 2
    for v in (mid, -mid, mid * (1 + 1e-9), mid * (1 - 1e-9), qo.E4M3[:127], np.array([0.0, -0.0, np.nan])):
        want = torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
        got = qo.to_e4m3(v)
        if np.isnan(v).any():
            want, got = want & 0x7F, got & 0x7F
        # torch goes through fp32, where mid * (1 +- 1e-9) is the tie itself
        if np.array_equal(v.astype(np.float32).astype(np.float64), v, equal_nan=True):
            assert np.array_equal(got, want)
        else:
            assert np.all(np.abs(qo.E4M3[got] - v) <= np.abs(qo.E4M3[want] - v) + 1e-12)


def test_scale_is_the_smallest_that_holds():
    for k in (-127, -126, -10, 0, 3, 119):
        top = 448.0 * 2.0 ** k
        assert qo.scale_byte(np.array(top)) == k + 127
        assert qo.scale_byte(np.array(np.nextafter(top, np.inf))) == k + 128
    assert qo.scale_byte(np.array(0.0)) == 0


@pytest.mark.parametrize("K", [8, 128, 136, 320])
def test_quantised_values_are_near(K):
    rng = np.random.default_rng(K)
    x = rng.normal(size=(5, K)) * 10.0 ** rng.integers(-6, 6, size=(5, 1))
    data, scale = qo.quantize(x)
    assert not data[:, K:].any()
    y = qo.dequantize(data, scale, K)
    s = np.repeat(2.0 ** (scale.astype(float) - 127), 128, 1)[:, :K]
    assert np.all(np.abs(y - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * s))


def test_rotation_by_one_axis_is_a_complex_product():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(6, 2, 32))
    y = qo.qk_norm_rope(x, (6, 1, 1), (32, 0, 0), "none", None, None, 0.0)
    z = x[..., 0::2] + 1j * x[..., 1::2]
    turn = np.exp(1j * np.arange(6)[:, None, None] * 10000.0 ** (-np.arange(16) / 16))
    assert np.allclose(y[..., 0::2] + 1j * y[..., 1::2], z * turn, atol=1e-12)


def test_axes_are_independent_and_relative():
    """The product of a query and a key depends on the difference of their places alone, axis by axis."""
    rng = np.random.default_rng(2)
    q, k = rng.normal(size=32), rng.normal(size=32)
    places, dims = (3, 4, 5), (8, 12, 12)
    grid = np.broadcast_to(q, (60, 1, 32)), np.broadcast_to(k, (60, 1, 32))
    rq, rk = (qo.qk_norm_rope(np.array(g), places, dims, "none", None, None, 0.0)[:, 0] for g in grid)
    at = lambda t, y, x: (t * 4 + y) * 5 + x   # noqa: E731
    assert np.isclose(rq[at(1, 2, 3)] @ rk[at(0, 1, 1)], rq[at(2, 3, 4)] @ rk[at(1, 2, 2)])
    assert not np.isclose(rq[at(1, 2, 3)] @ rk[at(0, 1, 1)], rq[at(1, 2, 3)] @ rk[at(1, 1, 1)])


def test_factor_table_is_what_the_rotation_uses():
    f = qo.rope_factors((2, 3, 4), (8, 4, 6), (1, 0, 5), (1, 0.5, 2))
    assert f.shape == (2 * 4 + 3 * 2 + 4 * 3, 2)
    assert np.allclose(f[0], [np.cos(1), np.sin(1)]) and np.allclose(f[2 * 4 + 2 * 2], [np.cos(1.0), np.sin(1.0)])
    assert np.allclose(f[2 * 4 + 3 * 2 + 3 * 1], [np.cos(7.0), np.sin(7.0)])
