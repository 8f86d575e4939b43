"""Pins of the oracle's MXFP4 functions: the format's table, worked blocks, exact
decoding, and agreement with nearest-number search."""
import numpy as np
import pytest

import oracle


def block(*v):
    return np.array([list(v) + [0.0] * (32 - len(v))])


def test_element_table():
    """Code k of E2M1: exponent bits k >> 1, mantissa bit k & 1, bias 1, subnormal at 0."""
    for k in range(8):
        e, m = k >> 1, k & 1
        assert oracle.E2M1[k] == (m / 2 if e == 0 else (1 + m / 2) * 2.0 ** (e - 1))


def test_worked_block():
    # max 5.5: floor(log2) = 2, X = 1; ties go to the even code, 5 -> 4
    x = block(5.5, -0.25, 0.25, 0.75, -1.25, 1.75, 2.5, -3.5, 5.0, 0.26, -2.51, -0.0)
    codes, scales = oracle.quant_mx4(x)
    assert scales.shape == (1, 16) and scales[0, 0] == 127 and (scales[0, 1:] == 0).all()
    want = [6.0, -0.0, 0.0, 1.0, -1.0, 2.0, 2.0, -4.0, 4.0, 0.5, -3.0, -0.0]
    v = oracle.mx4_values(codes, scales)[0, :12]
    assert v.tolist() == want and np.signbit(v).tolist() == np.signbit(want).tolist()
    # codes of the first four values: 6 -> 7, -0 -> 8, 0 -> 0, 1 -> 2, even k in the low nibble
    assert codes[0, 0] == 0x87 and codes[0, 1] == 0x20


def test_scale_of_powers_and_saturation():
    for e in (-20, -1, 0, 7, 100):
        for top, value in ((1.0, 1.0), (1.24, 1.0), (1.9999, 1.5), (1.75, 1.5)):
            codes, scales = oracle.quant_mx4(block(top * 2.0 ** e))
            assert scales[0, 0] == e - 2 + 127
            assert oracle.mx4_values(codes, scales)[0, 0] == value * 2.0 ** e
    assert oracle.quant_mx4(block(2.0 ** -130))[1][0, 0] == 0
    assert oracle.mx4_values(*oracle.quant_mx4(block(2.0 ** -127)))[0, 0] == 2.0 ** -127


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_non_finite_block(bad):
    x = np.ones((1, 64))
    x[0, 33] = bad
    codes, scales = oracle.quant_mx4(x)
    assert scales[0, 0] == 125 and scales[0, 1] == 255 and (codes[0, 16:] == 0).all()
    v = oracle.mx4_values(codes, scales)
    assert (v[0, :32] == 1).all() and np.isnan(v[0, 32:]).all()


def test_nearest_number():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((50, 256)) * np.exp2(rng.integers(-9, 9, (50, 1)))
    codes, scales = oracle.quant_mx4(x)
    v = oracle.mx4_values(codes, scales)
    X = np.repeat(np.exp2(scales[:, :8] - 127.0), 32, axis=1)
    grid = np.concatenate([-oracle.E2M1, oracle.E2M1])
    assert np.array_equal(np.abs(x - v), np.abs(x[..., None] - X[..., None] * grid).min(-1))
    top = np.abs(x).reshape(50, 8, 32).max(2)
    assert (4 * X[:, ::32] <= top).all() and (top < 8 * X[:, ::32]).all()
    # what is on the grid stays
    assert np.array_equal(oracle.mx4_values(*oracle.quant_mx4(v)), v)


def test_linear_by_hand():
    a, w = oracle.quant_mx4(block(6.0, 1.0, -2.0)), oracle.quant_mx4(block(0.5, 3.0, 1.0, 4.0))
    y, mag = oracle.mx4_linear(*a, *w)
    assert y[0, 0] == 6 * .5 + 3 - 2 and mag[0, 0] == 6 * .5 + 3 + 2


def test_residual_rmsnorm():
    rng = np.random.default_rng(1)
    x, r = (rng.standard_normal((4, 64)).astype(np.float16) for _ in range(2))
    g, p, t = (rng.standard_normal(64).astype(np.float16) for _ in range(3))
    h, n = oracle.residual_rmsnorm(x, g, r, 0.0, "fp16", p, t, 0.5)
    b = r.astype(np.float64)
    b = b / np.sqrt((b ** 2).mean(1, keepdims=True)) * p * t
    assert np.allclose(h, x + 0.5 * b, rtol=2.0 ** -10, atol=2.0 ** -24)
    hw = h.astype(np.float64)
    assert np.allclose(n, hw / np.sqrt((hw ** 2).mean(1, keepdims=True)) * g, rtol=2.0 ** -23)
    # without a residual it is the norm alone, and rows of zeros stay zero at eps = 0
    x[2] = 0
    h, n = oracle.residual_rmsnorm(x, g, eps=0.0)
    assert h is x and (n[2] == 0).all() and np.isfinite(n).all()
