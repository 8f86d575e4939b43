"""Pins of the oracle's serving operators: closed forms and identities (CPU)."""
import numpy as np
import pytest

import oracle


def rng(seed):
    return np.random.default_rng(seed)


@pytest.mark.parametrize("D", [64, 128])
def test_rotation_is_a_complex_product(D):
    x, p = rng(1).standard_normal((9, 3, D)), np.array([0, 1, 2, 17, 703, 4096, 10 ** 5, 10 ** 6, 2 ** 31 - 1])
    y = oracle.rope(x, p, 500000.0)
    j = np.arange(D // 2)
    z = (x[..., :D // 2] + 1j * x[..., D // 2:]) * np.exp(1j * p[:, None, None] * 500000.0 ** (-2 * j / D))
    # 10^9 rad carry an error of 2^-53 of themselves into the angle
    assert np.allclose(y[..., :D // 2], z.real, atol=1e-6) and np.allclose(y[..., D // 2:], z.imag, atol=1e-6)
    assert np.array_equal(y[0], x[0])


def test_rotated_products_depend_on_the_distance():
    q, k = rng(2).standard_normal((1, 1, 128)), rng(3).standard_normal((1, 1, 128))
    dots = [np.sum(oracle.rope(q, np.array([a + 5])) * oracle.rope(k, np.array([a]))) for a in (0, 1, 77, 5000)]
    assert np.allclose(dots, dots[0], rtol=1e-10)


@pytest.mark.parametrize("causal", [True, False])
def test_one_head_per_key_head_is_the_prefill(causal):
    q, k, v = (rng(4 + i).standard_normal((33, 2, 64)).astype(np.float16) for i in range(3))
    o, a = oracle.grouped_attention(q, k, v, causal)
    ref = oracle.attention_prefill(q, k, v, causal).astype(np.float64)
    assert np.all(np.abs(o - ref) <= 2.0 ** -11 * np.abs(ref) + 2.0 ** -25)
    assert np.all(a >= np.abs(o) - 1e-12)


def test_groups_read_their_key_head():
    q, k, v = rng(7).standard_normal((5, 6, 64)), rng(8).standard_normal((9, 2, 64)), rng(9).standard_normal((9, 2, 64))
    o, _ = oracle.grouped_attention(q, k, v)
    for h in range(6):
        one, _ = oracle.grouped_attention(q[:, h:h + 1], k[:, h // 3:h // 3 + 1], v[:, h // 3:h // 3 + 1])
        assert np.array_equal(o[:, h:h + 1], one)


def test_last_token_sees_last_key():
    q, k, v = (rng(10 + i).standard_normal((7, 1, 64)) for i in range(3))
    whole, _ = oracle.grouped_attention(q, k, v)
    part, _ = oracle.grouped_attention(q[4:], k, v)                    # a chunk: the same rows
    assert np.allclose(part, whole[4:], rtol=0, atol=1e-14)
    short, _ = oracle.grouped_attention(q, k[:3], v[:3])               # fewer keys than tokens
    assert not short[:4].any() and np.allclose(short[4], v[0])
    none, _ = oracle.grouped_attention(q, k[:0], v[:0], False)
    assert not none.any()


def test_cache_rows():
    cache = rng(13).standard_normal((4, 2, 16, 64))
    got = oracle.cache_rows(cache, np.array([3, 0, -1]), 20)
    assert np.array_equal(got[:16], cache[3].transpose(1, 0, 2)) and np.array_equal(got[16:], cache[0].transpose(1, 0, 2)[:4])
    assert oracle.cache_rows(cache, np.array([-1]), 0).shape == (0, 2, 64)
