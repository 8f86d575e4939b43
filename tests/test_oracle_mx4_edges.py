"""Pins of the oracle's MXFP4 functions on rows that are not finite."""
import numpy as np
import pytest

import oracle


@pytest.mark.parametrize("post", [False, True])
def test_residual_rmsnorm_nan_row(post):
    """The norm of a row with a NaN is NaN all over; with an infinity, the rest is zeros."""
    x, r = np.ones((3, 64), np.float16), np.ones((3, 64), np.float16)
    g = np.ones(64, np.float16)
    r[0, 5], r[1, 5] = np.nan, np.inf
    with np.errstate(invalid="ignore"):
        h, n = oracle.residual_rmsnorm(x, g, r, post_gamma=g if post else None)
    assert np.isnan(n[0]).all() and np.isnan(n[1, 5]) and np.isfinite(n[2]).all()
    # (post norm: infinity / infinity is a NaN of h, and then of its whole row)
    assert np.isnan(n[1]).all() if post else (np.delete(n[1], 5) == 0).all()
