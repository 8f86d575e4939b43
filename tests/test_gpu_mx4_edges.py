"""GPU parity of the MXFP4 calls at the edges of their definitions: vectors with
infinities, gates far below zero, the largest calls."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_34867_amd as p4q
from gpu_util import Guarded, bits, check_canaries, dev, first_mismatch, to_gpu, to_np
from test_gpu_mx4 import f64, rows, store

pytestmark = pytest.mark.gpu


# --------------------------------------------------------------------------- residual norm
# (widths that leave threads without a part of the row, and 4096, which does not)
@pytest.mark.parametrize("d", [32, 1056, 4096, 5120])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("bad", ["gate", "post_gamma"])
@pytest.mark.parametrize("at", [0, 7, 8, 31])
@pytest.mark.parametrize("value", [np.inf, np.nan])
def test_norm_non_finite_vectors(d, dtype, bad, at, value):
    """An infinity or a NaN of the gate or of the post norm's weight reaches the rows as the
    definition says, wherever in the vector it stands: an infinite h makes its block NaN and
    the rest of its row zeros."""
    M = 5
    x, r = rows(1, M, d, dtype, 1.0), rows(2, M, d, dtype, 1.0)
    r[:, at] = store(1.0, dtype)
    v = np.ones(d)
    v[at] = value
    v = store(v, dtype)
    one = store(np.ones(d), dtype)
    gh = Guarded((M, d), torch.float16 if dtype == "fp16" else torch.bfloat16, "h")
    codes, scales, h = p4q.residual_rmsnorm_quant(to_gpu(x, dtype), to_gpu(one, dtype), to_gpu(r, dtype), h_out=gh.t,
                                                  **{bad: to_gpu(v, dtype)})
    torch.cuda.synchronize()
    check_canaries(gh)
    with np.errstate(invalid="ignore", over="ignore"):
        rh, n = oracle.residual_rmsnorm(x, one, r, dtype=dtype, **{bad: v})
        rc, rs = oracle.quant_mx4(n.astype(np.float64))
    got, ref = f64(to_np(h), dtype), f64(rh, dtype)
    assert np.array_equal(got, ref, equal_nan=True)
    assert (m := first_mismatch(to_np(scales), rs)) is None, f"scales: {m}"
    assert (m := first_mismatch(to_np(codes), rc)) is None, f"codes: {m}"
