"""GPU parity of every kernel of MXFP4 products in the ways that it is taken: whole and cut
tiles, stores past the caches and not, work-groups that go on to a next tile
(test_mx4_choice.py says which size reaches what)."""
import numpy as np
import pytest
import torch

import mx4_sizes as sizes
import oracle
import paper_2609_34867_amd as p4q
from gpu_util import Guarded, bits, check_canaries, first_mismatch, to_np
from test_gpu_mx4 import HALF, TINY, TORCH, check_nearest, exact_operands, f64, gated_reference, gpu, operand, store

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kernel,M,N,K", sizes.LINEAR)
def test_linear(kernel, M, N, K):
    a, w = exact_operands(M + N + K, M, N, K)
    ref, _ = oracle.mx4_linear(*a, *w)
    for dtype in ("bf16", "fp16"):
        g = Guarded((M, N), TORCH[dtype], "y")
        y = p4q.mx4_linear(*gpu(a), *gpu(w), y=g.t)
        torch.cuda.synchronize()
        check_canaries(g)
        assert (m := first_mismatch(bits(to_np(y)), bits(store(ref, dtype)))) is None, f"{dtype}: {m}"


@pytest.mark.parametrize("kernel,M,N,K", sizes.GATED)
def test_gated(kernel, M, N, K):
    a, w = operand(M, M, K, 123, 125), operand(N, 2 * N, K, 121, 123)
    ref, tol = gated_reference(a, w, N, K, exact=True)
    for dtype in ("bf16", "fp16"):
        g = Guarded((M, N), TORCH[dtype], "y")
        y = p4q.mx4_gated_linear(*gpu(a), *gpu(w), y=g.t)
        torch.cuda.synchronize()
        check_canaries(g)
        err = np.abs(f64(to_np(y), dtype) - ref)
        lim = tol + HALF[dtype] * (np.abs(ref) + tol) + TINY[dtype]
        assert (err <= lim).all(), f"{dtype}: {(err > lim).sum()} values, worst {np.max(err / lim)}"


@pytest.mark.parametrize("kernel,M,N,K", sizes.QUANTIZED)
def test_gated_quant(kernel, M, N, K):
    a, w = operand(M, M, K, 123, 125), operand(N, 2 * N, K, 121, 123)
    ref, tol = gated_reference(a, w, N, K, exact=True)
    gc = Guarded((M, N // 2), torch.uint8, "codes")
    gs = Guarded((M, oracle.mx4_scale_stride(N)), torch.uint8, "scales")
    codes, scales = p4q.mx4_gated_linear_quant(*gpu(a), *gpu(w), codes=gc.t, scales=gs.t)
    torch.cuda.synchronize()
    check_canaries(gc, gs)
    check_nearest(to_np(codes), to_np(scales), ref, tol + np.abs(ref) * 2.0 ** -23 + 2.0 ** -150)


# rows of y at half lines of a wider buffer, and not
@pytest.mark.parametrize("kernel", list(sizes.SLOTS))
def test_linear_rows_in_a_wider_buffer(kernel):
    M, N, K = next(c[1:] for c in sizes.LINEAR if c[0] == kernel and c[2] % 32 == 0)
    a, w = exact_operands(1, M, N, K)
    ga, gw = gpu(a), gpu(w)
    ref = p4q.mx4_linear(*ga, *gw, out_dtype=torch.float16)
    for ld, first in ((N + 64, 32), (N + 32, 0), (N + 32, 8), (N + 5, 2)):
        wide = torch.full((M, ld), 7.0, dtype=torch.float16, device=ref.device)
        p4q.mx4_linear(*ga, *gw, y=wide[:, first:first + N])
        assert torch.equal(wide[:, first:first + N], ref), (ld, first)
        assert bool((wide[:, :first] == 7).all()) and bool((wide[:, first + N:] == 7).all())
