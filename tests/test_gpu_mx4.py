"""GPU parity of the MXFP4 calls (quantizer, residual norm, linear, gated linear)
against the oracle.

Codes, scales, residual rows and products of operands whose sums are exact in
fp32 have to match bit for bit.  Other products are held to the error of fp32
sums: K terms, each addition off by at most 2^-23 of the magnitudes summed (one
unit in the last place, so that truncating hardware is covered), and half a
step of the output type."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_34867_amd as p4q
from gpu_util import Guarded, bits, check_canaries, dev, first_mismatch, to_gpu, to_np

pytestmark = pytest.mark.gpu

HALF = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"fp16": 2.0 ** -25, "bf16": 2.0 ** -134}        # half the smallest step
TORCH = {"fp16": torch.float16, "bf16": torch.bfloat16}


def store(x, dtype):
    """float values -> storage array of dtype."""
    return oracle.round_out(np.asarray(x, dtype=np.float32), dtype)


def rows(seed, M, K, dtype="fp16", spread=3.0):
    """Rows whose blocks have very different magnitudes, zeros and ties among them."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((M, K // 32, 32)) * np.exp2(rng.integers(-3, 4, (M, K // 32, 1)) * spread / 3)
    x[rng.random((M, K // 32)) < 0.05] = 0.0
    on_grid = rng.random((M, K // 32)) < 0.2
    x[on_grid] = np.round(x[on_grid] * 4) / 4
    return store(x.reshape(M, K), dtype)


def f64(x, dtype):
    return oracle.as_f32(x, dtype).astype(np.float64)


# --------------------------------------------------------------------------- quantizer
def check_quant(x, dtype, ldx=None, ldv=None):
    M, K = x.shape
    xt = to_gpu(x, dtype)
    if ldx:
        wide = torch.full((M, ldx), float("nan"), dtype=xt.dtype, device=dev())
        wide[:, :K] = xt
        xt = wide[:, :K]
    gc = Guarded((M, K // 2), torch.uint8, "codes")
    gs = Guarded((M, oracle.mx4_scale_stride(K)), torch.uint8, "scales")
    gv = Guarded((M, ldv or K), TORCH[dtype], "values")
    p4q.quant_mx4(xt, codes=gc.t, scales=gs.t, values=gv.t[:, :K])
    codes, scales = p4q.quant_mx4(xt)
    torch.cuda.synchronize()
    check_canaries(gc, gs, gv)
    assert torch.equal(codes, gc.t) and torch.equal(scales, gs.t)
    rc, rs = oracle.quant_mx4(f64(x, dtype))
    assert (m := first_mismatch(to_np(scales), rs)) is None, f"scales: {m}"
    assert (m := first_mismatch(to_np(codes), rc)) is None, f"codes: {m}"
    rv, v = oracle.mx4_values(rc, rs), f64(to_np(gv.t[:, :K]), dtype)
    assert np.array_equal(np.isnan(rv), np.isnan(v)) and np.array_equal(rv[~np.isnan(rv)], v[~np.isnan(v)])


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_quant_every_bit_pattern(dtype):
    """Every 16-bit number, once among its neighbours and once below other maxima."""
    u = np.arange(65536, dtype=np.uint16)
    x = u.view(np.float16) if dtype == "fp16" else u
    check_quant(x.reshape(-1, 32), dtype)
    finite = u[np.isfinite(f64(x[None], dtype)[0])]
    rng = np.random.default_rng(1)
    for _ in range(3):
        y = rng.permutation(finite)[:len(finite) // 1024 * 1024].reshape(-1, 1024)
        check_quant(y.view(np.float16) if dtype == "fp16" else y, dtype)


@pytest.mark.parametrize("M,K", [(1, 32), (3, 64), (7, 480), (5, 544), (129, 4096), (2, 131072), (70001, 64)])
def test_quant_sizes(M, K):
    check_quant(rows(M + K, M, K, "bf16"), "bf16")


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_quant_values_in_place(dtype):
    x = rows(12, 50, 1056, dtype)
    t = to_gpu(x, dtype)
    codes, scales = p4q.quant_mx4(t, values=t)
    rc, rs = oracle.quant_mx4(f64(x, dtype))
    assert np.array_equal(to_np(codes), rc) and np.array_equal(to_np(scales), rs)
    assert np.array_equal(f64(to_np(t), dtype), oracle.mx4_values(rc, rs))
    # what is on the grid stays
    again = p4q.quant_mx4(t)
    assert np.array_equal(oracle.mx4_values(*(to_np(z) for z in again)), oracle.mx4_values(rc, rs))


def test_quant_row_gaps():
    check_quant(rows(2, 9, 96), "fp16", ldx=104, ldv=128)
    check_quant(rows(3, 33, 1056), "fp16", ldx=1064, ldv=1056)


# --------------------------------------------------------------------------- residual norm
def check_norm(M, d, dtype, fmt, r=True, post=False, gate=False, alpha=1.0, eps=1e-5, clip=1.0, seed=0, x=None,
               into=None):
    rng = np.random.default_rng(seed + M * d)
    x = store(rng.standard_normal((M, d)) * np.where(rng.random(d) < 0.01, 20, 1), dtype) if x is None else x
    b = store(rng.standard_normal((M, d)), dtype) if r else None
    vec = lambda m, s: store(m + s * rng.standard_normal(d), dtype)  # noqa: E731
    gamma, pg, gt = vec(1, .1), vec(1, .1) if post else None, vec(0, .5) if gate else None
    up = lambda t: None if t is None else to_gpu(t, dtype)  # noqa: E731
    xt, bt = up(x), up(b)
    gc = Guarded((M, d // 2), torch.uint8, "codes")
    gs = Guarded((M, oracle.mx4_scale_stride(d)) if fmt == "mx4" else (M,), torch.uint8 if fmt == "mx4" else torch.float32,
                 "scales")
    gh, gv = Guarded((M, d), TORCH[dtype], "h"), Guarded((M, d), TORCH[dtype], "values")
    h_out = {"x": xt, "r": bt, None: gh.t}[into] if r else None
    codes, scales, h = p4q.residual_rmsnorm_quant(xt, up(gamma), bt, eps=eps, fmt=fmt, clip=clip, post_gamma=up(pg),
                                                  gate=up(gt), alpha=alpha, h_out=h_out, codes=gc.t, scales=gs.t,
                                                  values=gv.t)
    torch.cuda.synchronize()
    check_canaries(gc, gs, gh, gv)
    assert h is (h_out if r else xt)
    rh, n = oracle.residual_rmsnorm(x, gamma, b, eps, dtype, pg, gt, alpha)
    assert (m := first_mismatch(bits(to_np(h)), bits(rh))) is None, f"h: {m}"
    values = f64(to_np(gv.t), dtype)
    if fmt == "mx4":
        rc, rs = oracle.quant_mx4(n.astype(np.float64))
        assert (m := first_mismatch(to_np(scales), rs)) is None, f"scales: {m}"
        rv = oracle.mx4_values(rc, rs)
    else:
        rc, rs = oracle.rmsnorm_quant(rh, gamma, float(np.float32(eps)), dtype, clip)
        # one rounding on each side
        assert np.allclose(to_np(scales), rs, rtol=2.0 ** -23, atol=0)
        rv = oracle.unpack_int4(rc).astype(np.float64) * to_np(scales).astype(np.float64)[:, None]
    assert (m := first_mismatch(to_np(codes), rc)) is None, f"codes: {m}"
    ref = f64(store(rv, dtype), dtype)
    assert np.array_equal(ref, values, equal_nan=True)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("fmt", ["mx4", "int4"])
@pytest.mark.parametrize("post,gate,alpha", [(False, False, 1.0), (True, False, 0.5), (False, True, 0.22), (True, True, -1.0)])
def test_norm_forms(dtype, fmt, post, gate, alpha):
    check_norm(37, 1056, dtype, fmt, post=post, gate=gate, alpha=alpha)


@pytest.mark.parametrize("M,d", [(1, 32), (1, 4096), (5, 96), (65, 2080), (3, 5120), (2, 6176), (4, 8192), (2, 12288), (3, 16384),
                                 (3000, 4096)])
def test_norm_widths(M, d):
    check_norm(M, d, "bf16", "mx4")
    check_norm(M, d, "fp16", "int4", post=True, clip=0.7)


@pytest.mark.parametrize("fmt", ["mx4", "int4"])
def test_norm_without_residual_and_in_place(fmt):
    check_norm(33, 544, "fp16", fmt, r=False)
    check_norm(33, 544, "fp16", fmt, into="x")
    check_norm(33, 544, "bf16", fmt, into="r", post=True)


@pytest.mark.parametrize("fmt", ["mx4", "int4"])
@pytest.mark.parametrize("eps", [0.0, 1e-5])
def test_norm_zero_rows(fmt, eps):
    x = rows(5, 9, 512)
    x[[0, 4, 8]] = 0
    check_norm(9, 512, "fp16", fmt, r=False, eps=eps, x=x)


def test_norm_non_finite_rows():
    """A row with an infinity or a NaN is its own trouble: MXFP4 blocks of it hold
    NaN or 0, the others are as they would be without it."""
    x = rows(6, 6, 256)
    bad = x.copy()
    bad[1, 40], bad[3, 0] = np.inf, np.nan
    g = to_gpu(np.ones(256, np.float16))
    outs = []
    for a in (x, bad):
        v = torch.empty(6, 256, dtype=torch.float16, device=dev())
        outs.append((*p4q.residual_rmsnorm_quant(to_gpu(a), g, values=v), v))
    keep = [0, 2, 4, 5]
    for a, b in zip(*outs):
        assert torch.equal(a[keep].view(torch.uint8), b[keep].view(torch.uint8))
    codes, scales, _, v = (to_np(t) for t in outs[1])
    assert scales[1, 1] == 255 and np.isnan(v[1, 32:64]).all() and (v[1, :32] == 0).all()
    assert (scales[3, :8] == 255).all() and np.isnan(v[3]).all()


def test_norm_row_gaps():
    M, d, ld = 21, 320, 352
    x, r = rows(7, M, ld), rows(8, M, ld)
    g = to_gpu(store(np.ones(d), "fp16"))
    xt, rt = to_gpu(x), to_gpu(r)
    h, v = torch.full((M, ld), 7.0, dtype=torch.float16, device=dev()), torch.full((M, ld), 7.0, dtype=torch.float16, device=dev())
    codes, scales, _ = p4q.residual_rmsnorm_quant(xt[:, :d], g, rt[:, :d], h_out=h[:, :d], values=v[:, :d])
    rh, n = oracle.residual_rmsnorm(x[:, :d], np.ones(d, np.float16), r[:, :d])
    rc, rs = oracle.quant_mx4(n.astype(np.float64))
    assert np.array_equal(to_np(codes), rc) and np.array_equal(to_np(scales), rs)
    assert np.array_equal(bits(to_np(h[:, :d].contiguous())), bits(rh))
    assert bool((h[:, d:] == 7).all()) and bool((v[:, d:] == 7).all())


# --------------------------------------------------------------------------- products
def operand(seed, R, K, lo=126, hi=128):
    """Random codes under scale bytes lo .. hi; the padding holds the byte of NaN."""
    rng = np.random.default_rng(seed)
    codes = rng.integers(0, 256, (R, K // 2)).astype(np.uint8)
    scales = np.full((R, oracle.mx4_scale_stride(K)), 255, dtype=np.uint8)
    scales[:, :K // 32] = rng.integers(lo, hi + 1, (R, K // 32))
    return codes, scales


def exact_operands(seed, M, N, K):
    """Operands whose partial sums are exact in fp32 in any order: multiples of
    2^-4 below 2^20."""
    a, w = operand(seed, M, K), operand(seed + 1, N, K)
    assert 36 * 4 * K < 2 ** 20
    return a, w


def gpu(op):
    return tuple(to_gpu(t) for t in op)


def fp32_sums(K):
    return (K + 8) * 2.0 ** -23


SIZES = [(1, 1, 32), (1, 33, 64), (3, 5, 96), (16, 32, 256), (17, 31, 288), (31, 65, 480), (32, 64, 512), (33, 100, 1056),
         (64, 256, 4096), (65, 129, 544), (128, 128, 1024), (130, 257, 1120), (257, 300, 320), (300, 520, 1568),
         (1, 4096, 4096), (5, 1000, 5120), (513, 768, 768), (1025, 1031, 1056), (2049, 2080, 512),
         (4100, 4200, 96), (3000, 6200, 1184), (16400, 1030, 288),
         # several sizes of tile (mx4_sizes.py reaches each), with rows, columns and k past the last whole one
         (1300, 67, 96), (1290, 61, 1312), (130, 6211, 96), (4100, 1050, 800), (4090, 1056, 1056), (1300, 6211, 288),
         (1000, 8219, 96), (1000, 8224, 1056), (4100, 3003, 288), (4097, 3000, 1056),
         # where two parts of a work-group share k: the second with as many stages, with fewer
         (1030, 61, 3040), (1030, 61, 5120), (1030, 130, 6176), (200, 4100, 1312), (387, 2500, 3040), (1030, 1001, 1312)]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear_exact(M, N, K):
    a, w = exact_operands(M + N + K, M, N, K)
    ref, _ = oracle.mx4_linear(*a, *w)
    for dtype in ("bf16", "fp16"):
        g = Guarded((M, N), TORCH[dtype], "y")
        y = p4q.mx4_linear(*gpu(a), *gpu(w), y=g.t)
        torch.cuda.synchronize()
        check_canaries(g)
        assert (m := first_mismatch(bits(to_np(y)), bits(store(ref, dtype)))) is None, f"{dtype}: {m}"


def check_product(y, ref, mag, K, dtype):
    err = np.abs(f64(to_np(y), dtype) - ref)
    tol = fp32_sums(K) * mag + HALF[dtype] * (np.abs(ref) + fp32_sums(K) * mag) + TINY[dtype]
    assert (err <= tol).all(), f"{(err > tol).sum()} values, worst {np.max(err / tol)}"


@pytest.mark.parametrize("M,N,K", [(1, 77, 13824), (4, 160, 131072), (16, 96, 11008), (200, 160, 4096), (700, 260, 2080),
                                   (1100, 40, 32768)])
def test_linear_rounding(M, N, K):
    x, w = rows(M, M, K, "bf16"), rows(N, N, K, "bf16")
    a, b = oracle.quant_mx4(f64(x, "bf16")), oracle.quant_mx4(f64(w, "bf16") * 2.0 ** -6)
    ref, mag = oracle.mx4_linear(*a, *b)
    check_product(p4q.mx4_linear(*gpu(a), *gpu(b)), ref, mag, K, "bf16")


@pytest.mark.parametrize("M", [3, 40, 600, 66000])
def test_linear_row_gaps(M):
    N, K = 200, 288
    a, w = exact_operands(3, M, N, K)
    ref = store(oracle.mx4_linear(*a, *w)[0], "fp16")
    for ld, first in ((N + 8, 0), (N + 3, 0), (N + 16, 2), (N + 24, 8), (N + 24, 0), (N + 56, 32)):
        wide = torch.full((M, ld), 7.0, dtype=torch.float16, device=dev())
        p4q.mx4_linear(*gpu(a), *gpu(w), y=wide[:, first:first + N])
        assert np.array_equal(bits(to_np(wide[:, first:first + N].contiguous())), bits(ref)), (ld, first)
        assert bool((wide[:, :first] == 7).all()) and bool((wide[:, first + N:] == 7).all())


@pytest.mark.parametrize("M", [2, 50, 400, 66000])
def test_linear_nan_and_extreme_scales(M):
    N, K = 130, 608
    a, w = exact_operands(4, M, N, K)
    ref = oracle.mx4_linear(*a, *w)[0]
    # NaN blocks reach their own row or column alone
    a[1][M - 1, 18], w[1][5, 0] = 255, 255
    y = f64(to_np(p4q.mx4_linear(*gpu(a), *gpu(w), out_dtype=torch.float16)), "fp16")
    nan = np.zeros((M, N), bool)
    nan[M - 1], nan[:, 5] = True, True
    assert np.array_equal(np.isnan(y), nan)
    assert np.array_equal(y[~nan], f64(store(ref, "fp16"), "fp16")[~nan])
    # the largest and the smallest bytes against each other, and sums below 2^-126
    (ac, _), (wc, _) = a, w
    for lo, hi in ((254, 0), (0, 254), (200, 54), (126, 128), (60, 60), (120, 1)):
        sa, sw = np.full_like(a[1], lo), np.full_like(w[1], hi)
        y = p4q.mx4_linear(*gpu((ac, sa)), *gpu((wc, sw)))
        ref = oracle.mx4_linear(ac, sa, wc, sw)[0]
        assert np.array_equal(bits(to_np(y)), bits(store(ref, "bf16"))), (lo, hi)


@pytest.mark.parametrize("M,N", [(1030, 200), (387, 2504)])
def test_linear_shared_k(M, N):
    """Row gaps, NaN blocks in either part of k, far scales, where two parts share it."""
    K = 3040
    a, w = exact_operands(7, M, N, K)
    ref = oracle.mx4_linear(*a, *w)[0]
    for ld, first in ((N + 3, 0), (N + 24, 8)):
        wide = torch.full((M, ld), 7.0, dtype=torch.float16, device=dev())
        p4q.mx4_linear(*gpu(a), *gpu(w), y=wide[:, first:first + N])
        assert np.array_equal(bits(to_np(wide[:, first:first + N].contiguous())), bits(store(ref, "fp16"))), (ld, first)
        assert bool((wide[:, :first] == 7).all()) and bool((wide[:, first + N:] == 7).all())
    a[1][M - 1, 94], a[1][2, 3], w[1][5, 0], w[1][N - 1, 60] = 255, 255, 255, 255
    y = f64(to_np(p4q.mx4_linear(*gpu(a), *gpu(w))), "bf16")
    nan = np.zeros((M, N), bool)
    nan[[2, M - 1]], nan[:, [5, N - 1]] = True, True
    assert np.array_equal(np.isnan(y), nan)
    assert np.array_equal(y[~nan], f64(store(ref, "bf16"), "bf16")[~nan])
    for lo, hi in ((254, 0), (126, 128)):
        sa, sw = np.full_like(a[1], lo), np.full_like(w[1], hi)
        y = p4q.mx4_linear(*gpu((a[0], sa)), *gpu((w[0], sw)))
        assert np.array_equal(bits(to_np(y)), bits(store(oracle.mx4_linear(a[0], sa, w[0], sw)[0], "bf16"))), (lo, hi)


def gated_reference(a, w, N, K, exact):
    s, mag = oracle.mx4_linear(*a, *w)
    g, u = s[:, :N], s[:, N:]
    dg, du = (0 * g, 0 * u) if exact else (fp32_sums(K) * mag[:, :N], fp32_sums(K) * mag[:, N:])
    e = np.exp(-np.abs(g))
    sig = np.where(g >= 0, 1 / (1 + e), e / (1 + e))
    y = g * sig * u
    # |SiLU'| <= 1.1; in fp32: exp of an argument rounded twice (|g| 2^-23) and five operations
    tol = 1.1 * dg * (np.abs(u) + du) + np.abs(g * sig) * du + (np.abs(g) + 8) * 2.0 ** -23 * np.abs(y)
    return y, tol


GATED = [(1, 32, 32), (1, 33, 64), (7, 1, 96), (16, 64, 1056), (33, 100, 288), (40, 352, 4096), (130, 129, 320), (300, 260, 544),
         (520, 512, 512), (1030, 1056, 288), (2050, 1030, 256),
         (4100, 2112, 96), (2900, 3011, 544), (1300, 64, 96), (1290, 61, 1056), (390, 8224, 96), (1000, 4128, 1056),
         (700, 8219, 288), (700, 8224, 1056)]


@pytest.mark.parametrize("M,N,K", GATED)
def test_gated(M, N, K):
    a, w = operand(M, M, K, 123, 125), operand(N, 2 * N, K, 121, 123)
    ref, tol = gated_reference(a, w, N, K, exact=True)
    for dtype in ("bf16", "fp16"):
        gy = Guarded((M, N), TORCH[dtype], "y")
        y = p4q.mx4_gated_linear(*gpu(a), *gpu(w), y=gy.t)
        torch.cuda.synchronize()
        check_canaries(gy)
        err = np.abs(f64(to_np(y), dtype) - ref)
        lim = tol + HALF[dtype] * (np.abs(ref) + tol) + TINY[dtype]
        assert (err <= lim).all(), f"{dtype}: {(err > lim).sum()} values, worst {np.max(err / lim)}"


@pytest.mark.parametrize("M", [2, 30, 200, 1300, 4100])
def test_gated_nan_blocks(M):
    """A NaN block of a row makes that row NaN; one of a gate or an up row, its output;
    quantized, every block that one of them enters."""
    N, K = 224, 320
    a, w = operand(8, M, K, 123, 125), operand(9, 2 * N, K, 121, 123)
    clean, held = (p4q.mx4_gated_linear(*gpu(a), *gpu(w)), p4q.mx4_gated_linear_quant(*gpu(a), *gpu(w)))
    a[1][M - 1, 9], w[1][3, 0], w[1][N + 40, 5] = 255, 255, 255
    nan = np.zeros((M, N), bool)
    nan[M - 1], nan[:, 3], nan[:, 40] = True, True, True
    y = to_np(p4q.mx4_gated_linear(*gpu(a), *gpu(w)))
    assert np.array_equal(np.isnan(f64(y, "bf16")), nan)
    assert np.array_equal(y[~nan], to_np(clean)[~nan])
    codes, scales = (to_np(t) for t in p4q.mx4_gated_linear_quant(*gpu(a), *gpu(w)))
    blocks = nan.reshape(M, -1, 32).any(2)
    assert np.array_equal(scales[:, :N // 32] == 255, blocks)
    assert (codes.reshape(M, -1, 16)[blocks] == 0).all() and (scales[:, N // 32:] == 0).all()
    assert np.array_equal(codes.reshape(M, -1, 16)[~blocks], to_np(held[0]).reshape(M, -1, 16)[~blocks])
    assert np.array_equal(scales[:, :N // 32][~blocks], to_np(held[1])[:, :N // 32][~blocks])


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_gated_far_gates(dtype):
    """Gates from far below zero, where SiLU vanishes, to far above, where it is the
    gate: no infinity or NaN where the product has none."""
    K, N = 32, 96
    ac, sa = np.zeros((40, 16), np.uint8), np.zeros((40, 16), np.uint8)
    wc, sw = np.zeros((2 * N, 16), np.uint8), np.zeros((2 * N, 16), np.uint8)
    ac[:, 0], sa[:, 0] = 0x02, 127                          # 1, 0, 0, ...
    wc[:, 0], sw[:, 0] = 0x02, 127
    wc[:N // 2, 0] = 0x0A                                   # half of the gates are negative
    sw[:N, 0] = 127 + np.tile(np.arange(-24, 24), 2)        # +- 2^-24 .. 2^23
    sw[N:, 0] = 127 - 9
    a, w = (ac, sa), (wc, sw)
    ref, tol = gated_reference(a, w, N, K, exact=True)
    y = f64(to_np(p4q.mx4_gated_linear(*gpu(a), *gpu(w), out_dtype=TORCH[dtype])), dtype)
    assert np.isfinite(y).all()
    assert (np.abs(y - ref) <= tol + HALF[dtype] * (np.abs(ref) + tol) + TINY[dtype]).all()


def check_nearest(codes, scales, ref, tol):
    """Each block's scale and codes are those of a value within tol of ref."""
    M, N = ref.shape
    top = np.abs(ref).reshape(M, -1, 32).max(2)
    slack = tol.reshape(M, -1, 32).max(2)
    byte = lambda t: np.maximum(np.frexp(np.maximum(t, 2.0 ** -140))[1] - 1 - 2, -127) + 127  # noqa: E731
    s = scales[:, :N // 32].astype(np.int64)
    assert ((s >= byte(top - slack)) & (s <= byte(top + slack))).all(), "scales"
    assert (scales[:, N // 32:] == 0).all(), "padding"
    v = oracle.mx4_values(codes, scales)
    X = np.repeat(np.exp2(s - 127.0), 32, axis=1)
    grid = np.concatenate([-oracle.E2M1[::-1], oracle.E2M1])
    best = np.min(np.abs(ref[..., None] - X[..., None] * grid), axis=-1) if M * N < 400000 else None
    if best is None:
        z = np.clip(np.abs(ref) / X, 0, 6)
        step = np.where(z < 2, .5, np.where(z < 4, 1., 2.))
        near = np.abs(np.round(z / step) * step - np.abs(ref) / X) * X
        best = near
    assert (np.abs(v - ref) <= best + 2 * tol).all(), "codes"


@pytest.mark.parametrize("M,N,K", [c for c in GATED if c[1] % 32 == 0] + [(3, 544, 96), (65, 1056, 512), (1000, 4128, 64), (900, 4224, 288)])
def test_gated_quant(M, N, K):
    a, w = operand(M, M, K, 123, 125), operand(N, 2 * N, K, 121, 123)
    ref, tol = gated_reference(a, w, N, K, exact=True)
    gc = Guarded((M, N // 2), torch.uint8, "codes")
    gs = Guarded((M, oracle.mx4_scale_stride(N)), torch.uint8, "scales")
    codes, scales = p4q.mx4_gated_linear_quant(*gpu(a), *gpu(w), codes=gc.t, scales=gs.t)
    torch.cuda.synchronize()
    check_canaries(gc, gs)
    check_nearest(to_np(codes), to_np(scales), ref, tol + np.abs(ref) * 2.0 ** -23 + 2.0 ** -150)


# --------------------------------------------------------------------------- together
def mlp_weights(d, f, seed=11):
    rng = np.random.default_rng(seed)
    w1 = oracle.quant_mx4(store(rng.standard_normal((2 * f, d)) * d ** -0.5, "bf16").view(np.uint16).astype(np.uint32).__lshift__(16)
                          .view(np.float32).astype(np.float64))
    w2 = oracle.quant_mx4(np.float64(np.float32(rng.standard_normal((d, f)) * f ** -0.5)))
    return w1, w2


def mlp(x, r, gamma, w1, w2, out=None):
    codes, scales, h = p4q.residual_rmsnorm_quant(x, gamma, r)
    mid = p4q.mx4_gated_linear_quant(codes, scales, *w1)
    return h, mid, p4q.mx4_linear(*mid, *w2, out_dtype=x.dtype, y=out)


@pytest.mark.parametrize("M", [1, 37, 600])
def test_feed_forward_half_of_a_layer(M):
    """Residual, norm, gate and up, down: each step against the oracle on what the
    step before gave."""
    d, f = 544, 1056
    w1, w2 = mlp_weights(d, f)
    x, r, gamma = rows(1, M, d, "bf16", 1.0), rows(2, M, d, "bf16", 1.0), store(np.ones(d), "bf16")
    h, mid, y = mlp(to_gpu(x, "bf16"), to_gpu(r, "bf16"), to_gpu(gamma, "bf16"), gpu(w1), gpu(w2))
    rh, n = oracle.residual_rmsnorm(x, gamma, r, dtype="bf16")
    assert np.array_equal(to_np(h), rh)
    a = oracle.quant_mx4(n.astype(np.float64))
    ref, tol = gated_reference(a, w1, f, d, exact=False)
    mid = tuple(to_np(t) for t in mid)
    check_nearest(*mid, ref, tol + np.abs(ref) * 2.0 ** -23)
    ref, mag = oracle.mx4_linear(*mid, *w2)
    check_product(y, ref, mag, f, "bf16")


@pytest.mark.parametrize("M", [4, 300])
def test_captured_and_replayed(M):
    """The run above in a graph, replayed over changing inputs on another stream than
    the one it was captured on, eager calls between the replays."""
    d, f = 288, 512
    w1, w2 = (gpu(w) for w in mlp_weights(d, f, 12))
    gamma = to_gpu(store(np.ones(d), "fp16"))
    x, r = (torch.zeros(M, d, dtype=torch.float16, device=dev()) for _ in range(2))
    inputs = [(to_gpu(rows(20 + i, M, d, "fp16", 1.0)), to_gpu(rows(30 + i, M, d, "fp16", 1.0))) for i in range(3)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        mlp(x, r, gamma, w1, w2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h, mid, y = mlp(x, r, gamma, w1, w2)
    for i in (0, 1, 2, 0):
        x.copy_(inputs[i][0])
        r.copy_(inputs[i][1])
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        side.synchronize()
        eh, emid, ey = mlp(*inputs[i], gamma, w1, w2)
        assert torch.equal(h, eh) and torch.equal(y, ey)
        assert all(torch.equal(a, b) for a, b in zip(mid, emid))


def test_another_stream():
    """Calls go to the current stream: on a side stream they wait for what was queued
    there."""
    M, d, f = 200, 544, 512
    w1, w2 = (gpu(w) for w in mlp_weights(d, f, 13))
    gamma = to_gpu(store(np.ones(d), "fp16"))
    x, r = to_gpu(rows(40, M, d, "fp16", 1.0)), to_gpu(rows(41, M, d, "fp16", 1.0))
    h, mid, y = mlp(x, r, gamma, w1, w2)
    late = torch.zeros_like(x)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        big = torch.randn(4096, 4096, device=dev())
        for _ in range(10):
            big = torch.mm(big, big).clamp(-1, 1)
        late.copy_(x)
        h2, mid2, y2 = mlp(late, r, gamma, w1, w2)
    side.synchronize()
    assert torch.equal(h, h2) and torch.equal(y, y2) and all(torch.equal(a, b) for a, b in zip(mid, mid2))


def test_two_streams_at_once():
    """Nothing is shared between calls."""
    M, N, K = 600, 1030, 1056
    ops = [(gpu(operand(50 + i, M, K)), gpu(operand(60 + i, N, K))) for i in range(2)]
    ref = [p4q.mx4_linear(*a, *w) for a, w in ops]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(20):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(p4q.mx4_linear(*ops[i][0], *ops[i][1]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, ref[i]) for y in got[i])


def test_refusals_enqueue_nothing():
    x = torch.full((4, 64), 3.0, dtype=torch.float16, device=dev())
    codes, scales = torch.full((4, 32), 9, dtype=torch.uint8, device=dev()), torch.full((4, 16), 9, dtype=torch.uint8, device=dev())
    with pytest.raises(p4q.P4QError, match="K=0|multiple of 32"):
        p4q.quant_mx4(x[:, :48], codes=codes[:, :24].contiguous(), scales=scales)
    with pytest.raises(p4q.P4QError, match="16-byte aligned rows"):
        p4q.quant_mx4(torch.zeros(4, 72, dtype=torch.float16, device=dev())[:, 4:68], codes=codes, scales=scales)
    with pytest.raises(p4q.P4QError, match="cannot replace"):
        p4q.mx4_gated_linear_quant(codes, scales, *(torch.zeros(128, n, dtype=torch.uint8, device=dev()) for n in (32, 16)), codes=codes)
    with pytest.raises(p4q.P4QError, match="M=0"):
        p4q.quant_mx4(x[:0])
    with pytest.raises(p4q.P4QError, match="clip"):
        p4q.residual_rmsnorm_quant(x, x[0], clip=0.5, codes=codes, scales=scales)
    torch.cuda.synchronize()
    assert bool((codes == 9).all()) and bool((scales == 9).all())
