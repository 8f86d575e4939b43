"""Host-side refusals of the MXFP4 calls at the C ABI (CPU only): the addresses below
are never dereferenced."""
import ctypes
import os

import pytest

from paper_2609_34867_amd import _lib as L
from paper_2609_34867_amd import mx4_scale_stride

P = 0x10000
BAD, UNSUPPORTED = L.P4Q_ERR_INVALID_ARG, L.P4Q_ERR_UNSUPPORTED
FLOATS = ("alpha", "eps", "clip")


@pytest.fixture(scope="module", autouse=True)
def built_library():
    if not os.path.exists(L.LIB_PATH):
        from paper_2609_34867_amd.build import build
        build()


def call(fn, a, kw):
    assert set(kw) <= set(a)
    a.update(kw)
    return getattr(L.lib(), fn)(*[ctypes.c_float(x) if n in FLOATS else x for n, x in a.items()], None)


def quant(**kw):
    return call("p4q_quant_mx4", dict(dt=0, M=4, K=64, x=P, ldx=64, codes=P, scales=P, values=None, ldv=0), kw)


def linear(**kw):
    return call("p4q_mx4_linear", dict(M=4, N=8, K=64, ac=P, sa=P, wc=P, sw=P, dt=0, y=P, ldy=8), kw)


def gated(**kw):
    return call("p4q_mx4_gated_linear", dict(M=4, N=8, K=64, ac=P, sa=P, wc=P, sw=P, dt=0, y=P, ldy=8), kw)


def gated_quant(**kw):
    return call("p4q_mx4_gated_linear_quant", dict(M=4, N=32, K=64, ac=P, sa=P, wc=P, sw=P, codes=2 * P, scales=2 * P), kw)


def norm(**kw):
    return call("p4q_residual_rmsnorm_quant",
                dict(dt=0, fmt=1, M=4, d=64, x=P, ldx=64, r=2 * P, ldr=64, post=None, gate=None, alpha=1.0, gamma=P, eps=1e-5,
                     clip=1.0, h=3 * P, ldh=64, codes=P, scales=P, values=None, ldv=0), kw)


def refused(fn, kw, status):
    assert fn(**kw) == status
    assert L.lib().p4q_last_error() != b""


@pytest.mark.parametrize("kw,status", [
    (dict(dt=2), UNSUPPORTED), (dict(M=0), BAD), (dict(M=-1), BAD), (dict(K=0), BAD), (dict(K=48), BAD),
    (dict(K=131104, ldx=131104), UNSUPPORTED), (dict(M=1 << 26), UNSUPPORTED), (dict(M=1 << 25, K=1024, ldx=1024), UNSUPPORTED),
    (dict(x=None), BAD), (dict(codes=None), BAD), (dict(scales=None), BAD), (dict(x=P + 8), BAD), (dict(ldx=56), BAD),
    (dict(ldx=68), BAD), (dict(codes=P + 4), BAD), (dict(scales=P + 8), BAD), (dict(values=P, ldv=56), BAD),
    (dict(values=P, ldv=65), BAD), (dict(values=P + 2, ldv=64), BAD),
    (dict(values=P, ldv=72), BAD)])
def test_quant_refusals(kw, status):
    refused(quant, kw, status)


PRODUCT = [(dict(M=0), BAD), (dict(N=0), BAD), (dict(K=0), BAD), (dict(K=80), BAD), (dict(K=-32), BAD),
           (dict(M=(1 << 20) + 1), UNSUPPORTED), (dict(N=(1 << 22) + 32, ldy=1 << 23), UNSUPPORTED), (dict(K=131104), UNSUPPORTED),
           (dict(ac=None), BAD), (dict(sa=None), BAD), (dict(wc=None), BAD), (dict(sw=None), BAD), (dict(ac=P + 8), BAD),
           (dict(sa=P + 4), BAD), (dict(wc=P + 8), BAD), (dict(sw=P + 1), BAD)]
OUT = [(dict(dt=5), UNSUPPORTED), (dict(y=None), BAD), (dict(y=P + 2), BAD), (dict(ldy=7), BAD), (dict(ldy=-8), BAD)]


@pytest.mark.parametrize("fn", [linear, gated])
@pytest.mark.parametrize("kw,status", PRODUCT + OUT)
def test_product_refusals(fn, kw, status):
    refused(fn, kw, status)


@pytest.mark.parametrize("kw,status", [(k, s) for k, s in [({a: b for a, b in kw.items() if a != "ldy"}, s) for kw, s in PRODUCT]] + [
    (dict(N=8), BAD), (dict(N=48), BAD), (dict(codes=None), BAD), (dict(scales=None), BAD), (dict(codes=P + 8), BAD),
    (dict(scales=P + 8), BAD), (dict(codes=P), BAD), (dict(scales=P), BAD)])
def test_gated_quant_refusals(kw, status):
    refused(gated_quant, kw, status)


@pytest.mark.parametrize("kw,status", [
    (dict(dt=3), UNSUPPORTED), (dict(fmt=2), UNSUPPORTED), (dict(fmt=-1), UNSUPPORTED), (dict(M=0), BAD), (dict(d=0), BAD),
    (dict(d=40), BAD), (dict(d=16416, ldx=16416, ldr=16416, ldh=16416), UNSUPPORTED), (dict(M=1 << 23), UNSUPPORTED),
    (dict(x=None), BAD), (dict(gamma=None), BAD), (dict(codes=None), BAD), (dict(scales=None), BAD), (dict(h=None), BAD),
    (dict(r=None), BAD), (dict(r=None, h=None, alpha=0.5), BAD), (dict(r=None, h=None, gate=P), BAD),
    (dict(r=None, h=None, post=P), BAD), (dict(x=P + 8), BAD), (dict(r=P + 8), BAD), (dict(h=P + 8), BAD), (dict(ldx=56), BAD),
    (dict(ldr=60), BAD), (dict(ldh=0), BAD), (dict(values=P, ldv=32), BAD), (dict(h=P, ldh=72), BAD), (dict(h=2 * P, ldh=72), BAD),
    (dict(gamma=P + 8), BAD), (dict(post=P + 2), BAD), (dict(gate=P + 4), BAD), (dict(codes=P + 8), BAD), (dict(scales=P + 8), BAD),
    (dict(fmt=0, scales=P + 2), BAD), (dict(eps=-1e-5), BAD), (dict(eps=2.0), BAD), (dict(eps=float("nan")), BAD),
    (dict(alpha=float("inf")), BAD), (dict(alpha=float("nan")), BAD), (dict(clip=0.5), BAD), (dict(fmt=0, clip=0.0), BAD),
    (dict(fmt=0, clip=float("nan")), BAD)])
def test_norm_refusals(kw, status):
    refused(norm, kw, status)


def test_scale_stride():
    f = L.lib().p4q_mx4_scale_stride
    assert [f(k) for k in (-32, 0, 16, 33, 131104)] == [0] * 5
    for K in (32, 480, 512, 544, 4096, 11008, 131072):
        assert f(K) == mx4_scale_stride(K) == -(-K // 512) * 16
