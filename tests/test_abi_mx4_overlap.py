"""Results of the MXFP4 calls that share memory with another operand are refused at the
C ABI (CPU only): the addresses below are never dereferenced."""
import ctypes
import os

import pytest

from paper_2609_34867_amd import _lib as L

S = 1 << 20                                                 # further apart than any operand below
FLOATS = ("alpha", "eps", "clip")


@pytest.fixture(scope="module", autouse=True)
def built_library():
    if not os.path.exists(L.LIB_PATH):
        from paper_2609_34867_amd.build import build
        build()


CALLS = {
    "p4q_quant_mx4": dict(dt=0, M=4, K=64, x=S, ldx=96, codes=2 * S, scales=3 * S, values=4 * S, ldv=96),
    "p4q_mx4_linear": dict(M=4, N=48, K=64, ac=S, sa=2 * S, wc=3 * S, sw=4 * S, dt=0, y=5 * S, ldy=96),
    "p4q_mx4_gated_linear": dict(M=4, N=48, K=64, ac=S, sa=2 * S, wc=3 * S, sw=4 * S, dt=0, y=5 * S, ldy=96),
    "p4q_mx4_gated_linear_quant": dict(M=4, N=64, K=64, ac=S, sa=2 * S, wc=3 * S, sw=4 * S, codes=5 * S, scales=6 * S),
    "p4q_residual_rmsnorm_quant": dict(dt=0, fmt=1, M=4, d=64, x=S, ldx=96, r=2 * S, ldr=96, post=3 * S, gate=4 * S, alpha=1.0,
                                       gamma=5 * S, eps=1e-5, clip=1.0, h=6 * S, ldh=96, codes=7 * S, scales=8 * S, values=9 * S,
                                       ldv=96),
}
ROW = 2 * 96                                                # bytes between the rows of x, r, h, values and y


def refused(fn, **kw):
    a = dict(CALLS[fn])
    assert set(kw) <= set(a)
    a.update(kw)
    assert getattr(L.lib(), fn)(*[ctypes.c_float(x) if n in FLOATS else x for n, x in a.items()], None) == L.P4Q_ERR_INVALID_ARG
    message = L.lib().p4q_last_error().decode()
    assert "overlap" in message or "cannot replace" in message, message


@pytest.mark.parametrize("kw", [
    dict(values=S + ROW), dict(values=S - ROW), dict(values=S + 2 * 32), dict(codes=S), dict(codes=S + 3 * ROW), dict(scales=S),
    dict(codes=4 * S), dict(scales=4 * S + 3 * ROW), dict(scales=2 * S), dict(scales=2 * S + 4 * 32 - 16), dict(codes=3 * S + 4 * 16 - 16),
    dict(values=None, ldv=2 ** 63 - 1, codes=S)])
def test_quantizer(kw):
    refused("p4q_quant_mx4", **kw)


@pytest.mark.parametrize("fn,rows", [("p4q_mx4_linear", 48), ("p4q_mx4_gated_linear", 96)])
@pytest.mark.parametrize("name,at", [("ac", 1), ("sa", 2), ("wc", 3), ("sw", 4)])
def test_products(fn, rows, name, at):
    refused(fn, y=at * S)
    refused(fn, y=at * S - 3 * ROW)                         # the last row
    n, width = (4 if at < 3 else rows), (32 if at % 2 else 16)
    refused(fn, y=at * S + n * width - 4)                   # the operand's last bytes


@pytest.mark.parametrize("name", ["codes", "scales"])
@pytest.mark.parametrize("at", [1, 2, 3, 4])
def test_quantized_product(name, at):
    refused("p4q_mx4_gated_linear_quant", **{name: at * S})
    refused("p4q_mx4_gated_linear_quant", **{name: at * S + 16})


def test_quantized_product_results():
    refused("p4q_mx4_gated_linear_quant", codes=6 * S)
    refused("p4q_mx4_gated_linear_quant", scales=5 * S + 4 * 32 - 16)


@pytest.mark.parametrize("kw", [
    dict(values=6 * S), dict(values=6 * S + ROW), dict(values=S), dict(values=2 * S), dict(values=5 * S), dict(values=4 * S),
    dict(h=S + ROW), dict(h=2 * S + 2 * 32), dict(h=3 * S), dict(h=5 * S + 64), dict(codes=6 * S), dict(codes=S), dict(codes=8 * S),
    dict(scales=9 * S), dict(scales=3 * S), dict(scales=7 * S + 16), dict(fmt=0, scales=6 * S), dict(fmt=0, scales=7 * S + 124),
    # without a residual x is the result
    dict(r=None, h=None, post=None, gate=None, values=S),
    dict(r=None, ldr=2 ** 63 - 1, h=None, ldh=-2 ** 63, post=None, gate=None, values=S)])
def test_norm(kw):
    refused("p4q_residual_rmsnorm_quant", **kw)
