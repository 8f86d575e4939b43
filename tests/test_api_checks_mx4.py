"""Host-side argument checks of the MXFP4 calls' Python binding (CPU): every error is
raised before the library is called."""
import pytest
import torch

import paper_2609_34867_amd.api as api


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    def forbidden():
        raise AssertionError("the library was called before the argument checks")
    monkeypatch.setattr(api, "lib", forbidden)


def f16(*shape):
    return torch.zeros(shape, dtype=torch.float16)


def u8(*shape):
    return torch.zeros(shape, dtype=torch.uint8)


def raises(match, fn, *a, **k):
    with pytest.raises(ValueError, match=match):
        fn(*a, **k)


GPU = "must live on the GPU"
X, G = f16(6, 96), f16(96)
C, S = u8(6, 48), u8(6, 16)


def test_quant_checks():
    raises(GPU, api.quant_mx4, X)
    raises(GPU, api.quant_mx4, X, C, S, X)
    raises("2-D", api.quant_mx4, G)
    raises("x must be", api.quant_mx4, X.float())
    raises("unit column stride", api.quant_mx4, f16(96, 6).t())
    raises("codes must have shape", api.quant_mx4, X, u8(6, 47))
    raises("codes must be", api.quant_mx4, X, torch.zeros(6, 48, dtype=torch.int8))
    raises("scales must have shape", api.quant_mx4, X, C, u8(6, 3))
    raises("scales must be contiguous", api.quant_mx4, X, C, u8(16, 6).t())
    raises("values must have shape", api.quant_mx4, X, values=f16(6, 64))
    raises("values must be", api.quant_mx4, X, values=X.bfloat16())


def test_norm_checks():
    fn = api.residual_rmsnorm_quant
    raises(GPU, fn, X, G)
    raises(GPU, fn, X, G, X, post_gamma=G, gate=G, alpha=0.5, h_out=X, codes=C, scales=S, values=X)
    raises(GPU, fn, X, G, X, fmt="int4", scales=torch.zeros(6))
    raises("2-D", fn, G, G)
    raises("fmt must be", fn, X, G, fmt="fp8")
    raises("x must be", fn, X.float(), G)
    for name in ("post_gamma", "gate"):
        raises(f"{name} must be", fn, X, G, X, **{name: f16(95)})
        raises(f"{name} must be", fn, X, G, X, **{name: G.bfloat16()})
        raises("need r", fn, X, G, **{name: G})
    raises("gamma must be", fn, X, f16(2, 96)[:, 0])
    raises("need r", fn, X, G, h_out=X)
    raises("need r", fn, X, G, alpha=0.5)
    raises("r must have shape", fn, X, G, f16(5, 96))
    raises("r must be", fn, X, G, X.bfloat16())
    raises("h_out must have shape", fn, X, G, X, h_out=f16(6, 64))
    raises("values must have shape", fn, X, G, values=f16(6, 64))
    raises("codes must have shape", fn, X, G, codes=u8(6, 96))
    raises("scales must have shape", fn, X, G, scales=u8(6, 3))
    raises("scales must have shape", fn, X, G, fmt="int4", scales=u8(6, 16))
    raises("scales must be", fn, X, G, fmt="int4", scales=torch.zeros(6, dtype=torch.float64))


W, SW = u8(10, 48), u8(10, 16)


@pytest.mark.parametrize("fn,N", [(api.mx4_linear, 10), (api.mx4_gated_linear, 5)])
def test_product_checks(fn, N):
    raises(GPU, fn, C, S, W, SW)
    raises(GPU, fn, C, S, W, SW, y=f16(6, N))
    raises("a_codes must be", fn, C.char(), S, W, SW)
    raises("a_codes must be", fn, u8(48, 6).t(), S, W, SW)
    raises("w_codes must be", fn, C, S, u8(480), SW)
    raises("a_scales must be", fn, C, u8(6, 3), W, SW)
    raises("w_scales must be", fn, C, S, W, u8(10, 32))
    raises("w_scales must be", fn, C, S, W, SW.char())
    raises("disagree on K", fn, C, S, u8(10, 64), SW)
    raises("y must have shape", fn, C, S, W, SW, y=f16(6, N + 1))
    raises("y must be", fn, C, S, W, SW, y=torch.zeros(6, N))
    raises("out_dtype", fn, C, S, W, SW, out_dtype=torch.float32)


def test_gated_checks():
    raises("as many up rows", api.mx4_gated_linear, C, S, u8(9, 48), u8(9, 16))
    fn, w, sw = api.mx4_gated_linear_quant, u8(128, 48), u8(128, 16)
    raises(GPU, fn, C, S, w, sw)
    raises(GPU, fn, C, S, w, sw, u8(6, 32), u8(6, 16))
    raises("as many up rows", fn, C, S, u8(9, 48), u8(9, 16))
    raises("disagree on K", fn, C, S, u8(128, 32), sw)
    raises("codes must have shape", fn, C, S, w, sw, u8(6, 64))
    raises("scales must have shape", fn, C, S, w, sw, u8(6, 32), u8(6, 2))


# ------------------------------------------------------------------ another device than the current one
class Recorder:
    """Stands in for the library: keeps what each call is given."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*a):
            self.calls.append((name, a))
            return 0
        return call


def test_calls_on_another_device_pass_everything_on(monkeypatch):
    """Tensors of a device that is not current: the call is made again, with that
    device current and the same arguments."""
    from contextlib import contextmanager
    rec, entered = Recorder(), []

    @contextmanager
    def device(d):
        entered.append(d)
        yield

    monkeypatch.setattr(api, "lib", lambda: rec)
    monkeypatch.setattr(api, "_stream", lambda d: 7)
    monkeypatch.setattr(api.torch.cuda, "device", device)
    h, v = f16(6, 96), f16(6, 96)
    w, sw = u8(128, 48), u8(128, 16)
    calls = [
        lambda: api.quant_mx4(X, C, S, v),
        lambda: api.residual_rmsnorm_quant(X, G, h, 1e-3, "int4", 0.5, G, G, 0.25, h, C, torch.zeros(6), v),
        lambda: api.residual_rmsnorm_quant(X, G),
        lambda: api.mx4_linear(C, S, W, SW, torch.float16),
        lambda: api.mx4_linear(C, S, W, SW, y=f16(6, 10)),
        lambda: api.mx4_gated_linear(C, S, W, SW, torch.float16),
        lambda: api.mx4_gated_linear_quant(C, S, w, sw, u8(6, 32), u8(6, 16)),
    ]
    for call in calls:
        got = []
        for away in (False, True):
            answers = [away, False]                       # not current, then current
            monkeypatch.setattr(api, "_elsewhere", lambda *t: answers.pop(0))
            rec.calls.clear()
            entered.clear()
            call()
            assert entered == ([torch.device("cpu")] if away else [])
            # (addresses of the tensors made in each call differ)
            got.append([(n, [x for x in a if not (isinstance(x, int) and x > 1 << 20)]) for n, a in rec.calls])
        assert got[0] == got[1] and len(got[0]) == 1


def test_new_outputs(monkeypatch):
    monkeypatch.setattr(api, "lib", lambda: Recorder())
    monkeypatch.setattr(api, "_stream", lambda d: 7)
    monkeypatch.setattr(api, "_elsewhere", lambda *t: False)
    said = lambda *ts: [(tuple(t.shape), t.dtype) for t in ts]  # noqa: E731
    held = [((6, 48), torch.uint8), ((6, 16), torch.uint8)]
    assert said(*api.quant_mx4(X)) == held
    codes, scales, h = api.residual_rmsnorm_quant(X, G)
    assert said(codes, scales) == held and h is X
    codes, scales, h = api.residual_rmsnorm_quant(X, G, X, fmt="int4")
    assert said(codes, scales, h) == [held[0], ((6,), torch.float32), ((6, 96), torch.float16)]
    assert said(api.mx4_linear(C, S, W, SW)) == [((6, 10), torch.bfloat16)]
    assert said(api.mx4_gated_linear(C, S, W, SW, torch.float16)) == [((6, 5), torch.float16)]
    assert said(*api.mx4_gated_linear_quant(C, S, u8(128, 48), u8(128, 16))) == [((6, 32), torch.uint8), ((6, 16), torch.uint8)]
