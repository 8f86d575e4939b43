"""Host-side argument checks of the serving calls' Python binding (CPU): every
error is raised before the library is called."""
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


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def raises(match, fn, *a, **k):
    with pytest.raises(ValueError, match=match):
        fn(*a, **k)


GPU = "must live on the GPU"
Q, K, V, CU = f16(6, 256), f16(6, 128), f16(6, 128), i32(3)
KC, VC, TABLE, LENS = f16(8, 2, 16, 64), f16(8, 2, 16, 64), i32(2, 4), i32(2)


def cache_checks(fn, args, q, kc, vc, table):
    """The checks that every call over a cache makes; q, kc, vc, table: their places among args."""
    def put(**at):
        return [at.get({q: "q", kc: "kc", vc: "vc", table: "table"}.get(i), a) for i, a in enumerate(args)]
    raises("q must be fp16 or bf16", fn, *put(q=torch.zeros(6, 256)))
    raises("share a shape", fn, *put(vc=f16(8, 2, 32, 64)))
    raises("share a shape", fn, *put(kc=f16(8, 2, 1024), vc=f16(8, 2, 1024)))
    raises("caches must have q's dtype", fn, *put(kc=KC.bfloat16()))
    raises("must be contiguous", fn, *put(kc=f16(8, 16, 2, 64).transpose(1, 2)))
    raises("block_table must be", fn, *put(table=TABLE.long()))
    raises("block_table must be", fn, *put(table=i32(8)))
    raises("block_table must be", fn, *put(table=i32(4, 2).t()))


def test_append_checks():
    ok = (Q, K, V, CU, TABLE, KC, VC, 4)
    raises(GPU, api.rope_append, *ok)
    raises(GPU, api.rope_append, *ok, cache_lens=LENS, positions=i32(6), q_out=Q, k_out=K)
    cache_checks(api.rope_append, ok, 0, 5, 6, 4)
    raises("not a multiple", api.rope_append, Q, K, V, CU, TABLE, KC, VC, 3)
    raises("q must have shape", api.rope_append, f16(6, 255), K, V, CU, TABLE, KC, VC, 4)
    raises("k must have shape", api.rope_append, Q, f16(5, 128), V, CU, TABLE, KC, VC, 4)
    raises("v must have shape", api.rope_append, Q, K, f16(6, 64), CU, TABLE, KC, VC, 4)
    raises("k must be", api.rope_append, Q, K.bfloat16(), V, CU, TABLE, KC, VC, 4)
    raises("unit column stride", api.rope_append, f16(256, 6).t(), K, V, CU, TABLE, KC, VC, 4)
    raises("cu_seqlens must be", api.rope_append, Q, K, V, i32(2), TABLE, KC, VC, 4)
    raises("cache_lens must be", api.rope_append, *ok, cache_lens=i32(3))
    raises("positions must be", api.rope_append, *ok, positions=torch.zeros(6, dtype=torch.int64))
    raises("q_out must have shape", api.rope_append, *ok, q_out=f16(5, 256))
    raises("k_out must be", api.rope_append, *ok, k_out=torch.zeros(6, 128))


def test_packed_checks():
    def call(q=Q, k=K, v=V, cu=CU, Hq=4, Hk=2, **kw):
        return api.attention_packed(q, k, v, cu, Hq, Hk, 64, **kw)
    raises(GPU, call)
    raises(GPU, call, cu_seqlens_k=i32(3), k=f16(9, 128), v=f16(9, 128), out=f16(6, 256))
    raises("q must be fp16 or bf16", call, q=torch.zeros(6, 256))
    raises("q must have shape", call, q=f16(6, 192))
    raises("v must have shape", call, v=f16(7, 128))
    raises("cu_seqlens_k is needed", call, k=f16(9, 128), v=f16(9, 128))
    raises("cu_seqlens must have shape", call, cu=i32(1))
    raises("cu_seqlens must be", call, cu=CU.long())
    raises("cu_seqlens_k must be", call, cu_seqlens_k=i32(4))
    raises("out must have shape", call, out=f16(6, 128))
    raises("out must be", call, out=f16(6, 256).bfloat16())
    raises("workspace must be", call, workspace=f16(6))


def test_paged_checks():
    ok = (Q, KC, VC, CU, TABLE, LENS, 4)
    raises(GPU, api.attention_prefill_paged, *ok)
    cache_checks(api.attention_prefill_paged, ok, 0, 1, 2, 4)
    raises("cu_seqlens must be", api.attention_prefill_paged, Q, KC, VC, i32(4), TABLE, LENS, 4)
    raises("seq_lens must be", api.attention_prefill_paged, Q, KC, VC, CU, TABLE, i32(3), 4)
    raises("out must have shape", api.attention_prefill_paged, *ok, out=f16(5, 256))
    raises("workspace must be", api.attention_prefill_paged, *ok, workspace=f16(6))


def test_decode_checks():
    ok = (f16(2, 256), KC, VC, TABLE, LENS, 4)
    raises(GPU, api.attention_decode, *ok)
    cache_checks(api.attention_decode, ok, 0, 1, 2, 3)
    raises("q must have shape", api.attention_decode, f16(3, 256), KC, VC, TABLE, LENS, 4)
    raises("seq_lens must be", api.attention_decode, f16(2, 256), KC, VC, TABLE, LENS.long(), 4)
    raises("out must have shape", api.attention_decode, *ok, out=f16(2, 128))
    raises("workspace must be", api.attention_decode, *ok, workspace=f16(6))


def test_sizes_past_32_bits_are_refused():
    """They would reach the library without their upper bits: 2^32 + 64 keys as 64."""
    ok = (f16(2, 256), KC, VC, TABLE, LENS, 4)
    for n in (2 ** 32 + 64, 2 ** 31, -2 ** 32 + 64):
        raises("max_len = .* does not fit", api.attention_decode, *ok, max_len=n)
        raises("max_len = .* does not fit", api.attention_decode_workspace, 2, 4, 2, 64, n, "cuda")
        raises("B = .* does not fit", api.attention_decode_workspace, n, 4, 2, 64, 64, "cuda")


# ------------------------------------------------------------------ another device than the current one
class Recorder:
    """Stands in for the library: keeps what each call is given."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*a):
            self.calls.append((name, a))
            return 4096 if name.endswith("_bytes") else 0
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
    ws = torch.zeros(4096, dtype=torch.uint8)
    calls = [
        lambda: api.rope_append(Q, K, V, CU, TABLE, KC, VC, 4, cache_lens=LENS, positions=i32(6), rope_base=5e5,
                                q_out=f16(6, 256), k_out=f16(6, 128)),
        lambda: api.attention_packed(Q, f16(9, 128), f16(9, 128), CU, 4, 2, 64, causal=False, cu_seqlens_k=CU,
                                     out=f16(6, 256), workspace=ws),
        lambda: api.attention_prefill_paged(Q, KC, VC, CU, TABLE, LENS, 4, causal=False, out=f16(6, 256), workspace=ws),
        lambda: api.attention_decode(f16(2, 256), KC, VC, TABLE, LENS, 4, max_len=33, out=f16(2, 256), workspace=ws),
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


def test_stream_handle_without_torchs_private_call(monkeypatch):
    """A torch build that lacks it: the current stream object's handle."""
    import importlib.util
    from types import SimpleNamespace
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    spec = importlib.util.spec_from_file_location("paper_2609_34867_amd.api_of_such_a_build", api.__file__)
    other = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(other)
    asked = []
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d: asked.append(d) or SimpleNamespace(cuda_stream=77))
    assert other._stream(torch.device("cuda", 3)) == 77 and asked == [torch.device("cuda", 3)]
