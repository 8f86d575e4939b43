"""Host-side refusals of the serving calls at the C ABI, and their workspace sizes
(CPU only): the addresses below are never dereferenced."""
import ctypes
import os
import subprocess
import sys

import pytest

from paper_2609_34867_amd import _lib as L

P = 0x10000
INT_MAX = 2 ** 31 - 1
BAD, UNSUPPORTED, ROOM = L.P4Q_ERR_INVALID_ARG, L.P4Q_ERR_UNSUPPORTED, L.P4Q_ERR_WORKSPACE


@pytest.fixture(scope="module", autouse=True)
def built_library():
    if not os.path.exists(L.LIB_PATH):
        from paper_2609_34867_amd.build import build
        build()


def append(**kw):
    a = dict(dt=0, T=4, B=2, Hq=4, Hk=2, D=64, q=P, ldq=256, k=P, ldk=128, v=P, ldv=128, cu=P, lens=P, pos=None,
             base=1e4, qo=2 * P, ldqo=256, ko=None, ldko=0, kc=P, vc=P, pages=8, page=16, table=P, width=4)
    a.update(kw)
    return L.lib().p4q_rope_append(*[ctypes.c_float(x) if n == "base" else x for n, x in a.items()], None)


def packed(**kw):
    a = dict(dt=0, T=4, Tk=4, B=2, Hq=4, Hk=2, D=64, q=P, ldq=256, k=P, ldk=128, v=P, ldv=128, cu=P, cuk=None,
             out=P, ldo=256, causal=1, ws=None, ws_bytes=0)
    a.update(kw)
    return L.lib().p4q_attention_packed(*a.values(), None)


def paged(**kw):
    a = dict(dt=0, T=4, B=2, Hq=4, Hk=2, D=64, q=P, ldq=256, kc=P, vc=P, pages=8, page=16, table=P, width=4, cu=P,
             lens=P, out=P, ldo=256, causal=1, ws=None, ws_bytes=0)
    a.update(kw)
    return L.lib().p4q_attention_prefill_paged(*a.values(), None)


def decode(**kw):
    a = dict(dt=0, B=2, Hq=4, Hk=2, D=64, q=P, ldq=256, kc=P, vc=P, pages=8, page=16, table=P, width=4, lens=P,
             max_len=64, out=P, ldo=256, ws=None, ws_bytes=0)
    a.update(kw)
    return L.lib().p4q_attention_decode(*a.values(), None)


HEADS = [(dict(dt=7), UNSUPPORTED), (dict(B=0), BAD), (dict(Hq=0), BAD), (dict(Hk=0), BAD), (dict(Hq=5), BAD),
         (dict(D=0), BAD), (dict(D=96), UNSUPPORTED), (dict(B=65536), UNSUPPORTED),
         (dict(Hq=1026, ldq=1026 * 64), UNSUPPORTED), (dict(q=None), BAD), (dict(q=P + 8), BAD), (dict(ldq=248), BAD),
         (dict(ldq=260), BAD), (dict(ldq=1 << 24), UNSUPPORTED)]
ROWS = [(dict(T=0), BAD), (dict(T=-1), BAD), (dict(T=(1 << 24) + 1), UNSUPPORTED), (dict(T=1 << 24, Hq=1024, Hk=1024), UNSUPPORTED), (dict(cu=None), BAD), (dict(cu=P + 2), BAD)]
KEYS = [(dict(k=None), BAD), (dict(v=None), BAD), (dict(k=P + 2), BAD), (dict(v=P + 8), BAD), (dict(ldk=64), BAD),
        (dict(ldv=132), BAD), (dict(ldk=1 << 24), UNSUPPORTED)]
CACHE = [(dict(kc=None), BAD), (dict(vc=None), BAD), (dict(kc=P + 8), BAD), (dict(table=None), BAD), (dict(table=P + 1), BAD),
         (dict(pages=0), BAD), (dict(width=0), BAD), (dict(page=8), UNSUPPORTED), (dict(page=48), UNSUPPORTED),
         (dict(page=8192), UNSUPPORTED), (dict(page=0), UNSUPPORTED), (dict(width=1 << 26), UNSUPPORTED)]
OUT = [(dict(out=None), BAD), (dict(out=P + 8), BAD), (dict(ldo=128), BAD), (dict(ldo=258), BAD)]
CAUSAL = [(dict(causal=2), BAD), (dict(causal=-1), BAD)]


def refused(call, kw, status):
    assert call(**kw) == status
    assert L.lib().p4q_last_error() != b""


@pytest.mark.parametrize("kw,status", HEADS + ROWS + KEYS + CACHE + [
    (dict(qo=None), BAD), (dict(qo=P + 4), BAD), (dict(ldqo=128), BAD), (dict(ko=P + 8, ldko=128), BAD),
    (dict(ko=P, ldko=64), BAD), (dict(lens=P + 2), BAD), (dict(pos=P + 1), BAD), (dict(base=1.0), BAD),
    (dict(base=float("nan")), BAD), (dict(base=float("inf")), BAD), (dict(qo=P, ldqo=512), BAD),
    (dict(ko=P, ldko=256), BAD)])
def test_append_refusals(kw, status):
    refused(append, kw, status)


@pytest.mark.parametrize("kw,status", HEADS + ROWS + KEYS + OUT + CAUSAL + [
    (dict(Tk=-1), BAD), (dict(Tk=5), BAD), (dict(Tk=(1 << 24) + 1, cuk=P), UNSUPPORTED), (dict(cuk=P + 2), BAD)])
def test_packed_refusals(kw, status):
    refused(packed, kw, status)


@pytest.mark.parametrize("kw,status", HEADS + ROWS + CACHE + OUT + CAUSAL + [(dict(lens=None), BAD), (dict(lens=P + 2), BAD)])
def test_paged_refusals(kw, status):
    refused(paged, kw, status)


@pytest.mark.parametrize("kw,status", HEADS + CACHE + OUT + [
    (dict(lens=None), BAD), (dict(lens=P + 2), BAD), (dict(max_len=0), BAD), (dict(max_len=65), BAD),
    (dict(), ROOM), (dict(max_len=1), ROOM), (dict(max_len=4096, width=256), ROOM), (dict(max_len=4096, width=256, ws=P, ws_bytes=100), ROOM),
    (dict(max_len=4096, width=256, ws=P + 8, ws_bytes=1 << 30), BAD)])
def test_decode_refusals(kw, status):
    refused(decode, kw, status)


@pytest.mark.parametrize("args", [(INT_MAX, INT_MAX, INT_MAX, INT_MAX, 64, INT_MAX), (0, 1, 1, 1, 64, 64),
                                  (1 << 24, 65535, 1024, 1, 128, INT_MAX), (1 << 24, 65535, 1024, 1024, 128, INT_MAX),
                                  (1, 1, 4, 3, 64, 64), (1, 1, 4, 4, 96, 1 << 20), (1, 1, 1, 1, 64, -1),
                                  (1, 1, 1, 1, 64, 2 ** 40)])
def test_prompt_workspace_extremes(args):
    """Refused shapes need none, full devices neither; no size overflows."""
    assert L.lib().p4q_attention_prompt_workspace_bytes(*args) == 0


@pytest.mark.parametrize("args", [(INT_MAX, INT_MAX, INT_MAX, 64, INT_MAX), (0, 1, 1, 64, 64), (65535, 1024, 1024, 128, 1 << 29),
                                  (1, 4, 3, 64, 64), (1, 4, 4, 96, 4096), (1, 4, 4, 64, 0), (1, 4, 4, 64, 1 << 30)])
def test_decode_workspace_extremes(args):
    assert L.lib().p4q_attention_decode_workspace_bytes(*args) == 0


@pytest.mark.parametrize("B,Hq,Hk,D,max_len", [(1, 1, 1, 64, 1), (5, 2, 2, 128, 100), (65535, 16, 1, 64, 128), (64, 64, 8, 128, 1 << 29)])
def test_every_decode_call_has_room_for_two_parts_of_each_share(B, Hq, Hk, D, max_len):
    """Short calls too: a work-group's share may begin and end within a sequence."""
    n = L.lib().p4q_attention_decode_workspace_bytes(B, Hq, Hk, D, max_len)
    groups = min(512, B * Hk * -(-(Hq // Hk) // 16) * -(-max_len // 128))     # of 256 compute units
    assert n >= 32768 + 2 * groups * 16 * (D + 2) * 4


def test_workspaces_where_keys_are_split():
    assert L.lib().p4q_attention_prompt_workspace_bytes(1, 1, 8, 8, 128, 1 << 29) > 8 * 128 * 4
    assert L.lib().p4q_attention_decode_workspace_bytes(1, 8, 8, 128, 1 << 29) > 32768 + 8 * 16 * 128 * 4


def test_these_pass_under_sanitizers(tmp_path):
    """This file against the library with its host code under the sanitizers."""
    if os.environ.get("P4Q_LIBRARY"):
        return                                        # the run inside
    from test_abi_sanitized import HIPCC, build_sanitized, runtime
    if not os.path.exists(HIPCC):
        pytest.fail("hipcc not found: the sanitized ABI build needs the ROCm toolchain")
    rt = runtime()
    assert rt, "the ROCm compiler's AddressSanitizer runtime was not found"
    logs = str(tmp_path / "sanitizer")
    env = dict(os.environ, LD_PRELOAD=rt, P4Q_LIBRARY=build_sanitized(),
               ASAN_OPTIONS=f"detect_leaks=0:halt_on_error=1:log_path={logs}",
               UBSAN_OPTIONS=f"halt_on_error=1:print_stacktrace=1:log_path={logs}")
    p = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), "-q", "-p", "no:cacheprovider"],
                       env=env, capture_output=True, text=True, timeout=600)
    reports = "".join(f.read_text() for f in tmp_path.glob("sanitizer*"))
    assert p.returncode == 0 and not reports, f"rc {p.returncode}:\n{reports[:4000]}\n{p.stdout[-3000:]}"
