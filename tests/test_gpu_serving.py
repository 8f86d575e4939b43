"""GPU parity of the serving calls (rope_append, attention_packed,
attention_prefill_paged, attention_decode) against the oracle in float64.

Tolerances, from the arithmetic (eps: of the 16-bit type; half a step is eps / 2):
  rotation: x cos a - x' sin a with sine and cosine of an angle reduced in 64 bits,
    within 2^-22 of theirs, products and sum in fp32: 2^-21 (|x| + |x'|), and the
    output's rounding, eps / 2 |y|;
  attention: with A = sum_j P_j |v_j|, the weights' rounding moves the result by at
    most eps / 2 A; a score of D products in fp32 is within D 2^-24 |q||k| / sqrt(D) of its
    value, and exp2 within 2^-22, which moves weight and sum by as much, relatively
    (twice); fp32 sums of m weights and products: m 2^-24 A each; fp16 weights below
    2^-24 of a scaled 2^7: m 2^-32 max|v|; the output's rounding, eps / 2 (|o| + all that)."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_34867_amd as p4q
from gpu_util import Guarded, check_canaries, dev

pytestmark = pytest.mark.gpu
DT = {"fp16": torch.float16, "bf16": torch.bfloat16}


def gen(seed):
    return torch.Generator(device=dev()).manual_seed(seed)


def randn(g, dtype, *shape, std=1.0):
    return (std * torch.randn(*shape, generator=g, device=dev())).to(DT[dtype])


def f64(t):
    return t.double().cpu().numpy()


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device=dev())


def cu_of(lens):
    return ints(np.concatenate([[0], np.cumsum(lens)]).tolist())


def assert_within(got, ref, bound, what=""):
    err = np.abs(got - ref)
    bad = np.argwhere(~(err <= bound))
    if bad.size:
        i = tuple(bad[0])
        raise AssertionError(f"{what}: {len(bad)} of {err.size} out of tolerance, first {i}: {got[i]} vs {ref[i]}, "
                             f"off by {err[i]}, allowed {bound[i]}")


def attention_bound(q, k, v, O, A, dtype):
    """q [n, Hq, D], k and v [m, Hk, D] (float64): the bound of the module's docstring."""
    eps, D, m = torch.finfo(DT[dtype]).eps, q.shape[-1], max(1, k.shape[0])
    G = q.shape[1] // k.shape[1]
    knorm = np.sqrt((k ** 2).sum(-1)).max(0) if k.shape[0] else np.zeros(k.shape[1])
    vmax = np.abs(v).max((0, 2)) if v.shape[0] else np.zeros(v.shape[1])
    score = 2 * (D * 2.0 ** -24 * np.sqrt((q ** 2).sum(-1)) * np.repeat(knorm, G) / np.sqrt(D) + 2.0 ** -22)
    inner = (eps / 2 + score[:, :, None] + 2 * m * 2.0 ** -24) * A
    if dtype == "fp16":
        inner = inner + m * 2.0 ** -32 * np.repeat(vmax, G)[None, :, None]
    return inner + eps / 2 * (np.abs(O) + inner) + 2.0 ** -25      # 2^-25: half an fp16 subnormal


def make_cache(g, dtype, key_lens, Hk, D, P, spare=3, width=None, fill=float("nan")):
    """(k_cache, v_cache, table): pages dealt in any order; rows past a sequence's keys, and pages of
    none, hold `fill`.  Unused table entries are outside the cache."""
    used = [-(-n // P) for n in key_lens]
    pages = sum(used) + spare
    kc = torch.full((pages, Hk, P, D), fill, dtype=DT[dtype], device=dev())
    vc = kc.clone()
    width = width or max(max(used), 1) + 1
    table = np.full((len(key_lens), width), -1, np.int32)
    order, at = torch.randperm(pages, generator=g, device=dev()).cpu().numpy(), 0
    for b, n in enumerate(key_lens):
        table[b, :used[b]] = order[at:at + used[b]]
        for j in range(used[b]):
            r = min(P, n - j * P)
            page = int(order[at + j])
            kc[page, :, :r] = randn(g, dtype, Hk, r, D)
            vc[page, :, :r] = randn(g, dtype, Hk, r, D)
        at += used[b]
    return kc, vc, torch.from_numpy(table).to(dev())


def make_cache_flat(g, dtype, B, width, Hk, D, P):
    """(k_cache, v_cache, table) full of keys, `width` pages for each of B sequences, dealt in any order."""
    kc, vc = (randn(g, dtype, B * width, Hk, P, D) for _ in range(2))
    return kc, vc, torch.randperm(B * width, generator=g, device=dev()).to(torch.int32).view(B, width)


def check_attention(got, q, keys, lens, Hq, D, dtype, causal=True):
    """got [T, Hq D] against the oracle; keys(b) gives k, v [m, Hk, D] in float64."""
    got, q = f64(got).reshape(-1, Hq, D), f64(q).reshape(-1, Hq, D)
    at = 0
    for b, n in enumerate(lens):
        k, v = keys(b)
        O, A = oracle.grouped_attention(q[at:at + n], k, v, causal)
        assert_within(got[at:at + n], O, attention_bound(q[at:at + n], k, v, O, A, dtype), f"sequence {b}")
        at += n


# ------------------------------------------------------------------ rotation and append
@pytest.mark.parametrize("dtype,Hq,Hk,D,P,lens,past,spots,pad", [
    ("fp16", 4, 4, 128, 16, [1], [0], None, 0),
    ("bf16", 40, 40, 128, 16, [1], [700], None, 0),                        # a decode step
    ("fp16", 6, 2, 64, 32, [1, 1, 0, 1], [15, 16, 7, 31], None, 2),        # page edges, an idle sequence
    ("bf16", 8, 1, 128, 64, [37, 0, 100, 1], [0, 5, 60, 64], "pruned", 5),
    ("fp16", 5, 5, 64, 16, [0, 0, 3], [0, 0, 0], "far", 0),
    ("fp16", 32, 8, 128, 256, [260], [255], "far", 1),
    ("bf16", 3, 1, 64, 4096, [70] * 70, [3] * 70, None, 9),                # more than 64 sequences
])
def test_rope_append(dtype, Hq, Hk, D, P, lens, past, spots, pad):
    g = gen(11)
    T, B = sum(lens) + pad, len(lens)
    totals = [n + m for n, m in zip(lens, past)]
    kc, vc, table = make_cache(g, dtype, totals, Hk, D, P, fill=1.5)
    kc0, vc0 = kc.clone(), vc.clone()
    qkv = randn(g, dtype, T, (Hq + 2 * Hk) * D + 8)                         # wider than its heads
    q, k, v = qkv[:, :Hq * D], qkv[:, Hq * D:(Hq + Hk) * D], qkv[:, (Hq + Hk) * D:(Hq + 2 * Hk) * D]
    place = np.concatenate([np.arange(m, m + n) for n, m in zip(lens, past)] + [np.zeros(pad)]).astype(np.int64)
    positions = None
    if spots == "pruned":
        place = np.cumsum(np.arange(T) % 7 + 1)
        positions = ints(place.tolist())
    if spots == "far":
        place = 2 ** 31 - 1 - 37 * np.arange(T)
        positions = ints(place.tolist())
    gq, gk = Guarded((T, Hq * D), DT[dtype], "q_out"), Guarded((T, Hk * D), DT[dtype], "k_out")
    gq.t.fill_(3), gk.t.fill_(3)
    got = p4q.rope_append(q, k, v, cu_of(lens), table, kc, vc, Hq, cache_lens=ints(past), positions=positions,
                          rope_base=500000.0, q_out=gq.t, k_out=gk.t)
    assert got[0] is gq.t and got[1] is gk.t
    check_canaries(gq, gk)
    n, eps = sum(lens), torch.finfo(DT[dtype]).eps
    for x, y, heads in ((q, gq.t, Hq), (k, gk.t, Hk)):
        assert (y[n:] == 3).all()                                           # behind the last sequence
        x = f64(x[:n]).reshape(n, heads, D)
        ref = oracle.rope(x, place[:n], 500000.0)
        size = np.abs(x) + np.abs(np.roll(x, D // 2, axis=-1))
        # a position of 2^31 carries 2^31 2^-53 (and theta's error as much again) into the angle
        bound = (2.0 ** -21 + 2.0 ** -20) * size + eps / 2 * np.abs(ref) + 2.0 ** -25
        assert_within(f64(y[:n]).reshape(n, heads, D), ref, bound)
    # the cache: the call's rows hold k_out and v bit for bit, every other row is as it was
    tab, at = table.cpu().numpy(), 0
    for b in range(B):
        for i in range(lens[b]):
            s = past[b] + i
            kc0[tab[b, s // P], :, s % P] = gk.t[at].view(Hk, D)
            vc0[tab[b, s // P], :, s % P] = v[at].view(Hk, D)
            at += 1
    assert torch.equal(kc, kc0) and torch.equal(vc, vc0)


def test_rope_append_in_place_and_defaults():
    """q_out = q and k_out = k; no cache_lens, no positions; v not touched."""
    Hq, Hk, D, P, lens = 6, 2, 128, 16, [20, 3]
    g = gen(12)
    kc, vc, table = make_cache(g, "fp16", lens, Hk, D, P, fill=0)
    qkv = randn(g, "fp16", 23, (Hq + 2 * Hk) * D)
    w = qkv.clone()
    cols = (slice(0, Hq * D), slice(Hq * D, (Hq + Hk) * D), slice((Hq + Hk) * D, None))
    q_ref, k_none = p4q.rope_append(*(w[:, c] for c in cols), cu_of(lens), table, kc, vc, Hq)
    assert k_none is None and torch.equal(w, qkv)
    kc2, vc2 = torch.zeros_like(kc), torch.zeros_like(vc)
    p4q.rope_append(*(w[:, c] for c in cols), cu_of(lens), table, kc2, vc2, Hq, cache_lens=ints([0, 0]),
                    positions=ints(list(range(20)) + [0, 1, 2]), q_out=w[:, cols[0]], k_out=w[:, cols[1]])
    assert torch.equal(w[:, cols[0]], q_ref) and torch.equal(w[:, cols[2]], qkv[:, cols[2]])
    assert torch.equal(w[:20, cols[1]].view(20, Hk, D)[:16], kc2[table[0, 0]].transpose(0, 1))
    keep = [int(p) for p in table[table >= 0]]
    assert torch.equal(kc2[keep][:, :, :3], kc[keep][:, :, :3])


def test_rope_append_out_of_range_places_are_dropped():
    """Table entries outside the cache, places past the table or negative: those
    tokens are rotated and not appended; nothing else is written."""
    Hq, Hk, D, P = 2, 1, 64, 16
    g = gen(13)
    kc = torch.full((5, Hk, P, D), 2.0, dtype=torch.float16, device=dev())
    vc = kc.clone()
    table = ints([0, -1, 4, 5, 2 ** 31 - 1, -2 ** 31]).view(3, 2).contiguous()
    lens, past = [40, 40, 30], [0, -8, 20]
    T = sum(lens)
    qkv = randn(g, "fp16", T, 4 * D)
    args = (qkv[:, :2 * D], qkv[:, 2 * D:3 * D], qkv[:, 3 * D:], cu_of(lens), table)
    k_out = torch.zeros(T, D, dtype=torch.float16, device=dev())
    q_out, _ = p4q.rope_append(*args, kc, vc, Hq, cache_lens=ints(past), k_out=k_out)
    assert torch.isfinite(q_out).all() and k_out.any(1).all()
    assert torch.equal(kc[0, 0], k_out[:16]) and torch.equal(vc[0, 0], qkv[:16, 3 * D:])
    # sequence 1: tokens 8 .. 23 take places 0 .. 15 of page 4
    assert torch.equal(kc[4, 0], k_out[48:64])
    assert (kc[1:4] == 2).all() and (vc[1:4] == 2).all()


def test_rope_append_nonfinite_values():
    """v goes through bit for bit (NaN, infinities, -0); rotated pairs with an
    infinity are what the formula gives."""
    D = 64
    q = torch.zeros(1, D, dtype=torch.float16, device=dev())
    v = torch.tensor([float("nan"), float("inf"), -float("inf"), -0.0] * 16, dtype=torch.float16, device=dev())[None]
    k = q.clone()
    k[0, 3] = float("inf")
    kc, vc = (torch.zeros(1, 1, 16, D, dtype=torch.float16, device=dev()) for _ in range(2))
    p4q.rope_append(q, k, v, ints([0, 1]), ints([0]).view(1, 1), kc, vc, 1, cache_lens=ints([0]))
    assert torch.equal(vc[0, 0, 0].view(torch.int16), v[0].view(torch.int16))
    p4q.rope_append(q, k, v, ints([0, 1]), ints([0]).view(1, 1), kc, vc, 1, cache_lens=ints([1]))
    row = kc[0, 0, 1]
    assert row[3] == float("inf") and row[3 + D // 2] == float("inf") and torch.isfinite(row).sum() == D - 2


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("Hq,Hk,D,lens", [(8, 8, 128, [7001, 1, 0, 6003, 5999]), (16, 8, 64, [9001, 12000, 0, 3, 8999])])
@pytest.mark.parametrize("in_place", [False, True])
def test_rope_append_of_more_than_128_mib(dtype, Hq, Hk, D, lens, in_place):
    """Calls that write more than 128 MiB go past the last-level cache: bit for bit what the same tokens
    give sequence by sequence in calls that write less, and what attention then reads."""
    g, P, B, pad = gen(14), 64, len(lens), 9
    T, past = sum(lens) + pad, [5, 0, 3, 64, 100]
    totals = [n + m for n, m in zip(lens, past)]
    kc, vc, table = make_cache(g, dtype, totals, Hk, D, P, fill=0.5)
    kc2, vc2 = kc.clone(), vc.clone()
    qkv = randn(g, dtype, T, (Hq + 2 * Hk) * D)
    cols = (slice(0, Hq * D), slice(Hq * D, (Hq + Hk) * D), slice((Hq + Hk) * D, None))
    place = torch.randint(0, 100000, (T,), generator=g, device=dev()).to(torch.int32)
    token = (Hq + 3 * Hk) * D * 2
    assert T * token > 1 << 27 > max(lens) * token                        # the launcher's threshold
    # sequence by sequence
    q_ref, k_ref = torch.full((T, Hq * D), 3.0, dtype=DT[dtype], device=dev()), torch.full((T, Hk * D), 3.0, dtype=DT[dtype], device=dev())
    at = 0
    for b, n in enumerate(lens):
        if n:
            r = slice(at, at + n)
            p4q.rope_append(*(qkv[r, c] for c in cols), ints([0, n]), table[b:b + 1], kc2, vc2, Hq, cache_lens=ints(past[b:b + 1]),
                            positions=place[r], q_out=q_ref[r], k_out=k_ref[r])
        at += n
    # in one call
    wide = qkv.clone()
    if in_place:
        q_out, k_out = wide[:, cols[0]], wide[:, cols[1]]
        q_ref[at:], k_ref[at:] = q_out[at:], k_out[at:]
    else:
        gq, gk = Guarded((T, Hq * D), DT[dtype], "q_out"), Guarded((T, Hk * D), DT[dtype], "k_out")
        q_out, k_out = gq.t.fill_(3), gk.t.fill_(3)
    p4q.rope_append(*(wide[:, c] for c in cols), cu_of(lens), table, kc, vc, Hq, cache_lens=ints(past), positions=place,
                    q_out=q_out, k_out=k_out)
    got = [p4q.attention_decode(q_out[:B], *c, table, ints(totals), Hq, max_len=max(totals)) for c in ((kc, vc), (kc2, vc2))]
    if not in_place:
        check_canaries(gq, gk)
    for a, b in ((q_out, q_ref), (k_out, k_ref), (kc, kc2), (vc, vc2), got, (wide[:, cols[2]], qkv[:, cols[2]])):
        assert torch.equal(a, b)


# ------------------------------------------------------------------ packed prompts
def packed_case(seed, dtype, Hq, Hk, D, lens, key_lens=None, causal=True, pad=0, std=1.0):
    g = gen(seed)
    own = key_lens is None
    key_lens = lens if own else key_lens
    T, Tk = sum(lens) + pad, sum(key_lens) + pad
    q = randn(g, dtype, T, Hq * D, std=std)
    kv = randn(g, dtype, Tk, 2 * Hk * D, std=std)
    kv[sum(key_lens):] = float("nan")                                       # behind the last sequence
    go = Guarded((T, Hq * D), DT[dtype], "out")
    go.t.fill_(7)
    p4q.attention_packed(q, kv[:, :Hk * D], kv[:, Hk * D:], cu_of(lens), Hq, Hk, D, causal,
                         cu_seqlens_k=None if own else cu_of(key_lens), out=go.t)
    check_canaries(go)
    assert (go.t[sum(lens):] == 7).all()
    ends = np.concatenate([[0], np.cumsum(key_lens)])
    kv64 = f64(kv).reshape(-1, 2, Hk, D)
    check_attention(go.t, q, lambda b: (kv64[ends[b]:ends[b + 1], 0], kv64[ends[b]:ends[b + 1], 1]), lens, Hq, D, dtype, causal)


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 257])
@pytest.mark.parametrize("D", [64, 128])
def test_packed_lengths(n, D):
    packed_case(20 + n, "fp16", 2, 2, D, [n, 3, n])


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("Hq,Hk,D", [(4, 4, 128), (8, 2, 128), (7, 1, 128), (12, 4, 64), (40, 1, 64), (130, 1, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_packed_heads(dtype, Hq, Hk, D, causal):
    packed_case(40, dtype, Hq, Hk, D, [70, 0, 1, 33, 0, 150], causal=causal, pad=3)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("Hq,Hk,D", [(2, 2, 128), (6, 2, 64)])
def test_packed_other_key_lengths(causal, Hq, Hk, D):
    """More keys than tokens (a chunk), fewer (first rows see nothing), none at all."""
    packed_case(41, "bf16", Hq, Hk, D, [5, 100, 64, 90, 1, 0, 33], [300, 40, 64, 0, 513, 20, 1], causal=causal, pad=2)


def test_packed_no_keys():
    packed_case(42, "fp16", 2, 1, 64, [3, 4], [0, 0])
    packed_case(42, "fp16", 2, 1, 128, [3, 4], [0, 0], causal=False)


def test_packed_many_sequences():
    """More than 64, lengths from none to 140, so that the search runs over several batches."""
    lens = [(37 * i) % 141 if i % 5 else 0 for i in range(150)]
    packed_case(43, "fp16", 2, 1, 64, lens, pad=1)


@pytest.mark.parametrize("dtype,std", [("fp16", 3.0), ("bf16", 3.0)])
def test_packed_large_logits(dtype, std):
    packed_case(44, dtype, 2, 1, 128, [300, 160], std=std)


@pytest.mark.parametrize("Hq,Hk,D,lens,keys", [(8, 8, 128, [3], [5000]), (8, 2, 128, [40, 1], [3001, 2500]),
                                               (4, 1, 64, [130], [4100]), (2, 2, 128, [1], [70001])])
def test_packed_few_rows_over_many_keys(Hq, Hk, D, lens, keys):
    """Keys split among work-groups and joined; and the same call without a workspace."""
    assert p4q.attention_prompt_workspace(sum(lens), len(lens), Hq, Hk, D, sum(keys), dev()) is not None
    packed_case(45, "bf16", Hq, Hk, D, lens, keys)
    packed_case(46, "fp16", Hq, Hk, D, lens, keys, causal=False)
    g = gen(47)
    q, k, v = randn(g, "fp16", sum(lens), Hq * D), randn(g, "fp16", sum(keys), Hk * D), randn(g, "fp16", sum(keys), Hk * D)
    args = (q, k, v, cu_of(lens), Hq, Hk, D)
    split = p4q.attention_packed(*args, cu_seqlens_k=cu_of(keys))
    again = p4q.attention_packed(*args, cu_seqlens_k=cu_of(keys))
    whole = p4q.attention_packed(*args, cu_seqlens_k=cu_of(keys), workspace=torch.empty(0, dtype=torch.uint8, device=dev()))
    assert torch.equal(split, again)
    # both within fp16 weights and sums of the same scores
    assert (split.float() - whole.float()).abs().max() <= 2 * 2.0 ** -10 * v.float().abs().max()


def test_packed_sequences_do_not_meet():
    """A sequence's result does not change with its neighbours, NaN among them."""
    Hq, Hk, D, lens = 4, 2, 128, [50, 77, 130]
    g = gen(48)
    qkv = randn(g, "fp16", sum(lens), (Hq + 2 * Hk) * D)
    parts = lambda t: (t[:, :Hq * D], t[:, Hq * D:(Hq + Hk) * D], t[:, (Hq + Hk) * D:])
    ref = p4q.attention_packed(*parts(qkv), cu_of(lens), Hq, Hk)
    for b in range(3):
        bad, at = qkv.clone(), sum(lens[:b])
        bad[at:at + lens[b]] = float("nan")
        out = p4q.attention_packed(*parts(bad), cu_of(lens), Hq, Hk)
        rows = torch.ones(sum(lens), dtype=torch.bool, device=dev())
        rows[at:at + lens[b]] = False
        assert torch.equal(out[rows], ref[rows]) and torch.isnan(out[~rows]).all()


def test_packed_masked_keys_and_values_do_not_leak():
    """Keys past a token's mask: non-finite keys reach no earlier token at all,
    non-finite values none whose mask ends 64 or more keys before them (here, with
    rows and keys aligned, 32)."""
    Hq, Hk, D, n = 2, 1, 128, 200
    g = gen(49)
    q, k, v = randn(g, "bf16", n, Hq * D), randn(g, "bf16", n, D), randn(g, "bf16", n, D)
    ref = p4q.attention_packed(q, k, v, cu_of([n]), Hq, Hk)
    for row in (1, 40, 64, 130, 199):
        k2, v2 = k.clone(), v.clone()
        k2[row], v2[row] = float("nan"), float("inf")
        out = p4q.attention_packed(q, k2, v, cu_of([n]), Hq, Hk)
        assert torch.equal(out[:row], ref[:row]) and torch.isnan(out[row:]).all()
        out = p4q.attention_packed(q, k, v2, cu_of([n]), Hq, Hk)
        assert torch.equal(out[:max(0, row - 32)], ref[:max(0, row - 32)])
        assert not torch.isfinite(out[row:]).any()


@pytest.mark.parametrize("more", [1, 17, 33, 63])
@pytest.mark.parametrize("Hq,Hk", [(1, 1), (2, 1), (3, 1)])
def test_packed_masked_values_do_not_leak_in_a_chunk(Hq, Hk, more):
    """The same where the tokens follow `more` earlier keys, so that the ends of
    masks, rows and tiles fall anywhere."""
    D, n = 64, 150
    g = gen(52)
    q, k, v = randn(g, "fp16", n, Hq * D), randn(g, "fp16", n + more, D), randn(g, "fp16", n + more, D)
    args = (cu_of([n]), Hq, Hk, D)
    ref = p4q.attention_packed(q, k, v, *args, cu_seqlens_k=cu_of([n + more]))
    for j in (more, more + 31, more + 66, n + more - 1):                   # seen from token j - more on
        v2 = v.clone()
        v2[j] = float("nan")
        out = p4q.attention_packed(q, k, v2, *args, cu_seqlens_k=cu_of([n + more]))
        clean = max(0, j - more - 63)
        assert torch.equal(out[:clean], ref[:clean]) and torch.isnan(out[j - more:]).all()


def test_packed_bad_lists_stay_inside():
    """cu_seqlens that do not ascend or leave the rows: nothing outside out is
    written, the process lives."""
    Hq, Hk, D, T = 2, 1, 64, 40
    g = gen(50)
    q, kv = randn(g, "fp16", T, Hq * D), randn(g, "fp16", T, 2 * D)
    for cu in ([0, 30, 10, 40], [-5, 20, 10 ** 9, 2 ** 31 - 1], [40, 0, 40, 0], [0, -2 ** 31, 2 ** 31 - 1, 5]):
        go = Guarded((T, Hq * D), torch.float16, "out")
        p4q.attention_packed(q, kv[:, :D], kv[:, D:], ints(cu), Hq, Hk, D, out=go.t, cu_seqlens_k=ints(cu[::-1]))
        check_canaries(go)


def test_packed_offsets_pass_32_bits():
    """Rows far into a buffer of more than 2^31 elements, strides near 2^24."""
    Hq, Hk, D, n = 2, 1, 128, 150
    ld = (1 << 24) - 8
    g = gen(51)
    q, k, v = randn(g, "fp16", n, Hq * D), randn(g, "fp16", n, D), randn(g, "fp16", n, D)
    ref = p4q.attention_packed(q, k, v, cu_of([n - 9, 9]), Hq, Hk)
    big = torch.full(((n - 1) * ld + 6 * D,), float("nan"), dtype=torch.float16, device=dev())
    rows = big.as_strided((n, 6 * D), (ld, 1))
    rows[:, :2 * D], rows[:, 2 * D:3 * D], rows[:, 3 * D:4 * D] = q, k, v
    p4q.attention_packed(rows[:, :2 * D], rows[:, 2 * D:3 * D], rows[:, 3 * D:4 * D], cu_of([n - 9, 9]), Hq, Hk,
                         out=rows[:, 4 * D:])
    assert torch.equal(rows[:, 4 * D:], ref) and torch.equal(rows[:, :2 * D], q)


def far_scores(dtype, D, scale, sign, rows, keys, Hq, Hk, seed):
    """q [rows, Hq D] all sign 2^a, k [keys, Hk D] in rows of 2^b n with 1 <= n <= 255 and a + b = scale:
    every score is D 2^scale n / sqrt(D), exact in fp32, and two different ones are 700 and more apart in
    units of log 2, so that a row's result is the mean of the values of its largest scores."""
    b = min(8, scale)
    n = np.random.default_rng(seed).integers(1, 256, (keys, Hk))
    k = np.repeat(n[:, :, None] * 2.0 ** b, D, axis=2).reshape(keys, Hk * D)
    q = torch.full((rows, Hq * D), sign * 2.0 ** (scale - b), dtype=DT[dtype], device=dev())
    return q, torch.from_numpy(k).to(dev()).to(DT[dtype]), randn(gen(seed), dtype, keys, Hk * D)


def far_bound(O, A, dtype):
    """Equal weights of the largest scores (rounded once each: eps / 2), fp32 sums, the output's rounding."""
    eps = torch.finfo(DT[dtype]).eps
    inner = (eps / 2 + 2.0 ** -20) * A
    return inner + eps / 2 * (np.abs(O) + inner) + 2.0 ** -25


@pytest.mark.parametrize("dtype,D,scale", [("fp16", 128, 6), ("fp16", 64, 15), ("fp16", 128, 19), ("fp16", 64, 23),
                                           ("bf16", 128, 6), ("bf16", 64, 24), ("bf16", 128, 40), ("bf16", 64, 90)])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("lens,keys", [([150, 40], [150, 70]), ([3], [5000])])
def test_packed_far_scores(dtype, D, scale, sign, lens, keys):
    """Finite scores of any size, whole and split: 2^28 and more in units of log 2 among them, which
    no fp32 product with log2(e) holds to within a weight's range."""
    Hq, Hk = 4, 2
    q, k, v = far_scores(dtype, D, scale, sign, sum(lens), sum(keys), Hq, Hk, 53)
    for causal in (True, False):
        out = f64(p4q.attention_packed(q, k, v, cu_of(lens), Hq, Hk, D, causal, cu_seqlens_k=cu_of(keys))).reshape(-1, Hq, D)
        at = np.concatenate([[0], np.cumsum(lens)]), np.concatenate([[0], np.cumsum(keys)])
        for b in range(len(lens)):
            rows, cols = slice(at[0][b], at[0][b + 1]), slice(at[1][b], at[1][b + 1])
            O, A = oracle.grouped_attention(f64(q)[rows].reshape(-1, Hq, D), f64(k)[cols].reshape(-1, Hk, D),
                                            f64(v)[cols].reshape(-1, Hk, D), causal)
            assert_within(out[rows], O, far_bound(O, A, dtype), f"sequence {b}")


# ------------------------------------------------------------------ prompts over the cache
def paged_case(seed, dtype, Hq, Hk, D, P, lens, key_lens, causal=True, pad=0, width=None):
    g = gen(seed)
    kc, vc, table = make_cache(g, dtype, key_lens, Hk, D, P, width=width)
    T = sum(lens) + pad
    q = randn(g, dtype, T, Hq * D)
    go = Guarded((T, Hq * D), DT[dtype], "out")
    go.t.fill_(7)
    p4q.attention_prefill_paged(q, kc, vc, cu_of(lens), table, ints(key_lens), Hq, causal, out=go.t)
    check_canaries(go)
    assert (go.t[sum(lens):] == 7).all()
    tab, k64, v64 = table.cpu().numpy(), f64(kc), f64(vc)
    check_attention(go.t, q, lambda b: tuple(oracle.cache_rows(c, tab[b], key_lens[b]) for c in (k64, v64)), lens, Hq, D,
                    dtype, causal)


@pytest.mark.parametrize("P", [16, 32, 64, 128, 1024])
@pytest.mark.parametrize("Hq,Hk,D", [(2, 2, 128), (8, 2, 128), (6, 1, 64)])
def test_paged_pages(P, Hq, Hk, D):
    paged_case(60, "fp16", Hq, Hk, D, P, [17, 0, 90, 1, 64], [17, 30, 201, 257, 1000], pad=2)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
def test_paged_masks(dtype, causal):
    """Fewer keys than tokens, none, one."""
    paged_case(61, dtype, 4, 2, 128, 16, [40, 33, 5, 130], [12, 0, 1, 129], causal=causal)


@pytest.mark.parametrize("Hq,Hk,D,lens,keys", [(8, 8, 128, [3], [5000]), (8, 2, 64, [40, 1, 7], [3001, 100, 65])])
def test_paged_few_rows_over_many_keys(Hq, Hk, D, lens, keys):
    paged_case(62, "bf16", Hq, Hk, D, 16, lens, keys)
    paged_case(63, "fp16", Hq, Hk, D, 128, lens, keys, width=4096)          # a table of far more than is used


def test_paged_is_packed():
    """The same keys, packed or paged: the same bits."""
    Hq, Hk, D, P, lens, keys = 4, 2, 128, 16, [100, 7, 64], [150, 30, 64]
    g = gen(64)
    kc, vc, table = make_cache(g, "bf16", keys, Hk, D, P)
    q = randn(g, "bf16", sum(lens), Hq * D)
    flat = [torch.cat([c[table[b, :-(-m // P)].long()].transpose(1, 2).reshape(-1, Hk * D)[:m] for b, m in enumerate(keys)])
            for c in (kc, vc)]
    none = torch.empty(0, dtype=torch.uint8, device=dev())
    a = p4q.attention_packed(q, *flat, cu_of(lens), Hq, Hk, cu_seqlens_k=cu_of(keys), workspace=none)
    b = p4q.attention_prefill_paged(q, kc, vc, cu_of(lens), table, ints(keys), Hq, workspace=none)
    assert torch.equal(a, b)


def test_paged_bad_pages_give_nan_where_they_are_seen():
    """An entry outside the cache, or a length past the table: tokens that see
    such a key are NaN, earlier ones and other sequences are not touched."""
    Hq, Hk, D, P, lens, keys = 2, 1, 128, 16, [100, 50], [100, 50]
    g = gen(65)
    kc, vc, table = make_cache(g, "fp16", keys, Hk, D, P)
    q = randn(g, "fp16", 150, Hq * D)
    ref = p4q.attention_prefill_paged(q, kc, vc, cu_of(lens), table, ints(keys), Hq)
    for col, entry in ((2, -1), (5, kc.shape[0]), (6, 2 ** 31 - 1), (0, -2 ** 31)):
        bad = table.clone()
        bad[0, col] = entry
        out = p4q.attention_prefill_paged(q, kc, vc, cu_of(lens), bad, ints(keys), Hq)
        assert torch.isnan(out[P * col:100]).all() and torch.isfinite(out[:max(0, P * col)]).all()
        assert torch.equal(out[:max(0, P * col - 32)], ref[:max(0, P * col - 32)]) and torch.equal(out[100:], ref[100:])
    over = ints([2 ** 31 - 1, 50])                                          # all see keys past the table
    out = p4q.attention_prefill_paged(q, kc, vc, cu_of(lens), table, over, Hq)
    assert torch.isnan(out[:100]).all() and torch.equal(out[100:], ref[100:])
    out = p4q.attention_prefill_paged(q, kc, vc, cu_of(lens), table, ints([-7, 50]), Hq)
    assert not out[:100].any() and torch.equal(out[100:], ref[100:])


@pytest.mark.parametrize("dtype,Hq,Hk,D,P", [("fp16", 8, 8, 128, 64), ("bf16", 8, 2, 64, 16)])
def test_paged_bad_pages_in_split_keys_give_nan_where_they_are_seen(dtype, Hq, Hk, D, P):
    """The same where the keys of a row tile are split among work-groups and joined: the bad entry in the
    first, a middle and the last of them, a length past the table (every split knows), and the call
    without a workspace."""
    g, lens, keys = gen(66), [70, 5], [5000, 3000]
    width = -(-5000 // P)
    kc, vc, table = make_cache(g, dtype, keys, Hk, D, P, width=width)
    q = randn(g, dtype, 75, Hq * D)
    ws = p4q.attention_prompt_workspace(75, 2, Hq, Hk, D, width * P, dev())
    assert ws is not None
    ws.fill_(255)
    none = torch.empty(0, dtype=torch.uint8, device=dev())
    refs = [p4q.attention_prefill_paged(q, kc, vc, cu_of(lens), table, ints(keys), Hq, workspace=w) for w in (ws, none)]
    assert not (ws == 255).all() and all(torch.isfinite(r).all() for r in refs)          # split, and joined

    def check(tab, have, first):
        """Tokens of sequence 0 see keys [0, have[0] - 69 + i); those that see key `first` are NaN."""
        clean = min(70, max(0, first - (have[0] - 70)))
        for w, ref in zip((ws, none), refs):
            out = p4q.attention_prefill_paged(q, kc, vc, cu_of(lens), tab, ints(have), Hq, workspace=w)
            assert torch.isnan(out[clean:70]).all() and torch.isfinite(out[:clean]).all(), (first, clean)
            assert torch.equal(out[70:], ref[70:])
            if have == keys:                                                             # (64 keys: a tile)
                assert torch.equal(out[:max(0, clean - 64)], ref[:max(0, clean - 64)])

    for key in (0, 63, 64, 2500, 4900, 4950, 4999):
        for entry in (-1, kc.shape[0], -2 ** 31):
            bad = table.clone()
            bad[0, key // P] = entry
            check(bad, keys, key // P * P)
    full = table.clone()                                                                 # every page there
    full[0] = table[0, 0]
    for m in (width * P + 1, width * P + 40, 2 ** 31 - 1):
        check(full, [m, 3000], width * P)


# ------------------------------------------------------------------ decode
def decode_case(seed, dtype, Hq, Hk, D, P, key_lens, max_len=None, width=None, std=1.0):
    g = gen(seed)
    kc, vc, table = make_cache(g, dtype, key_lens, Hk, D, P, width=width)
    B = len(key_lens)
    q = randn(g, dtype, B, Hq * D, std=std)
    go = Guarded((B, Hq * D), DT[dtype], "out")
    p4q.attention_decode(q, kc, vc, table, ints(key_lens), Hq, max_len=max_len, out=go.t)
    check_canaries(go)
    tab, k64, v64 = table.cpu().numpy(), f64(kc), f64(vc)
    check_attention(go.t, q, lambda b: tuple(oracle.cache_rows(c, tab[b], key_lens[b]) for c in (k64, v64)), [1] * B, Hq, D, dtype)
    return q, kc, vc, table, go.t


@pytest.mark.parametrize("P", [16, 32, 64, 256, 4096])
@pytest.mark.parametrize("Hq,Hk,D", [(2, 2, 128), (8, 2, 128), (16, 1, 64), (3, 3, 64)])
def test_decode_lengths(P, Hq, Hk, D):
    """Around the edges of tiles, rounds and chunks; none and one."""
    decode_case(70, "fp16", Hq, Hk, D, P, [0, 1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 256, 257, 600])


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("Hq,Hk,D", [(40, 40, 128), (14, 2, 64), (17, 1, 128), (24, 1, 128), (71, 1, 64), (32, 8, 128)])
def test_decode_heads(dtype, Hq, Hk, D):
    decode_case(71, dtype, Hq, Hk, D, 32, [77, 0, 1000])


@pytest.mark.parametrize("dtype,Hq,Hk,D", [("fp16", 1, 1, 128), ("bf16", 8, 1, 128), ("fp16", 9, 1, 64), ("bf16", 20, 1, 64),
                                           ("fp16", 12, 1, 128)])
def test_decode_split_over_long_keys(dtype, Hq, Hk, D):
    """Many chunks, joined by the last; sequences of one chunk and of none beside them."""
    assert p4q.attention_decode_workspace(3, Hq, Hk, D, 20000, dev()) is not None
    decode_case(72, dtype, Hq, Hk, D, 64, [20000, 100, 0], max_len=20000)
    decode_case(73, dtype, Hq, Hk, D, 16, [9001], width=2048)


@pytest.mark.parametrize("B,Hq,Hk,D,most", [(5, 2, 2, 128, 100), (3, 40, 4, 64, 60), (70, 24, 24, 64, 120), (70, 24, 12, 128, 128),
                                            (200, 16, 16, 64, 1), (130, 5, 5, 64, 33)])
def test_decode_short_keys_shared_unevenly(B, Hq, Hk, D, most):
    """Short sequences of different lengths, fewer and more of them than
    work-groups: their shares begin and end within sequences, and all sums of
    parts stay in the workspace."""
    lens = [(37 * i) % (most + 1) for i in range(B - 1)] + [most]
    g = gen(79)
    kc, vc, table = make_cache(g, "fp16", lens, Hk, D, 16)
    q = randn(g, "fp16", B, Hq * D)
    n = p4q.attention_decode_workspace(B, Hq, Hk, D, most, dev()).numel()
    ws = Guarded((n,), torch.uint8, "workspace")
    ws.t.zero_()
    out = p4q.attention_decode(q, kc, vc, table, ints(lens), Hq, max_len=most, workspace=ws.t)
    ws.check()
    assert not ws.t[:32768].any()
    tab, k64, v64 = table.cpu().numpy(), f64(kc), f64(vc)
    check_attention(out, q, lambda b: tuple(oracle.cache_rows(c, tab[b], lens[b]) for c in (k64, v64)), [1] * B, Hq, D, "fp16")


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_decode_large_logits(dtype):
    decode_case(74, dtype, 4, 1, 128, 16, [500, 3000], std=8.0)


def test_decode_workspace_serves_call_after_call():
    """One workspace for calls of different lengths, its counters zero again
    after each; results do not depend on what it held, nor on the run."""
    Hq, Hk, D = 8, 2, 128
    q, kc, vc, table, _ = decode_case(75, "bf16", Hq, Hk, D, 32, [5000, 300, 4097], max_len=5000)
    ws = p4q.attention_decode_workspace(3, Hq, Hk, D, 5000, dev())
    ws[32768:] = 255
    ref = p4q.attention_decode(q, kc, vc, table, ints([5000, 300, 4097]), Hq, max_len=5000)
    for lens in ([5000, 300, 4097], [700, 0, 4097], [5000, 300, 4097]):
        out = p4q.attention_decode(q, kc, vc, table, ints(lens), Hq, max_len=5000, workspace=ws)
        assert not ws[:32768].any()
    assert torch.equal(out, ref)


def test_decode_bad_pages_and_lengths_give_nan():
    Hq, Hk, D, P = 4, 2, 64, 16
    q, kc, vc, table, ref = decode_case(76, "fp16", Hq, Hk, D, P, [3000, 40, 64], max_len=3000)
    for b, col, entry in ((0, 0, -1), (0, 187, kc.shape[0]), (1, 2, 2 ** 31 - 1), (2, 3, -2 ** 31)):
        bad = table.clone()
        bad[b, col] = entry
        out = p4q.attention_decode(q, kc, vc, bad, ints([3000, 40, 64]), Hq, max_len=3000)
        others = [i for i in range(3) if i != b]
        assert torch.isnan(out[b]).all() and torch.equal(out[others], ref[others])
    out = p4q.attention_decode(q, kc, vc, table, ints([3001, 40, -64]), Hq, max_len=3000)
    assert torch.isnan(out[0]).all() and torch.equal(out[1], ref[1]) and not out[2].any()
    out = p4q.attention_decode(q, kc, vc, table, ints([2 ** 31 - 1, 40, 64]), Hq)
    assert torch.isnan(out[0]).all()
    assert (out[1:].float() - ref[1:].float()).abs().max() <= 2.0 ** -8      # another split of the keys


def test_decode_nonfinite_keys_and_values():
    """A NaN key or an infinite value among the seen ones shows; the queries of
    another key head do not see it."""
    Hq, Hk, D, P = 4, 2, 128, 16
    q, kc, vc, table, ref = decode_case(77, "bf16", Hq, Hk, D, P, [300], max_len=300)
    page = int(table[0, 7])
    k2, v2 = kc.clone(), vc.clone()
    k2[page, 1, 3], v2[page, 0, 3, 5] = float("nan"), float("inf")
    out = p4q.attention_decode(q, k2, vc, table, ints([300]), Hq, max_len=300)
    assert torch.isnan(out[0, 2 * D:]).all() and torch.equal(out[0, :2 * D], ref[0, :2 * D])
    out = p4q.attention_decode(q, kc, v2, table, ints([300]), Hq, max_len=300)
    assert (out[0, [5, D + 5]] == float("inf")).all() and torch.isfinite(out).sum() == Hq * D - 2


@pytest.mark.parametrize("dtype,D,scale", [("fp16", 128, 6), ("fp16", 64, 15), ("fp16", 128, 19), ("fp16", 64, 23),
                                           ("bf16", 128, 6), ("bf16", 64, 24), ("bf16", 128, 40), ("bf16", 64, 90)])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("keys", [[40, 600], [9001]])
def test_decode_far_scores(dtype, D, scale, sign, keys):
    """Finite scores of any size (as test_packed_far_scores), in whole units and in parts."""
    Hq, Hk, P = 4, 2, 64
    kc, vc, table = make_cache(gen(84), dtype, keys, Hk, D, P, fill=0)
    tab, want = table.cpu().numpy(), []
    for b, m in enumerate(keys):
        q, k, v = far_scores(dtype, D, scale, sign, len(keys), m, Hq, Hk, 85 + b)
        for j in range(0, m, P):
            n = min(P, m - j)
            kc[tab[b, j // P], :, :n] = k[j:j + n].view(n, Hk, D).transpose(0, 1)
            vc[tab[b, j // P], :, :n] = v[j:j + n].view(n, Hk, D).transpose(0, 1)
        want.append(oracle.grouped_attention(f64(q)[:1].reshape(1, Hq, D), f64(k).reshape(m, Hk, D), f64(v).reshape(m, Hk, D)))
    out = f64(p4q.attention_decode(q, kc, vc, table, ints(keys), Hq)).reshape(-1, Hq, D)
    for b, (O, A) in enumerate(want):
        assert_within(out[b:b + 1], O, far_bound(O, A, dtype), f"sequence {b}")


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("Hq,Hk,D", [(4, 4, 128), (16, 1, 128), (24, 2, 64)])
def test_decode_weights_are_not_rounded_to_16_bits(dtype, Hq, Hk, D):
    """Flat rows, where one rounding per weight would show: weights in two pieces (the first within 2 eps
    below, the second rounded: eps / 2 of that) are within eps^2 of themselves (fp16: or m 2^-32 max|v| in all); scores, sums and output as in the module's docstring."""
    g, lens, P = gen(90), [7, 33, 100, 180], 16
    kc, vc, table = make_cache(g, dtype, lens, Hk, D, P)
    q = randn(g, dtype, 4, Hq * D, std=0.05)
    out = f64(p4q.attention_decode(q, kc, vc, table, ints(lens), Hq)).reshape(-1, Hq, D)
    tab, k64, v64, q64, eps = table.cpu().numpy(), f64(kc), f64(vc), f64(q).reshape(-1, Hq, D), torch.finfo(DT[dtype]).eps
    for b, m in enumerate(lens):
        k, v = (oracle.cache_rows(c, tab[b], m) for c in (k64, v64))
        O, A = oracle.grouped_attention(q64[b:b + 1], k, v)
        G, norm = Hq // Hk, np.sqrt((q64[b:b + 1] ** 2).sum(-1))
        score = 2 * (D * 2.0 ** -24 * norm * np.repeat(np.sqrt((k ** 2).sum(-1)).max(0), G) / np.sqrt(D) + 2.0 ** -22)
        inner = (eps ** 2 + score[:, :, None] + 2 * m * 2.0 ** -24) * A
        if dtype == "fp16":
            inner = inner + m * 2.0 ** -32 * np.repeat(np.abs(v).max((0, 2)), G)[None, :, None]
        assert_within(out[b:b + 1], O, inner + eps / 2 * (np.abs(O) + inner) + 2.0 ** -25, f"sequence {b}")


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_decode_keys_without_weight_add_nothing(dtype):
    """One key 10^3 and more above all others in units of log 2, whose weights are 0 in fp32: its value row,
    here zeros, is the result, however many others there are."""
    Hq, Hk, D, P, n = 2, 1, 64, 4096, 300000
    pages = -(-n // P)
    kc = torch.ones(pages, Hk, P, D, dtype=DT[dtype], device=dev())
    vc, table = torch.full_like(kc, 9.0), torch.arange(pages, device=dev(), dtype=torch.int32).view(1, -1)
    q = torch.full((1, Hq * D), 64.0, dtype=DT[dtype], device=dev())        # scores 512, and four times as much
    for at in (0, 12345, n - 1):
        k, v = kc.clone(), vc.clone()
        k[at // P, :, at % P], v[at // P, :, at % P] = 4.0, 0.0
        assert not p4q.attention_decode(q, k, v, table, ints([n]), Hq).any()


@pytest.mark.parametrize("dtype,Hq,Hk,D,P,lens", [
    ("bf16", 32, 8, 128, 32, [16000, 16, 700, 0, 1, 9000, 33, 2500, 4097, 120, 64, 11000, 5, 300]),    # shares of parts and whole units
    ("fp16", 64, 8, 128, 256, [40001]),                                                                # one long sequence
    ("fp16", 24, 1, 64, 64, [70000, 0, 12345, 31]),                                                    # two passes over one key head
    ("bf16", 40, 40, 128, 16, [1217, 672, 900, 1100])])
def test_decode_many_long_units(dtype, Hq, Hk, D, P, lens):
    """More than 16 tiles for every compute unit, in units of more than 16 on the mean, which one work-group
    per compute unit shares: units in parts over many work-groups, parts and whole units in one, and
    all of them joined.  Sampled heads against the oracle; nothing around the workspace is written,
    its counters are zero again, and neither what its other bytes hold nor the run shows."""
    cus = torch.cuda.get_device_properties(dev()).multi_processor_count
    heads = Hk * -(-(Hq // Hk) // 16)
    tiles = sum(2 + -(-n // 32) for n in lens) * heads
    assert tiles > 16 * cus and tiles > 16 * len(lens) * heads
    g, B, most = gen(91), len(lens), max(lens)
    kc, vc, table = make_cache(g, dtype, lens, Hk, D, P)
    q = randn(g, dtype, B, Hq * D)
    outs = []
    for fill in (0, 255):
        ws = Guarded((p4q.attention_decode_workspace(B, Hq, Hk, D, most, dev()).numel(),), torch.uint8, "workspace")
        ws.t[:32768], ws.t[32768:] = 0, fill
        out = Guarded((B, Hq * D), DT[dtype], "out")
        p4q.attention_decode(q, kc, vc, table, ints(lens), Hq, max_len=most, out=out.t, workspace=ws.t)
        check_canaries(ws, out)
        assert not ws.t[:32768].any() and not (ws.t[32768:] == fill).all()      # parts have been there
        outs.append(out.t)
    assert torch.equal(*outs)
    got, q64, G = f64(outs[0]).reshape(B, Hq, D), f64(q).reshape(B, Hq, D), Hq // Hk
    for b, m in enumerate(lens):
        pages = table[b, :-(-m // P)].long()
        for hk in {0, Hk // 2, Hk - 1}:
            k, v = (f64(c[pages, hk].reshape(-1, 1, D)[:m]) for c in (kc, vc))
            mine = slice(hk * G, (hk + 1) * G)
            O, A = oracle.grouped_attention(q64[b:b + 1, mine], k, v)
            assert_within(got[b:b + 1, mine], O, attention_bound(q64[b:b + 1, mine], k, v, O, A, dtype), f"sequence {b}, key head {hk}")
    # Every tile once: with q = 0 and value rows that name their tile, O counts them.  Equal weights, sums of
    # whole numbers, one division, one product and the output's rounding.
    for b, m in enumerate(lens):
        at = torch.arange(m, device=dev())
        vc[table[b, at // P].long(), :, at % P] = torch.eye(D, dtype=DT[dtype], device=dev())[at // 32 % D][:, None]
    out = f64(p4q.attention_decode(torch.zeros_like(q), kc, vc, table, ints(lens), Hq, max_len=most)).reshape(B, Hq, D)
    for b, m in enumerate(lens):
        ref = np.bincount(np.arange(m) // 32 % D, minlength=D) / max(1, m)
        assert_within(out[b], np.broadcast_to(ref, (Hq, D)), np.broadcast_to((torch.finfo(DT[dtype]).eps / 2 + 2.0 ** -21) * ref, (Hq, D)),
                      f"sequence {b}, counts")


def test_offsets_in_the_cache_pass_32_bits():
    """A cache of more than 2^31 elements: append to, attend over and decode from
    its last pages."""
    Hq, Hk, D, P = 16, 8, 128, 4096
    pages = 2 ** 31 // (Hk * P * D) + 3
    g = gen(78)
    kc, vc = (torch.empty(pages, Hk, P, D, dtype=torch.bfloat16, device=dev()) for _ in range(2))
    small = [torch.zeros(2, Hk, P, D, dtype=torch.bfloat16, device=dev()) for _ in range(2)]
    n = 100
    table, table2 = ints([[pages - 1, 0]]), ints([[1, 0]])
    qkv = randn(g, "bf16", n, (Hq + 2 * Hk) * D)
    parts = (qkv[:, :Hq * D], qkv[:, Hq * D:(Hq + Hk) * D], qkv[:, (Hq + Hk) * D:])
    q, _ = p4q.rope_append(*parts, cu_of([n]), table, kc, vc, Hq)
    p4q.rope_append(*parts, cu_of([n]), table2, *small, Hq)
    assert torch.equal(kc[-1, :, :n], small[0][1, :, :n]) and torch.equal(vc[-1, :, :n], small[1][1, :, :n])
    for call in (lambda k, v, t: p4q.attention_prefill_paged(q, k, v, cu_of([n]), t, ints([n]), Hq),
                 lambda k, v, t: p4q.attention_decode(q[:1], k, v, t, ints([n]), Hq, max_len=n)):
        assert torch.equal(call(kc, vc, table), call(*small, table2))


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype,Hq,Hk,D,P", [("fp16", 8, 8, 128, 16), ("bf16", 8, 2, 128, 64), ("fp16", 6, 1, 64, 32)])
def test_a_conversation(dtype, Hq, Hk, D, P):
    """Pruned prompts (rotated by their positions in the unpruned ones), a decode
    step for each, a second turn of some, more steps: every output against
    attention over all that was said, in 64 bits, on the rotated rows that the
    first call gave."""
    g = gen(80)
    B, prompt = 3, [70, 129, 33]
    kc, vc, _ = make_cache(g, dtype, [300] * B, Hk, D, P, fill=0)
    kc.fill_(float("nan")), vc.fill_(float("nan"))
    width = -(-300 // P) + 1
    table = torch.randperm(kc.shape[0], generator=g, device=dev())[:B * (width - 1)].to(torch.int32).view(B, -1)
    table = torch.cat([table, ints([[-1]] * B)], 1).contiguous()
    said = [[np.zeros((0, Hk, D))] * 2 for _ in range(B)]
    have, where = [0] * B, [0] * B

    def turn(lens, step):
        T = sum(lens)
        qkv = randn(g, dtype, T, (Hq + 2 * Hk) * D)
        gaps = torch.randint(1, 5, (T,), generator=g, device=dev()).cpu().numpy()
        at, spots = 0, np.zeros(T, np.int64)
        for b, n in enumerate(lens):
            spots[at:at + n] = where[b] + np.cumsum(gaps[at:at + n])
            where[b] = int(spots[at + n - 1]) if n else where[b]
            at += n
        q, k, v = qkv[:, :Hq * D], qkv[:, Hq * D:(Hq + Hk) * D], qkv[:, (Hq + Hk) * D:]
        k_out = torch.empty(T, Hk * D, dtype=DT[dtype], device=dev())
        qr, _ = p4q.rope_append(q, k, v, cu_of(lens), table, kc, vc, Hq, cache_lens=ints(have),
                                positions=ints(spots.tolist()), k_out=k_out)
        k64, v64, at = f64(k_out).reshape(T, Hk, D), f64(v).reshape(T, Hk, D), 0
        for b, n in enumerate(lens):
            said[b] = [np.concatenate([said[b][0], k64[at:at + n]]), np.concatenate([said[b][1], v64[at:at + n]])]
            have[b] += n
            at += n
        outs = []
        if step:
            outs.append(p4q.attention_decode(qr, kc, vc, table, ints(have), Hq))
        if all(have[b] == lens[b] for b in range(B)):
            outs.append(p4q.attention_packed(qr, k_out, v, cu_of(lens), Hq, Hk, D))
        outs.append(p4q.attention_prefill_paged(qr, kc, vc, cu_of(lens), table, ints(have), Hq))
        for out in outs:
            check_attention(out, qr, lambda b: said[b], lens, Hq, D, dtype)

    turn(prompt, False)
    for _ in range(3):
        turn([1] * B, True)
    turn([20, 0, 41], False)
    turn([1] * B, True)


def test_captured_steps():
    """Append and decode captured once and replayed while the lengths grow, with
    eager work and a second graph on its own workspace between the replays."""
    Hq, Hk, D, P, B = 8, 2, 128, 16, 4
    g = gen(81)
    start = [600, 0, 31, 1500]
    kc, vc, _ = make_cache(g, "bf16", [1600] * B, Hk, D, P, fill=0)
    table = torch.arange(B * 100, device=dev(), dtype=torch.int32).view(B, 100).contiguous()
    for c in (kc, vc):
        c.copy_(randn(g, "bf16", *c.shape))
    qkv = torch.empty(B, (Hq + 2 * Hk) * D, dtype=torch.bfloat16, device=dev())
    have, lens, cu = ints(start), ints([n + 1 for n in start]), cu_of([1] * B)
    q_out, out = torch.empty(B, Hq * D, dtype=torch.bfloat16, device=dev()), torch.empty(B, Hq * D, dtype=torch.bfloat16, device=dev())
    parts = (qkv[:, :Hq * D], qkv[:, Hq * D:(Hq + Hk) * D], qkv[:, (Hq + Hk) * D:])

    def step(ws, k, v):
        p4q.rope_append(*parts, cu, table, k, v, Hq, cache_lens=have, q_out=q_out)
        p4q.attention_decode(q_out, k, v, table, lens, Hq, out=out, workspace=ws)

    wss = [p4q.attention_decode_workspace(B, Hq, Hk, D, 1600, dev()) for _ in range(3)]
    qkv.zero_()
    warm = [c.clone() for c in (kc, vc)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(wss[0], *warm)
    torch.cuda.synchronize()
    graphs = []
    for ws in wss[:2]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step(ws, kc, vc)
    kc2, vc2 = kc.clone(), vc.clone()
    for i in range(6):
        qkv.copy_(randn(g, "bf16", *qkv.shape))
        step(wss[2], kc2, vc2)
        eager = out.clone()
        out.zero_()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(kc, kc2), i
        have += 1
        lens += 1


def test_another_stream():
    """Calls go to the current stream: on a side stream they wait for what was
    queued there, and a captured prompt call replays."""
    Hq, Hk, D, lens = 4, 2, 128, [40, 100]
    g = gen(82)
    qkv = randn(g, "fp16", 140, (Hq + 2 * Hk) * D)
    parts = lambda t: (t[:, :Hq * D], t[:, Hq * D:(Hq + Hk) * D], t[:, (Hq + Hk) * D:])
    ref = p4q.attention_packed(*parts(qkv), cu_of(lens), Hq, Hk)
    cu, late = cu_of(lens), torch.zeros_like(qkv)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        big = torch.randn(4096, 4096, device=dev())
        for _ in range(10):
            big = torch.mm(big, big).clamp(-1, 1)
        late.copy_(qkv)
        out = p4q.attention_packed(*parts(late), cu, Hq, Hk)
    side.synchronize()
    assert torch.equal(out, ref)
    graph, got = torch.cuda.CUDAGraph(), torch.empty_like(ref)
    with torch.cuda.graph(graph):
        p4q.attention_packed(*parts(late), cu, Hq, Hk, out=got)
    for _ in range(3):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, ref)


@pytest.mark.parametrize("B", [1, 70])
def test_an_idle_batch(B):
    """No sequence has a token, or a key: padding is left as it was, decode gives zeros."""
    Hq, Hk, D, P, T = 4, 2, 64, 16, 30
    g = gen(92)
    kc, vc, table = make_cache(g, "fp16", [20] * B, Hk, D, P, fill=1.5)
    kc0, vc0 = kc.clone(), vc.clone()
    qkv = randn(g, "fp16", T, (Hq + 2 * Hk) * D)
    q, k, v = qkv[:, :Hq * D], qkv[:, Hq * D:(Hq + Hk) * D], qkv[:, (Hq + Hk) * D:]
    cu, none = cu_of([0] * B), ints([0] * B)
    outs = [torch.full((T, n * D), 7.0, dtype=torch.float16, device=dev()) for n in (Hq, Hk, Hq, Hq)]
    p4q.rope_append(q, k, v, cu, table, kc, vc, Hq, cache_lens=ints([20] * B), q_out=outs[0], k_out=outs[1])
    p4q.attention_packed(q, k, v, cu, Hq, Hk, D, out=outs[2])
    p4q.attention_prefill_paged(q, kc, vc, cu, table, ints([20] * B), Hq, out=outs[3])
    assert all((o == 7).all() for o in outs) and torch.equal(kc, kc0) and torch.equal(vc, vc0)
    out = p4q.attention_decode(randn(g, "fp16", B, Hq * D), kc, vc, table, none, Hq)
    assert not out.any()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_the_largest_group(dtype):
    """1024 query heads on one key head: packed, over the cache, decode."""
    packed_case(93, dtype, 1024, 1, 64, [3, 0, 9, 1], pad=1)
    paged_case(94, dtype, 1024, 1, 64, 16, [2, 1], [40, 300])
    decode_case(95, dtype, 1024, 1, 64, 16, [77, 0, 300])


def test_many_sequences():
    """Batches of thousands, where a sequence is found many steps into the lists."""
    B, Hq, Hk, D, P = 5000, 2, 1, 64, 16
    g = gen(96)
    lens = [(7 * i) % 4 for i in range(B)]
    have = [(5 * i) % 40 for i in range(B)]
    qkv = randn(g, "fp16", sum(lens), (Hq + 2 * Hk) * D)
    q, k, v = qkv[:, :Hq * D], qkv[:, Hq * D:(Hq + Hk) * D], qkv[:, (Hq + Hk) * D:]
    kc, vc, table = make_cache_flat(g, "fp16", B, 3, Hk, D, P)
    q_out, k_out = p4q.rope_append(q, k, v, cu_of(lens), table, kc, vc, Hq, cache_lens=ints(have), k_out=torch.empty(sum(lens), Hk * D, dtype=torch.float16, device=dev()))
    total = [n + m for n, m in zip(lens, have)]
    packed = p4q.attention_packed(q_out, k_out, v, cu_of(lens), Hq, Hk, D)
    paged = p4q.attention_prefill_paged(q_out, kc, vc, cu_of(lens), table, ints(total), Hq)
    ones = randn(g, "fp16", B, Hq * D)
    step = p4q.attention_decode(ones, kc, vc, table, ints(total), Hq)
    ends = np.concatenate([[0], np.cumsum(lens)])
    k64, v64, kc64, vc64 = f64(k_out).reshape(-1, Hk, D), f64(v).reshape(-1, Hk, D), f64(kc), f64(vc)
    tab = table.cpu().numpy()
    for b in [*range(0, B, 97), 63, 64, 65, 4095, 4096, B - 1]:
        r, n = slice(ends[b], ends[b + 1]), lens[b]
        cached = [oracle.cache_rows(c, tab[b], total[b]) for c in (kc64, vc64)]
        assert np.array_equal(cached[0][have[b]:], k64[r]) and np.array_equal(cached[1][have[b]:], v64[r])
        check_attention(packed[r], q_out[r], lambda _: (k64[r], v64[r]), [n], Hq, D, "fp16")
        check_attention(paged[r], q_out[r], lambda _: cached, [n], Hq, D, "fp16")
        check_attention(step[b:b + 1], ones[b:b + 1], lambda _: cached, [1], Hq, D, "fp16")
