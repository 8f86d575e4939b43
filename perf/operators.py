"""The serving path's attention over a paged key-value cache, as cases to measure.

Each case is one call that a serving program makes per decoder layer once the
pruned prompt's q|k|v projections are there:

  append         p4q.rope_append: q and k rotated by their positions, k and v
                 appended to the paged cache
  packed         p4q.attention_packed: attention of whole prompts of different
                 lengths, packed one behind the other
  prefill_paged  p4q.attention_prefill_paged: a further turn's or a chunk's
                 tokens over the keys of the cache
  decode         p4q.attention_decode: one new token per sequence over the cache

run() computes them in plain torch operations in 32 bits, or, with `own`, by
the framework's calls.

The cache holds k and v as [pages, key heads, page size, D]; row b of the block
table lists the pages of sequence b in order.  Lengths are drawn from the
case's own number `mix`, log-uniformly from lo to hi with hi among them, so
that they are part of the case.
"""
from __future__ import annotations

import itertools
import math
import random

import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
# (query heads, key heads, head dimension): 7B, 13B, grouped ones, one shared key head, narrow heads
HEADS = [(32, 32, 128), (40, 40, 128), (32, 8, 128), (64, 8, 128), (28, 4, 128), (24, 1, 128),
         (20, 20, 64), (32, 8, 64), (14, 2, 64)]
MAX_PAIRS = 2.2e9            # padded query-key pairs of a prompt call, all heads
MAX_KEYS = 1.9e8             # padded key values that a call over the cache reads
MAX_ROWS = 1.4e8             # values of an append call, or of a prompt call's rows


def listed():
    return [
        # the decode step of one sequence, 13B layer: launch-bound
        dict(name="append_13b_decode_b1", kind="append", Hq=40, Hk=40, D=128, B=1, lo=1, hi=1,
             past=700, page=16, spots="next", base=10000.0, keep_k=False, pad=0, mix=1, dtype="fp16"),
        # 16 pruned images and their questions, 7B layer; the kept tokens rotate by their positions
        # in the unpruned prompt
        dict(name="append_7b_pruned_b16", kind="append", Hq=32, Hk=32, D=128, B=16, lo=656, hi=704,
             past=0, page=64, spots="pruned", base=10000.0, keep_k=True, pad=0, mix=2, dtype="fp16"),
        # one pruned image with an odd text length, 13B layer
        dict(name="packed_13b_b1", kind="packed", Hq=40, Hk=40, D=128, B=1, lo=371, hi=371, more_lo=0,
             more_hi=0, causal=True, pad=0, mix=3, dtype="bf16"),
        # tiles of a vision tower: 577 tokens each, narrow heads, every token sees every other
        dict(name="packed_tower_b10", kind="packed", Hq=20, Hk=20, D=64, B=10, lo=577, hi=577,
             more_lo=0, more_hi=0, causal=False, pad=0, mix=4, dtype="fp16"),
        # prompts from a few tokens to an unpruned image in one call, grouped heads, a padded batch
        dict(name="packed_ragged_b16", kind="packed", Hq=32, Hk=8, D=128, B=16, lo=9, hi=2003,
             more_lo=0, more_hi=0, causal=True, pad=37, mix=5, dtype="fp16"),
        # one long prompt (several unpruned images), grouped heads
        dict(name="packed_long_b1", kind="packed", Hq=32, Hk=8, D=128, B=1, lo=8191, hi=8191, more_lo=0,
             more_hi=0, causal=True, pad=0, mix=6, dtype="bf16"),
        # the second question about 8 cached pruned images, 7B layer
        dict(name="paged_7b_turn2_b8", kind="prefill_paged", Hq=32, Hk=32, D=128, B=8, lo=17, hi=90,
             past_lo=650, past_hi=1400, causal=True, page=16, pad=0, mix=7, dtype="fp16"),
        # a chunk of a long prompt, grouped heads
        dict(name="paged_chunk_b1", kind="prefill_paged", Hq=32, Hk=8, D=128, B=1, lo=2048, hi=2048,
             past_lo=30001, past_hi=30001, causal=True, page=64, pad=0, mix=8, dtype="bf16"),
        # decode of one sequence, 13B layer: the smallest call
        dict(name="decode_13b_b1", kind="decode", Hq=40, Hk=40, D=128, B=1, lo=371, hi=371, page=16,
             mix=9, dtype="fp16"),
        # decode of 16 pruned images, 7B layer
        dict(name="decode_7b_b16", kind="decode", Hq=32, Hk=32, D=128, B=16, lo=672, hi=1217, page=64,
             mix=10, dtype="bf16"),
        # a serving batch of very different lengths, grouped heads
        dict(name="decode_ragged_b64", kind="decode", Hq=32, Hk=8, D=128, B=64, lo=16, hi=16000, page=32,
             mix=11, dtype="bf16"),
        # one very long sequence, grouped heads
        dict(name="decode_long_b1", kind="decode", Hq=64, Hk=8, D=128, B=1, lo=131071, hi=131071,
             page=256, mix=12, dtype="fp16"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "packed", "packed", "prefill_paged", "decode", "decode"])
    Hq, Hk, D = rng.choice(HEADS)
    case = dict(kind=kind, Hq=Hq, Hk=Hk, D=D, B=_log_int(rng, 1, 64), mix=rng.randint(1, 1 << 30),
                dtype=rng.choice(["fp16", "bf16"]))
    if kind == "append":
        step = rng.random() < 0.4                              # a decode step, or prompts
        hi = 1 if step else _log_int(rng, 1, 8191)
        case.update(lo=1 if step else rng.choice([0, 1, max(1, hi // 4)]), hi=hi,
                    past=rng.choice([0, _log_int(rng, 1, 1000), _log_int(rng, 1, 200000)]),
                    spots=rng.choice(["next", "pruned"]), base=rng.choice([10000.0, 500000.0]),
                    keep_k=not step, pad=rng.choice([0, 0, rng.randint(1, 40)]))
        case["B"] = max(1, min(case["B"], int(MAX_ROWS / ((Hq + 2 * Hk) * D * hi))))
    elif kind == "packed":
        hi = _log_int(rng, 1, 8191)
        case.update(lo=rng.choice([0, 1, max(1, hi // 4), hi]), hi=hi, causal=rng.random() < 0.8,
                    pad=rng.choice([0, 0, rng.randint(1, 300)]))
        # mostly a prompt over itself; also one over more keys than it has tokens, or fewer
        more = rng.choice([0, 0, 0, rng.randint(1, 700), -rng.randint(1, 2 * hi)])
        case.update(more_lo=min(0, more), more_hi=max(0, more))
        case["B"] = max(1, min(case["B"], int(MAX_PAIRS / (Hq * hi * (hi + case["more_hi"])))))
        if Hq * hi * (hi + case["more_hi"]) > MAX_PAIRS:
            case.update(hi=4001, lo=min(case["lo"], 4001))
        # a full square costs twice its causal half
        case["causal"] = case["causal"] or 2 * case["B"] * Hq * case["hi"] ** 2 > MAX_PAIRS
    elif kind == "prefill_paged":
        hi = _log_int(rng, 1, 2048)
        past = min(_log_int(rng, 1, 30001), int(MAX_KEYS / (Hk * D)) - hi)
        case.update(lo=rng.choice([0, 1, hi]), hi=hi, past_lo=rng.choice([0, past]), past_hi=past,
                    causal=rng.random() < 0.9, pad=rng.choice([0, 0, rng.randint(1, 40)]))
        if Hq * hi * (hi + past) > MAX_PAIRS:
            hi = max(1, int(MAX_PAIRS / (Hq * (hi + past))))
            case.update(hi=hi, lo=min(case["lo"], hi))
        case["B"] = max(1, min(case["B"], int(MAX_PAIRS / (Hq * hi * (hi + past))),
                               int(MAX_KEYS / ((hi + past) * Hk * D))))
    else:
        hi = _log_int(rng, 1, 131071)
        case.update(lo=rng.choice([0, 1, max(1, hi // 8), hi]), hi=hi)
        if hi * Hk * D > MAX_KEYS:
            case.update(hi=16001, lo=min(case["lo"], 16001))
        case["B"] = max(1, min(case["B"], int(MAX_KEYS / (case["hi"] * Hk * D))))
    if kind in ("packed", "prefill_paged"):
        case["B"] = max(1, min(case["B"], int(MAX_ROWS / ((Hq + Hk) * D * case["hi"]))))
    if kind != "packed":
        case["page"] = rng.choice([16, 32, 64, 128, 256])
    return case


# --------------------------------------------------------------------------- lengths
def _lens(case):
    """Tokens of each sequence in the call (decode: keys in the cache)."""
    rng = random.Random(case["mix"])
    lo, hi = case["lo"], case["hi"]
    lens = [hi] + [hi if lo == hi else 0 if lo == 0 and rng.random() < 0.2 else _log_int(rng, max(1, lo), hi)
                   for _ in range(case["B"] - 1)]
    rng.shuffle(lens)
    return lens


def _key_lens(case):
    """Keys that each sequence's last token may see."""
    rng = random.Random(case["mix"] + 1)
    lens = _lens(case)
    if case["kind"] == "packed":
        return [max(0, n + rng.randint(case["more_lo"], case["more_hi"])) for n in lens]
    if case["kind"] == "prefill_paged":
        return [n + rng.randint(case["past_lo"], case["past_hi"]) for n in lens]
    if case["kind"] == "append":
        return [n + rng.randint(case["past"] // 2, case["past"]) for n in lens]
    return lens


def _cu(lens):
    return _ints([0, *itertools.accumulate(lens)])


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# --------------------------------------------------------------------------- inputs
def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _rows(g, dt, rows, heads, D, scale):
    """Projected rows: N(0, scale^2) with a few large channels per head, as keys and queries have."""
    x = scale * _randn(g, rows, heads, D)
    x[:, :, torch.randperm(D, generator=g, device="cuda")[:3]] *= 3.0
    return x.to(dt)


def _cache(g, case, dt, key_lens):
    """A cache whose pages are dealt in any order, and the table with two columns to spare."""
    P, Hk, D = case["page"], case["Hk"], case["D"]
    used = [-(-n // P) for n in key_lens]
    pages = sum(used) + 3
    k = _rows(g, dt, pages * P, Hk, D, 1.0).view(pages, P, Hk, D).transpose(1, 2).contiguous()
    v = _randn(g, pages, Hk, P, D).to(dt)
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    width = max(used) + 2
    col = torch.arange(width, device="cuda")
    first, n = _cu(used)[:-1, None], _ints(used)[:, None]
    table = torch.where(col < n, order[(first + col).clamp(max=pages - 1).long()], -1)
    return k, v, table.contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    Hq, Hk, D, kind = case["Hq"], case["Hk"], case["D"], case["kind"]
    lens, key_lens = _lens(case), _key_lens(case)
    st = {"case": case, "most": max(lens), "most_keys": max(key_lens), "tokens": sum(lens),
          "lens": _ints(lens), "key_lens": _ints(key_lens), "cu": _cu(lens)}
    T = sum(lens) + case.get("pad", 0) if kind != "decode" else case["B"]
    if kind == "append":
        qkv = torch.cat([_rows(g, dt, T, Hq + Hk, D, 1.0), _randn(g, T, Hk, D).to(dt)], 1).view(T, -1)
        st.update(q=qkv[:, :Hq * D], k=qkv[:, Hq * D:(Hq + Hk) * D], v=qkv[:, (Hq + Hk) * D:])
        st["k_cache"], st["v_cache"], st["table"] = _cache(g, case, dt, key_lens)
        st["cached"] = st["key_lens"] - st["lens"]
        st["positions"] = None
        if case["spots"] == "pruned":
            # kept tokens of an unpruned prompt: ascending, with gaps
            at = torch.cumsum(torch.randint(1, 9, (T,), generator=g, device="cuda"), 0)
            start = torch.searchsorted(st["cu"][1:], torch.arange(T, device="cuda", dtype=torch.int32),
                                       right=True).clamp(max=case["B"] - 1)
            first = at[st["cu"][:-1].long().clamp(max=T - 1)][start]
            st["positions"] = (at - first + st["cached"][start] + 1).to(torch.int32)
        st["q_out"] = torch.zeros(T, Hq * D, dtype=dt, device="cuda")
        st["k_out"] = torch.zeros(T, Hk * D, dtype=dt, device="cuda") if case["keep_k"] else None
        return st
    # queries a little sharper than keys: attention rows from flat to peaked
    st["q"] = _rows(g, dt, T, Hq, D, 1.0).view(T, Hq * D)
    st["out"] = torch.zeros(T, Hq * D, dtype=dt, device="cuda")
    if kind == "packed":
        keys = sum(key_lens) + case["pad"]
        kv = torch.cat([_rows(g, dt, keys, Hk, D, 1.0), _randn(g, keys, Hk, D).to(dt)], 1).view(keys, -1)
        st.update(k=kv[:, :Hk * D], v=kv[:, Hk * D:], cu_keys=_cu(key_lens))
    else:
        st["k_cache"], st["v_cache"], st["table"] = _cache(g, case, dt, key_lens)
    return st


# --------------------------------------------------------------------------- one pass
def run(st):
    kind = st["case"]["kind"]
    if own:
        return _run_own(st)
    if kind == "append":
        return _plain_append(st)
    if kind == "packed":
        return _plain_packed(st)
    if kind == "prefill_paged":
        return _plain_prefill_paged(st)
    return _plain_decode(st)


def _run_own(st):
    import paper_2609_34867_amd as p4q

    case = st["case"]
    Hq, Hk, D, kind = case["Hq"], case["Hk"], case["D"], case["kind"]
    if kind == "append":
        p4q.rope_append(st["q"], st["k"], st["v"], st["cu"], st["table"], st["k_cache"], st["v_cache"], Hq,
                        cache_lens=st["cached"], positions=st["positions"], rope_base=case["base"],
                        q_out=st["q_out"], k_out=st["k_out"])
        return _append_outputs(st)
    if kind == "packed":
        return p4q.attention_packed(st["q"], st["k"], st["v"], st["cu"], Hq, Hk, D=D, causal=case["causal"],
                                    cu_seqlens_k=st["cu_keys"], out=st["out"])
    if kind == "prefill_paged":
        return p4q.attention_prefill_paged(st["q"], st["k_cache"], st["v_cache"], st["cu"], st["table"],
                                           st["key_lens"], Hq, causal=case["causal"], out=st["out"])
    if "workspace" not in st:                # a program makes it once
        st["workspace"] = p4q.attention_decode_workspace(case["B"], Hq, Hk, D, st["most_keys"], st["q"].device)
    return p4q.attention_decode(st["q"], st["k_cache"], st["v_cache"], st["table"], st["key_lens"], Hq,
                                max_len=st["most_keys"], out=st["out"], workspace=st["workspace"])


def _append_outputs(st):
    out = {"q": st["q_out"], "k_cache": st["k_cache"], "v_cache": st["v_cache"]}
    if st["k_out"] is not None:
        out["k"] = st["k_out"]
    return out


def _tokens(st):
    """(sequence, place in it) of each token of the call."""
    n = torch.arange(st["tokens"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(st["cu"][1:], n, right=True)
    return seq, n - st["cu"][seq]


def _plain_append(st):
    case = st["case"]
    Hq, Hk, D, P, T = case["Hq"], case["Hk"], case["D"], case["page"], st["tokens"]
    seq, i = _tokens(st)
    slot = (st["cached"][seq] + i).long()
    at = slot if st["positions"] is None else st["positions"][:T]
    theta = case["base"] ** (-2.0 * torch.arange(D // 2, device="cuda", dtype=torch.float64) / D)
    angle = at.double()[:, None] * theta                       # far positions: in 64 bits
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def rotate(x, heads):
        a, b = x[:T].view(T, heads, 2, D // 2).float().unbind(2)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(x.dtype)

    q, k = rotate(st["q"], Hq), rotate(st["k"], Hk)
    st["q_out"][:T] = q.view(T, Hq * D)
    if st["k_out"] is not None:
        st["k_out"][:T] = k.view(T, Hk * D)
    page = st["table"][seq, slot // P].long()
    st["k_cache"][page, :, slot % P] = k
    st["v_cache"][page, :, slot % P] = st["v"][:T].view(T, Hk, D)
    return _append_outputs(st)


def _attend(q, k, v, q_lens, k_lens, causal):
    """softmax(q k^T / sqrt(D)) v in 32 bits, sequences padded to one length: q [B, Hk, G, Lq, D],
    k and v [B, Hk, Lk, D].  With `causal`, a sequence's last token sees its last key.  Rows that see
    nothing are zero."""
    B, Hk, G, Lq, D = q.shape
    Lk = k.shape[2]
    i = torch.arange(Lq, device="cuda")[:, None]
    j = torch.arange(Lk, device="cuda")
    seen = j < k_lens[:, None, None]
    if causal:
        seen = seen & (j <= i + (k_lens - q_lens)[:, None, None])
    s = torch.matmul(q.reshape(B, Hk, G * Lq, D) * D ** -0.5, k.transpose(2, 3).contiguous())
    s = s.view(B, Hk, G, Lq, Lk).masked_fill_(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).min)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hk, G * Lq, Lk), v).view(B, Hk, G, Lq, D)
    return o / total.masked_fill(total == 0, 1.0)


def _padded(x, cu, lens, most, heads, D):
    """[rows, heads * D] packed -> [B, heads, most, D] in 32 bits; rows past a length are any row's."""
    at = cu[:-1, None] + torch.minimum(torch.arange(most, device="cuda", dtype=torch.int32),
                                       (lens[:, None] - 1).clamp(min=0))
    at = at.clamp(max=max(0, x.shape[0] - 1)).long()
    return x[at].float().view(len(lens), most, heads, D).transpose(1, 2)


def _queries(st):
    case = st["case"]
    Hq, Hk, D = case["Hq"], case["Hk"], case["D"]
    q = _padded(st["q"], st["cu"], st["lens"], st["most"], Hq, D)
    return q.reshape(case["B"], Hk, Hq // Hk, st["most"], D)


def _store(st, o):
    """[B, Hk, G, most, D] -> the packed rows of `out`; rows behind the last sequence stay."""
    case = st["case"]
    seq, i = _tokens(st)
    o = o.to(st["out"].dtype).reshape(case["B"], case["Hq"], st["most"], case["D"])
    st["out"][:st["tokens"]] = o[seq, :, i].reshape(st["tokens"], -1)
    return st["out"]


def _cached(cache, table, most):
    """The first `most` keys of every sequence, in 32 bits: [B, Hk, most, D]."""
    P, Hk, D = cache.shape[2], cache.shape[1], cache.shape[3]
    n = -(-most // P)
    x = cache[table[:, :n].clamp(min=0).long()].transpose(1, 2)
    return x.reshape(table.shape[0], Hk, n * P, D)[:, :, :most].float()


def _plain_packed(st):
    case = st["case"]
    if st["most_keys"] == 0:
        return st["out"]
    k, v = (_padded(st[x], st["cu_keys"], st["key_lens"], st["most_keys"], case["Hk"], case["D"]) for x in "kv")
    return _store(st, _attend(_queries(st), k, v, st["lens"], st["key_lens"], case["causal"]))


def _plain_prefill_paged(st):
    case = st["case"]
    k, v = (_cached(st[x], st["table"], st["most_keys"]) for x in ("k_cache", "v_cache"))
    return _store(st, _attend(_queries(st), k, v, st["lens"], st["key_lens"], case["causal"]))


def _plain_decode(st):
    case = st["case"]
    B, Hq, Hk, D = case["B"], case["Hq"], case["Hk"], case["D"]
    k, v = (_cached(st[x], st["table"], st["most_keys"]) for x in ("k_cache", "v_cache"))
    q = st["q"].float().view(B, Hk, Hq // Hk, 1, D)
    o = _attend(q, k, v, torch.ones_like(st["key_lens"]), st["key_lens"], False)
    st["out"].copy_(o.view(B, Hq * D))
    return st["out"]


# --------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    lens, key_lens = _lens(case), _key_lens(case)
    if case["kind"] == "append":
        return _exact_append(st, lens, key_lens)
    Hq, Hk, D = case["Hq"], case["Hk"], case["D"]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    if case["kind"] == "decode":
        lens = [1] * case["B"]
    row = key_row = 0
    for b, (n, m) in enumerate(zip(lens, key_lens)):
        if n and m:
            if case["kind"] == "packed":
                k, v = (st[x][key_row:key_row + m].reshape(m, Hk, D).double() for x in "kv")
            else:
                pages = st["table"][b, :-(-m // case["page"])].long()
                k, v = (st[x].transpose(1, 2)[pages].reshape(-1, Hk, D)[:m].double()
                        for x in ("k_cache", "v_cache"))
            last = torch.arange(n, device="cuda") + (m - n if case.get("causal", True) else m)
            hidden = torch.arange(m, device="cuda") > last[:, None]
            for h in range(Hq):
                c = h * D
                z = st["q"][row:row + n, c:c + D].double() @ k[:, h * Hk // Hq].T / math.sqrt(D)
                z[hidden] = -math.inf
                w = torch.exp(z - torch.logsumexp(z, 1, keepdim=True))
                w[last < 0] = 0.0
                out[row:row + n, c:c + D] = w @ v[:, h * Hk // Hq]
                del z, w
        row += n
        key_row += m
    return out


def _exact_append(st, lens, key_lens):
    case = st["case"]
    Hq, Hk, D, P = case["Hq"], case["Hk"], case["D"], case["page"]
    q_out, k_cache, v_cache = (st[x].double() for x in ("q_out", "k_cache", "v_cache"))
    k_out = torch.zeros(st["k"].shape, dtype=torch.float64, device="cuda")
    turn = torch.exp(torch.arange(D // 2, device="cuda", dtype=torch.float64) * (-2.0 / D * math.log(case["base"])))
    row = 0
    for b, (n, m) in enumerate(zip(lens, key_lens)):
        if n:
            slots = torch.arange(m - n, m, device="cuda")
            at = slots if st["positions"] is None else st["positions"][row:row + n]
            spin = torch.polar(torch.ones_like(turn), turn * at.double()[:, None])[:, None]   # e^(i p theta)
            for x, y, heads in ((st["q"], q_out, Hq), (st["k"], k_out, Hk)):
                a, c = x[row:row + n].reshape(n, heads, D).double().chunk(2, -1)
                z = torch.complex(a, c) * spin
                y[row:row + n] = torch.cat([z.real, z.imag], -1).reshape(n, heads * D)
            page = st["table"][b].long()[slots // P]
            k_cache[page, :, slots % P] = k_out[row:row + n].reshape(n, Hk, D)
            v_cache[page, :, slots % P] = st["v"][row:row + n].reshape(n, Hk, D).double()
            row += n
    out = {"q": q_out, "k_cache": k_cache, "v_cache": v_cache}
    if case["keep_k"]:
        out["k"] = k_out
    return out


# --------------------------------------------------------------------------- cost
def work(case):
    Hq, Hk, D, kind = case["Hq"], case["Hk"], case["D"], case["kind"]
    lens, key_lens = _lens(case), _key_lens(case)
    T = sum(lens)
    if kind == "append":
        values = T * (2 * Hq + 4 * Hk + (Hk if case["keep_k"] else 0)) * D
        return {"bytes": 2 * values + 8 * T, "flops": 3 * T * (Hq + Hk) * D}
    if kind == "decode":
        pairs, rows = sum(key_lens), case["B"]
    else:
        pairs, rows = 0, T
        for n, m in zip(lens, key_lens):
            if case["causal"]:
                first = max(0, n - m)                         # rows before it see nothing
                pairs += (m - n + first + 1 + m) * (n - first) // 2
            else:
                pairs += n * m
    return {"bytes": 2 * D * (2 * Hq * rows + 2 * Hk * sum(key_lens)) + 4 * sum(key_lens) // case.get("page", 64),
            "flops": 4 * D * Hq * pairs}
