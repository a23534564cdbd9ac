"""Rotated and normed keys into the paged cache, and attention over it with shaped scores: what they are measured on.

The paged cache of grouped-query attention holds a key and a value row per token and kv head, in pages of 16
tokens, as bf16 or as e4m3 bytes with a scale per page and head. Three operators work on it:

``append``   a step's queries, keys and values as the projection leaves them: root-mean-square norm of each query
             and key head, rotation by the token's position (or by several positions: time, height, width), queries
             to an array, keys and values into their slots
``prefill``  attention of packed ragged prompts, or chunks of prompts behind a context, over the paged cache
``decode``   attention of one token per sequence over the paged cache

Both attentions shape the scores: a cap by tanh, a bias that grows with distance, a window, documents (a token sees
nothing before its document's start) and, for prompts, a prefix that every token sees.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
POOL = 1.25          # physical pages per page needed, as a server keeps some free
TABLE = 140000       # positions that the table of cosines and sines covers
THETA = 500000.0
EPS = 1e-6


def listed():
    """A case's lengths are drawn from ``lens_seed``: ``lo..hi`` new tokens behind ``ctx_lo..ctx_hi`` earlier ones."""
    return [
        # the decode step's rows, one per request: latency
        dict(name="append_decode", op="append", batch=64, lo=1, hi=1, ctx_lo=500, ctx_hi=4000, q_heads=32, kv_heads=8, dim=128,
             rot=128, pairs=False, norm=True, axes=1, fp8=False, lens_seed=1),
        # a batch of prompts: bytes
        dict(name="append_prompts", op="append", batch=24, lo=30, hi=1400, ctx_lo=0, ctx_hi=0, q_heads=32, kv_heads=8, dim=128,
             rot=128, pairs=False, norm=True, axes=1, fp8=False, lens_seed=2),
        # images among text, positions of three axes, into a quantised cache
        dict(name="append_axes", op="append", batch=7, lo=200, hi=1300, ctx_lo=0, ctx_hi=900, q_heads=28, kv_heads=4, dim=128,
             rot=128, pairs=False, norm=False, axes=3, fp8=True, lens_seed=3),
        # short ragged prompts together, capped scores
        dict(name="prefill_short", op="prefill", batch=24, lo=1, hi=700, ctx_lo=0, ctx_hi=0, q_heads=32, kv_heads=8, dim=128,
             cap=50.0, slopes=False, window=0, docs=0, prefix=False, fp8=False, lens_seed=4),
        # one long prompt, capped scores: tensor work
        dict(name="prefill_prompt", op="prefill", batch=1, lo=8192, hi=8192, ctx_lo=0, ctx_hi=0, q_heads=32, kv_heads=8, dim=128,
             cap=50.0, slopes=False, window=0, docs=0, prefix=False, fp8=False, lens_seed=5),
        # prompts of a model without rotation: a bias by distance, a kv head for each query head
        dict(name="prefill_distance", op="prefill", batch=4, lo=1500, hi=2900, ctx_lo=0, ctx_hi=0, q_heads=32, kv_heads=32, dim=128,
             cap=0.0, slopes=True, window=0, docs=0, prefix=False, fp8=False, lens_seed=6),
        # one chunk of a prompt behind a long context: few rows, many keys
        dict(name="prefill_chunk", op="prefill", batch=1, lo=300, hi=300, ctx_lo=60000, ctx_hi=60000, q_heads=32, kv_heads=8, dim=128,
             cap=0.0, slopes=False, window=0, docs=0, prefix=False, fp8=False, lens_seed=7),
        # several documents in a row of tokens, a prefix seen by all, small heads
        dict(name="prefill_documents", op="prefill", batch=6, lo=700, hi=4000, ctx_lo=0, ctx_hi=0, q_heads=14, kv_heads=2, dim=64,
             cap=0.0, slopes=False, window=0, docs=300, prefix=True, fp8=False, lens_seed=8),
        # chunks behind contexts in a quantised cache, capped scores in a window
        dict(name="prefill_fp8", op="prefill", batch=8, lo=400, hi=1000, ctx_lo=1000, ctx_hi=8000, q_heads=32, kv_heads=8, dim=128,
             cap=30.0, slopes=False, window=4096, docs=0, prefix=False, fp8=True, lens_seed=9),
        # a single short request, capped scores: latency
        dict(name="decode_one", op="decode", batch=1, lo=1, hi=1, ctx_lo=516, ctx_hi=516, q_heads=32, kv_heads=8, dim=128, cap=50.0,
             slopes=False, window=0, docs=0, fp8=False, lens_seed=10),
        # a decode batch, capped scores: the cache's bytes
        dict(name="decode_batch", op="decode", batch=64, lo=1, hi=1, ctx_lo=511, ctx_hi=4095, q_heads=32, kv_heads=8, dim=128, cap=50.0,
             slopes=False, window=0, docs=0, fp8=False, lens_seed=11),
        # long contexts in a quantised cache, a bias by distance: the split over the tokens
        dict(name="decode_long", op="decode", batch=8, lo=1, hi=1, ctx_lo=32767, ctx_hi=131071, q_heads=32, kv_heads=8, dim=128, cap=0.0,
             slopes=True, window=0, docs=0, fp8=True, lens_seed=12),
    ]


def draw(rng):
    """One more case of the same ranges."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["append", "append", "prefill", "prefill", "prefill", "decode", "decode"])
    seed = rng.randrange(1 << 30)
    fp8 = rng.random() < 0.3
    heads = rng.choice([(32, 8), (32, 8), (64, 8), (28, 4), (16, 16), (24, 8), (8, 1), (40, 8)])
    dim = 128 if fp8 else rng.choice([128, 128, 64])
    if op == "append":
        hi = log(1, 1400)
        rot = rng.choice([dim, dim, dim // 2])
        case = dict(op=op, batch=max(1, min(log(1, 200), 16000 // hi)), lo=max(1, hi // rng.choice([1, 3, 50])), hi=hi,
                    ctx_lo=0, ctx_hi=rng.choice([0, 1]) * log(16, 30000), rot=rot, pairs=rng.random() < 0.3, norm=rng.random() < 0.6,
                    axes=rng.choice([1, 1, 3]))
    else:
        cap = rng.choice([0.0, 20.0, 50.0])
        case = dict(op=op, cap=cap, slopes=rng.random() < 0.3, window=rng.choice([0, 0, 128, 1000, 4096]), docs=rng.choice([0, 0, 200]))
        if op == "decode":
            hi = log(16, 60000)
            dim = 128 if fp8 else rng.choice([dim, dim, 256])
            case.update(batch=max(1, min(log(1, 200), int(6.0e5 / hi))), lo=1, hi=1, ctx_lo=max(0, hi // rng.choice([1, 2, 8]) - 1), ctx_hi=hi - 1)
        else:
            hi, ctx = log(1, 4000), rng.choice([0, 0, 1]) * log(32, 16000)
            batch = max(1, min(log(1, 24), int(1.0e9 / (heads[0] * hi * (hi / 2 + ctx))), int(5.0e5 / (heads[1] * (hi + ctx) / 4))))
            case.update(batch=batch, lo=max(1, hi // rng.choice([1, 3, 50])), hi=hi, ctx_lo=ctx // 2, ctx_hi=ctx, prefix=rng.random() < 0.2)
    return dict(case, q_heads=heads[0], kv_heads=heads[1], dim=dim, fp8=fp8, lens_seed=seed)


# ---- what a case's numbers say (functions of the case alone) ---------------------------------------

def _lens(case):
    """Per sequence (length after the step, tokens of the step)."""
    g = np.random.default_rng(case["lens_seed"])
    new = g.integers(case["lo"], case["hi"], size=case["batch"], endpoint=True)
    return new + g.integers(case["ctx_lo"], case["ctx_hi"], size=case["batch"], endpoint=True), new


def _masks(case):
    """(first visible key of each of the step's tokens or None, prefix lengths or None)."""
    L, n = _lens(case)
    g = np.random.default_rng(case["lens_seed"] + 1)
    first = prefix = None
    if case["docs"]:        # documents of about that many tokens, one behind the other in each sequence
        parts = []
        for b in range(len(L)):
            starts = np.cumsum(g.integers(1, 2 * case["docs"], size=int(L[b]) // case["docs"] * 2 + 4))
            starts = np.concatenate([[0], starts[starts < L[b]]])
            pos = np.arange(L[b] - n[b], L[b])
            parts.append(starts[np.searchsorted(starts, pos, side="right") - 1])
        first = np.concatenate(parts)
    if case.get("prefix"):
        prefix = np.minimum(g.integers(0, np.maximum(L // 2, 1), endpoint=True), L)
    return first, prefix


def _ranges(case):
    """Per sequence, the arrays (lo, hi) of the keys that its tokens see: lo <= j < hi."""
    L, n = _lens(case)
    first, prefix = _masks(case)
    out, at = [], 0
    for b in range(len(L)):
        p = np.arange(L[b] - n[b], L[b])
        lo, hi = np.zeros_like(p), p + 1
        if prefix is not None:
            hi = np.maximum(hi, prefix[b])
        if case["window"]:
            lo = np.maximum(lo, p - case["window"] + 1)
        if first is not None:
            lo = np.maximum(lo, first[at:at + n[b]])
        at += n[b]
        out.append((lo, hi))
    return out


def _slopes(heads):
    return [2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)]


# ---- inputs ---------------------------------------------------------------------------------------

def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _pages(L, rng):
    need = -(-L // PAGE)
    pool = int(math.ceil(POOL * need.sum())) + 1
    perm = rng.permutation(pool).astype(np.int32)
    table = np.full((len(L), int(need.max())), -1, dtype=np.int32)
    at = 0
    for b in range(len(L)):
        table[b, :need[b]] = perm[at:at + need[b]]
        at += need[b]
    return table, pool


def _cache(case, gen, pool, table, L):
    """A cache whose tokens are random and whose other slots hold NaN: (cache, scales or None)."""
    shape = (pool, case["kv_heads"], PAGE, case["dim"])
    cache = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    for i in range(0, pool, 4096):
        cache[i:i + 4096] = _randn(gen, *cache[i:i + 4096].shape)
    live = np.zeros((pool, PAGE), dtype=bool)
    for b in range(len(L)):
        need = -(-int(L[b]) // PAGE)
        live[table[b, :need]] = True
        live[table[b, need - 1], (int(L[b]) - 1) % PAGE + 1:] = False
    dead = torch.from_numpy(~live).cuda()[:, None, :, None]
    if not case["fp8"]:
        return cache.masked_fill_(dead, float("nan")), None
    scale = cache.abs().amax(dim=(2, 3)).float() / 448.0
    out = torch.empty(shape, dtype=torch.float8_e4m3fn, device="cuda")
    for i in range(0, pool, 4096):
        out[i:i + 4096] = (cache[i:i + 4096].float() / scale[i:i + 4096, :, None, None]).to(torch.float8_e4m3fn)
    out.view(torch.uint8).masked_fill_(dead, 0xFF)
    return out, scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    st = dict(case=case)
    if own:
        from paper_2605_06068_b200 import binding
        st["pda"] = binding
    L, n = _lens(case)
    Hq, Hkv, D, B, T = case["q_heads"], case["kv_heads"], case["dim"], case["batch"], int(n.sum())
    table, pool = _pages(L, rng)

    if case["op"] == "append":
        rot = case["rot"]
        qkv = _randn(gen, T, Hq + 2 * Hkv, D)       # the projection's output; its parts are strided views
        qkv *= torch.rand((T, Hq + 2 * Hkv, 1), generator=gen, device="cuda") * 3 + 0.1
        pos = np.concatenate([np.arange(L[b] - n[b], L[b]) for b in range(B)])
        slots = np.concatenate([table[b, p // PAGE] * PAGE + p % PAGE for b in range(B) for p in [np.arange(L[b] - n[b], L[b])]])
        half = rot // 2
        if case["axes"] == 3:                       # an image of 32 columns after 64 tokens of text, and so on
            image = pos % 512 >= 64
            row = (pos % 512 - 64) // 32
            pos = np.stack([pos, np.where(image, pos - pos % 512 + 64 + row, pos), np.where(image, pos - pos % 512 + 64 + pos % 32, pos)])
            parts = [half // 4, (half - half // 4) // 2]
            axis = [0] * parts[0] + [1] * parts[1] + [2] * (half - sum(parts))
        else:
            axis = [0] * half
        angle = torch.arange(TABLE, dtype=torch.float64, device="cuda")[:, None] * THETA ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        cos_sin = torch.cat([angle.cos(), angle.sin()], dim=1).float()
        if case["fp8"]:
            bytes_ = torch.randint(0, 64, (2, pool, Hkv, PAGE, D), generator=gen, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn)
            k_cache, v_cache = bytes_[0].clone(), bytes_[1].clone()
            k_scale, v_scale = (torch.rand((2, pool, Hkv), generator=gen, device="cuda") * 0.01 + 0.02).unbind(0)
            st.update(k_scale0=k_scale.contiguous(), v_scale0=v_scale.contiguous(), k_scale=k_scale.clone(), v_scale=v_scale.clone())
        else:
            k_cache, v_cache = _randn(gen, pool, Hkv, PAGE, D), _randn(gen, pool, Hkv, PAGE, D)
        norms = [_randn(gen, D) * 0.2 + 1 if case["norm"] else None for _ in range(2)]
        st.update(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:], positions=_ints(pos), axis=axis, cos_sin=cos_sin,
                  slots=_ints(slots), k_cache=k_cache, v_cache=v_cache, q_norm=norms[0], k_norm=norms[1],
                  out=torch.zeros((T, Hq, D), dtype=torch.bfloat16, device="cuda"))
        return st

    k_cache, k_scale = _cache(case, gen, pool, table, L)
    v_cache, v_scale = _cache(case, gen, pool, table, L)
    first, prefix = _masks(case)
    q = _randn(gen, T, Hq, D) * 4                  # scores of +-15, as trained heads have them
    st.update(q=q, k_cache=k_cache, v_cache=v_cache, k_scale=k_scale, v_scale=v_scale, table=_ints(table), seq_lens=_ints(L),
              lens=[int(x) for x in L], new=[int(x) for x in n], max_q=int(n.max()), scale=1.0 / math.sqrt(D),
              cu_q=_ints(np.concatenate([[0], np.cumsum(n)])), first=None if first is None else _ints(first),
              prefix=None if prefix is None else _ints(prefix), slopes=torch.tensor(_slopes(Hq), device="cuda") if case["slopes"] else None,
              lo_hi=[(_ints(lo), _ints(hi)) for lo, hi in _ranges(case)], out=torch.zeros((T, Hq, D), dtype=torch.bfloat16, device="cuda"))
    if own and case["op"] == "prefill":
        st["workspace"] = st["pda"].prefill_workspace(Hq, D)
    if own and case["op"] == "decode":
        # few units: their tokens are cut so that there are about four for each of the 148 SMs; none shorter than 64 tokens
        units, longest = B * Hkv, int(L.max())
        chunk = 0
        if units < 2 * 148:
            chunk = max(64, -(-longest * units // (4 * 148)) // 64 * 64)
            chunk = 0 if chunk >= longest else chunk
        st.update(chunk=chunk, part_o=None, part_lse=None, counters=None)
        if chunk:
            c = st["pda"].max_chunks(longest, chunk)
            st.update(part_o=torch.empty((B, Hq, c, D), device="cuda"), part_lse=torch.empty((B, Hq, c), device="cuda"),
                      counters=st["pda"].new_workspace(B, Hkv))
    return st


def run(st):
    return globals()[("_own_" if own else "_plain_") + st["case"]["op"]](st)


# ---- the framework's calls ------------------------------------------------------------------------

def _own_append(st):
    case = st["case"]
    st["pda"].rope_kv_append(st["q"], st["k"], st["v"], st["positions"], st["cos_sin"], st["k_cache"], st["v_cache"], st["slots"],
                             q_norm=st["q_norm"], k_norm=st["k_norm"], eps=EPS, interleaved=case["pairs"],
                             freq_axis=st["axis"] if case["axes"] > 1 else None, out=st["out"], k_scale=st.get("k_scale"),
                             v_scale=st.get("v_scale"))
    return _append_outputs(st)


def _own_prefill(st):
    case = st["case"]
    return st["pda"].paged_prefill_attention(st["q"], st["k_cache"], st["v_cache"], st["table"], st["seq_lens"], st["cu_q"], st["max_q"],
                                             st["scale"], softcap=case["cap"], slopes=st["slopes"], window=case["window"],
                                             prefix_lens=st["prefix"], first_keys=st["first"], out=st["out"], k_scale=st["k_scale"],
                                             v_scale=st["v_scale"], workspace=st["workspace"])


def _own_decode(st):
    case = st["case"]
    return st["pda"].paged_biased_decode_attention(st["q"], st["k_cache"], st["v_cache"], st["table"], st["seq_lens"], st["scale"],
                                                   softcap=case["cap"], slopes=st["slopes"], window=case["window"], first_keys=st["first"],
                                                   chunk_tokens=st["chunk"], out=st["out"], part_o=st["part_o"], part_lse=st["part_lse"],
                                                   workspace=st["counters"], k_scale=st["k_scale"], v_scale=st["v_scale"])


# ---- plain forms ----------------------------------------------------------------------------------

def _append_outputs(st):
    scales = (st["k_scale"], st["v_scale"]) if st["case"]["fp8"] else ()
    return (st["out"], st["k_cache"], st["v_cache"]) + scales


def _plain_rotated(x, weight, cos, sin, case):
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * weight.float()
    rot = case["rot"]
    c, s = cos[:, None, :], sin[:, None, :]
    if case["pairs"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    return torch.cat([y, x[..., rot:]], dim=-1)


def _plain_append(st):
    case = st["case"]
    half = case["rot"] // 2
    pos = st["positions"].long()
    if case["axes"] > 1:
        pos = pos[torch.tensor(st["axis"], device="cuda")].T               # [T, half]
        col = torch.arange(half, device="cuda")[None, :]
        cos, sin = st["cos_sin"][pos, col], st["cos_sin"][pos, half + col]
    else:
        cos, sin = st["cos_sin"][pos, :half], st["cos_sin"][pos, half:]
    st["out"].copy_(_plain_rotated(st["q"], st["q_norm"], cos, sin, case))
    k, v = _plain_rotated(st["k"], st["k_norm"], cos, sin, case), st["v"]
    slots = st["slots"].long()
    page, slot = slots // PAGE, slots % PAGE
    if not case["fp8"]:
        st["k_cache"][page, :, slot] = k.to(torch.bfloat16)
        st["v_cache"][page, :, slot] = v
        return _append_outputs(st)
    opening = slot == 0                       # a page's scale is that of its first row
    for rows, cache, before, scale in ((k, st["k_cache"], st["k_scale0"], st["k_scale"]), (v.float(), st["v_cache"], st["v_scale0"], st["v_scale"])):
        top = rows[opening].abs().amax(dim=-1)
        scale.copy_(before)
        scale[page[opening]] = torch.where(top > 0, top * 2 / 448, 1.0)
        cache[page, :, slot] = (rows / scale[page][:, :, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
    return _append_outputs(st)


def _plain_rows(st, b, g, which):
    """Keys or values of sequence b and kv head g, in 32 bits."""
    L = st["lens"][b]
    pages = st["table"][b, :(L + PAGE - 1) // PAGE].long()
    rows = st[which + "_cache"][pages, g].float()
    if st["case"]["fp8"]:
        rows = rows * st[which + "_scale"][pages, g][:, None, None]
    return rows.flatten(0, 1)[:L]


def _plain_attention(st):
    case = st["case"]
    G = case["q_heads"] // case["kv_heads"]
    at = 0
    for b, (L, n) in enumerate(zip(st["lens"], st["new"])):
        j = torch.arange(L, device="cuda")
        lo, hi = st["lo_hi"][b]
        hidden = (j < lo[:, None]) | (j >= hi[:, None])                      # [n, L]
        distance = (torch.arange(L - n, L, device="cuda")[:, None] - j).abs() if case["slopes"] else None
        for g in range(case["kv_heads"]):
            q = st["q"][at:at + n, g * G:(g + 1) * G].float()
            s = (q.flatten(0, 1) @ _plain_rows(st, b, g, "k").T).view(n, G, L) * st["scale"]
            if case["cap"]:
                s = case["cap"] * torch.tanh(s / case["cap"])
            if case["slopes"]:
                s = s - st["slopes"][g * G:(g + 1) * G, None] * distance[:, None, :]
            s = s.masked_fill(hidden[:, None, :], float("-inf"))
            top = s.amax(dim=-1, keepdim=True)
            p = torch.exp(s - torch.where(top == float("-inf"), 0.0, top))   # (a row that sees nothing is zero)
            total = p.sum(dim=-1, keepdim=True)
            o = (p.flatten(0, 1) @ _plain_rows(st, b, g, "v")).view(n, G, -1) / torch.where(total == 0, 1.0, total)
            st["out"][at:at + n, g * G:(g + 1) * G] = o.to(torch.bfloat16)
        at += n
    return st["out"]


_plain_prefill = _plain_decode = _plain_attention


# ---- the operators' definitions in 64 bits --------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    return _exact_append(st, case) if case["op"] == "append" else _exact_attention(st, case)


def _exact_append(st, case):
    T, D, half = st["q"].shape[0], case["dim"], case["rot"] // 2
    freq = torch.arange(half, device="cuda")
    table = st["cos_sin"].double()
    where = st["positions"].long().reshape(case["axes"], T)[torch.tensor(st["axis"], device="cuda")]     # [half, T]
    turn = torch.complex(table[where, freq[:, None]], table[where, half + freq[:, None]]).T[:, None, :]
    even = torch.arange(half, device="cuda") * (2 if case["pairs"] else 1)
    odd = even + (1 if case["pairs"] else half)

    def rotated(x, weight):
        x = x.double()
        if weight is not None:
            x = x / (x.square().sum(-1, keepdim=True) / D + EPS).sqrt() * weight.double()
        z = torch.complex(x[..., even], x[..., odd]) * turn
        x = x.clone()
        x[..., even], x[..., odd] = z.real, z.imag
        return x

    q, slots = rotated(st["q"], st["q_norm"]), st["slots"].tolist()
    page = torch.tensor([s // PAGE for s in slots], device="cuda")
    slot = torch.tensor([s % PAGE for s in slots], device="cuda")
    outs, scales = [q], []
    for name, rows in (("k", rotated(st["k"], st["k_norm"])), ("v", st["v"].double())):
        cache = st[name + "_cache"].double()
        if case["fp8"]:
            scale = st[name + "_scale0"].double()
            for t, s in enumerate(slots):
                if s % PAGE == 0:
                    top = rows[t].abs().amax(-1)
                    scale[s // PAGE] = torch.where(top == 0, torch.ones_like(top), top / 224)
            rows = (rows / scale[page].unsqueeze(-1)).clamp(-448, 448)
            scales.append(scale)
        cache[page, :, slot] = rows
        outs.append(cache)
    return tuple(outs + scales)


def _exact_attention(st, case):
    Hq, Hkv, D = case["q_heads"], case["kv_heads"], case["dim"]
    out = torch.zeros((st["q"].shape[0], Hq, D), dtype=torch.float64, device="cuda")
    first, prefix = _masks(case)
    at = 0
    for b in range(case["batch"]):
        L, n = st["lens"][b], st["new"][b]
        j = torch.arange(L, device="cuda")
        page, slot = st["table"][b, j // PAGE].long(), j % PAGE
        pos = torch.arange(L - n, L, device="cuda")
        for h in range(Hq):
            g = h * Hkv // Hq
            k, v = st["k_cache"][page, g, slot].double(), st["v_cache"][page, g, slot].double()
            if case["fp8"]:
                k, v = k * st["k_scale"][page, g].double()[:, None], v * st["v_scale"][page, g].double()[:, None]
            for i in range(0, n, 2048):
                p = pos[i:i + 2048, None]
                s = st["q"][at + i:at + i + len(p), h].double() @ k.T * st["scale"]
                if case["cap"]:
                    s = torch.tanh(s / case["cap"]) * case["cap"]
                if case["slopes"]:
                    s = s - st["slopes"][h].double() * (p - j).abs()
                see = j <= p
                if prefix is not None:
                    see = see | (j < int(prefix[b]))
                if case["window"]:
                    see = see & (p - j < case["window"])
                if first is not None:
                    see = see & (j >= st["first"][at + i:at + i + len(p), None])
                w = torch.where(see, torch.exp(s - torch.where(see, s, -1e300).amax(1, keepdim=True)), 0.0)
                out[at + i:at + i + len(p), h] = w @ v / w.sum(1, keepdim=True)
        at += n
    return out


def work(case):
    """Each input read once, each output written once; the products over the visible pairs."""
    L, n = _lens(case)
    Hq, Hkv, D, T = case["q_heads"], case["kv_heads"], case["dim"], int(n.sum())
    elem = 1 if case["fp8"] else 2
    if case["op"] == "append":
        angles = min(T, TABLE) * case["rot"] * 4
        rows = T * D * (4 * Hq + 2 * Hkv * (2 + elem))
        opened = int((-(-L // PAGE) - -(-(L - n) // PAGE)).sum()) if case["fp8"] else 0
        return dict(bytes=rows + angles + 4 * T * (case["axes"] + 1) + 8 * Hkv * opened, flops=T * (Hq + Hkv) * (3 * case["rot"] + (4 * D if case["norm"] else 0)))
    pairs = keys = pages = 0
    for lo, hi in _ranges(case):
        pairs += int(np.maximum(hi - lo, 0).sum())
        keys += int(hi.max() - lo.min())
        pages += int(-(-hi.max() // PAGE) - lo.min() // PAGE)
    masks = (T if case["docs"] else 0) + (len(L) if case.get("prefix") else 0) + (Hq if case["slopes"] else 0)
    bytes_ = 4 * T * Hq * D + keys * 2 * Hkv * D * elem + 4 * (pages + 2 * len(L) + masks) + (8 * Hkv * pages if case["fp8"] else 0)
    return dict(bytes=bytes_, flops=4 * D * Hq * pairs)
