"""The latent-attention operators and the step tables: what they are measured on.

A latent cache holds one row ``[c | r]`` per token (``c``: the latent vector, ``r``: the rotary key part),
shared by all query heads, in pages. Four operators work on it:

``tables``   block-table rows, slot map, positions and cumulative counts of a step, from request lengths
``append``   the step's rows into their slots, optionally with the latent's RMS norm
``absorbed`` attention of one or a few query tokens per sequence over the paged latent cache
``expanded`` causal attention over packed ragged sequences with per-head keys/values and the shared rotary key
"""
import math

import numpy as np
import torch

own = False

ROPE, NOPE, VDIM = 64, 128, 128      # rotary part, per-head key part without it, per-head value
POOL = 1.25                          # physical pages per page needed, as a server keeps some free


def listed():
    """A case's ``lens`` are drawn from ``lens_seed`` between ``lo`` and ``hi``."""
    return [
        # a decode step's tables: every request grows by one token
        dict(name="tables_decode", op="tables", batch=256, lo=512, hi=4096, new_lo=1, new_hi=1, page=64, pad=0, lens_seed=1),
        # a step of chunked prompts next to decoding requests, token arrays padded to a fixed capacity
        dict(name="tables_prompts", op="tables", batch=96, lo=1, hi=4096, new_lo=0, new_hi=2048, page=16, pad=1000, lens_seed=2),
        # the decode step's rows, one per request
        dict(name="append_decode", op="append", tokens=256, latent=512, page=64, norm=True, lens_seed=3),
        # a prompt batch's rows, latents already normed
        dict(name="append_prompts", op="append", tokens=16411, latent=512, page=16, norm=False, lens_seed=4),
        # a single short request on one of eight shards of the heads: latency
        dict(name="absorbed_one", op="absorbed", batch=1, heads=16, tokens=1, lo=517, hi=517, latent=512, page=64, lens_seed=5),
        # a decode batch on a shard with 16 heads: the cache's bytes
        dict(name="absorbed_h16", op="absorbed", batch=64, heads=16, tokens=1, lo=512, hi=4096, latent=512, page=64, lens_seed=6),
        # a decode batch with all 128 heads on one GPU: bytes and tensor work in balance
        dict(name="absorbed_h128", op="absorbed", batch=128, heads=128, tokens=1, lo=512, hi=4096, latent=512, page=64, lens_seed=7),
        # long contexts, few sequences, small pages: the split over the tokens
        dict(name="absorbed_long", op="absorbed", batch=8, heads=32, tokens=1, lo=32768, hi=131072, latent=512, page=16, lens_seed=8),
        # a block of draft tokens per sequence is verified: tensor work
        dict(name="absorbed_verify", op="absorbed", batch=32, heads=64, tokens=5, lo=300, hi=8000, latent=512, page=64, lens_seed=9),
        # short ragged prompts together
        dict(name="expanded_short", op="expanded", batch=24, heads=16, lo=1, hi=700, ctx_lo=0, ctx_hi=0, lens_seed=10),
        # one long prompt
        dict(name="expanded_prompt", op="expanded", batch=1, heads=32, lo=8192, hi=8192, ctx_lo=0, ctx_hi=0, lens_seed=11),
        # prompt chunks over longer contexts
        dict(name="expanded_chunks", op="expanded", batch=4, heads=16, lo=500, hi=1024, ctx_lo=1000, ctx_hi=16384, lens_seed=12),
    ]


def draw(rng):
    """One more case of the same ranges."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["tables", "append", "absorbed", "absorbed", "expanded", "expanded"])
    seed = rng.randrange(1 << 30)
    if op == "tables":
        new_hi = rng.choice([1, 1, 7, 2048])
        return dict(op=op, batch=log(1, 96 if new_hi == 2048 else 700), lo=1, hi=log(64, 8192), new_lo=rng.choice([0, 1]),
                    new_hi=new_hi, page=rng.choice([16, 32, 64]), pad=rng.choice([0, 0, 333]), lens_seed=seed)
    if op == "append":
        return dict(op=op, tokens=log(1, 16000), latent=rng.choice([256, 512]), page=rng.choice([16, 32, 64]),
                    norm=rng.random() < 0.5, lens_seed=seed)
    if op == "absorbed":
        heads, tokens = rng.choice([(8, 1), (16, 1), (32, 1), (64, 1), (128, 1), (16, 3), (32, 8), (64, 2), (128, 4), (24, 1)])
        hi = log(64, 40000)
        most = 2.0e7 / (heads * tokens * hi)      # (half of the pairs of the largest listed case, for lengths near hi)
        batch = max(1, min(log(1, 160), int(most), int(6.0e5 / hi)))
        return dict(op=op, batch=batch, heads=heads, tokens=tokens, lo=max(tokens, hi // rng.choice([1, 2, 8])), hi=max(tokens, hi),
                    latent=rng.choice([256, 512, 512]), page=rng.choice([16, 32, 64]), lens_seed=seed)
    hi, ctx = log(8, 4000), rng.choice([0, 0, 1]) * log(32, 8000)
    heads = rng.choice([4, 16, 32])
    batch = max(1, min(log(1, 24), 300 // heads, int(1.0e9 / (heads * hi * (hi / 2 + ctx))), int(5.0e5 / (heads * (hi + ctx)))))
    return dict(op=op, batch=batch, heads=heads, lo=max(1, hi // rng.choice([1, 3, 50])), hi=hi, ctx_lo=ctx // 2, ctx_hi=ctx, lens_seed=seed)


def _lens(case):
    """Per sequence (length after the step, tokens of the step); a function of the case alone."""
    g = np.random.default_rng(case["lens_seed"])
    if case["op"] == "tables":
        new = g.integers(case["new_lo"], case["new_hi"], size=case["batch"], endpoint=True)
        old = g.integers(case["lo"], case["hi"], size=case["batch"], endpoint=True)
        return old + new, new
    if case["op"] == "absorbed":
        n = g.integers(case["lo"], case["hi"], size=case["batch"], endpoint=True)
        return n, np.minimum(n, case["tokens"])
    new = g.integers(case["lo"], case["hi"], size=case["batch"], endpoint=True)
    return new + g.integers(case["ctx_lo"], case["ctx_hi"], size=case["batch"], endpoint=True), new


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    st = dict(case=case)
    if own:
        from paper_2605_06068_b200 import binding
        st["pda"] = binding

    def ints(a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()

    if case["op"] == "tables":
        L, n = _lens(case)
        P = case["page"]
        held, need = -(-(L - n) // P), -(-L // P)
        pool = int(math.ceil(POOL * need.sum())) + 1
        perm = rng.permutation(pool).astype(np.int32)
        table = np.full((len(L), int(need.max()) + 2), -1, dtype=np.int32)
        at = 0
        for b in range(len(L)):
            table[b, :held[b]] = perm[at:at + held[b]]
            at += held[b]
        cap = int(n.sum()) + case["pad"]
        st.update(seq_lens=ints(L), new_lens=ints(n), table0=ints(table), table=ints(table), free_pages=ints(perm[at:]),
                  free_count=ints([pool - at]), free_out=ints([0]), cu=ints(np.zeros(len(L) + 1)), slots=ints(np.zeros(max(cap, 1))),
                  positions=ints(np.zeros(max(cap, 1))))
        return st
    if case["op"] == "append":
        T, R, P = case["tokens"], case["latent"], case["page"]
        pages = int(math.ceil(POOL * T / P)) + 1
        # the projection's output [c | r] in one buffer, as the layer leaves it: both parts are strided views
        new = _randn(gen, T, R + ROPE)
        new[:, :R] *= torch.rand((T, 1), generator=gen, device="cuda") * 3 + 0.1
        st.update(c_new=new[:, :R], r_new=new[:, R:], cache=_randn(gen, pages, P, R + ROPE),
                  slots=ints(rng.permutation(pages * P)[:T]), weight=_randn(gen, R) * 0.2 + 1 if case["norm"] else None)
        return st
    L, n = _lens(case)
    if case["op"] == "absorbed":
        R, P, H, T, B = case["latent"], case["page"], case["heads"], case["tokens"], case["batch"]
        need = -(-L // P)
        pool = int(math.ceil(POOL * need.sum())) + 1
        perm = rng.permutation(pool).astype(np.int32)
        table = np.full((B, int(need.max())), -1, dtype=np.int32)
        cache = torch.full((pool, P, R + ROPE), float("nan"), dtype=torch.bfloat16, device="cuda")
        at = 0
        for b in range(B):
            table[b, :need[b]] = perm[at:at + need[b]]
            at += need[b]
        used = torch.from_numpy(perm[:at].astype(np.int64)).cuda()
        cache[used] = _randn(gen, at, P, R + ROPE)
        last = torch.from_numpy(table[np.arange(B), need - 1].astype(np.int64)).cuda()      # tails of the last pages hold nothing
        tail = torch.arange(P, device="cuda")[None, :] >= ints((L - 1) % P + 1)[:, None]
        cache[last] = cache[last].masked_fill(tail[:, :, None], float("nan"))
        # q_latent as the batched product over heads leaves it ([H, B*T, R]), q_rope as a slice of the heads' queries
        ql = _randn(gen, H, B * T, R).permute(1, 0, 2).unflatten(0, (B, T))
        qr = _randn(gen, B, T, H, NOPE + ROPE)[..., NOPE:]
        st.update(q_latent=ql, q_rope=qr, cache=cache, table=ints(table), seq_lens=ints(L), lens=[int(x) for x in L],
                  scale=1.0 / math.sqrt(NOPE + ROPE), out=torch.zeros((B, T, H, R), dtype=torch.bfloat16, device="cuda"))
        if own:
            st["workspace"] = st["pda"].latent_workspace(B, H, T, R)
        return st
    H, tq, tk = case["heads"], int(n.sum()), int(L.sum())
    kv = _randn(gen, tk, H, NOPE + VDIM)                # the up-projection's output: keys and values of a head together
    st.update(q=_randn(gen, tq, H, NOPE + ROPE), k_nope=kv[..., :NOPE], v=kv[..., NOPE:], k_rope=_randn(gen, tk, ROPE),
              cu_q=ints(np.concatenate([[0], np.cumsum(n)])), cu_k=ints(np.concatenate([[0], np.cumsum(L)])),
              q_lens=[int(x) for x in n], k_lens=[int(x) for x in L], max_q=int(n.max()), scale=1.0 / math.sqrt(NOPE + ROPE),
              out=torch.zeros((tq, H, VDIM), dtype=torch.bfloat16, device="cuda"))
    return st


def run(st):
    return globals()[("_own_" if own else "_plain_") + st["case"]["op"]](st)


# ---- the framework's calls ------------------------------------------------------------------------

def _own_tables(st):
    st["pda"].paged_build_tables(st["seq_lens"], st["new_lens"], st["case"]["page"], st["free_pages"], st["free_count"],
                                 st["table"], st["cu"], st["slots"], positions=st["positions"], free_count_out=st["free_out"])
    return st["table"], st["cu"], st["slots"], st["positions"], st["free_out"]


def _own_append(st):
    st["pda"].latent_append(st["c_new"], st["r_new"], st["cache"], st["slots"], norm_weight=st["weight"], eps=1e-6)
    return st["cache"]


def _own_absorbed(st):
    return st["pda"].paged_latent_attention(st["q_latent"], st["q_rope"], st["cache"], st["table"], st["seq_lens"], st["scale"],
                                            out=st["out"], workspace=st["workspace"])


def _own_expanded(st):
    return st["pda"].latent_prefill_attention(st["q"], st["k_nope"], st["k_rope"], st["v"], st["cu_q"], st["cu_k"], st["max_q"],
                                              st["scale"], out=st["out"])


# ---- plain forms ----------------------------------------------------------------------------------

def _plain_tables(st):
    L, n, P = st["seq_lens"].long(), st["new_lens"].long(), st["case"]["page"]
    cap = st["slots"].numel()
    held, need = (L - n + P - 1) // P, (L + P - 1) // P
    taken = torch.cumsum(need - held, 0) - (need - held)
    col = torch.arange(st["table0"].shape[1], device="cuda")[None, :]
    fresh = (col >= held[:, None]) & (col < need[:, None])
    at = st["free_count"].long() - 1 - (taken[:, None] + col - held[:, None])
    table = torch.where(fresh, st["free_pages"][at.clamp(0, st["free_pages"].numel() - 1)], st["table0"])
    cu = torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), torch.cumsum(n, 0)])
    t = torch.arange(cap, device="cuda")
    b = torch.searchsorted(cu[1:], t, right=True).clamp(max=L.numel() - 1)
    live = t < cu[-1]
    pos = torch.where(live, t - cu[b] + L[b] - n[b], 0)
    slot = torch.where(live, table[b, pos // P].long() * P + pos % P, -1)
    pos = torch.where(live, pos, -1)
    left = st["free_count"] - (need - held).sum().int()
    return table, cu.int(), slot.int(), pos.int(), left


def _plain_append(st):
    c = st["c_new"].float()
    if st["weight"] is not None:
        c = c * torch.rsqrt((c * c).mean(dim=1, keepdim=True) + 1e-6) * st["weight"].float()
    row = torch.cat([c.to(torch.bfloat16), st["r_new"]], dim=1)
    cache = st["cache"]
    cache.view(-1, cache.shape[2])[st["slots"].long()] = row
    return cache


def _plain_absorbed(st):
    R, P, T = st["case"]["latent"], st["case"]["page"], st["case"]["tokens"]
    for b, L in enumerate(st["lens"]):
        pages = st["table"][b, :(L + P - 1) // P].long()
        rows = st["cache"][pages].flatten(0, 1)[:L].float()
        q = torch.cat([st["q_latent"][b], st["q_rope"][b]], dim=-1).float()
        s = (q.flatten(0, 1) @ rows.T).view(T, -1, L) * st["scale"]
        if T > 1:
            hidden = torch.arange(L, device="cuda")[None, :] > torch.arange(T, device="cuda")[:, None] + (L - T)
            s = s.masked_fill(hidden[:, None, :], float("-inf"))
        p = torch.exp(s - s.amax(dim=-1, keepdim=True))
        o = (p.flatten(0, 1) @ rows[:, :R]).view(T, -1, R) / p.sum(dim=-1, keepdim=True)
        st["out"][b] = o.to(torch.bfloat16)
    return st["out"]


def _plain_expanded(st):
    q0 = k0 = 0
    for nq, nk in zip(st["q_lens"], st["k_lens"]):
        hidden = torch.arange(nk, device="cuda")[None, :] > torch.arange(nq, device="cuda")[:, None] + (nk - nq)
        kr = st["k_rope"][k0:k0 + nk].float()
        for h in range(st["case"]["heads"]):
            q = st["q"][q0:q0 + nq, h].float()
            s = (q[:, :NOPE] @ st["k_nope"][k0:k0 + nk, h].float().T + q[:, NOPE:] @ kr.T) * st["scale"]
            s = s.masked_fill(hidden, float("-inf"))
            p = torch.exp(s - s.amax(dim=-1, keepdim=True))
            o = p @ st["v"][k0:k0 + nk, h].float() / p.sum(dim=-1, keepdim=True)
            st["out"][q0:q0 + nq, h] = o.to(torch.bfloat16)
        q0, k0 = q0 + nq, k0 + nk
    return st["out"]


# ---- the operators' definitions in 64 bits --------------------------------------------------------

def exact(case, seed):
    if case["op"] == "tables":
        return None     # whole numbers
    st = prepare(case, seed)
    if case["op"] == "append":
        cache = st["cache"].double()
        pages, P, W = cache.shape
        flat, R = cache.view(pages * P, W), case["latent"]
        c = st["c_new"].double()
        if case["norm"]:
            c = c / torch.sqrt((c ** 2).sum(1, keepdim=True) / R + 1e-6) * st["weight"].double()
        where = st["slots"].long()
        flat[where, :R] = c
        flat[where, R:] = st["r_new"].double()
        return cache
    if case["op"] == "absorbed":
        B, T, H, R, P = case["batch"], case["tokens"], case["heads"], case["latent"], case["page"]
        out = torch.zeros((B, T, H, R), dtype=torch.float64, device="cuda")
        for b in range(B):
            L = st["lens"][b]
            j = torch.arange(L, device="cuda")
            rows = st["cache"][st["table"][b, j // P].long(), j % P].double()
            for t in range(T):
                live = rows[:L - T + 1 + t]
                s = (live[:, :R] @ st["q_latent"][b, t].double().T + live[:, R:] @ st["q_rope"][b, t].double().T) * st["scale"]
                out[b, t] = torch.softmax(s, dim=0).T @ live[:, :R]
        return out
    tq, H = st["q"].shape[:2]
    out = torch.zeros((tq, H, VDIM), dtype=torch.float64, device="cuda")
    cq, ck = st["cu_q"].tolist(), st["cu_k"].tolist()
    for b in range(case["batch"]):
        nq, nk = cq[b + 1] - cq[b], ck[b + 1] - ck[b]
        for h in range(H):
            k = torch.cat([st["k_nope"][ck[b]:ck[b + 1], h], st["k_rope"][ck[b]:ck[b + 1]]], dim=1).double()
            v = st["v"][ck[b]:ck[b + 1], h].double()
            for i in range(0, nq, 2048):
                n = min(2048, nq - i)
                s = st["q"][cq[b] + i:cq[b] + i + n, h].double() @ k.T * st["scale"]
                s += torch.triu(torch.full_like(s, float("-inf")), diagonal=nk - nq + i + 1)
                out[cq[b] + i:cq[b] + i + n, h] = torch.softmax(s, dim=1) @ v
    return out


def work(case):
    """Each input read once, each output written once; the products over the visible pairs."""
    if case["op"] == "append":
        row = case["latent"] + ROPE
        return dict(bytes=case["tokens"] * (4 * row + 4) + (2 * case["latent"] if case["norm"] else 0),
                    flops=case["tokens"] * case["latent"] * (4 if case["norm"] else 0))
    L, n = _lens(case)
    if case["op"] == "tables":
        P, tokens, B = case["page"], int(n.sum()), len(L)
        fresh = int((-(-L // P) - -(-(L - n) // P)).sum())
        touched = int((-(-L // P) - (L - n) // P)[n > 0].sum())      # page ids behind the step's tokens
        return dict(bytes=4 * (3 * B + 3 + 2 * fresh + touched + 2 * (tokens + case["pad"])), flops=4 * tokens)
    if case["op"] == "absorbed":
        R, rows = case["latent"], case["heads"] * case["tokens"]
        pairs = sum(int(x) * case["tokens"] - case["tokens"] * (case["tokens"] - 1) // 2 for x in L) * case["heads"]
        pages = int((-(-L // case["page"])).sum())
        return dict(bytes=int(L.sum()) * (R + ROPE) * 2 + len(L) * rows * (2 * R + ROPE) * 2 + 4 * (pages + len(L)),
                    flops=2 * pairs * (2 * R + ROPE))
    H, tq, tk = case["heads"], int(n.sum()), int(L.sum())
    pairs = sum(int(q) * int(k) - int(q) * (int(q) - 1) // 2 for k, q in zip(L, n))
    return dict(bytes=2 * (tq * H * (NOPE + ROPE + VDIM) + tk * (H * (NOPE + VDIM) + ROPE)) + 8 * (len(L) + 1),
                flops=2 * H * pairs * (NOPE + ROPE + VDIM))
