"""The ends of the ranges that the calls over the paged cache allow: caps of any size, rows far below the cap, scales of zero, rows
that see nothing, sums joined where scores are large, chunks beyond any sequence, value scales of any size. Plain references in
64 bits."""
import numpy as np
import pytest
import torch

import shaped_util as U
from paper_2605_06068_b200 import binding as pda

pytestmark = pytest.mark.gpu

GENERIC = pda.PDA_FLAG_FORCE_GENERIC
INT_MAX = 2 ** 31 - 1


def randn(seed, *shape, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(torch.bfloat16)


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def cum(n):
    return ints([0] + list(np.cumsum(n)))


def nan(*shape):
    return torch.full(shape, float("nan"), device="cuda")


# ---- chunks beyond any sequence ---------------------------------------------------------------------

@pytest.mark.parametrize("chunk,room", [(1 << 30, 9), (1 << 20, 4100), ((1 << 31) - 16, 3), (32, 64)])
def test_chunks_that_start_beyond_32_bits(chunk, room):
    """Partial buffers with room for more chunks than any sequence has: the chunks' places pass 2^31."""
    lens, Hq, Hkv, D = [200, 0, 17, 1999], 4, 2, 128
    c = U.Cache(lens, Hkv, D, seed=1)
    q = randn(2, 4, Hq, D)
    args = q.cuda(), c.k_cache, c.v_cache, c.dev_table, ints(lens), 0.1
    ref, tol = U.reference(c, q, [1] * 4, 0.1, decode=True)
    parts = lambda: dict(chunk_tokens=chunk, part_o=nan(4, Hq, room, D), part_lse=nan(4, Hq, room))
    status = ints([0])
    for workspace in (pda.new_workspace(4, Hkv), None):
        U.check(pda.paged_biased_decode_attention(*args, workspace=workspace, status=status, **parts()), ref, tol, "shaped")
    U.check(pda.paged_decode_step(args[0], None, None, *args[1:], workspace=pda.new_workspace(4, Hkv), status=status, **parts()), ref, tol, "step")
    for flags in (0, GENERIC):
        po, pl = pda.paged_decode_attention(*args, flags=flags, status=status, **parts())
        U.check(pda.paged_decode_reduce(po, pl, ints(lens), chunk), ref, tol, "attention and reduce")
    for flags in (0, pda.PDA_FLAG_MQ_MMA_SYNC):
        kw = dict(chunk_tokens=chunk, part_o=nan(4, 1, Hq, room, D), part_lse=nan(4, 1, Hq, room))
        out = pda.paged_verify_attention(args[0][:, None].contiguous(), *args[1:], flags=flags, status=status, **kw)
        U.check(out[:, 0], ref, tol, "verify")
    assert int(status.item()) == 0


def test_decode_lengths_up_to_the_last():
    """2^31 - 1 tokens by a table that names the same pages again, of which a window sees the last ones."""
    D, L = 64, INT_MAX
    c = U.Cache([64], 1, D, seed=3, extra=0)
    table = c.dev_table[:1, :4].repeat(1, 1 << 25)
    q = randn(4, 1, 2, D)
    status = ints([0])
    call = lambda **kw: pda.paged_biased_decode_attention(q.cuda(), c.k_cache, c.v_cache, table, ints([L]), 0.125, window=100, status=status, **kw)
    j = torch.arange(L - 100, L) % 64
    for h in range(2):
        ref, tol = U.attend(q[:, h], c.k[0][j, 0], c.v[0][j, 0], torch.tensor([0]), torch.tensor([100]), torch.tensor([99]), 0.125)
        U.check(call()[:, h], ref, tol, "whole")
        for workspace in (pda.new_workspace(1, 1), None):
            kw = dict(chunk_tokens=1 << 30, part_o=nan(1, 2, 5, D), part_lse=nan(1, 2, 5), workspace=workspace)
            U.check(call(**kw)[:, h], ref, tol, "in chunks")
    assert int(status.item()) == 0


# ---- caps of any size -------------------------------------------------------------------------------

def capped(q, k, v, live, scale, cap, slope=0.0, dist=None, byte=None):
    """(out, tol) of one head: rows q [n,D] over k, v [L,D], ``live`` [n,L]. Scores in 32 bits: the product is off by
    (D + 3) 2^-24 scale sum |q_d k_d|, the cap by 2^-20 of the score (an odd polynomial whose error is relative, or exponential and
    reciprocal where the tangent is not small: eight roundings of 2^-24 and two functions of 2^-22), and where a polynomial's error
    is absolute by 2^-17 of the cap, for caps up to 128: 2^-10 at most. The rest as in shaped_util.attend. ``byte``: [n,L] bounds of
    16-bit weights' steps."""
    q, k, v = q.double(), k.double(), v.double()
    s = (q @ k.T) * scale
    e = (q.shape[1] + 3) * 2.0 ** -24 * abs(scale) * (q.abs() @ k.abs().T)
    if cap > 0:
        e = e * (1 - torch.tanh((s.abs() - e).clamp(min=0) / cap) ** 2)      # (the largest slope of the tangent on the way)
        s = cap * torch.tanh(s / cap)
        e = e + 2.0 ** -20 * s.abs() + (cap * 2.0 ** -17 if cap <= 128 else 0.0)
    if dist is not None:
        s = s - slope * dist
        e = e + 2.0 ** -22 * (abs(slope) * dist + s.abs())
    w = torch.softmax(torch.where(live, s, float("-inf")), 1)
    o, A, we = w @ v, w @ v.abs(), w * e
    tol = U.EPS * o.abs() + (2 * U.EPS + k.shape[0] * 2.0 ** -24 + 2.0 ** -12) * A + 2 * (we @ v.abs() + we.sum(1, keepdim=True) * o.abs())
    if byte is not None:
        tol = tol + byte
    return o, 1.01 * tol


def run_caps(how, D, fp8, cap, scale, seed, slopes=None, spread=4.0, near=None):
    """Two sequences; ``near``: products q.k scale / cap spread over this range, by one number of a query and one of a key."""
    lens, new, Hq, Hkv = [300, 70], ([300, 40] if how != "decode" else [1, 1]), 4, 2
    c = U.Cache(lens, Hkv, D, fp8=fp8, seed=seed)
    T = sum(new)
    q = randn(seed + 1, T, Hq, D, scale=spread)
    if near is not None:
        g = np.random.default_rng(seed)
        rows = torch.zeros(c.k_cache.shape)
        for b, L in enumerate(lens):
            x = torch.as_tensor(g.uniform(*near, size=(L, Hkv))).to(U.E4M3 if fp8 else torch.bfloat16)
            for j in range(L):
                rows[int(c.table[b, j // 16]), :, j % 16, 0] = x[j].float()
            c.k[b] = torch.zeros((L, Hkv, D), dtype=torch.float64)
            c.k[b][:, :, 0] = x.double()
        c.k_cache = rows.to(c.k_cache.dtype).cuda()
        if fp8:
            c.k_scale = torch.ones_like(c.k_scale)
        q = torch.zeros((T, Hq, D), dtype=torch.bfloat16)
        q[:, :, 0] = 8.0
        scale = float(np.float32(cap / 8.0))
    dev_slopes = None if slopes is None else torch.tensor(slopes, device="cuda")
    status = ints([0])
    kw = dict(softcap=cap, slopes=dev_slopes, status=status, flags=GENERIC if how == "generic" else 0, **c.args())
    if how == "decode":
        out = pda.paged_biased_decode_attention(q.cuda(), c.k_cache, c.v_cache, c.dev_table, ints(lens), scale, **kw)
    else:
        out = pda.paged_prefill_attention(q.cuda(), c.k_cache, c.v_cache, c.dev_table, ints(lens), cum(new), max(new), scale, **kw)
    assert int(status.item()) == 0
    at = 0
    for b, n in enumerate(new):
        pos, j = torch.arange(n) + lens[b] - n, torch.arange(lens[b])
        live, dist = j[None, :] <= pos[:, None], (pos[:, None] - j[None, :]).abs().double()
        for h in range(Hq):
            k, v = c.k[b][:, h // 2], c.v[b][:, h // 2]
            byte = 2.0 ** -25 * c.byte * live.sum(1, keepdim=True) if fp8 and how == "decode" else None
            ref, tol = capped(q[at:at + n, h], k, v, live, float(np.float32(scale)), float(np.float32(cap)), 0.0 if slopes is None else float(np.float32(slopes[h])), dist, byte)
            U.check(out[at:at + n, h], ref, tol, f"cap {cap} sequence {b} head {h}")
        at += n


WAYS = [("prompt", 128, False), ("prompt", 64, False), ("prompt", 128, True), ("generic", 96, False), ("generic", 64, True), ("decode", 128, False),
        ("decode", 256, False), ("decode", 128, True)]


@pytest.mark.parametrize("how,D,fp8", WAYS)
@pytest.mark.parametrize("cap", [1.0, 30.0, 120.0, 135.0, 1000.0, 4100.0, 1e4, 1e6, 1e8, 1e20, 2e38])
def test_scores_far_below_a_cap_are_left_alone(how, D, fp8, cap):
    for slopes in (None, [0.3, 0.0, 0.05, -0.01]):
        run_caps(how, D, fp8, cap, D ** -0.5, seed=50, slopes=slopes)


@pytest.mark.parametrize("how,D,fp8", WAYS)
@pytest.mark.parametrize("cap,near", [(20.0, (-1.5, 1.5)), (130.0, (2.0, 4.0)), (1000.0, (3.0, 6.0)), (1000.0, (0.6, 0.64)), (2000.0, (-0.001, 0.001)), (1e5, (5.0, 9.0)), (1e-30, (-2.0, 2.0))])
def test_scores_about_a_cap(how, D, fp8, cap, near):
    run_caps(how, D, fp8, cap, 0.0, seed=51, near=near)


# ---- rows far below the cap -------------------------------------------------------------------------

def signed_prompt(fp8, cap, vscale, signs, new, first=None, D=128, order=None, seed=5):
    """A prompt whose scores are +-cap (or near zero) by ``signs`` [L] of its keys, values of the size ``vscale``: one kv head, two
    query heads, of which the second sees the opposite scores. Returns (got, ref, tol)."""
    L = len(signs)
    c = U.Cache([L], 1, D, seed=seed)
    rows = torch.zeros(c.k_cache.shape)
    for j, s in enumerate(signs):
        rows[int(c.table[0, j // 16]), 0, j % 16] = 8.0 * float(s)
    values = torch.where(c.v_cache.cpu().isnan(), 0.0, c.v_cache.cpu().float())
    kw = {}
    if fp8:
        k_cache, v_cache = rows.to(U.E4M3).cuda(), values.to(U.E4M3).cuda()
        one = torch.ones((rows.shape[0], 1), device="cuda")
        kw = dict(k_scale=one, v_scale=one * vscale)
        values = v_cache.cpu().double() * vscale
    else:
        k_cache, v_cache = rows.to(torch.bfloat16).cuda(), (values * vscale).to(torch.bfloat16).cuda()
        values = v_cache.cpu().double()
    v = torch.stack([values[int(c.table[0, j // 16]), 0, j % 16] for j in range(L)])
    q = torch.full((new, 2, D), 8.0, dtype=torch.bfloat16)
    q[:, 1] = -8.0
    status = ints([0])
    got = pda.paged_prefill_attention(q.cuda(), k_cache, v_cache, c.dev_table, ints([L]), ints([0, new]), new, 1.0, softcap=cap, status=status,
                                      first_keys=None if first is None else ints(first), **kw)
    assert int(status.item()) == 0
    pos, j = torch.arange(new) + L - new, torch.arange(L)
    live = j[None, :] <= pos[:, None]
    if first is not None:
        live &= j[None, :] >= torch.tensor(first)[:, None]
    ref, tol = torch.zeros((new, 2, D), dtype=torch.float64), torch.zeros((new, 2, D), dtype=torch.float64)
    some = live.any(1)
    for h, sign in enumerate((1.0, -1.0)):
        s = cap * torch.tanh(sign * torch.tensor(signs, dtype=torch.float64) * 64 * D / cap)
        # scores off by 2^-20 of the cap (and by 2^-17 of it where a polynomial takes them): the same for equal scores
        e = cap * (2.0 ** -20 + 2.0 ** -17)
        w = torch.softmax(torch.where(live, s[None, :], float("-inf"))[some], 1)
        o, A = w @ v, w @ v.abs()
        ref[some, h] = o
        tol[some, h] = 1.01 * (U.EPS * o.abs() + (2 * U.EPS + L * 2.0 ** -24 + 2.0 ** -12 + 4 * e) * A)
    return got, ref, tol


SIZES = [(True, 2.0 ** -8), (True, 2.0 ** -14), (True, 2.0 ** -22), (True, 2.0 ** -40), (False, 1.0), (False, 2.0 ** -30), (False, 2.0 ** -45), (True, 2.0 ** 30), (False, 2.0 ** 40)]


@pytest.mark.parametrize("cap", [5.0, 20.0, 40.0, 50.0, 51.9, 60.0])
@pytest.mark.parametrize("fp8,vscale", SIZES)
def test_rows_all_of_whose_scores_lie_at_the_negative_cap(cap, fp8, vscale):
    g = np.random.default_rng(3)
    U.check(*signed_prompt(fp8, cap, vscale, [-1.0], 1))
    U.check(*signed_prompt(fp8, cap, vscale, [-1.0] * 300, 300))
    # the first tokens see only the lowest scores, later ones higher and higher ones, 64 and more keys on
    steps = [-1.0] * 100 + [0.0] * 30 + [1.0] + [-1.0] * 170
    U.check(*signed_prompt(fp8, cap, vscale, steps, 300))
    U.check(*signed_prompt(fp8, cap, vscale, list(g.choice([-1.0, -1.0, -1.0, 0.0, 1.0], size=700)), 700))


@pytest.mark.parametrize("fp8,vscale", SIZES)
def test_low_rows_whose_keys_are_split(fp8, vscale):
    """Few rows: the tiles are shared by a block's halves, or cut along the keys; some rows see keys of one share only."""
    U.check(*signed_prompt(fp8, 50.0, vscale, [-1.0] * 400, 5, first=[0, 390, 200, 0, INT_MAX]))
    U.check(*signed_prompt(fp8, 50.0, vscale, [-1.0] * 150 + [1.0] + [-1.0] * 249, 5, first=[0, 390, 200, 120, 151]))
    U.check(*signed_prompt(fp8, 50.0, vscale, [-1.0] * 3000, 60, first=[50 * i for i in range(59)] + [2999]))
    U.check(*signed_prompt(fp8, 50.0, vscale, [-1.0] * 1000 + [0.0] + [-1.0] * 1000 + [1.0] + [-1.0] * 998, 60, first=[50 * i for i in range(59)] + [2999]))


# ---- a scale of zero --------------------------------------------------------------------------------

@pytest.mark.parametrize("D,fp8", [(128, False), (128, True), (64, False), (64, True)])
@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-30, -0.2])
def test_prefix_without_slopes_whatever_the_scale(D, fp8, scale):
    lens, new, prefix = [170, 240, 60], [150, 40, 60], [170, 230, 33]
    c = U.Cache(lens, 2, D, fp8=fp8, seed=8)
    q = randn(9, sum(new), 4, D)
    for flags in (0, GENERIC):
        out = pda.paged_prefill_attention(q.cuda(), c.k_cache, c.v_cache, c.dev_table, ints(lens), cum(new), 150, scale, prefix_lens=ints(prefix), flags=flags, **c.args())
        U.check(out, *U.reference(c, q, new, scale, prefix=prefix))


def test_prefix_and_slopes_that_a_small_scale_does_not_bear():
    """Biases of 2^70 and more of keys behind the token itself: the nearest key's weight is all there is."""
    lens, new, prefix = [200, 90], [150, 40], [170, 60]
    c = U.Cache(lens, 2, 128, seed=8)
    q = randn(9, sum(new), 4, 128)
    first = [p + 3 if p + 3 < 170 else 0 for p in range(50, 200)] + [0] * 40      # (rows that see keys behind themselves alone)
    status = ints([0])
    for slope in (2.0 ** 70, 2.0 ** 100):
        slopes = torch.tensor([slope, 0.0, slope, 0.1], device="cuda")
        for scale in (1e-17, 1e-3):
            for flags in (0, GENERIC):
                out = pda.paged_prefill_attention(q.cuda(), c.k_cache, c.v_cache, c.dev_table, ints(lens), cum(new), 150, scale, slopes=slopes,
                                                  prefix_lens=ints(prefix), first_keys=ints(first), flags=flags, status=status)
                U.check(out[:, [1, 3]], *(x[:, [1, 3]] for x in U.reference(c, q, new, scale, slopes=slopes.cpu().double(), prefix=prefix, first=first)))
                at = 0
                for b, (lo, hi) in enumerate(U.visible(lens, new, 0, prefix, first)):
                    pos = torch.arange(new[b]) + lens[b] - new[b]
                    near = torch.minimum(torch.maximum(pos, lo), hi - 1)
                    for h in (0, 2):
                        ref = c.v[b][near, h // 2]
                        U.check(out[at:at + new[b], h], ref, 1.01 * 3 * U.EPS * ref.abs(), f"{slope} {scale} {flags}")
                    at += new[b]
    assert int(status.item()) == 0


# ---- rows that see nothing --------------------------------------------------------------------------

def unseen(c, lens, new, window, prefix, first, how):
    """Tables and caches in which nothing that no token sees can be used: ids outside the cache, or pages of NaN."""
    see = U.visible(lens, new, window, prefix, first)
    table = c.dev_table.clone()
    for b, (lo, hi) in enumerate(see):
        for i in range(-(-lens[b] // 16)):
            if not ((lo < hi) & (lo < 16 * i + 16) & (hi > 16 * i)).any():
                if how == "ids":
                    table[b, i] = -1 if i % 2 else c.k_cache.shape[0] + i
                else:
                    for cache in (c.k_cache, c.v_cache):
                        cache.view(torch.uint8)[int(c.table[b, i])] = 0xFF
                    for scale in (c.k_scale, c.v_scale):
                        if scale is not None:
                            scale[int(c.table[b, i])] = float("nan")
    return table


CASES = [
    # trailing rows that see nothing (padding), of a block, of a half and of whole blocks
    ([128], [128], 0, None, [0] * 64 + [INT_MAX] * 64),
    ([700], [700], 0, None, [0] * 10 + [INT_MAX] * 690),
    # leading ones, with a window and without
    ([300], [300], 40, None, [INT_MAX] * 150 + [0] * 150),
    ([300, 90], [300, 60], 0, None, [250] * 250 + [255] * 20 + [270] * 30 + [INT_MAX] * 30 + [64] * 30),
    # in the middle, in several places
    ([400], [400], 30, None, [0] * 40 + [INT_MAX] * 100 + [0] * 10 + [390] * 240 + [0] * 10),
    ([400], [400], 0, None, [16 * (i // 16) if i // 50 % 2 else INT_MAX for i in range(400)]),
    # all of them
    ([200, 33], [200, 20], 0, None, [INT_MAX] * 200 + [0] * 20),
    # rows that see keys behind themselves alone, and none between
    ([500], [300], 0, [450], [400] * 20 + [0] * 5 + [420] * 200 + [INT_MAX] * 60 + [499] * 15),
    # rows before their sequence
    ([100], [150], 5, None, [0] * 60 + [INT_MAX] * 30 + [0] * 60),
    # many keys and few rows: blocks that are cut
    ([4000, 2500], [60, 20], 0, None, [INT_MAX] * 10 + [3900 + i for i in range(20)] + [INT_MAX] * 10 + [3990] * 20 + [2490] * 10 + [INT_MAX] * 10),
    ([4000], [40], 0, [1000], [0] * 10 + [3000] * 10 + [INT_MAX] * 20),
]


@pytest.mark.parametrize("how", ["ids", "pages"])
@pytest.mark.parametrize("kw", [dict(), dict(softcap=9.0), dict(slopes=[0.1, 0.02, 0.0, 0.3])])
@pytest.mark.parametrize("D,fp8", [(128, False), (128, True), (64, False)])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_pages_that_no_row_sees(case, D, fp8, kw, how):
    lens, new, window, prefix, first = CASES[case]
    Hq, Hkv = 4, 2
    c = U.Cache(lens, Hkv, D, fp8=fp8, seed=case)
    table = unseen(c, lens, new, window, prefix, first, how)
    q = randn(case + 1, sum(new), Hq, D)
    dev = dict(kw, slopes=torch.tensor(kw["slopes"], device="cuda")) if "slopes" in kw else kw
    status = ints([0])
    out = pda.paged_prefill_attention(q.cuda(), c.k_cache, c.v_cache, table, ints(lens), cum(new), max(new), 0.1, window=window, first_keys=ints(first),
                                      prefix_lens=None if prefix is None else ints(prefix), status=status, **c.args(), **dev)
    assert int(status.item()) == 0
    slopes = None if "slopes" not in kw else dev["slopes"].cpu().double()
    U.check(out, *U.reference(c, q, new, 0.1, kw.get("softcap", 0.0), slopes, window, prefix, first))


def test_pages_that_no_row_sees_in_many_sequences():
    """More row blocks than are listed, half of them without a row that sees anything."""
    g = np.random.default_rng(9)
    new = [int(x) for x in g.integers(1, 40, size=400)]
    lens = [n + int(x) for n, x in zip(new, g.integers(0, 60, size=400))]
    first = []
    for b, (L, n) in enumerate(zip(lens, new)):
        first += [INT_MAX] * n if b % 2 else [int(g.integers(0, L - n + i + 2)) for i in range(n)]
    c = U.Cache(lens, 2, 64, seed=9)
    table = unseen(c, lens, new, 0, None, first, "ids")
    q = randn(10, sum(new), 4, 64)
    status = ints([0])
    out = pda.paged_prefill_attention(q.cuda(), c.k_cache, c.v_cache, table, ints(lens), cum(new), max(new), 0.1, first_keys=ints(first), status=status)
    assert int(status.item()) == 0
    U.check(out, *U.reference(c, q, new, 0.1, first=first))


# ---- sums that are joined ---------------------------------------------------------------------------

@pytest.mark.parametrize("shape", ["plain", "bias", "e4m3"])
@pytest.mark.parametrize("L", [300, 4000])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_equal_scores_of_2_28_in_different_shares(shape, L, sign):
    """The largest score stands twice, in shares of the keys that are joined afterwards (the halves of a block, or parts of it): both
    weigh the same. In one of them a score that is less by one step came first, and the sums are relative to that one."""
    D, fp8, hidden = 128, shape == "e4m3", -15 * 2 ** 25
    # z = c s passes 2^28 from a score to the next one, 32 further on
    for scale in np.arange(0.6925, 0.6929, 1e-7, dtype=np.float32):
        factor = float(np.float32(1.4426950408889634 * float(scale)))
        top = -(-int(2 ** 28 / factor) // 32) * 32
        if 0 <= top * factor - 2 ** 28 < 4 and (top - 32) * factor < 2 ** 28 - 20:
            break
    else:
        raise AssertionError("no such scale")
    where = {10: top - 32, 100: top, L - 5: top} if sign > 0 else {10: -top, 100: 32 - top, L - 5: 32 - top}
    # products that add up to a score exactly: digits to the base 16 of score / 32 as keys, their places' values as the query
    c = U.Cache([L], 1, D, seed=2)
    rows = torch.zeros(c.k_cache.shape)
    for j in range(L):
        s = abs(where.get(j, hidden)) // 32
        for d in range(6):
            rows[int(c.table[0, j // 16]), 0, j % 16, d] = (s >> 4 * d & 15) * (1 if where.get(j, hidden) > 0 else -1)
    values = torch.where(c.v_cache.cpu().isnan(), 0.0, c.v_cache.cpu().float())
    q = torch.zeros((3, 2, D), dtype=torch.bfloat16)
    q[:, :, :6] = torch.tensor([32.0 * 16 ** d for d in range(6)])
    dtype, kw = (U.E4M3, dict(k_scale=torch.ones((rows.shape[0], 1), device="cuda"), v_scale=torch.ones((rows.shape[0], 1), device="cuda"))) if fp8 else (torch.bfloat16, {})
    if shape == "bias":
        kw["slopes"] = torch.zeros(2, device="cuda")
    k_cache, v_cache = rows.to(dtype).cuda(), values.to(dtype).cuda()
    out = pda.paged_prefill_attention(q.cuda(), k_cache, v_cache, c.dev_table, ints([L]), ints([0, 3]), 3, float(scale), **kw)
    host = v_cache.cpu().double()
    a, b = (host[int(c.table[0, j // 16]), 0, j % 16] for j in (100, L - 5))
    ref = ((a + b) / 2)[None, None].expand(3, 2, D)
    # the third score weighs 2^-30 of the others at most
    U.check(out, ref, 1.01 * (U.EPS * ref.abs() + (2 * U.EPS + L * 2.0 ** -24 + 2.0 ** -12) * ((a.abs() + b.abs()) / 2)[None, None]) + 2.0 ** -24, "joined")


# ---- e4m3 decoding: value scales of any size --------------------------------------------------------

@pytest.mark.parametrize("vscale", [2.0 ** -8, 2.0 ** -14, 2.0 ** -22, 2.0 ** -40, 2.0 ** -90, 2.0 ** 8, 2.0 ** 40, "pages"])
@pytest.mark.parametrize("kw", [dict(), dict(softcap=20.0), dict(slopes=[0.02, 0.0, 0.3, 0.001])])
def test_decode_value_scales_of_any_size(vscale, kw):
    """Weights are held in 16 bits together with the value scale: relative to the largest of the products."""
    lens, Hq, Hkv, D = [1, 17, 300, 3000], 4, 2, 128
    c = U.Cache(lens, Hkv, D, fp8=True, seed=11)
    g = np.random.default_rng(12)
    per_page = torch.as_tensor(2.0 ** g.uniform(-60, 20, size=c.v_scale.shape) if vscale == "pages" else np.full(c.v_scale.shape, vscale)).float()
    if vscale == "pages":
        per_page[::3] = 0.0                        # (pages of zeros may have any scale)
    stored = c.scales[1]
    for b, L in enumerate(lens):
        pages = torch.as_tensor(c.table[b].astype(np.int64))[torch.arange(L) // 16]
        c.v[b] = c.v[b] / stored[pages].double()[:, :, None] * per_page[pages].double()[:, :, None]
    c.v_scale = per_page.cuda()
    q = randn(13, len(lens), Hq, D, scale=2.0)
    scale = D ** -0.5
    dev = dict(kw, slopes=torch.tensor(kw["slopes"], device="cuda")) if "slopes" in kw else kw
    status = ints([0])
    for chunk in (0, 64):
        parts = dict(chunk_tokens=64, part_o=nan(4, Hq, 47, D), part_lse=nan(4, Hq, 47), workspace=pda.new_workspace(4, Hkv)) if chunk else {}
        out = pda.paged_biased_decode_attention(q.cuda(), c.k_cache, c.v_cache, c.dev_table, ints(lens), scale, status=status, **c.args(), **dev, **parts)
        assert int(status.item()) == 0
        for b, L in enumerate(lens):
            pages = torch.as_tensor(c.table[b].astype(np.int64))[torch.arange(L) // 16]
            dist = (L - 1 - torch.arange(L)).double()
            for h in range(Hq):
                k, v = c.k[b][:, h // 2], c.v[b][:, h // 2]
                ref, tol = U.attend(q[b:b + 1, h], k, v, torch.tensor([0]), torch.tensor([L]), torch.tensor([L - 1]), scale, kw.get("softcap", 0.0),
                                    0.0 if "slopes" not in kw else float(dev["slopes"][h]))
                # each product w_j scale_j off by half a step of 2^-24 of the largest such product, times the byte
                s = (q[b, h].double() @ k.T) * scale
                s = kw["softcap"] * torch.tanh(s / kw["softcap"]) if "softcap" in kw else s
                w = torch.softmax(s - (0.0 if "slopes" not in kw else float(dev["slopes"][h])) * dist, 0)
                product = w * per_page[pages, h // 2].double()
                byte = torch.where(per_page[pages, h // 2][:, None] > 0, v / per_page[pages, h // 2].double()[:, None], 0.0).abs()
                step = 2.0 ** -25 * product.max() * byte.sum(0, keepdim=True) * 1.01
                U.check(out[b:b + 1, h], ref, tol + step + 1e-38, f"{vscale} sequence {b} head {h} chunk {chunk}")


@pytest.mark.parametrize("vscale", [1.0, 2.0 ** -30])
def test_low_rows_of_small_heads(vscale):
    steps = [-1.0] * 100 + [0.0] * 30 + [1.0] + [-1.0] * 170
    for cap in (30.0, 50.0):
        U.check(*signed_prompt(False, cap, vscale, steps, 300, D=64))
        U.check(*signed_prompt(False, cap, vscale, [-1.0] * 400, 5, first=[0, 390, 200, 0, INT_MAX], D=64))


def test_captured_calls_with_low_rows_and_rows_that_see_nothing():
    """Replayed as they were captured, and with other lengths, masks and queries in the same buffers."""
    L, n = 900, 300
    c = U.Cache([L], 2, 128, seed=21)
    q, lens, cu = randn(22, n, 8, 128, scale=8.0).cuda(), ints([L]), ints([0, n])
    first = ints([INT_MAX if i % 7 == 3 else i for i in range(n)])
    ws, out = pda.prefill_workspace(8, 128), torch.empty((n, 8, 128), dtype=torch.bfloat16, device="cuda")
    call = lambda o: pda.paged_prefill_attention(q, c.k_cache, c.v_cache, c.dev_table, lens, cu, n, 0.5, softcap=50.0, first_keys=first, workspace=ws, out=o)
    call(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for step in range(3):
        if step:
            q.copy_(randn(23 + step, n, 8, 128, scale=8.0))
            lens.fill_(L - 100 * step)
            cu.copy_(ints([0, n - 50 * step]))
        out.fill_(7.0)
        graph.replay()
        want = torch.full_like(out, 7.0)
        call(want)
        assert torch.equal(out, want)
