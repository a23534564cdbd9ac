"""The rotating cache append and attention with shaped scores on the GPU, against plain references in 64 bits."""
import numpy as np
import pytest
import torch

import shaped_util as U
from paper_2605_06068_b200 import binding as pda

pytestmark = pytest.mark.gpu

GENERIC = pda.PDA_FLAG_FORCE_GENERIC


def randn(seed, *shape, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(torch.bfloat16)


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def cum(n):
    return ints([0] + list(np.cumsum(n)))


# ---- append ----------------------------------------------------------------------------------------

def table_of(positions, rot, theta=10000.0):
    half = rot // 2
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * theta ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


def run_append(T, Hq, Hkv, D, rot, seed=0, fp8=False, norm=True, interleaved=False, axes=1, lens=None, skip=(), in_place=False,
               layout="head", packed=True, eps=1e-6):
    """Sequences ``lens`` = [(context, new), ...] one behind the other (or T single tokens), slots of permuted pages."""
    g = np.random.default_rng(seed)
    if lens is None:
        lens = [(int(g.integers(0, 300)), 1) for _ in range(T)]
    assert sum(n for _, n in lens) == T
    need = [-(-(c + n) // 16) for c, n in lens]
    n_pages = sum(need) + 2
    perm = g.permutation(n_pages)
    slots, pos, at = [], [], 0
    for (c, n), m in zip(lens, need):
        pages = perm[at:at + m]
        at += m
        slots += [int(pages[j // 16]) * 16 + j % 16 for j in range(c, c + n)]
        pos += list(range(c, c + n))
    for t in skip:
        slots[t] = -1
    P = max(700, max(pos) + 1)
    table = table_of(P, rot)
    if axes > 1:
        pos = g.integers(0, P, size=(axes, T))
        axis = [int(a) for a in g.integers(0, axes, size=rot // 2)]
        at_pos = torch.as_tensor(pos)[torch.tensor(axis)].T
    else:
        axis = None
        at_pos = torch.as_tensor(np.array(pos))[:, None].expand(-1, rot // 2)
    col = torch.arange(rot // 2)[None, :]
    cos, sin = table[at_pos, col], table[at_pos, rot // 2 + col]
    heads = Hq + 2 * Hkv
    qkv = randn(seed + 1, T, heads, D, scale=2.0)
    parts = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    weights = [randn(seed + 2 + i, D, scale=0.3) + 1 if norm else None for i in range(2)]
    dev = qkv.cuda()
    q, k, v = dev[:, :Hq], dev[:, Hq:Hq + Hkv], dev[:, Hq + Hkv:]
    if not packed:
        q, k, v = (x.permute(1, 0, 2).contiguous().permute(1, 0, 2) for x in (q, k, v))     # [heads, tokens, D] storage
    store = torch.uint8 if fp8 else torch.int16
    raw = torch.randint(0, 100, (2, n_pages, Hkv, 16, D), dtype=store, generator=torch.Generator().manual_seed(seed))
    before = raw.clone()
    caches = [raw[i].permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3) if layout == "slot" else raw[i].cuda() for i in range(2)]
    if not fp8:
        caches = [c.view(torch.bfloat16) for c in caches]
    scales = [torch.rand((n_pages, Hkv), generator=torch.Generator().manual_seed(seed + 9)) * 0.02 + 0.01 for _ in range(2)] if fp8 else [None] * 2
    dev_scales = [s if s is None else s.cuda() for s in scales]
    out = q if in_place else torch.full((T, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    status = ints([0])
    got = pda.rope_kv_append(q, k, v, ints(pos) if rot else None, table.cuda() if rot else None, *caches, ints(slots),
                             q_norm=None if not norm else weights[0].cuda(), k_norm=None if not norm else weights[1].cuda(), eps=eps,
                             interleaved=interleaved, freq_axis=axis, out=out, k_scale=dev_scales[0], v_scale=dev_scales[1], status=status)
    torch.cuda.synchronize()
    assert got is out and int(status.item()) == 0
    live = [t for t in range(T) if slots[t] >= 0]
    ref_q, size_q = U.rotate(parts[0], weights[0], eps, cos, sin, rot, interleaved)
    ref_k, size_k = U.rotate(parts[1], weights[1], eps, cos, sin, rot, interleaved)
    # half a step of bf16 and, relative to the operands, 2^-20 of 32-bit arithmetic (the norm's sum, two products, a sum)
    tol = lambda ref, size: U.EPS * ref.abs() + 2.0 ** -20 * size + 1e-37
    U.check(out[live], ref_q[live], tol(ref_q, size_q)[live], "q")
    for t in skip:
        want = parts[0][t] if in_place else torch.full((Hq, D), 7.0, dtype=torch.bfloat16)
        assert torch.equal(out[t].cpu(), want)
    untouched = torch.ones((n_pages, 16), dtype=torch.bool)
    page, slot = torch.tensor([slots[t] // 16 for t in live]), torch.tensor([slots[t] % 16 for t in live])
    if live:
        untouched[page, slot] = False
    for i, (rows, size) in enumerate(((ref_k, size_k), (parts[2].double(), parts[2].double().abs()))):
        host = caches[i].cpu()
        same = host.view(store).permute(0, 2, 1, 3)[untouched] == before[i].permute(0, 2, 1, 3)[untouched]
        assert same.all(), "slots that are not in the map were written"
        if not live:
            continue
        here = host[page, :, slot]
        if not fp8:
            if i == 1:
                assert torch.equal(here.view(torch.int16), parts[2][live].view(torch.int16)), "v"
            U.check(here, rows[live], tol(rows, size)[live], "k v"[2 * i])
            continue
        scale = scales[i].double().clone()
        for t in live:
            if slots[t] % 16 == 0:
                top = rows[t].abs().amax(-1)
                scale[slots[t] // 16] = torch.where(top > 0, top * 2 / 448, 1.0)
        got_scale = dev_scales[i].cpu().double()
        assert ((got_scale - scale).abs() <= 2.0 ** -18 * scale).all(), "scales"
        ratio = (rows[live] / scale[page][:, :, None]).clamp(-448, 448)
        bytes_ = here.view(U.E4M3).double()
        # half a step of e4m3 (2^-4 of a normal value, 2^-10 of a subnormal one) and the ratio's 32-bit error
        bound = 2.0 ** -4 * ratio.abs() + 2.0 ** -10 + 2.0 ** -16 * (ratio.abs() + size[live] / scale[page][:, :, None])
        U.check(bytes_, ratio, bound, "k v"[2 * i] + " bytes")


@pytest.mark.parametrize("Hq,Hkv,D,rot", [(32, 8, 128, 128), (8, 1, 64, 64), (14, 2, 64, 32), (28, 4, 128, 64), (5, 5, 96, 96),
                                          (8, 4, 256, 256), (3, 1, 32, 32), (16, 2, 192, 48), (2, 2, 160, 0), (1, 1, 224, 16)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_heads_and_dims(Hq, Hkv, D, rot, interleaved):
    run_append(37, Hq, Hkv, D, rot, seed=D + rot, interleaved=interleaved, skip=(5, 36), layout="slot" if Hq % 2 else "head")


@pytest.mark.parametrize("T", [1, 2, 63, 1000])
@pytest.mark.parametrize("norm", [False, True])
def test_append_lengths(T, norm):
    run_append(T, 32, 8, 128, 128, seed=T, norm=norm, lens=[(3, T)])


def test_append_layouts_and_in_place():
    run_append(50, 12, 4, 128, 128, seed=1, packed=False, layout="slot")
    run_append(50, 12, 4, 128, 64, seed=2, in_place=True, skip=(0, 7), interleaved=True)
    run_append(50, 12, 4, 64, 64, seed=3, packed=False, in_place=True)


@pytest.mark.parametrize("axes", [2, 3, 4])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_axes(axes, interleaved):
    run_append(90, 12, 4, 128, 128, seed=axes, axes=axes, interleaved=interleaved, lens=[(0, 40), (17, 50)])


@pytest.mark.parametrize("D,rot,norm,interleaved", [(128, 128, True, False), (128, 64, False, True), (64, 64, False, False), (96, 32, True, False), (256, 256, True, True)])
def test_append_e4m3(D, rot, norm, interleaved):
    """Pages opened by the call and by earlier ones, sequences that begin and end inside pages."""
    run_append(200, 10, 3, D, rot, seed=D, fp8=True, norm=norm, interleaved=interleaved, lens=[(0, 1), (15, 2), (16, 1), (5, 100), (0, 64), (33, 20), (48, 12)])
    run_append(9, 8, 2, D, rot, seed=D + 1, fp8=True, norm=norm, interleaved=interleaved, layout="slot", skip=(3,))


def test_append_e4m3_axes_and_zero_rows():
    run_append(64, 8, 2, 128, 128, seed=4, fp8=True, axes=3, lens=[(0, 64)])
    T, D = 20, 128
    z = torch.zeros((T, 4, D), dtype=torch.bfloat16, device="cuda")
    cache = torch.full((2, 2, 1, 16, D), 0x55, dtype=torch.uint8, device="cuda")
    scale = torch.full((2, 2, 1), 9.0, device="cuda")
    pda.rope_kv_append(z[:, :2], z[:, 2:3], z[:, 3:], None, None, cache[0], cache[1], ints(range(T)), k_scale=scale[0], v_scale=scale[1])
    assert (scale == 1).all() and (cache[:, 0] == 0).all() and (cache[:, 1, :, :4] == 0).all() and (cache[:, 1, :, 4:] == 0x55).all()


@pytest.mark.parametrize("fp8", [False, True])
def test_append_matches_the_plain_append(fp8):
    """Without norm and rotation the rows are those that the framework's own append writes, bit for bit."""
    B, n, Hkv, D = 3, 21, 4, 128
    lens = [21, 40, 37]
    g = np.random.default_rng(0)
    table = ints(g.permutation(12)[:9].reshape(3, 3))
    k, v, q = randn(1, B, n, Hkv, D).cuda(), randn(2, B, n, Hkv, D).cuda(), randn(3, B * n, 8, D).cuda()
    make = lambda: [torch.zeros((12, Hkv, 16, D), dtype=torch.uint8 if fp8 else torch.bfloat16, device="cuda") for _ in range(2)]
    scales = lambda: [torch.full((12, Hkv), 0.03, device="cuda") for _ in range(2)]
    a, b, sa, sb = make(), make(), scales(), scales()
    if fp8:
        pda.kv_append_tokens_fp8(k, v, *a, *sa, table, ints(lens))
    else:
        pda.kv_append_tokens(k, v, *a, table, ints(lens))
    host = table.cpu().numpy()
    slots = [int(host[s, j // 16]) * 16 + j % 16 for s, L in enumerate(lens) for j in range(L - n, L)]
    out = pda.rope_kv_append(q, k.flatten(0, 1), v.flatten(0, 1), None, None, *b, ints(slots), k_scale=sb[0] if fp8 else None, v_scale=sb[1] if fp8 else None)
    for x, y in zip(a + sa, b + sb):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    assert torch.equal(out, q)


def test_append_bad_positions_and_slots():
    T, D = 6, 64
    x = randn(1, T, 4, D).cuda()
    cache = [torch.zeros((2, 1, 16, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    status, out = ints([0]), torch.full((T, 2, D), 7.0, dtype=torch.bfloat16, device="cuda")
    args = lambda pos, slots: (x[:, :2], x[:, 2:3], x[:, 3:], ints(pos), table_of(10, D).cuda(), *cache, ints(slots))
    pda.rope_kv_append(*args([0, 10, -1, 3, 2 ** 31 - 1, 9], [0, 1, 2, -1, 4, 5]), out=out, status=status)
    assert int(status.item()) == 2                               # PDA_DEV_BAD_SEQ_LEN
    assert (out[[1, 2, 4]] == 0).all() and (out[3] == 7).all() and (out[[0, 5]] != 0).any()
    assert (cache[0][0, 0, [1, 2, 3, 4]] == 0).all() and torch.equal(cache[1][0, 0, 5], x[5, 3])
    status.zero_()
    pda.rope_kv_append(*args([0] * 6, [31, 32, 2 ** 31 - 1, -5, 6, 7]), out=out, status=status)
    assert int(status.item()) == 1                               # PDA_DEV_BAD_PAGE
    assert torch.equal(cache[1][1, 0, 15], x[0, 3]) and torch.equal(out[:3], x[:3, :2])
    assert (out[3] == 7).all()


# ---- decode ----------------------------------------------------------------------------------------

def run_decode(lens, Hq, Hkv, D, seed=0, fp8=False, softcap=0.0, slopes=None, window=0, first=None, chunk=0, workspace=True, flags=0,
               layout="head", scale=None, spread=2.0):
    c = U.Cache(lens, Hkv, D, fp8=fp8, seed=seed, layout=layout)
    B = len(lens)
    q = randn(seed + 1, B, Hq, D, scale=spread)
    scale = D ** -0.5 if scale is None else scale
    kw = {}
    if chunk:
        mc = max(1, pda.max_chunks(max(max(lens), 1), chunk))
        nan = lambda *s: torch.full(s, float("nan"), device="cuda")
        kw = dict(chunk_tokens=chunk, part_o=nan(B, Hq, mc, D), part_lse=nan(B, Hq, mc),
                  workspace=pda.new_workspace(B, Hkv * -(-(Hq // Hkv) // 8)) if workspace else None)
    status = ints([0])
    dev_slopes = None if slopes is None else torch.tensor(slopes, dtype=torch.float32, device="cuda")
    dev_first = None if first is None else ints(first)
    for _ in range(2 if chunk else 1):          # (the second call finds the workspace as the first left it)
        out = torch.full((B, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        got = pda.paged_biased_decode_attention(q.cuda(), c.k_cache, c.v_cache, c.dev_table, ints(lens), scale, softcap=softcap,
                                                slopes=dev_slopes, window=window, first_keys=dev_first, out=out, flags=flags,
                                                status=status, **c.args(), **kw)
        assert got is out and int(status.item()) == 0
        ref, tol = U.reference(c, q, [1] * B, scale, softcap, None if slopes is None else dev_slopes.cpu().double(), window, None, first, decode=True)
        U.check(out, ref, tol, f"chunk {chunk}")
    if chunk and workspace:
        assert int(kw["workspace"].abs().sum().item()) == 0


LENS = [1, 2, 15, 16, 17, 63, 64, 65, 129, 500, 0, 1000]


@pytest.mark.parametrize("Hq,Hkv,D,fp8", [(32, 8, 128, False), (8, 8, 64, False), (7, 1, 128, False), (8, 2, 256, False), (28, 4, 128, True),
                                          (20, 1, 128, False), (24, 2, 64, False), (6, 2, 96, False), (4, 2, 64, True), (12, 1, 256, True)])
@pytest.mark.parametrize("shape", ["plain", "cap", "slopes", "cap+slopes"])
def test_decode_shapes(Hq, Hkv, D, fp8, shape):
    kw = dict(softcap=7.0 if "cap" in shape else 0.0, slopes=[0.5 ** (h % 9 + 1) for h in range(Hq)] if "slopes" in shape else None)
    run_decode(LENS, Hq, Hkv, D, seed=Hq + D, fp8=fp8, **kw)


@pytest.mark.parametrize("Hq,Hkv,D,fp8", [(32, 8, 128, False), (20, 2, 64, False), (8, 2, 256, False), (28, 4, 128, True)])
@pytest.mark.parametrize("chunk,workspace", [(16, True), (64, True), (64, False), (2048, True)])
def test_decode_split(Hq, Hkv, D, fp8, chunk, workspace):
    run_decode(LENS, Hq, Hkv, D, seed=chunk, fp8=fp8, softcap=5.0, slopes=[0.01 * h for h in range(Hq)], window=100, chunk=chunk, workspace=workspace)


@pytest.mark.parametrize("flags", [0, GENERIC])
@pytest.mark.parametrize("chunk", [0, 64])
def test_decode_masks(flags, chunk):
    first = [0, 1, 20, 16, 5, 62, 64, -3, 128, 499, 3, 2 ** 31 - 1]      # (some see nothing)
    run_decode(LENS, 16, 4, 128, seed=3, first=first, chunk=chunk, flags=flags)
    run_decode(LENS, 16, 4, 128, seed=4, first=first, window=33, softcap=30.0, chunk=chunk, flags=flags)
    run_decode(LENS, 16, 4, 128, seed=5, window=1, chunk=chunk, flags=flags)


def test_decode_layouts_scales_and_generic():
    run_decode(LENS, 16, 4, 128, seed=6, layout="slot", softcap=50.0)
    run_decode(LENS, 16, 4, 128, seed=7, scale=-0.1)
    run_decode(LENS, 16, 4, 128, seed=8, scale=0.0, softcap=3.0)
    run_decode(LENS, 16, 4, 128, seed=9, flags=GENERIC, softcap=4.0, slopes=[0.1 * h for h in range(16)])
    run_decode(LENS, 16, 4, 128, seed=9, flags=GENERIC, fp8=True, softcap=4.0, window=77)
    run_decode([700, 3000], 8, 2, 128, seed=10, softcap=2.0, scale=3.0)        # far into the cap


def test_decode_without_shapes_is_decode():
    """Nothing capped, biased or masked: the bits of paged_decode_attention."""
    c = U.Cache(LENS, 8, 128, seed=1)
    q = randn(2, len(LENS), 32, 128).cuda()
    a = pda.paged_biased_decode_attention(q, c.k_cache, c.v_cache, c.dev_table, ints(LENS), 0.1)
    b = pda.paged_decode_attention(q, c.k_cache, c.v_cache, c.dev_table, ints(LENS), 0.1)
    assert torch.equal(a, b)


def test_decode_bad_pages_and_lengths():
    lens = [100, 100, 100]
    for flags in (0, GENERIC):
        c = U.Cache(lens, 2, 128, seed=1)
        q = randn(2, 3, 8, 128).cuda()
        good = pda.paged_biased_decode_attention(q, c.k_cache, c.v_cache, c.dev_table, ints(lens), 0.1, softcap=5.0, flags=flags)
        status = ints([0])
        c.dev_table[1, 3] = c.k_cache.shape[0]
        out = pda.paged_biased_decode_attention(q, c.k_cache, c.v_cache, c.dev_table, ints(lens), 0.1, softcap=5.0, status=status, flags=flags)
        assert int(status.item()) == 1 and (out[1] == 0).all() and torch.equal(out[[0, 2]], good[[0, 2]])
        out = pda.paged_biased_decode_attention(q, c.k_cache, c.v_cache, c.dev_table, ints(lens), 0.1, softcap=5.0, window=30, status=ints([0]), flags=flags)
        assert (out[1] != 0).any()                                 # (the page is before the window: it is not looked at)
        status.zero_()
        out = pda.paged_biased_decode_attention(q, c.k_cache, c.v_cache, c.dev_table, ints([100, 100, 1 << 20]), 0.1, softcap=5.0, status=status, flags=flags)
        assert int(status.item()) == 2 and (out[2] == 0).all() and torch.equal(out[0], good[0])


def test_decode_nan_and_infinite_scores():
    lens = [200, 200, 200, 200]
    for flags in (0, GENERIC):
        for chunk in (0, 64):
            c = U.Cache(lens, 1, 128, seed=1)
            kw = {}
            if chunk:
                kw = dict(chunk_tokens=64, part_o=torch.empty((4, 8, 4, 128), device="cuda"), part_lse=torch.empty((4, 8, 4), device="cuda"), workspace=pda.new_workspace(4, 1))
            q = randn(2, 4, 8, 128).abs().cuda()
            call = lambda **k: pda.paged_biased_decode_attention(q, c.k_cache, c.v_cache, c.dev_table, ints(lens), 0.1, softcap=5.0, flags=flags, **kw, **k)
            good = call()
            rows = c.k_cache[:, 0]
            at = lambda b, j: (int(c.table[b, j // 16]), j % 16)
            rows[at(1, 70)] = float("nan")
            rows[at(2, 70)] = float("inf")                         # (capped: a score of 5)
            rows[at(3, 70)] = float("-inf")
            out = call()
            assert torch.equal(out[0], good[0]) and out[1].isnan().all() and out[2:].isfinite().all()
            out = call(window=200 - 71)                            # (it is not seen)
            assert out.isfinite().all()
            nocap = pda.paged_biased_decode_attention(q, c.k_cache, c.v_cache, c.dev_table, ints(lens), 0.1, flags=flags, **kw)
            assert nocap[0].isfinite().all() and nocap[1].isnan().all() and nocap[2].isnan().all() and nocap[3].isfinite().all()


# ---- prompts ---------------------------------------------------------------------------------------

def run_prefill(new, ctx, Hq, Hkv, D, seed=0, fp8=False, softcap=0.0, slopes=None, window=0, prefix=None, first=None, flags=0,
                layout="head", scale=None, spread=2.0, q_layout="packed", out_pad=0, gap=0, loose=0, workspace=True):
    """``gap`` rows of q and out before, between and behind the sequences that belong to none."""
    lens = [n + c for n, c in zip(new, ctx)]
    c = U.Cache(lens, Hkv, D, fp8=fp8, seed=seed, layout=layout)
    T = sum(new)
    q = randn(seed + 1, T, Hq, D, scale=spread)
    scale = D ** -0.5 if scale is None else scale
    dev_slopes = None if slopes is None else torch.tensor(slopes, dtype=torch.float32, device="cuda")
    qd = q.cuda()
    if q_layout == "heads":
        qd = qd.permute(1, 0, 2).contiguous().permute(1, 0, 2)
    elif q_layout == "buffer":
        big = torch.full((T, Hq + 3, D + 16), float("nan"), dtype=torch.bfloat16, device="cuda")
        big[:, 1:Hq + 1, 8:D + 8] = qd
        qd = big[:, 1:Hq + 1, 8:D + 8]
    buf = torch.full((T, Hq, D + out_pad), 7.0, dtype=torch.bfloat16, device="cuda")
    out = buf[:, :, :D]
    status = ints([0])
    got = pda.paged_prefill_attention(qd, c.k_cache, c.v_cache, c.dev_table, ints(lens), cum(new), max(new + [0]) + loose, scale, softcap=softcap,
                                      slopes=dev_slopes, window=window, prefix_lens=None if prefix is None else ints(prefix),
                                      first_keys=None if first is None else ints(first), out=out, flags=flags, status=status, **c.args())
    torch.cuda.synchronize()
    assert got is out and int(status.item()) == 0
    ref, tol = U.reference(c, q, new, scale, softcap, None if slopes is None else dev_slopes.cpu().double(), window, prefix, first)
    U.check(out, ref, tol)
    assert (buf[:, :, D:] == 7).all()
    return out


NEW = [1, 5, 0, 33, 64, 130, 300]
CTX = [0, 20, 40, 0, 127, 200, 3]


@pytest.mark.parametrize("Hq,Hkv,D,fp8", [(8, 2, 128, False), (4, 4, 128, False), (7, 1, 64, False), (16, 1, 128, False), (8, 2, 128, True),
                                          (6, 2, 64, False), (3, 1, 96, False), (2, 1, 256, False), (4, 2, 64, True), (10, 2, 128, True)])
@pytest.mark.parametrize("shape", ["plain", "cap", "slopes", "cap+slopes"])
def test_prefill_shapes(Hq, Hkv, D, fp8, shape):
    kw = dict(softcap=7.0 if "cap" in shape else 0.0, slopes=[0.5 ** (h % 9 + 1) for h in range(Hq)] if "slopes" in shape else None)
    run_prefill(NEW, CTX, Hq, Hkv, D, seed=Hq + D, fp8=fp8, **kw)


@pytest.mark.parametrize("flags", [0, GENERIC])
@pytest.mark.parametrize("fp8", [False, True])
def test_prefill_masks(flags, fp8):
    g = np.random.default_rng(0)
    T = sum(NEW)
    prefix = [0, 7, 40, 33, 1000, 250, 150]
    docs = []
    for n, c in zip(NEW, CTX):
        docs += [(p // 37) * 37 for p in range(c, c + n)]
    for i, kw in enumerate((dict(window=1), dict(window=50), dict(window=128, softcap=6.0), dict(prefix=prefix), dict(first=docs),
                            dict(prefix=prefix, first=docs, window=60, slopes=[0.1 * h for h in range(8)]),
                            dict(first=list(g.integers(-5, 400, size=T)), prefix=prefix, softcap=3.0))):
        run_prefill(NEW, CTX, 8, 2, 128, seed=20 + i, flags=flags, fp8=fp8, **kw)


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 127, 128, 129, 255, 256, 257, 511, 513, 1000])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (8, 2), (5, 1)])
def test_prefill_lengths(n, Hq, Hkv):
    run_prefill([n], [0], Hq, Hkv, 128, seed=n)
    run_prefill([n, n], [16 * (n % 5), 333], Hq, Hkv, 64, seed=n + 1, softcap=20.0)


def test_prefill_layouts():
    run_prefill(NEW, CTX, 8, 2, 128, seed=1, layout="slot", q_layout="heads", out_pad=8)
    run_prefill(NEW, CTX, 6, 2, 64, seed=2, q_layout="buffer", out_pad=64, loose=1000)
    run_prefill(NEW, CTX, 8, 2, 128, seed=3, scale=-0.2)
    run_prefill(NEW, CTX, 8, 2, 128, seed=4, scale=0.0, slopes=[0.3] * 8)
    run_prefill([200, 300], [0, 100], 8, 2, 128, seed=5, softcap=2.0, scale=3.0)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("kw", [dict(scale=0.0), dict(scale=1e-30), dict(scale=-0.1), dict(softcap=4.0), dict(scale=0.0, softcap=4.0)])
def test_prefill_bias_within_a_prefix(fp8, kw):
    """Keys behind the token itself, by their distance, whatever the products weigh; slopes of either sign."""
    run_prefill([150, 40], [30, 200], 4, 2, 128, seed=9, fp8=fp8, prefix=[170, 240], slopes=[0.3, 0.0, -0.02, 0.05], **kw)


def test_prefill_many_small_and_few_long():
    g = np.random.default_rng(5)
    run_prefill(list(g.integers(0, 40, size=300)), list(g.integers(0, 100, size=300)), 4, 2, 64, seed=6, softcap=10.0)
    run_prefill([1, 3, 20], [3000, 5000, 7001], 8, 2, 128, seed=7)
    run_prefill([16], [9000], 8, 1, 128, seed=8, softcap=30.0, window=4000)


def test_prefill_more_query_tokens_than_keys():
    """A chunk longer than its sequence: its first rows stand before the sequence and see nothing."""
    for flags in (0, GENERIC):
        c = U.Cache([20, 0, 150], 2, 128, seed=1)
        new = [50, 10, 200]
        q = randn(2, sum(new), 4, 128)
        for prefix in (None, [20, 3, 100]):
            out = pda.paged_prefill_attention(q.cuda(), c.k_cache, c.v_cache, c.dev_table, ints([20, 0, 150]), cum(new), 200, 0.1, flags=flags,
                                              prefix_lens=None if prefix is None else ints(prefix))
            U.check(out, *U.reference(c, q, new, 0.1, prefix=prefix))
            assert (out[:30] == 0).all() and (out[50:60] == 0).all()
        for window in (2 ** 31 - 1, 2 ** 31 - 30, 1):
            out = pda.paged_prefill_attention(q.cuda(), c.k_cache, c.v_cache, c.dev_table, ints([20, 0, 150]), cum(new), 200, 0.1, flags=flags, window=window)
            U.check(out, *U.reference(c, q, new, 0.1, window=window))


def test_prefill_rows_outside_the_sequences():
    """Rows before the first and behind the last sequence stay as they were, whatever q holds there."""
    for flags in (0, GENERIC):
        c = U.Cache([60, 70], 2, 128, seed=1)
        q = randn(2, 140, 4, 128)
        qd = q.cuda()
        qd[:20] = float("nan")
        qd[60:] = float("inf")
        out = torch.full((140, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        pda.paged_prefill_attention(qd, c.k_cache, c.v_cache, c.dev_table, ints([60, 70]), ints([20, 50, 60]), 30, 0.1, out=out, softcap=9.0, flags=flags)
        assert (out[:20] == 7).all() and (out[60:] == 7).all()
        U.check(out[20:60], *U.reference(c, q[20:60], [30, 10], 0.1, softcap=9.0))


def test_prefill_bad_pages_and_spans():
    lens, new = [300, 300, 300], [40, 40, 40]
    for flags in (0, GENERIC):
        c = U.Cache(lens, 2, 128, seed=1)
        q = randn(2, 120, 8, 128).cuda()
        call = lambda lens=lens, cu=(0, 40, 80, 120), mq=40, **k: pda.paged_prefill_attention(q, c.k_cache, c.v_cache, c.dev_table, ints(lens), ints(cu), mq, 0.1, flags=flags, **k)
        good = call()
        status = ints([0])
        out = call(lens=[300, 1 << 24, 300], status=status)
        assert int(status.item()) == 2 and (out[40:80] == 0).all() and torch.equal(out[:40], good[:40]) and torch.equal(out[80:], good[80:])
        status.zero_()
        out = call(cu=(0, 40, 80, 200), status=status, out=torch.full_like(q, 7.0))
        assert int(status.item()) == 2 and torch.equal(out[:80], good[:80]) and (out[80:] == 0).all()
        status.zero_()
        out = call(mq=39, status=status, out=torch.full_like(q, 7.0))
        assert int(status.item()) == 2 and all((out[i:i + 39] == 0).all() for i in (0, 40, 80))
        c.dev_table[1, 3] = -1
        status.zero_()
        out = call(status=status)
        assert int(status.item()) == 1 and (out[40:80] == 0).all() and torch.equal(out[:40], good[:40]) and torch.equal(out[80:], good[80:])
        status.zero_()
        out = call(window=64, status=status)                       # (the page is before the window: it is not looked at)
        assert int(status.item()) == 0 and (out[40:80] != 0).any()


def test_prefill_nan_and_infinite_scores():
    lens, new = [200] * 4, [100] * 4
    for flags in (0, GENERIC):
        c = U.Cache(lens, 1, 128, seed=1)
        q = randn(2, 400, 8, 128).abs().cuda()
        call = lambda **k: pda.paged_prefill_attention(q, c.k_cache, c.v_cache, c.dev_table, ints(lens), cum(new), 100, 0.1, flags=flags, **k).view(4, 100, 8, 128)
        rows = c.k_cache[:, 0]
        at = lambda b, j: (int(c.table[b, j // 16]), j % 16)
        good = {kw: call(**dict(kw)) for kw in ((), (("softcap", 5.0),), (("slopes", None),))}
        rows[at(1, 150)] = float("nan")
        rows[at(2, 150)] = float("inf")
        rows[at(3, 150)] = float("-inf")
        for kw, before in good.items():
            out = call(**dict(kw))
            capped = bool(dict(kw).get("softcap"))
            assert torch.equal(out[0], before[0]) and torch.equal(out[1:, :50], before[1:, :50])     # (position 150 is not seen by rows before it)
            assert out[1, 50:].isnan().all() and out[3].isfinite().all()
            assert out[2, 50:].isfinite().all() if capped else out[2, 50:].isnan().all()


@pytest.mark.parametrize("kw", [dict(), dict(slopes=[0.3, 0.01]), dict(softcap=3.0, slopes=[0.3, 0.01]), dict(slopes=[0.0, 0.0], prefix=[400, 0, 1900])])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("how", ["prompt", "generic", "decode"])
def test_scores_whose_steps_pass_every_threshold(kw, fp8, how):
    """Products up to 2^100: one step of such a score's 32-bit form is more than any weight's exponent may be off by. Each is
    the product of one number of a query and one of a key: 80 keys a sequence have different ones of either sign, the others
    zero. The numbers that count are so far apart that only the largest has a weight, or the same, and then their weights differ
    by their biases alone; both whatever the product's rounding."""
    if how == "decode" and "prefix" in kw:
        kw = {k: v for k, v in kw.items() if k != "prefix"}
    lens, new = ([400, 70, 2000], [300, 70, 20]) if how != "decode" else ([400, 70, 2000], [1, 1, 1])
    D, scale = 128, 0.0883883
    c = U.Cache(lens, 1, D, seed=71)
    g = np.random.default_rng(72)
    k0 = []
    for L in lens:
        x = torch.zeros(L, dtype=torch.float64)
        at = torch.as_tensor(g.permutation(L)[:min(L, 80)])
        x[at] = torch.as_tensor(np.concatenate([np.arange(8, 16) * 2.0 ** e for e in range(5)] + [-np.arange(8, 16) * 2.0 ** e for e in range(5)])[:len(at)])
        k0.append(x)                                # (four bits each: 8-bit pages hold them too)
    rows = torch.zeros(c.k_cache.shape, dtype=torch.bfloat16)
    values = c.v_cache.cpu().float()
    for b, L in enumerate(lens):
        for j in range(L):
            rows[int(c.table[b, j // 16]), 0, j % 16, 0] = k0[b][j]
    k_cache, v_cache, scales = rows.cuda(), c.v_cache, {}
    if fp8:
        k_cache, v_cache = rows.float().to(U.E4M3).cuda(), torch.where(values.isnan(), 0.0, values).to(U.E4M3).cuda()
        ones = torch.full((rows.shape[0], 1), 1.0, device="cuda")
        scales = dict(k_scale=ones * 0.7, v_scale=ones)
        values = v_cache.cpu().float()
    T = sum(new)
    q = torch.zeros((T, 2, D), dtype=torch.bfloat16)
    powers = np.array([24, 27, 28, 30, 31, 33, 40, 64, 90])
    if how == "decode" and fp8:                     # (queries are held in fp16 there: the rest is the scale's)
        scale *= 2.0 ** 40
        powers = np.minimum(powers - 40, 14)
    q[:, :, 0] = torch.as_tensor(2.0 ** g.choice(powers, size=(T, 2)) * g.choice([-1.0, 1.0, 1.5, -1.25], size=(T, 2))).to(torch.bfloat16)
    host = dict(kw, slopes=torch.tensor(kw.get("slopes", [0.0, 0.0]), dtype=torch.float32))
    dev = dict(kw)
    if "slopes" in kw:
        dev["slopes"] = host["slopes"].cuda()
    if "prefix" in kw:
        dev["prefix_lens"] = ints(dev.pop("prefix"))
    status = ints([0])
    flags = GENERIC if how == "generic" else 0
    if how == "decode":
        out = pda.paged_biased_decode_attention(q.cuda(), k_cache, v_cache, c.dev_table, ints(lens), scale, status=status, **dev, **scales)
    else:
        out = pda.paged_prefill_attention(q.cuda(), k_cache, v_cache, c.dev_table, ints(lens), cum(new), max(new), scale, status=status, flags=flags, **dev, **scales)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    see = U.visible(lens, new, 0, kw.get("prefix"))
    at = 0
    for b, n in enumerate(new):
        v = torch.stack([values[int(c.table[b, j // 16]), 0, j % 16] for j in range(lens[b])]).double()
        j, pos = torch.arange(lens[b]), torch.arange(n) + (lens[b] - n)
        live = (j[None, :] >= see[b][0][:, None]) & (j[None, :] < see[b][1][:, None])
        for h in range(2):
            s = q[at:at + n, h, :1].double() * (k0[b] * (0.7 if fp8 else 1.0))[None, :] * scale
            if kw.get("softcap"):
                s = kw["softcap"] * torch.tanh(s / kw["softcap"])
            bias = float(host["slopes"][h]) * (pos[:, None] - j[None, :]).abs()
            w = torch.softmax(torch.where(live, s - bias, float("-inf")), 1)
            # 16-bit weights and result; exponents off by 2^-22 of a bias with a weight and 2^-17 of a cap; 32-bit sums
            off = 2 * ((w * bias).max(1, keepdim=True).values * 2.0 ** -22 * lens[b] + kw.get("softcap", 0.0) * 2.0 ** -17)
            # decode, 8 bits: weights times the value scale held in fp16, 2^-25 of a value each
            small = 2.0 ** -25 * (live.double() @ v.abs()) if fp8 and how == "decode" else 0.0
            tol = (3 * U.EPS + lens[b] * 2.0 ** -24 + 2.0 ** -12 + 2 * off) * (w @ v.abs()) * 1.01 + small
            U.check(out[at:at + n, h], w @ v, tol, f"sequence {b} head {h}")
        at += n


# ---- few rows and many keys: blocks cut along the keys and joined -----------------------------------

@pytest.mark.parametrize("kw", [dict(), dict(softcap=6.0), dict(slopes=[0.01, 0.2, 0.0, 0.05]), dict(softcap=30.0, slopes=[0.003] * 4, window=1500),
                                dict(prefix=[2800, 100], window=900), dict(softcap=80.0)])
@pytest.mark.parametrize("D,fp8", [(128, False), (128, True), (64, False)])
def test_prefill_cut_along_the_keys(kw, D, fp8):
    run_prefill([70, 3], [3000, 2600], 4, 1, D, seed=31, fp8=fp8, **kw)


def test_prefill_cut_with_documents():
    """Rows that see keys of some parts only, or of none."""
    first = [3000 - 40 * i for i in range(60)] + [2 ** 31 - 1, 2500] + [0] * 8
    run_prefill([70], [3000], 8, 2, 128, seed=32, first=first)
    run_prefill([70], [3000], 8, 2, 128, seed=33, first=first, softcap=9.0, fp8=True)


def test_prefill_cut_bad_pages_and_nan():
    c = U.Cache([3000, 2900], 1, 128, seed=1)
    new = [40, 30]
    q = randn(2, 70, 8, 128).abs().cuda()
    call = lambda **k: pda.paged_prefill_attention(q, c.k_cache, c.v_cache, c.dev_table, ints([3000, 2900]), cum(new), 40, 0.1, **k)
    good = call()
    U.check(good, *U.reference(c, q.cpu(), new, 0.1))
    status = ints([0])
    c.dev_table[0, 20] = -7
    out = call(status=status)
    assert int(status.item()) == 1 and (out[:40] == 0).all() and torch.equal(out[40:], good[40:])
    c.dev_table[0, 20] = int(c.table[0, 20])
    row = int(c.table[1, 2880 // 16]), 0, 0                          # token 2880 of the second sequence: seen from row 50 on
    keep = c.k_cache[row].clone()
    for value in (float("nan"), float("inf")):
        c.k_cache[row] = value
        out = call()
        assert torch.equal(out[:50], good[:50]) and out[50:].isnan().all()
        assert call(softcap=5.0)[50:].isnan().all() == (value != float("inf"))
    c.k_cache[row] = keep
    assert torch.equal(call(), good)


def test_prefill_workspaces():
    """A workspace that holds anything, none at all, and a call that is not cut behind one that is."""
    c = U.Cache([3000], 2, 128, seed=1)
    q = randn(2, 50, 8, 128).cuda()
    args = q, c.k_cache, c.v_cache, c.dev_table, ints([3000]), ints([0, 50]), 50, 0.1
    ws = pda.prefill_workspace(8, 128)
    ws.fill_(0xFF)
    a = pda.paged_prefill_attention(*args, workspace=ws)
    ws.fill_(0x7F)
    b = pda.paged_prefill_attention(*args, workspace=ws)
    assert torch.equal(a, b)
    ref, tol = U.reference(c, q.cpu(), [50], 0.1)
    U.check(a, ref, tol)
    out = torch.empty_like(q)
    desc = pda._paged_caches(c.k_cache, c.v_cache, None, None, 128)
    rc = pda.lib().paged_prefill_attention(q.data_ptr(), 1024, 128, c.k_cache.data_ptr(), c.v_cache.data_ptr(), desc, None, None,
                                           c.dev_table.data_ptr(), c.dev_table.shape[1], args[4].data_ptr(), args[5].data_ptr(), 1, 8, 50, 50,
                                           pda.ScoreDesc(0.1, 0.0, None, 0), None, None, out.data_ptr(), 1024, 128, None, 0, 0, None,
                                           torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert rc == 0
    U.check(out, ref, tol)


# ---- sizes at the ends ------------------------------------------------------------------------------

@pytest.mark.parametrize("Hq,Hkv", [(128, 1), (100, 1), (130, 1), (66, 2), (12, 4)])
def test_prefill_groups(Hq, Hkv):
    """Groups that fill a tile's rows alone, that leave rows over, and one above what the tensor-core kernel takes."""
    run_prefill([9, 1, 20], [0, 50, 130], Hq, Hkv, 64, seed=Hq, softcap=8.0)


@pytest.mark.parametrize("kw", [dict(), dict(slopes=[0.1, 0.01]), dict(softcap=5.0)])
@pytest.mark.parametrize("fp8", [False, True])
def test_prefill_many_blocks(kw, fp8):
    """More row blocks than are listed, and just fewer, of sequences of very unequal lengths; empty ones among them."""
    g = np.random.default_rng(7)
    for n, hi in ((290, 30), (255, 5), (120, 2)):
        new = [int(x) for x in g.integers(0, hi, size=n)]
        new[3], new[7] = 600, 0
        run_prefill(new, [int(x) for x in g.integers(0, 60, size=n)], 2, 1, 128, seed=n, fp8=fp8, **kw)


def test_empty_calls_and_lengths_below_zero():
    c = U.Cache([30], 2, 128, seed=1)
    e = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")
    cs = table_of(8, 128).cuda()
    assert pda.rope_kv_append(e(0, 4, 128), e(0, 2, 128), e(0, 2, 128), ints([]), cs, c.k_cache, c.v_cache, ints([])).shape == (0, 4, 128)
    assert pda.paged_prefill_attention(e(0, 4, 128), c.k_cache, c.v_cache, c.dev_table, ints([30]), ints([0, 0]), 0, 0.1).shape == (0, 4, 128)
    none = torch.empty((0, 3), dtype=torch.int32, device="cuda")
    assert pda.paged_biased_decode_attention(e(0, 4, 128), c.k_cache, c.v_cache, none, ints([]), 0.1).shape == (0, 4, 128)
    q = randn(1, 5, 4, 128).cuda()
    for flags in (0, GENERIC):
        out = pda.paged_prefill_attention(q, c.k_cache, c.v_cache, c.dev_table, ints([-4]), ints([0, 5]), 5, 0.1, prefix_lens=ints([9]), flags=flags)
        assert (out == 0).all()
        assert (pda.paged_biased_decode_attention(q[:1], c.k_cache, c.v_cache, c.dev_table, ints([-4]), 0.1, flags=flags) == 0).all()


def test_decode_cut_finer_than_asked_for():
    """Sequences that are shorter than the partial buffers allow for are cut into as many chunks, of 2048 tokens at least."""
    for kw in (dict(), dict(fp8=True, softcap=9.0, slopes=[0.001 * h for h in range(4)])):
        run_decode([9000, 5000, 300, 0, 4097, 12288], 4, 1, 128, seed=40, chunk=4096, **kw)
    run_decode([9000, 2500], 10, 1, 128, seed=41, chunk=6000 // 16 * 16, window=3000)


def test_offsets_beyond_32_bits():
    """Caches of more than 2^31 elements: the pages in use are the last ones."""
    Hkv, D, n = 8, 128, 140000
    caches = [torch.empty((n, Hkv, 16, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    assert caches[0].numel() > 2 ** 31
    L = 200
    pages = list(range(n - 13, n))
    table = ints([pages])
    slots = ints([pages[j // 16] * 16 + j % 16 for j in range(L)])
    x = randn(3, L, 16 + 2 * Hkv, D).cuda()
    q = pda.rope_kv_append(x[:, :16], x[:, 16:16 + Hkv], x[:, 16 + Hkv:], None, None, *caches, slots)
    assert torch.equal(q, x[:, :16]) and torch.equal(caches[1][pages[3], :, 5], x[53, 16 + Hkv:])
    c = U.Cache.__new__(U.Cache)
    c.lens, c.fp8, c.byte = [L], False, 0.0
    c.k, c.v = [x[:, 16:16 + Hkv].cpu().double()], [x[:, 16 + Hkv:].cpu().double()]
    out = pda.paged_prefill_attention(q, *caches, table, ints([L]), ints([0, L]), L, 0.1, softcap=9.0)
    U.check(out, *U.reference(c, q.cpu(), [L], 0.1, 9.0))
    one = pda.paged_biased_decode_attention(q[-1:].contiguous(), *caches, table, ints([L]), 0.1, softcap=9.0)
    U.check(one, *U.reference(c, q[-1:].cpu(), [1], 0.1, 9.0, decode=True))


def test_calls_on_a_given_stream():
    c = U.Cache([500], 2, 128, seed=1)
    q = randn(2, 100, 8, 128).cuda()
    args = q, c.k_cache, c.v_cache, c.dev_table, ints([500]), ints([0, 100]), 100, 0.1
    want = pda.paged_prefill_attention(*args, softcap=7.0)
    dec = pda.paged_biased_decode_attention(q[-1:].contiguous(), *args[1:5], 0.1, softcap=7.0)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    a = pda.paged_prefill_attention(*args, softcap=7.0, stream=side)      # (output and workspace belong to that stream)
    b = pda.paged_biased_decode_attention(q[-1:].contiguous(), *args[1:5], 0.1, softcap=7.0, stream=side)
    side.synchronize()
    assert torch.equal(a, want) and torch.equal(b, dec)


def test_results_do_not_depend_on_timing_or_on_other_sequences():
    """The same bits call by call; and a sequence's bits whatever its neighbours' values are."""
    lens, new = [700, 333, 90], [200, 333, 7]
    for kw in (dict(), dict(softcap=10.0), dict(slopes=torch.tensor([0.02 * h for h in range(8)], device="cuda"))):
        c = U.Cache(lens, 2, 128, seed=1)
        q = randn(2, sum(new), 8, 128, scale=3.0).cuda()
        call = lambda: pda.paged_prefill_attention(q, c.k_cache, c.v_cache, c.dev_table, ints(lens), cum(new), 333, 0.1, **kw)
        a = call()
        assert all(torch.equal(a, call()) for _ in range(5))
        q[:200] *= 100
        b = call()
        assert torch.equal(a[200:], b[200:]) and not torch.equal(a[:200], b[:200])


# ---- the operators together ------------------------------------------------------------------------

@pytest.mark.parametrize("fp8", [False, True])
def test_a_prompt_and_its_decode_steps(fp8):
    """build_tables -> rope_kv_append -> prompt attention, then single tokens, against a model layer in 64 bits. The caches'
    rounded rows are read back for the reference, so that only the attention's own error counts."""
    Hq, Hkv, D, B, cap, P = 8, 2, 128, 3, 12.0, 512
    lens = np.array([40, 77, 1])
    cos_sin = table_of(P, D).cuda()
    store = torch.uint8 if fp8 else torch.bfloat16
    caches = [torch.zeros((40, Hkv, 16, D), dtype=store, device="cuda") for _ in range(2)]
    scales = [torch.ones((40, Hkv), device="cuda") if fp8 else None for _ in range(2)]
    table, count = torch.full((B, 10), -1, dtype=torch.int32, device="cuda"), ints([40])
    free = ints(np.random.default_rng(0).permutation(40))
    new = lens.copy()
    weights = [(randn(i, D, scale=0.2) + 1).cuda() for i in (1, 2)]
    for step in range(4):
        T = int(new.sum())
        cu, slots, pos = ints([0] * (B + 1)), ints([0] * T), ints([0] * T)
        pda.paged_build_tables(ints(lens), ints(new), 16, free, count, table, cu, slots, positions=pos)
        x = randn(10 + step, T, Hq + 2 * Hkv, D, scale=2.0).cuda()
        q = pda.rope_kv_append(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], pos, cos_sin, *caches, slots, q_norm=weights[0], k_norm=weights[1],
                               k_scale=scales[0], v_scale=scales[1])
        kw = dict(softcap=cap, k_scale=scales[0], v_scale=scales[1])
        if step == 0:
            out = pda.paged_prefill_attention(q, *caches, table, ints(lens), cu, int(new.max()), 0.2, **kw)
        else:
            out = pda.paged_biased_decode_attention(q, *caches, table, ints(lens), 0.2, **kw)
        c = U.Cache.__new__(U.Cache)
        c.lens, c.fp8, c.D, c.byte = [int(x) for x in lens], fp8, D, 448.0 if fp8 else 0.0
        c.k, c.v = [], []
        host = table.cpu().long()
        for rows, cache, scale in ((c.k, caches[0], scales[0]), (c.v, caches[1], scales[1])):
            vals = (cache.view(U.E4M3) if fp8 else cache).cpu().double()
            if fp8:
                vals = vals * scale.cpu().double()[:, :, None, None]
            for b, L in enumerate(c.lens):
                j = torch.arange(L)
                rows.append(vals[host[b][j // 16], :, j % 16])
        U.check(out, *U.reference(c, q.cpu(), [int(n) for n in new], 0.2, cap, decode=step > 0))
        new = np.ones(B, dtype=int)
        lens = lens + 1


def test_other_streams_and_captured_calls():
    lens, new = [200, 300], [60, 70]
    c = U.Cache(lens, 2, 128, seed=1)
    q = randn(2, 130, 8, 128).cuda()
    pos = ints(list(range(140, 200)) + list(range(230, 300)))
    slots = ints([int(c.table[b, j // 16]) * 16 + j % 16 for b in range(2) for j in range(lens[b] - new[b], lens[b])])
    kv = randn(3, 130, 4, 128).cuda()
    ws, cs = pda.prefill_workspace(8, 128), table_of(400, 128).cuda()
    args = ints(lens), cum(new)
    parts = dict(chunk_tokens=64, part_o=torch.empty((2, 8, 5, 128), device="cuda"), part_lse=torch.empty((2, 8, 5), device="cuda"), workspace=pda.new_workspace(2, 2))
    out, rot, dec = torch.zeros_like(q), torch.zeros_like(q), torch.zeros((2, 8, 128), dtype=torch.bfloat16, device="cuda")
    qd = randn(4, 2, 8, 128).cuda()

    def step():
        pda.rope_kv_append(q, kv[:, :2], kv[:, 2:], pos, cs, c.k_cache, c.v_cache, slots, out=rot)
        pda.paged_prefill_attention(rot, c.k_cache, c.v_cache, c.dev_table, *args, 70, 0.1, softcap=8.0, out=out, workspace=ws)
        pda.paged_biased_decode_attention(qd, c.k_cache, c.v_cache, c.dev_table, args[0], 0.1, softcap=8.0, out=dec, **parts)

    step()
    torch.cuda.synchronize()
    want = [x.clone() for x in (out, rot, dec)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (out, rot, dec)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for x in (out, rot, dec):
        x.zero_()
    q.mul_(-1)
    graph.replay()
    torch.cuda.synchronize()
    assert not torch.equal(rot, want[1]) and torch.equal(rot, -want[1])
    q.mul_(-1)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (out, rot, dec)))
