"""The latent-attention operators and the step tables on the GPU, against plain references in 64 bits."""
import numpy as np
import pytest
import torch

import latent_util as U
from paper_2605_06068_b200 import binding as pda

pytestmark = pytest.mark.gpu

GENERIC = pda.PDA_FLAG_FORCE_GENERIC


def randn(seed, *shape, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(torch.bfloat16)


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


# ---- step tables -----------------------------------------------------------------------------------

def run_tables(L, n, P, pad=0, spare=5, in_place=False, seed=0):
    L, n = list(map(int, L)), list(map(int, n))
    g = np.random.default_rng(seed)
    held = [-(-(a - b) // P) for a, b in zip(L, n)]
    need = [-(-a // P) for a in L]
    pool = sum(need) + spare
    perm = g.permutation(pool).astype(np.int32)
    table = np.full((len(L), max(need + [0]) + 2), -7, dtype=np.int32)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = perm[at:at + h]
        at += h
    free = perm[at:]
    cap = sum(n) + pad
    dt, cu = ints(table), torch.full((len(L) + 1,), -9, dtype=torch.int32, device="cuda")
    slots, pos = (torch.full((cap,), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    cnt, status = ints([len(free)]), ints([0])
    out = cnt if in_place else ints([-9])
    pda.paged_build_tables(ints(L), ints(n), P, ints(free), cnt, dt, cu, slots, positions=pos, free_count_out=None if in_place else out,
                           status=status)
    rt, rcu, rs, rp, rc = U.tables(L, n, P, free, len(free), table, cap)
    assert int(status.item()) == 0
    assert (dt.cpu().numpy() == rt).all() and cu.tolist() == rcu and slots.tolist() == rs and pos.tolist() == rp
    assert out.item() == rc


@pytest.mark.parametrize("P", [1, 16, 24, 64])
@pytest.mark.parametrize("in_place", [False, True])
def test_tables_small(P, in_place):
    run_tables([1, 16, 17, 64, 65, 100, 33, 0], [1, 16, 1, 0, 65, 36, 33, 0], P, pad=3, in_place=in_place)
    run_tables([1], [1], P, in_place=in_place)
    run_tables([500], [500], P, in_place=in_place)


@pytest.mark.parametrize("B", [31, 1024, 1025, 2500])
@pytest.mark.parametrize("in_place", [False, True])
def test_tables_many(B, in_place):
    g = np.random.default_rng(B)
    L = g.integers(0, 90, size=B)
    n = np.where(g.random(B) < 0.3, 1, g.integers(0, 90, size=B))
    run_tables(L, np.minimum(n, L), 16, pad=int(g.integers(0, 5000)), in_place=in_place, seed=B)


def test_tables_sums_beyond_32_bits_of_room():
    """A table whose rows have room for more tokens than 32 bits count (the sums are then kept in 64)."""
    B, stride = 40, 1 << 22
    table = torch.full((B, stride), -7, dtype=torch.int32, device="cuda")
    L, n = [5 + b for b in range(B)], [1 + b % 3 for b in range(B)]
    free = list(range(500, 600))
    held = [-(-(a - b) // 16) for a, b in zip(L, n)]
    host = np.full((B, 8), -7, dtype=np.int32)
    for b in range(B):
        host[b, :held[b]] = 3 * b + np.arange(held[b])
    table[:, :8] = ints(host)
    cu, slots, cnt = ints([0] * (B + 1)), ints([0] * (sum(n) + 2)), ints([100])
    pda.paged_build_tables(ints(L), ints(n), 16, ints(free), cnt, table, cu, slots)
    rt, rcu, rs, _, rc = U.tables(L, n, 16, free, 100, host, sum(n) + 2)
    assert (table[:, :8].cpu().numpy() == rt).all() and cu.tolist() == rcu and slots.tolist() == rs and cnt.item() == rc


def test_tables_refuse_on_the_device():
    P, free = 16, list(range(100, 110))

    def call(L, n, table=None, count=10, cap=64, freel=free, stride=4):
        B = len(L)
        dt = ints(np.full((B, stride), 5) if table is None else table)
        cu, slots, out, st = ints([0] * (B + 1)), ints([0] * cap), ints([0]), ints([0])
        pda.paged_build_tables(ints(L), ints(n), P, ints(freel), ints([count]), dt, cu, slots, free_count_out=out, status=st)
        return dt.cpu().numpy(), cu.tolist(), slots.tolist(), out.item(), st.item()

    # too few pages: nothing is taken
    t, cu, slots, cnt, st = call([64, 64, 64], [64, 64, 64], cap=200)
    assert st == 4 and (t == 5).all() and set(slots) == {-1} and cnt == 10 and cu == [0, 64, 128, 192]
    # a count beyond the list, and below zero
    assert call([64, 64, 64], [64, 64, 64], count=1000, cap=200)[4] == 4
    assert call([16], [16], count=-3)[4] == 4
    # too few slots
    t, cu, slots, cnt, st = call([20, 20], [20, 20], cap=39)
    assert st == 5 and (t == 5).all() and set(slots) == {-1} and cnt == 10
    # lengths that cannot be: the others go ahead
    for L, n in ((-1, 0), (5, 6), (5, -1), (65, 1)):
        t, cu, slots, cnt, st = call([3, L, 18], [3, n, 2])
        assert st == 2 and cu == [0, 3, 3, 5] and cnt == 8
        assert slots[:5] == [109 * 16, 109 * 16 + 1, 109 * 16 + 2, 108 * 16, 108 * 16 + 1]
    # page ids that no slot number can hold
    t, cu, slots, cnt, st = call([17, 3], [1, 1], table=[[5] * 4, [-4] * 4], freel=[2 ** 30] * 10)
    assert st == 1 and slots[:2] == [-1, -1]


@pytest.mark.parametrize("in_place", [False, True])
def test_tables_count_beyond_the_list(in_place):
    """A count beyond the list counts as the list's length from then on: no page is handed out twice."""
    free = list(range(100, 110))
    count, taken = ints([1000]), []
    for left in (7, 4, 1):
        cu, slots, table = ints([0, 0, 0]), ints([0] * 1500), ints(np.zeros((2, 8)))
        out = count if in_place else ints([0])
        pda.paged_build_tables(ints([17, 3]), ints([17, 3]), 16, ints(free), count, table, cu, slots, free_count_out=out)
        taken += table[0, :2].tolist() + table[1, :1].tolist()
        assert out.item() == left
        count = out
    assert taken == free[:0:-1]
    count, cu, slots, st = ints([-5]), ints([0, 0]), ints([0]), ints([0])
    pda.paged_build_tables(ints([1]), ints([1]), 16, ints(free), count, ints(np.zeros((1, 8))), cu, slots, status=st)
    assert count.item() == 0 and st.item() == 4


def test_tables_empty_batch():
    cu, slots, out = ints([9]), ints([9, 9]), ints([9])
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    pda.paged_build_tables(e, e, 16, ints([1, 2]), ints([2]), torch.empty((0, 4), dtype=torch.int32, device="cuda"), cu, slots, free_count_out=out)
    assert cu.tolist() == [0] and slots.tolist() == [-1, -1] and out.item() == 2


# ---- append ----------------------------------------------------------------------------------------

@pytest.mark.parametrize("T", [1, 5, 257])
@pytest.mark.parametrize("R,Dr,P", [(512, 64, 64), (8, 0, 1), (1024, 256, 16), (264, 8, 5)])
@pytest.mark.parametrize("norm", [False, True])
def test_append(T, R, Dr, P, norm):
    pages = T // P + 3
    buf = torch.cat([randn(1, T, R) * (torch.rand(T, 1) * 4 + 0.01), randn(2, T, Dr + 8)], dim=1).to(torch.bfloat16)
    cache = randn(3, pages, P, R + Dr + 16)[:, :, :R + Dr]           # rows with a gap behind them
    slots = np.random.default_rng(T).permutation(pages * P)[:T].astype(np.int32)
    slots[T // 2] = -1
    w = (randn(4, R, scale=0.3) + 1).to(torch.bfloat16)
    d = torch.empty((pages, P, R + Dr + 16), dtype=torch.bfloat16, device="cuda")[:, :, :R + Dr]
    d.copy_(cache)
    dbuf, status = buf.cuda(), ints([0])
    pda.latent_append(dbuf[:, :R], dbuf[:, R:R + Dr], d, ints(slots), norm_weight=w.cuda() if norm else None, eps=1e-5, status=status)
    c = buf[:, :R].double()
    if norm:
        c = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * w.double()
    ref = cache.clone().double()
    for t in range(T):
        if slots[t] >= 0:
            ref[slots[t] // P, slots[t] % P] = torch.cat([c[t], buf[t, R:R + Dr].double()])
    got = d.cpu().double()
    if norm:  # one rounding to bf16 and a few 32-bit ones
        assert ((got - ref).abs() <= ref.abs() * (U.EPS + 2.0 ** -18)).all()
        rest = torch.ones(pages * P, dtype=torch.bool)
        rest[slots[slots >= 0].astype(np.int64)] = False
        assert torch.equal(got.reshape(pages * P, -1)[rest], ref.reshape(pages * P, -1)[rest])
        assert torch.equal(got[..., R:], ref[..., R:])
    else:
        assert torch.equal(got, ref)
    assert status.item() == 0


def test_append_slot_beyond_the_cache():
    cache, status = torch.zeros((2, 16, 72), dtype=torch.bfloat16, device="cuda"), ints([0])
    pda.latent_append(randn(1, 3, 64).cuda(), randn(2, 3, 8).cuda(), cache, ints([32, 31, 2 ** 31 - 1]), status=status)
    assert status.item() == 1
    nz = cache.view(32, 72).abs().sum(1) != 0
    assert nz.tolist() == [False] * 31 + [True]


def test_append_all_zero_row_is_zero():
    cache = torch.ones((1, 16, 72), dtype=torch.bfloat16, device="cuda")
    z = torch.zeros((1, 64), dtype=torch.bfloat16, device="cuda")
    pda.latent_append(z, randn(2, 1, 8).cuda(), cache, ints([3]), norm_weight=torch.ones(64, dtype=torch.bfloat16, device="cuda"), eps=1e-6)
    assert (cache[0, 3, :64] == 0).all() and (cache[0, 2] == 1).all()


# ---- absorbed attention ----------------------------------------------------------------------------

def run_absorbed(lens, H, T, R, Dr, P, seed=1, flags=0, layout="plain", scale=None, spread=1.0, **kw):
    pg = U.Paged(lens, P, R, Dr, seed, spread=spread, **kw)
    B = len(lens)
    ql, qr = randn(seed + 1, B, T, H, R), randn(seed + 2, B, T, H, Dr)
    scale = 1.0 / np.sqrt(192.0) if scale is None else scale
    if layout == "plain":
        dql, dqr, out = ql.cuda(), qr.cuda(), torch.full((B, T, H, R), float("nan"), dtype=torch.bfloat16, device="cuda")
    else:  # heads outermost, as a batched product leaves them; the rotary part a slice
        dql = ql.permute(2, 0, 1, 3).contiguous().cuda().permute(1, 2, 0, 3)
        dqr = torch.cat([randn(9, B, T, H, 128), qr], dim=-1).cuda()[..., 128:]
        out = torch.full((H, B, T, R), float("nan"), dtype=torch.bfloat16, device="cuda").permute(1, 2, 0, 3)
    ws = pda.latent_workspace(B, H, T, R)
    ws.fill_(255)
    got = pda.paged_latent_attention(dql, dqr, pg.cache, pg.dtable, pg.dlens, scale, out=out, workspace=ws, flags=flags, status=pg.status)
    torch.cuda.synchronize()
    assert pg.status.item() == 0
    ref, tol = U.absorbed(ql, qr, pg.host, pg.table, lens, scale, R)
    U.check(got, ref, tol, f"lens {lens[:6]} H {H} T {T} R {R} P {P}")
    return pg, dql, dqr, ws, got


LENS = [1, 0, 17, 64, 65, 63, 128, 200, 16, 15]


@pytest.mark.parametrize("flags", [0, GENERIC])
@pytest.mark.parametrize("H", [1, 16, 24, 64, 128])
@pytest.mark.parametrize("P", [16, 64])
def test_absorbed_lengths(H, P, flags):
    run_absorbed(LENS, H, 1, 512, 64, P, flags=flags)


@pytest.mark.parametrize("R,Dr,P,H", [(128, 64, 16, 8), (256, 64, 32, 33), (384, 64, 128, 16), (512, 64, 256, 65), (512, 64, 8, 16),
                                      (512, 64, 48, 16), (64, 64, 16, 4), (200, 40, 7, 5), (1024, 0, 16, 3), (8, 8, 1, 2)])
def test_absorbed_shapes(R, Dr, P, H):
    run_absorbed([70, 1, 300, 129], H, 1, R, Dr, P, seed=R)


@pytest.mark.parametrize("T,H", [(2, 16), (3, 5), (5, 64), (16, 8), (7, 128), (40, 16)])
@pytest.mark.parametrize("layout", ["plain", "bmm"])
def test_absorbed_blocks_of_queries(T, H, layout):
    # among them sequences shorter than the block: query tokens before the first one have nothing to attend
    run_absorbed([T, T + 1, 1, 0, 64, 63 + T, 130, 300], H, T, 512, 64, 64, seed=T, layout=layout)


@pytest.mark.parametrize("lens,H,T", [([4000], 16, 1), ([3000, 1, 2000], 128, 1), ([5000, 4997], 32, 3), ([257] * 30, 64, 1)])
@pytest.mark.parametrize("P", [16, 64])
def test_absorbed_split_over_the_tokens(lens, H, T, P):
    run_absorbed(lens, H, T, 512, 64, P, seed=3)


def test_absorbed_many_sequences():
    g = np.random.default_rng(5)
    run_absorbed([int(x) for x in g.integers(0, 150, size=700)], 16, 1, 128, 64, 16, seed=5)


@pytest.mark.parametrize("spread,scale", [(30.0, 0.07), (1e-3, 0.07), (1.0, 0.0), (8.0, 1.0)])
def test_absorbed_peaked_and_flat_scores(spread, scale):
    run_absorbed([700, 65, 1300], 32, 1, 512, 64, 64, seed=6, spread=spread, scale=scale)


def test_absorbed_rising_scores():
    """Every block of tokens raises the running maximum far beyond the last one's, then it falls again."""
    L, H, R = 1024, 16, 512
    pg = U.Paged([L], 64, R, 64, 7)
    ql, qr = randn(8, 1, 1, H, R), randn(9, 1, 1, H, 64)
    ramp = torch.cat([torch.linspace(-60, 60, L // 2), torch.linspace(60, -60, L // 2)])
    host = pg.host.clone()
    for i in range(L // 64):
        rows = host[int(pg.table[0, i])].float()
        rows[:, :R] += ramp[i * 64:(i + 1) * 64, None] * ql[0, 0, i % H].float() / 100
        host[int(pg.table[0, i])] = rows.to(torch.bfloat16)
    pg.cache.copy_(host)
    got = pda.paged_latent_attention(ql.cuda(), qr.cuda(), pg.cache, pg.dtable, pg.dlens, 0.07)
    ref, tol = U.absorbed(ql, qr, host, pg.table, [L], 0.07, R)
    U.check(got, ref, tol)


def test_absorbed_more_row_blocks_than_run_at_once():
    run_absorbed([100, 70, 1, 230], 64, 100, 128, 64, 64, seed=31)         # 100 row blocks of 64: several rounds
    run_absorbed([500], 128, 40, 512, 64, 16, seed=32)


def test_absorbed_one_query_for_all_heads():
    """Query strides of zero (a broadcast over the heads), and a head count that no copy of several heads fits."""
    pg = U.Paged([130, 64], 64, 512, 64, 41)
    for T, H in ((1, 12), (3, 7)):
        ql, qr = randn(42, 2, T, 1, 512), randn(43, 2, T, 1, 64)
        got = pda.paged_latent_attention(ql.cuda().expand(2, T, H, 512), qr.cuda().expand(2, T, H, 64), pg.cache, pg.dtable, pg.dlens, 0.07,
                                         out=torch.empty((2, T, H, 512), dtype=torch.bfloat16, device="cuda"))
        ref, tol = U.absorbed(ql.expand(2, T, H, 512), qr.expand(2, T, H, 64), pg.host, pg.table, [130, 64], 0.07, 512)
        U.check(got, ref, tol)


@pytest.mark.parametrize("lens", [[300, 90], [64, 50], [100, 4000]])
def test_absorbed_nan_in_one_query_stays_there(lens):
    pg = U.Paged(lens, 64, 512, 64, 44)
    ql, qr = randn(45, 2, 1, 16, 512), randn(46, 2, 1, 16, 64)
    ref, tol = U.absorbed(ql, qr, pg.host, pg.table, lens, 0.07, 512)
    ql[1, 0, 3, 100] = float("nan")
    got = pda.paged_latent_attention(ql.cuda(), qr.cuda(), pg.cache, pg.dtable, pg.dlens, 0.07).cpu()
    assert torch.isnan(got[1, 0, 3]).all()
    got[1, 0, 3], ref[1, 0, 3] = 0, 0
    U.check(got, ref, tol)


def test_absorbed_workspace_reuse_across_shapes():
    """One workspace for calls of different shapes in a row: nothing in it outlives a call."""
    ws = pda.latent_workspace(64, 128, 1, 512)
    for i, (lens, H) in enumerate((([3000, 10], 128), ([900] * 40, 64), ([1] * 64, 128), ([5000], 128))):
        pg = U.Paged(lens, 64, 512, 64, 50 + i)
        ql, qr = randn(60 + i, len(lens), 1, H, 512), randn(70 + i, len(lens), 1, H, 64)
        got = pda.paged_latent_attention(ql.cuda(), qr.cuda(), pg.cache, pg.dtable, pg.dlens, 0.07, workspace=ws)
        ref, tol = U.absorbed(ql, qr, pg.host, pg.table, lens, 0.07, 512)
        U.check(got, ref, tol, str(i))


@pytest.mark.parametrize("flags", [0, GENERIC])
def test_absorbed_strides_of_the_cache(flags):
    run_absorbed([100, 33, 64], 16, 1, 512, 64, 16, flags=flags, slot_pad=8, page_pad=24)


@pytest.mark.parametrize("flags", [0, GENERIC])
def test_absorbed_bad_pages_and_lengths(flags):
    lens = [700, 300, 64, 500, 129]
    pg = U.Paged(lens, 64, 512, 64, 11)
    ql, qr = randn(1, 5, 1, 16, 512), randn(2, 5, 1, 16, 64)
    ref, tol = U.absorbed(ql, qr, pg.host, pg.table, lens, 0.07, 512)
    for seq, entry, value in ((0, 10, -1), (1, 0, pg.cache.shape[0]), (3, 3, -2 ** 31), (4, 2, 2 ** 31 - 1)):
        t = pg.dtable.clone()
        t[seq, entry] = value
        st = ints([0])
        got = pda.paged_latent_attention(ql.cuda(), qr.cuda(), pg.cache, t, pg.dlens, 0.07, status=st, flags=flags)
        assert st.item() == 1
        r, o = ref.clone(), tol.clone()
        r[seq], o[seq] = 0, 0
        U.check(got, r, o, f"bad page in {seq}")
    for seq, L in ((2, 64 * pg.table.shape[1] + 1), (0, 2 ** 31 - 1), (3, -5)):
        ls = list(lens)
        ls[seq] = L
        st = ints([0])
        got = pda.paged_latent_attention(ql.cuda(), qr.cuda(), pg.cache, pg.dtable, ints(ls), 0.07, status=st, flags=flags)
        assert st.item() == (2 if L > 0 else 0)
        r, o = ref.clone(), tol.clone()
        r[seq], o[seq] = 0, 0
        U.check(got, r, o, f"length {L}")


def test_absorbed_rows_that_are_not_there_do_not_matter():
    """112 rows in two blocks of 64: what earlier segments left behind the last row must not change the others'
    rounding. (Many sequences per CTA, the same call over and over between calls that leave other things behind.)"""
    lens = [int(x) for x in np.random.default_rng(4).integers(0, 1500, size=17)]
    pg, ql, qr, ws, first = run_absorbed(lens, 16, 7, 512, 64, 32, seed=61)
    first = first.clone()
    other, oql, oqr, ows, _ = run_absorbed([900] * 40, 64, 1, 512, 64, 64, seed=62, spread=20.0)
    for _ in range(10):
        pda.paged_latent_attention(oql, oqr, other.cache, other.dtable, other.dlens, 0.3, workspace=ows)
        got = pda.paged_latent_attention(ql, qr, pg.cache, pg.dtable, pg.dlens, 1.0 / np.sqrt(192.0), workspace=ws)
        assert torch.equal(got, first)


def test_absorbed_repeats_bit_for_bit_and_other_streams():
    pg, ql, qr, ws, first = run_absorbed([900, 77, 2500, 64], 32, 1, 512, 64, 64, seed=21)
    first = first.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a = pda.paged_latent_attention(ql, qr, pg.cache, pg.dtable, pg.dlens, 1.0 / np.sqrt(192.0))
    b = pda.paged_latent_attention(ql, qr, pg.cache, pg.dtable, pg.dlens, 1.0 / np.sqrt(192.0), stream=s, workspace=ws)
    s.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(a, first) and torch.equal(b, first)


def test_absorbed_far_offsets():
    """Pages whose offsets pass 2^31 elements."""
    R, W, P = 512, 576, 64
    page_stride = 2 ** 28                                    # elements; 10 pages span 5.4 GB
    n_pages = 10
    flat = torch.empty((n_pages - 1) * page_stride + P * W, dtype=torch.bfloat16, device="cuda")
    cache = flat.as_strided((n_pages, P, W), (page_stride, W, 1))
    host = randn(1, n_pages, P, W)
    cache.copy_(host)
    table = np.array([[9, 8, 2, 7, 0], [1, 9, 9, 9, 9]], dtype=np.int32)
    lens = [300, 50]
    ql, qr = randn(2, 2, 1, 16, R), randn(3, 2, 1, 16, 64)
    ref, tol = U.absorbed(ql, qr, host, table, lens, 0.07, R)
    for flags in (0, GENERIC):
        got = pda.paged_latent_attention(ql.cuda(), qr.cuda(), cache, ints(table), ints(lens), 0.07, flags=flags)
        U.check(got, ref, tol)
    pda.latent_append(randn(4, 1, R).cuda(), randn(5, 1, 64).cuda(), cache, ints([9 * P + 63]))
    assert torch.equal(cache[9, 63, :R].cpu(), randn(4, 1, R)[0]) and torch.equal(cache[9, 62].cpu(), host[9, 62])


# ---- expanded attention ----------------------------------------------------------------------------

def run_expanded(q_lens, k_lens, H, dims=(128, 64, 128), seed=1, flags=0, gap=0, scale=None, max_q=None, spread=1.0):
    dn, dr, dv = dims
    cq = [gap + int(x) for x in np.concatenate([[0], np.cumsum(q_lens)])]
    ck = [gap + int(x) for x in np.concatenate([[0], np.cumsum(k_lens)])]
    tq, tk = cq[-1] + gap, ck[-1] + gap
    scale = 1.0 / np.sqrt(dn + dr) if scale is None else scale
    q, kv, kr = randn(seed, tq, H, dn + dr), randn(seed + 1, tk, H, dn + dv, scale=spread), randn(seed + 2, tk, dr, scale=spread)
    if gap:
        for t, n in ((q, tq), (kv, tk), (kr, tk)):          # rows outside the sequences hold anything
            t[:gap] = float("nan")
            t[n - gap:] = float("nan")
    dq, dkv, dkr = q.cuda(), kv.cuda(), kr.cuda()
    out = torch.full((tq, H, dv), -5.0, dtype=torch.bfloat16, device="cuda")
    st = ints([0])
    got = pda.latent_prefill_attention(dq, dkv[..., :dn], dkr, dkv[..., dn:], ints(cq), ints(ck), max_q or max(q_lens), scale,
                                       out=out, flags=flags, status=st)
    torch.cuda.synchronize()
    assert st.item() == 0
    ref, tol = U.expanded(q, kv[..., :dn], kr, kv[..., dn:], cq, ck, scale)
    if gap:
        assert (got[:gap] == -5).all() and (got[tq - gap:] == -5).all()
    U.check(got[cq[0]:cq[-1]], ref[cq[0]:cq[-1]], tol[cq[0]:cq[-1]], f"q {q_lens[:5]} k {k_lens[:5]} H {H} {dims}")
    return dq, dkv, dkr, got


@pytest.mark.parametrize("flags", [0, GENERIC])
@pytest.mark.parametrize("lens", [[1], [2, 1, 3], [127, 128, 129], [255, 256, 257, 64], [400, 1, 31]])
def test_expanded_prompts(lens, flags):
    run_expanded(lens, lens, 3, flags=flags)


@pytest.mark.parametrize("q_lens,k_lens", [([1], [300]), ([5, 128, 1], [600, 128, 129]), ([200, 0, 10], [513, 40, 10]), ([130], [1000]),
                                           ([300, 7], [17, 0])])
def test_expanded_behind_a_context(q_lens, k_lens):
    # the last pair: more query tokens than keys, and none at all: rows without keys are zero
    run_expanded(q_lens, k_lens, 2, seed=4, gap=0)
    run_expanded(q_lens, k_lens, 2, seed=5, gap=3, max_q=max(q_lens) + 200)


@pytest.mark.parametrize("dims", [(64, 32, 64), (128, 64, 64), (128, 0, 128), (200, 8, 96), (512, 256, 512)])
def test_expanded_shapes(dims):
    run_expanded([40, 3], [70, 3], 2, dims=dims, seed=6)


@pytest.mark.parametrize("spread,scale", [(30.0, 0.07), (1e-3, 0.07), (1.0, 0.0), (4.0, 1.0)])
def test_expanded_peaked_and_flat_scores(spread, scale):
    run_expanded([300], [700], 2, seed=7, spread=spread, scale=scale)


def test_expanded_long():
    run_expanded([1500, 700], [1500, 2100], 2, seed=8)


def test_expanded_many_sequences():
    g = np.random.default_rng(3)
    n = [int(x) for x in g.integers(0, 40, size=200)]                        # more than are sorted
    run_expanded(n, [x + int(y) for x, y in zip(n, g.integers(0, 60, size=200))], 2, seed=11)
    run_expanded([200] * 100, [200] * 100, 1, seed=12)                       # as many tokens as make more blocks than that
    run_expanded([1] * 127 + [513], [30] * 127 + [600], 1, seed=13)


def test_expanded_many_heads():
    run_expanded([300, 1, 77, 520, 128], [300, 50, 77, 700, 128], 40, seed=14)   # several row blocks per pair of CTAs


def test_expanded_unequal_halves():
    """The two halves of a row block with 0, 1, 2 and many tiles of difference, in a row."""
    run_expanded([600, 256, 257, 130, 512, 385], [300, 2000, 257, 1500, 100, 385], 30, seed=15)


@pytest.mark.parametrize("q_lens,k_lens", [([1], [129]), ([256], [256]), ([24, 17], [4000, 2049]), ([129, 200], [900, 385]),
                                           ([700, 768], [3000, 768]), ([250, 256], [200, 130]), ([100], [60]), ([30, 0, 256], [1300, 500, 641])])
@pytest.mark.parametrize("spread", [1.0, 30.0])
def test_expanded_few_rows_behind_a_long_context(q_lens, k_lens, spread):
    """Row blocks of at most 256 rows, with room for each: odd and even numbers of tiles, rows that see the first few
    keys or none, the last block of a longer prompt; with a spread of 30 a row's weight lies on one key."""
    run_expanded(q_lens, k_lens, 3, seed=17, spread=spread)


@pytest.mark.parametrize("flags", [0, GENERIC])
def test_expanded_loose_bound_of_the_query_tokens(flags):
    """max_q far above what the sequences have, with few and with many of them."""
    most = (2 ** 31 - 1) // 2
    run_expanded([5, 130, 1], [70, 130, 9], 2, seed=18, max_q=most, flags=flags)
    run_expanded([3, 0, 1, 40] * 50, [9, 5, 1, 60] * 50, 2, seed=19, max_q=most, flags=flags)


def test_expanded_result_does_not_depend_on_the_bound():
    outs = [run_expanded([130, 300, 70] * 6, [1200, 2300, 900] * 6, 3, seed=22, max_q=m)[3] for m in (300, 513, 10000)]
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("long_at", [0, 77, 149])
@pytest.mark.parametrize("gap", [0, 700])
def test_expanded_one_long_among_many_short(long_at, gap):
    """More sequences than are listed, one of which has many row blocks."""
    g = np.random.default_rng(long_at)
    n = [int(x) for x in g.integers(0, 20, size=150)]
    n[long_at] = 2600
    run_expanded(n, [x + int(y) for x, y in zip(n, g.integers(0, 200, size=150))], 3, seed=20, gap=gap)


@pytest.mark.parametrize("flags", [0, GENERIC])
def test_expanded_bad_ranges_among_many(flags):
    """Sequences whose ranges are bad are reported and zeroed, also those without rows; the others are as they should be."""
    B, H = 150, 2
    n = [3] * B
    n[70] = 2600
    cq = [int(x) for x in np.concatenate([[0], np.cumsum(n)])]
    T = cq[-1]
    q, kn, kr, v = randn(1, T, H, 192), randn(2, T, H, 128), randn(3, T, 64), randn(4, T, H, 128)
    ref, tol = U.expanded(q, kn, kr, v, cq, cq, 0.07)
    d = [x.cuda() for x in (q, kn, kr, v)]

    def call(cq, ck, max_q):
        out, st = torch.full((T, H, 128), -5.0, dtype=torch.bfloat16, device="cuda"), ints([0])
        pda.latent_prefill_attention(*d, ints(cq), ints(ck), max_q, 0.07, out=out, flags=flags, status=st)
        return out.cpu().double(), st.item()

    x, st = call(cq, cq[:-1] + [T + 1], 2600)                # the last one's keys pass the array
    assert st == 2 and (x[T - 3:] == 0).all()
    U.check(x[:T - 3], ref[:T - 3], tol[:T - 3], "the others")
    x, st = call(cq, cq, 1000)                               # one has more rows than max_q: so many are zeroed
    a, b = cq[70], cq[71]
    assert st == 2 and (x[a:a + 1000] == 0).all() and (x[a + 1000:b] == -5).all()
    U.check(x[:a], ref[:a], tol[:a], "before")
    U.check(x[b:], ref[b:], tol[b:], "behind")
    no_rows = cq[:100] + [cq[100]] * 2 + cq[102:]            # sequence 100 has no rows, and keys out of range
    x, st = call(no_rows, [0] * 100 + [5, 0] + [0] * (B - 101), 2600)
    assert st == 2


@pytest.mark.parametrize("q_lens,k_lens,H", [([700, 300, 513], [5000, 4300, 4700], 41), ([8192], [8192], 6), ([257], [20000], 1),
                                             ([600, 40, 1100], [1500, 1024, 1100], 2), ([300] * 3, [12500, 130, 300], 30)])
@pytest.mark.parametrize("spread", [1.0, 20.0])
def test_expanded_many_keys(q_lens, k_lens, H, spread):
    """Long contexts, with several row blocks per pair of CTAs and with fewer than there are."""
    run_expanded(q_lens, k_lens, H, seed=21, spread=spread)


@pytest.mark.parametrize("token", [0, 31, 33, 70, 100, 2000, 4130])
def test_expanded_nan_among_many_keys(token):
    """A NaN in one key reaches the rows that see it and no other."""
    nq, nk, H = 600, 4200, 2
    q, kv, kr = randn(1, nq, H, 192), randn(2, nk, H, 256), randn(3, nk, 64)
    kv[token, 1, 5] = float("nan")
    out = pda.latent_prefill_attention(q.cuda(), kv[..., :128].cuda(), kr.cuda(), kv[..., 128:].cuda(), ints([0, nq]), ints([0, nk]), nq, 0.07)
    nan = out.float().isnan().any(-1).cpu()
    sees = torch.arange(nq) + nk - nq >= token
    assert not nan[:, 0].any() and (nan[:, 1] == sees).all()


def test_expanded_huge_values_behind_the_mask():
    """Later tokens' values near the largest number must not reach earlier rows."""
    nq = 200
    q, kv, kr = randn(1, nq, 2, 192), randn(2, nq, 2, 256), randn(3, nq, 64)
    kv[150:, :, 128:] = 3e38
    args = [x.cuda() for x in (q, kv, kr)]
    for flags in (0, GENERIC):
        got = pda.latent_prefill_attention(args[0], args[1][..., :128], args[2], args[1][..., 128:], ints([0, nq]), ints([0, nq]), nq, 0.07, flags=flags)
        ref, tol = U.expanded(q[:150], kv[:150, :, :128], kr[:150], kv[:150, :, 128:], [0, 150], [0, 150], 0.07)
        U.check(got[:150], ref, tol)


@pytest.mark.parametrize("token", [0, 5, 67, 130])
def test_expanded_nan_reaches_the_rows_that_see_it(token):
    nq = 300
    q, kv, kr = randn(1, nq, 2, 192), randn(2, nq, 2, 256), randn(3, nq, 64)
    ref, tol = U.expanded(q, kv[..., :128], kr, kv[..., 128:], [0, nq], [0, nq], 0.07)
    kv[token, 1, 17] = float("nan")
    args = [x.cuda() for x in (q, kv, kr)]
    for flags in (0, GENERIC):
        got = pda.latent_prefill_attention(args[0], args[1][..., :128], args[2], args[1][..., 128:], ints([0, nq]), ints([0, nq]), nq, 0.07, flags=flags).cpu()
        assert torch.isnan(got[token:, 1]).all()
        U.check(got[:, 0], ref[:, 0], tol[:, 0])
        if token:
            U.check(got[:token, 1], ref[:token, 1], tol[:token, 1])


@pytest.mark.parametrize("flags", [0, GENERIC])
def test_expanded_strides(flags):
    """Queries a part of wider rows, keys, values and output with the heads outermost."""
    lens, H = [70, 200], 3
    T = sum(lens)
    q, kn, kr, v = randn(1, T, H, 192), randn(2, T, H, 128), randn(3, T, 64), randn(4, T, H, 128)
    dq = torch.cat([q, randn(5, T, H, 64)], dim=-1).cuda()[..., :192]
    heads_out = lambda t: t.permute(1, 0, 2).contiguous().cuda().permute(1, 0, 2)
    dkr = torch.cat([randn(6, T, 512), kr], dim=-1).cuda()[:, 512:]
    out = torch.full((H, T, 128), -5.0, dtype=torch.bfloat16, device="cuda").permute(1, 0, 2)
    cu = [0, 70, 270]
    got = pda.latent_prefill_attention(dq, heads_out(kn), dkr, heads_out(v), ints(cu), ints(cu), 200, 0.07, out=out, flags=flags)
    ref, tol = U.expanded(q, kn, kr, v, cu, cu, 0.07)
    U.check(got, ref, tol)


def test_expanded_repeats_bit_for_bit_in_a_graph_and_on_other_streams():
    dq, dkv, dkr, first = run_expanded([300, 40, 700], [300, 90, 900], 8, seed=16)
    cq, ck = ints([0, 300, 340, 1040]), ints([0, 300, 390, 1290])
    call = lambda out, **kw: pda.latent_prefill_attention(dq, dkv[..., :128], dkr, dkv[..., 128:], cq, ck, 700, 1.0 / np.sqrt(192.0), out=out, **kw)
    s, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    outs = [torch.zeros_like(first) for _ in range(3)]
    torch.cuda.synchronize()
    call(outs[0], stream=s)
    call(outs[1], stream=s2)                        # two at once
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(outs[2])
    graph.replay()
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, first)


@pytest.mark.parametrize("flags", [0, GENERIC])
def test_expanded_bad_ranges(flags):
    tq = tk = 60
    q, kn, kr, v = randn(1, tq, 2, 192), randn(2, tk, 2, 128), randn(3, tk, 64), randn(4, tk, 2, 128)
    d = [x.cuda() for x in (q, kn, kr, v)]
    good_q, good_k = [0, 20, 40, 60], [0, 20, 40, 60]
    ref, tol = U.expanded(q, kn, kr, v, good_q, good_k, 0.07)
    for cq, ck, zero, skip in (([0, 20, 40, 61], good_k, [2], []), (good_q, [0, 20, 40, 61], [2], []), (good_q, [0, 20, 10, 60], [1, 2], []),
                               (good_q, [-3, 20, 40, 60], [0], []), ([-2, 20, 40, 60], good_k, [], [0])):
        out, st = torch.full((tq, 2, 128), -5.0, dtype=torch.bfloat16, device="cuda"), ints([0])
        pda.latent_prefill_attention(*d, ints(cq), ints(ck), 20 if cq[-1] == 60 else 21, 0.07, out=out, flags=flags, status=st)
        assert st.item() == 2
        r, o, x = ref.clone(), tol.clone(), out.cpu().double()
        if ck == [0, 20, 10, 60]:        # the last sequence's keys 10 .. 60 are a range of their own
            rr, oo = U.expanded(q, kn, kr, v, [40, 60], [10, 60], 0.07)
            r[40:], o[40:] = rr[40:], oo[40:]
            zero = [1]
        for b in zero:
            r[20 * b:20 * b + 20], o[20 * b:20 * b + 20] = 0, 0
        for b in skip:
            assert (x[20 * b:20 * b + 20] == -5).all()
            x[20 * b:20 * b + 20] = r[20 * b:20 * b + 20]
        U.check(x, r, o, f"{cq} {ck}")
    # more query tokens than max_q
    out, st = torch.full((tq, 2, 128), -5.0, dtype=torch.bfloat16, device="cuda"), ints([0])
    pda.latent_prefill_attention(*d, ints([0, 25, 45, 60]), ints([0, 25, 45, 60]), 20, 0.07, out=out, flags=flags, status=st)
    assert st.item() == 2 and (out[:20] == 0).all() and (out[20:25] == -5).all() and (out[25:] != -5).any()


# ---- together --------------------------------------------------------------------------------------

def test_prompts_then_decoding_steps():
    """Tables, append and both forms as a layer runs them, against the definition on the stored rows."""
    B, H, R, Dr, Dn, Dv, P = 4, 16, 512, 64, 128, 128, 16
    prompts, steps, pool = [37, 1, 160, 64], 4, 64
    scale = 1.0 / np.sqrt(Dn + Dr)
    wk, wv = randn(1, H, Dn, R, scale=R ** -0.5).cuda(), randn(2, H, Dv, R, scale=R ** -0.5).cuda()
    norm_w = (randn(3, R, scale=0.1) + 1).to(torch.bfloat16).cuda()
    cache = torch.full((pool, P, R + Dr), float("nan"), dtype=torch.bfloat16, device="cuda")
    table = torch.full((B, 16), -1, dtype=torch.int32, device="cuda")
    free, count, status = ints(np.random.default_rng(0).permutation(pool)), ints([pool]), ints([0])
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    ws = pda.latent_workspace(B, H, 1, R)
    for step in range(steps + 1):
        new = prompts if step == 0 else [1] * B
        n = sum(new)
        new_lens, cu, slots, pos = ints(new), ints([0] * (B + 1)), ints([0] * (n + 5)), ints([0] * (n + 5))
        lens = lens + new_lens
        pda.paged_build_tables(lens, new_lens, P, free, count, table, cu, slots, positions=pos, status=status)
        rows = randn(10 + step, n, R + Dr).cuda()
        pda.latent_append(rows[:, :R], rows[:, R:], cache, slots[:n], norm_weight=norm_w, eps=1e-6, status=status)
        q = randn(50 + step, n, H, Dn + Dr).cuda()
        if step == 0:
            stored = cache.view(-1, R + Dr)[slots[:n].long()]
            k_nope = torch.einsum("tr,hdr->thd", stored[:, :R].float(), wk.float()).to(torch.bfloat16)
            v = torch.einsum("tr,hdr->thd", stored[:, :R].float(), wv.float()).to(torch.bfloat16)
            out = pda.latent_prefill_attention(q, k_nope, stored[:, R:], v, cu, cu, max(new), scale, status=status)
        else:
            ql = torch.einsum("thd,hdr->thr", q[..., :Dn].float(), wk.float()).to(torch.bfloat16)
            o = pda.paged_latent_attention(ql, q[..., Dn:], cache, table, lens, scale, workspace=ws, status=status)
            out = torch.einsum("thr,hdr->thd", o.float(), wv.float())
        assert status.item() == 0
        at, where = 0, table.cpu().numpy()
        for b, L in enumerate(lens.tolist()):
            j = np.arange(L)
            stored = cache[torch.as_tensor(where[b, j // P].astype(np.int64)).cuda(), torch.as_tensor(j % P).cuda()].double()
            for h in range(H):
                k = torch.cat([stored[:, :R] @ wk[h].double().T, stored[:, R:]], dim=1)
                vv = stored[:, :R] @ wv[h].double().T
                for i in range(new[b]):
                    live = L - new[b] + i + 1
                    w = torch.softmax(k[:live] @ q[at + i, h].double() * scale, dim=0)
                    ref = w @ vv[:live]
                    # every rounding to bf16 on the way (keys or absorbed query, values or latent output, weights,
                    # output) is 2^-8 of values near 1: scores move by less than 5 * 2^-8, outputs by a tenth at most
                    assert float((out[at + i, h].double() - ref).abs().max()) < 0.1, (step, b, h, i)
            at += new[b]
    assert count.item() == pool - sum(-(-int(L) // P) for L in lens.tolist())


def test_step_in_a_graph():
    """A whole decode step captured once and replayed while the lengths grow on the device."""
    B, H, R, Dr, P, steps = 3, 16, 512, 64, 16, 20
    g = np.random.default_rng(1)
    start = [30, 1, 100]
    pg = U.Paged(start, P, R, Dr, 5, pages_extra=12)
    used = {int(x) for b, L in enumerate(start) for x in pg.table[b, :-(-L // P)]}
    free = [i for i in range(pg.cache.shape[0]) if i not in used]
    table = torch.full((B, 12), -1, dtype=torch.int32, device="cuda")
    table[:, :pg.table.shape[1]] = pg.dtable
    lens, one, count, status = ints(start), ints([1] * B), ints([len(free)]), ints([0])
    dfree, cu, slots = ints(free), ints([0] * (B + 1)), ints([0] * B)
    rows, ql, qr = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((B, R + Dr), (B, 1, H, R), (B, 1, H, Dr)))
    out, ws = torch.zeros((B, 1, H, R), dtype=torch.bfloat16, device="cuda"), pda.latent_workspace(B, H, 1, R)

    def step():
        pda.advance_seq_lens(lens)
        pda.paged_build_tables(lens, one, P, dfree, count, table, cu, slots, status=status)
        pda.latent_append(rows[:, :R], rows[:, R:], pg.cache, slots, status=status)
        pda.paged_latent_attention(ql, qr, pg.cache, table, lens, 0.07, out=out, workspace=ws, status=status)

    graph = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    with torch.cuda.graph(graph):
        step()
    for i in range(steps):
        rows.copy_(randn(100 + i, B, R + Dr))
        hq, hr = randn(200 + i, B, 1, H, R), randn(300 + i, B, 1, H, Dr)
        ql.copy_(hq)
        qr.copy_(hr)
        graph.replay()
        now = [L + 2 + i for L in start]
        assert lens.tolist() == now and status.item() == 0
        ref, tol = U.absorbed(hq, hr, pg.cache.cpu(), table.cpu().numpy(), now, 0.07, R)
        U.check(out, ref, tol, f"replay {i}")


def test_buffers_of_a_call_belong_to_its_stream(monkeypatch):
    """What a call on another stream allocates is not handed out on the current one while the call may still run."""
    import paper_2605_06068_b200.binding as binding
    real, seen = binding.lib(), {}

    class Recorder:
        def __getattr__(self, name):
            f = getattr(real, name)

            def call(*args):
                seen[name] = args
                return f(*args)
            return call if name == "paged_latent_attention" else f

    monkeypatch.setattr(binding, "lib", lambda: Recorder())
    pg = U.Paged([700, 40], 64, 512, 64, 50)
    ql, qr = randn(51, 2, 16, 512).cuda(), randn(52, 2, 16, 64).cuda()
    s = torch.cuda.Stream()
    first = pda.paged_latent_attention(ql, qr, pg.cache, pg.dtable, pg.dlens, 0.07)
    torch.cuda.synchronize()
    out = pda.paged_latent_attention(ql, qr, pg.cache, pg.dtable, pg.dlens, 0.07, stream=s)
    at, size = seen["paged_latent_attention"][18], seen["paged_latent_attention"][19]
    held = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(4)]   # of the current stream
    assert at not in [x.data_ptr() for x in held]
    torch.cuda.synchronize()
    assert torch.equal(out, first)


def test_calls_on_several_streams_at_once():
    """Both forms, the append and the tables on four streams at the same time, each with buffers of its own."""
    jobs = []
    for i, (lens, H) in enumerate((([2000, 5, 700], 128), ([300] * 50, 16), ([9000], 32))):
        pg = U.Paged(lens, 64, 512, 64, 80 + i)
        ql, qr = randn(83 + i, len(lens), 1, H, 512).cuda(), randn(86 + i, len(lens), 1, H, 64).cuda()
        ws, out = pda.latent_workspace(len(lens), H, 1, 512), torch.zeros_like(ql)
        jobs.append((lambda s, pg=pg, ql=ql, qr=qr, ws=ws, out=out: pda.paged_latent_attention(
            ql, qr, pg.cache, pg.dtable, pg.dlens, 0.07, out=out, workspace=ws, stream=s), out))
    q, kv, kr = randn(90, 900, 16, 192).cuda(), randn(91, 900, 16, 256).cuda(), randn(92, 900, 64).cuda()
    cu, out = ints([0, 600, 900]), torch.zeros((900, 16, 128), dtype=torch.bfloat16, device="cuda")
    jobs.append((lambda s: pda.latent_prefill_attention(q, kv[..., :128], kr, kv[..., 128:], cu, cu, 600, 0.07, out=out, stream=s), out))
    want = []
    for call, o in jobs:
        call(None)
        torch.cuda.synchronize()
        want.append(o.clone())
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(15):
        for (_, o), s in zip(jobs, streams):
            with torch.cuda.stream(s):
                o.zero_()
        for (call, _), s in zip(jobs, streams):
            call(s)
    torch.cuda.synchronize()
    for (_, o), w in zip(jobs, want):
        assert torch.equal(o, w)


def test_two_graphs_replayed_side_by_side():
    """Two captured calls with a workspace each, replayed on two streams."""
    pg, ql, qr, ws, first = run_absorbed([3000, 100], 64, 1, 512, 64, 64, seed=95)
    first = first.clone()
    graphs, outs = [], []
    for _ in range(2):
        w, o, g = pda.latent_workspace(2, 64, 1, 512), torch.zeros_like(first), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            pda.paged_latent_attention(ql, qr, pg.cache, pg.dtable, pg.dlens, 1.0 / np.sqrt(192.0), out=o, workspace=w)
        graphs.append((g, w))
        outs.append(o)
    streams = [torch.cuda.Stream() for _ in graphs]
    torch.cuda.synchronize()
    for _ in range(10):
        for (g, _), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, first)
