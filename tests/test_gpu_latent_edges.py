"""Latent attention and the step tables where they can go wrong: status words left by other calls, memory behind a
sequence, scores at the ends of the 32-bit range, bounds and strides that mean nothing."""
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


# ---- status words ----------------------------------------------------------------------------------

@pytest.mark.parametrize("lens", [[700, 1, 90], [3000, 10], [300] * 200])
def test_absorbed_with_a_status_word_that_holds_an_expired_wait(lens):
    """The word may be shared with other calls: what an earlier one left there does not keep this one from its work
    (records by sequence, few sequences over many spans, more sequences than spans; a workspace full of ones)."""
    pg = U.Paged(lens, 64, 512, 64, 3)
    ql, qr = randn(4, len(lens), 1, 16, 512), randn(5, len(lens), 1, 16, 64)
    ws, st = pda.latent_workspace(len(lens), 16, 1, 512), ints([3])
    ws.fill_(255)
    out = torch.full(ql.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    pda.paged_latent_attention(ql.cuda(), qr.cuda(), pg.cache, pg.dtable, pg.dlens, 0.07, out=out, workspace=ws, status=st)
    ref, tol = U.absorbed(ql, qr, pg.host, pg.table, lens, 0.07, 512)
    U.check(out, ref, tol)
    assert st.item() == 3


def test_an_expired_wait_stands_above_all_other_codes():
    """One status word for all calls of a step: a wait that expires after other trouble is seen, and stays."""
    def tables(st, count, cap):
        pda.paged_build_tables(ints([64]), ints([64]), 16, ints(range(10)), ints([count]), ints(np.zeros((1, 8))), ints([0, 0]),
                               ints([0] * max(cap, 1))[:cap], status=st)

    for before in (0, 1, 2, 4, 5):
        st = ints([before])
        pda.debug_wait_timeout(1, st)
        assert st.item() == 3
        tables(st, 1, 64)                        # too few pages
        tables(st, 10, 63)                       # too few slots
        assert st.item() == 3
    st = ints([1])
    tables(st, 1, 64)
    assert st.item() == 4
    tables(st, 10, 63)
    assert st.item() == 5
    tables(st, 1, 64)
    assert st.item() == 5


# ---- memory behind a sequence ----------------------------------------------------------------------

@pytest.mark.parametrize("q_lens,k_lens,H", [([40], [1000], 3),             # the keys of a small block split over the halves
                                             ([77], [77], 4), ([150, 9] * 40, [150, 300] * 40, 4),   # two heads at once
                                             ([530], [4600], 2),            # S in two runs
                                             ([300, 513], [700, 513], 60)])  # several row blocks per pair of CTAs
def test_expanded_bits_do_not_depend_on_the_queries_behind(q_lens, k_lens, H):
    """The rows that share a warp with a sequence's last ones are the next sequence's or anything: with other (finite,
    large) values there, the same bits. The keys' size grows, so that such a row's scores pass its first ones again
    and again."""
    B = len(q_lens)
    cq = [int(x) for x in np.concatenate([[0], np.cumsum(np.asarray(q_lens) + 50)])]    # 50 rows of nobody's behind each
    ck = [int(x) for x in np.concatenate([[0], np.cumsum(k_lens)])]
    q, kv, kr = randn(1, cq[-1], H, 192), randn(2, ck[-1], H, 256), randn(3, ck[-1], 64)
    for b in range(B):
        kv[ck[b]:ck[b + 1], :, :128] *= torch.linspace(0.2, 2, k_lens[b])[:, None, None]
    dkv, dkr = kv.cuda(), kr.cuda()
    outs = []
    for spread in (0.0, 1.0, 30.0):
        d = q.clone()
        out = torch.zeros((cq[-1], H, 128), dtype=torch.bfloat16, device="cuda")
        for b in range(B):
            end = cq[b] + q_lens[b]
            d[end:end + 50] = randn(100 + b, 50, H, 192) * spread
        dq = d.cuda()
        for b in range(0, B, 10):   # one call cannot leave rows between sequences out: a call for every tenth, at its place
            pda.latent_prefill_attention(dq[cq[b]:], dkv[..., :128], dkr, dkv[..., 128:], ints([0, q_lens[b]]), ints(ck[b:b + 2]),
                                         q_lens[b], 0.07, out=out[cq[b]:])
        outs.append(out)
        # all sequences in one call, their queries packed: behind each but the last stand the next one's
        packed = torch.cat([d[cq[b]:cq[b] + q_lens[b]] for b in range(B)] + [d[cq[-1] - 50:]]).cuda()
        cu = [int(x) for x in np.concatenate([[0], np.cumsum(q_lens)])]
        outs.append(pda.latent_prefill_attention(packed, dkv[..., :128], dkr, dkv[..., 128:], ints(cu), ints(ck), max(q_lens), 0.07,
                                                 out=torch.zeros((cu[-1] + 50, H, 128), dtype=torch.bfloat16, device="cuda")))
    for a, b in ((0, 2), (0, 4), (1, 3), (1, 5)):
        assert torch.equal(outs[a], outs[b])


def test_expanded_bits_do_not_depend_on_the_next_sequence():
    """The same first sequence before two different second ones."""
    n, k, H = [70, 33], [900, 60], 3
    q, kv, kr = randn(4, sum(n), H, 192), randn(5, sum(k), H, 256), randn(6, sum(k), 64)
    kv[:900, :, :128] *= torch.linspace(0.2, 2, 900)[:, None, None]
    outs = []
    for spread in (1.0, 40.0):
        q[70:] = randn(7, 33, H, 192) * spread
        outs.append(pda.latent_prefill_attention(q.cuda(), kv[..., :128].cuda(), kr.cuda(), kv[..., 128:].cuda(), ints([0, 70, 103]),
                                                 ints([0, 900, 960]), 70, 0.07)[:70])
    assert torch.equal(outs[0], outs[1])


# ---- scores at the ends of the range ---------------------------------------------------------------
# Scores made of powers of two are exact in 32 bits whatever their size, so that of a row's error bound (latent_util)
# all but the scores' part remains: the output's rounding 2^-8 |out|, the weights' 2 * 2^-8 A (theirs and their sum's),
# the 32-bit sums' L 2^-24 A, and the exponential's 2^-12 A (a polynomial's 7.5e-5 of every fourth pair is 2^-13.7).

def attend_exact(q, k, v, scale, n_keys):
    ref = U.attend(q, k, v, scale, n_keys)[0]
    A = U.attend(q, k, v.abs(), scale, n_keys)[0]
    return ref, 1.01 * (U.EPS * ref.abs() + (2 * U.EPS + k.shape[0] * 2.0 ** -24 + 2.0 ** -12) * A)


def levels(kind, n):
    """Scores of n tokens in units of the largest size, as a rotary key's one element."""
    c = torch.ones(n)
    if kind == "down":         # the first tokens weigh, those from the 64th on not
        c[min(64, n - 1):] = 2
        return -c
    if kind == "up":           # the reference rises by far, from below to above zero
        return torch.where(torch.arange(n) < n // 2, -1.0, 1.0)
    if kind == "late":         # the first 130 far below the rest
        c[:min(130, n - 1)] = 4
        return -c
    return c if kind == "plus" else -c


KINDS = ["minus", "plus", "down", "up", "late"]


def run_levels_absorbed(kind, log2_size, flags, lens=(700, 3000, 5, 64), H=16, T=1, R=512, P=64):
    """Scores of +-2^log2_size (times 1, 2 or 4): all of it from one rotary element, the latent part of the query zero."""
    pg = U.Paged(list(lens), P, R, 64, 9)
    half = log2_size // 2
    host = pg.host.clone()
    for b, L in enumerate(lens):
        c = levels(kind, L) * 2.0 ** half * 165 / 128
        j = np.arange(L)
        rows = host[torch.as_tensor(pg.table[b][j // P].astype(np.int64)), torch.as_tensor(j % P)]
        rows[:, R:] = 0
        rows[:, R] = c.to(torch.bfloat16)
        host[torch.as_tensor(pg.table[b][j // P].astype(np.int64)), torch.as_tensor(j % P)] = rows
    pg.cache.copy_(host)
    B = len(lens)
    ql, qr = torch.zeros((B, T, H, R), dtype=torch.bfloat16), torch.zeros((B, T, H, 64), dtype=torch.bfloat16)
    qr[..., 0] = 2.0 ** (log2_size - half - 3) * 141 / 128      # (the products are exact in 32 bits, and not times log2(e))
    got = pda.paged_latent_attention(ql.cuda(), qr.cuda(), pg.cache, pg.dtable, pg.dlens, 8.0, flags=flags, status=pg.status).cpu()
    assert pg.status.item() == 0
    for b, L in enumerate(lens):
        j = np.arange(L)
        rows = host[torch.as_tensor(pg.table[b][j // P].astype(np.int64)), torch.as_tensor(j % P)]
        n_keys = (torch.arange(T) + (L - T + 1)).clamp(min=0)
        ref, tol = attend_exact(torch.cat([ql[b, :, 0], qr[b, :, 0]], dim=-1), rows, rows[:, :R], 8.0, n_keys)
        for h in range(H):
            U.check(got[b, :, h], ref, tol, f"{kind} 2^{log2_size} sequence {b} head {h}")


def run_levels_expanded(kind, log2_size, flags, q_lens=(70, 530, 3), k_lens=(1000, 700, 300), H=2):
    half = log2_size // 2
    cq, ck = ([int(x) for x in np.concatenate([[0], np.cumsum(n)])] for n in (q_lens, k_lens))
    q, kr = torch.zeros((cq[-1], H, 192), dtype=torch.bfloat16), torch.zeros((ck[-1], 64), dtype=torch.bfloat16)
    kn, v = torch.zeros((ck[-1], H, 128), dtype=torch.bfloat16), randn(1, ck[-1], H, 128)
    # (141 * 165 / 2^14: exact in 32 bits, and not when multiplied by log2(e))
    q[..., 128] = 2.0 ** (log2_size - half - 3) * 141 / 128
    for b, n in enumerate(k_lens):
        kr[ck[b]:ck[b + 1], 0] = (levels(kind, n) * 2.0 ** half * 165 / 128).to(torch.bfloat16)
    st = ints([0])
    got = pda.latent_prefill_attention(q.cuda(), kn.cuda(), kr.cuda(), v.cuda(), ints(cq), ints(ck), max(q_lens), 8.0, flags=flags, status=st).cpu()
    assert st.item() == 0
    for b in range(len(q_lens)):
        n_keys = (torch.arange(q_lens[b]) + k_lens[b] - q_lens[b] + 1).clamp(min=0)
        for h in range(H):
            ref, tol = attend_exact(q[cq[b]:cq[b + 1], h], torch.cat([kn[ck[b]:ck[b + 1], h], kr[ck[b]:ck[b + 1]]], dim=1),
                                    v[ck[b]:ck[b + 1], h], 8.0, n_keys)
            U.check(got[cq[b]:cq[b + 1], h], ref, tol, f"{kind} 2^{log2_size} sequence {b} head {h}")




def minus_infinity_absorbed(marked, flags, H=16, R=512):
    """(out, rows) of one sequence whose marked tokens' scores pass the lowest 32-bit number."""
    n = len(marked)
    pg = U.Paged([n], 64, R, 64, 12)
    host = pg.host.clone()
    j = np.arange(n)
    at = torch.as_tensor(pg.table[0][j // 64].astype(np.int64)), torch.as_tensor(j % 64)
    rows = host[at]
    rows[:, R:] = 0
    rows[:, R] = torch.where(marked, -2.0 ** 100, 0.0).to(torch.bfloat16)
    host[at] = rows
    pg.cache.copy_(host)
    ql, qr = torch.zeros((1, 1, H, R), dtype=torch.bfloat16), torch.zeros((1, 1, H, 64), dtype=torch.bfloat16)
    qr[..., 0] = 2.0 ** 100
    return pda.paged_latent_attention(ql.cuda(), qr.cuda(), pg.cache, pg.dtable, pg.dlens, 0.5, flags=flags).cpu()[0, 0], rows


def minus_infinity_expanded(marked, nq, flags, H=2):
    n = len(marked)
    q, kn = torch.zeros((nq, H, 192), dtype=torch.bfloat16), torch.zeros((n, H, 128), dtype=torch.bfloat16)
    kr, v = torch.zeros((n, 64), dtype=torch.bfloat16), randn(2, n, H, 128)
    kr[:, 0] = torch.where(marked, -2.0 ** 100, 0.0).to(torch.bfloat16)
    q[..., 128] = 2.0 ** 100
    out = pda.latent_prefill_attention(q.cuda(), kn.cuda(), kr.cuda(), v.cuda(), ints([0, nq]), ints([0, n]), nq, 0.5, flags=flags).cpu()
    return out, q, torch.cat([kn[:, 0], kr], dim=1), v


def marks(kind, n):
    m = torch.zeros(n, dtype=torch.bool)
    if kind == "first":
        m[:200] = True
    elif kind == "most":
        m[:] = True
        m[n // 2] = False
    elif kind == "last":
        m[n // 3:] = True
    return m


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", [20, 28, 40, 101])
def test_plain_kernels_far_scores(kind, size):
    run_levels_absorbed(kind, size, GENERIC)
    run_levels_expanded(kind, size, GENERIC)


@pytest.mark.parametrize("kind", ["first", "most", "last"])
def test_plain_kernels_scores_below_the_range(kind):
    """Scores of -inf weigh nothing beside finite ones, wherever they stand."""
    n, nq = 700, 90
    marked = marks(kind, n)
    got, rows = minus_infinity_absorbed(marked, GENERIC)
    ref, tol = attend_exact(torch.zeros(1, 1), torch.zeros(int((~marked).sum()), 1), rows[~marked, :512], 1.0, (~marked).sum()[None])
    for h in range(got.shape[0]):
        U.check(got[h:h + 1], ref, tol)
    got, q, k, v = minus_infinity_expanded(marked, nq, GENERIC)
    for h in range(2):
        ref, tol = attend_exact(q[:, h], k, v[:, h], 0.5, torch.arange(nq) + n - nq + 1)
        U.check(got[:, h], ref, tol)


def test_plain_kernels_only_scores_below_the_range():
    """A row without any finite score has no softmax."""
    assert minus_infinity_absorbed(torch.ones(300, dtype=torch.bool), GENERIC)[0].isnan().all()
    assert minus_infinity_expanded(torch.ones(300, dtype=torch.bool), 40, GENERIC)[0].isnan().all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", [20, 27, 28, 31, 40, 101])
def test_absorbed_far_scores(kind, size):
    run_levels_absorbed(kind, size, 0)
    run_levels_absorbed(kind, size, 0, lens=(200, 66, 1, 2000), H=24, T=5)


def test_absorbed_far_scores_split_unevenly():
    """Equal scores far from zero over many spans, each with its own number of tokens: every token weighs the same."""
    for size in (24, 60, 101):
        run_levels_absorbed("minus", size, 0, lens=(4000, 1, 999), H=16)
        run_levels_absorbed("plus", size, 0, lens=(9000,), H=64)


@pytest.mark.parametrize("n", [100, 700, 5000])
@pytest.mark.parametrize("kind", ["first", "most", "last"])
def test_absorbed_scores_below_the_range(kind, n):
    marked = marks(kind, n) if n > 200 else torch.arange(n) % 3 == 0
    got, rows = minus_infinity_absorbed(marked, 0)
    ref, tol = attend_exact(torch.zeros(1, 1), torch.zeros(int((~marked).sum()), 1), rows[~marked, :512], 1.0, (~marked).sum()[None])
    for h in range(got.shape[0]):
        U.check(got[h:h + 1], ref, tol)


@pytest.mark.parametrize("n", [1, 60, 300, 5000])
def test_absorbed_only_scores_below_the_range(n):
    """A row without any finite score has no softmax: NaN, and not the zeros of a row that sees nothing."""
    assert minus_infinity_absorbed(torch.ones(n, dtype=torch.bool), 0)[0].isnan().all()


@pytest.mark.parametrize("lens", [[2, 1], [900, 2], [3000]])
@pytest.mark.parametrize("flags", [0, GENERIC])
def test_absorbed_infinite_query(lens, flags):
    """-inf scores throughout for one row, +inf for another, next to rows that see nothing and ordinary ones."""
    T, H = 4, 16
    pg = U.Paged(lens, 64, 512, 64, 14)
    host = pg.host.clone()
    host[..., 512:] = host[..., 512:].abs()
    pg.cache.copy_(host)
    ql, qr = randn(15, len(lens), T, H, 512), randn(16, len(lens), T, H, 64)
    ref, tol = U.absorbed(ql, qr, host, pg.table, lens, 0.07, 512)
    qr[:, 3, 2, 7], qr[:, 3, 9, 7] = float("-inf"), float("inf")
    got = pda.paged_latent_attention(ql.cuda(), qr.cuda(), pg.cache, pg.dtable, pg.dlens, 0.07, flags=flags).cpu()
    for h in (2, 9):
        assert got[:, 3, h].isnan().all()
        got[:, 3, h], ref[:, 3, h] = 0, 0
    U.check(got, ref, tol)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", [20, 27, 28, 29, 31, 40, 101])
def test_expanded_far_scores(kind, size):
    run_levels_expanded(kind, size, 0)                                              # one of them with its keys split over the halves
    run_levels_expanded(kind, size, 0, q_lens=(90, 200), k_lens=(4000, 129), H=60)  # two heads at once
    run_levels_expanded(kind, size, 0, q_lens=(300,), k_lens=(5000,), H=2)          # S in two runs


@pytest.mark.parametrize("scale", [2.0 ** -120, 2.0 ** -60, 2.0 ** 60, 2.0 ** 120])
def test_expanded_far_scales(scale):
    """Scores so small that only their scale makes them count, and the other way round."""
    n, H = 900, 2
    q, kr, v = torch.zeros((n, H, 192), dtype=torch.bfloat16), torch.zeros((n, 64), dtype=torch.bfloat16), randn(1, n, H, 128)
    kn = torch.zeros((n, H, 128), dtype=torch.bfloat16)
    half = -int(np.log2(scale)) // 2
    q[..., 128] = 2.0 ** half
    kr[:, 0] = (torch.arange(n) % 4 - 2).to(torch.bfloat16) * 2.0 ** half      # scores -2, -1, 0 and 1 times 1
    for flags in (0, GENERIC):
        got = pda.latent_prefill_attention(q.cuda(), kn.cuda(), kr.cuda(), v.cuda(), ints([0, n]), ints([0, n]), n, scale, flags=flags).cpu()
        for h in range(H):
            ref, tol = attend_exact(q[:, h], torch.cat([kn[:, h], kr], dim=1), v[:, h], scale, torch.arange(n) + 1)
            U.check(got[:, h], ref, tol)


@pytest.mark.parametrize("kind", ["first", "most", "last"])
@pytest.mark.parametrize("n,nq", [(700, 90), (5000, 300), (900, 900)])
def test_expanded_scores_below_the_range(kind, n, nq):
    marked = marks(kind, n)
    marked[0] = False                   # (each row sees one that is not)
    got, q, k, v = minus_infinity_expanded(marked, nq, 0)
    for h in range(2):
        ref, tol = attend_exact(q[:, h], k, v[:, h], 0.5, torch.arange(nq) + n - nq + 1)
        U.check(got[:, h], ref, tol)


@pytest.mark.parametrize("n,nq", [(1, 1), (300, 40), (300, 300), (2000, 70), (5000, 300), (30, 60)])
def test_expanded_only_scores_below_the_range(n, nq):
    """NaN where a row sees keys, zeros where it sees none."""
    got = minus_infinity_expanded(torch.ones(n, dtype=torch.bool), nq, 0)[0]
    sees = torch.arange(nq) + n - nq >= 0
    assert got[sees].isnan().all() and (got[~sees] == 0).all()


@pytest.mark.parametrize("flags", [0, GENERIC])
@pytest.mark.parametrize("n,nq", [(1000, 70), (4500, 600), (300, 300)])
def test_expanded_infinite_query(n, nq, flags):
    """-inf scores throughout for one row, +inf for another; the others are as they should be."""
    H, a, b = 2, nq // 3, nq - 1
    q, kv, kr = randn(1, nq, H, 192), randn(2, n, H, 256), randn(3, n, 64).abs()
    ref, tol = U.expanded(q, kv[..., :128], kr, kv[..., 128:], [0, nq], [0, n], 0.07)
    q[a, 1, 130], q[b, 1, 140] = float("-inf"), float("inf")
    got = pda.latent_prefill_attention(q.cuda(), kv[..., :128].cuda(), kr.cuda(), kv[..., 128:].cuda(), ints([0, nq]), ints([0, n]), nq, 0.07,
                                       flags=flags).cpu()
    for i in (a, b):
        assert got[i, 1].isnan().all()
        got[i, 1], ref[i, 1] = 0, 0
    U.check(got, ref, tol)


# ---- bounds and strides that mean nothing ----------------------------------------------------------

@pytest.mark.parametrize("flags", [0, GENERIC])
@pytest.mark.parametrize("max_q", [60, 61, 2 ** 30, 2 ** 31 - 1])
def test_expanded_any_bound_of_the_query_tokens_in_c(max_q, flags):
    """The C call takes any bound, however loose, whatever the number of heads."""
    T, H = 60, 5
    q, kv, kr = randn(1, T, H, 192).cuda(), randn(2, T, H, 256).cuda(), randn(3, T, 64).cuda()
    out, st, cu = torch.zeros((T, H, 128), dtype=torch.bfloat16, device="cuda"), ints([0]), ints([0, T])
    rc = pda.lib().latent_prefill_attention(q.data_ptr(), H * 192, 192, kv.data_ptr(), H * 256, 256, kr.data_ptr(), 64,
                                            kv[..., 128:].data_ptr(), H * 256, 256, cu.data_ptr(), cu.data_ptr(), 1, H, 128, 64, 128, max_q, T, T,
                                            0.07, out.data_ptr(), H * 128, 128, flags, st.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    ref, tol = U.expanded(q.cpu(), kv[..., :128].cpu(), kr.cpu(), kv[..., 128:].cpu(), [0, T], [0, T], 0.07)
    U.check(out, ref, tol)
    assert st.item() == 0


def test_append_one_row_of_any_stride():
    """A tensor of one row may carry any stride between rows, as one cut out of a wider buffer does."""
    buf, rope = randn(1, 601).cuda(), randn(2, 99).cuda()
    cache = torch.zeros((2, 16, 576), dtype=torch.bfloat16, device="cuda")
    pda.latent_append(buf.as_strided((1, 512), (601, 1)), rope.as_strided((1, 64), (99, 1)), cache, ints([17]))
    assert torch.equal(cache[1, 1], torch.cat([buf[:512], rope[:64]])) and int((cache.view(32, 576) != 0).any(1).sum()) == 1


@pytest.mark.parametrize("offset,pad", [(8, 0), (0, 8), (8, 24), (16, 0)])
@pytest.mark.parametrize("lens", [[70, 200, 1], [600]])
def test_expanded_output_aligned_to_16_bytes_only(offset, pad, lens):
    """Rows that begin at 16 but not at 32 bytes: by their base, by the tokens' or heads' stride."""
    H, T = 3, sum(lens)
    cu = [int(x) for x in np.concatenate([[0], np.cumsum(lens)])]
    q, kv, kr = randn(1, T, H, 192), randn(2, T, H, 256), randn(3, T, 64)
    buf = torch.full((offset + T * H * (128 + pad) + 64,), -5.0, dtype=torch.bfloat16, device="cuda")
    out = buf[offset:].as_strided((T, H, 128), (H * (128 + pad), 128 + pad, 1))
    pda.latent_prefill_attention(q.cuda(), kv[..., :128].cuda(), kr.cuda(), kv[..., 128:].cuda(), ints(cu), ints(cu), max(lens), 0.07, out=out)
    ref, tol = U.expanded(q, kv[..., :128], kr, kv[..., 128:], cu, cu, 0.07)
    U.check(out, ref, tol)
    out.fill_(-5.0)
    assert (buf == -5).all()                        # nothing between the rows, before or behind them


@pytest.mark.parametrize("lens", [[700, 3, 64], [4000], [60] * 200])
def test_absorbed_output_between_other_things(lens):
    """Rows at 16 bytes' alignment with gaps, written directly and by the merge."""
    B, H, R = len(lens), 5, 512
    pg = U.Paged(lens, 64, R, 64, 31)
    ql, qr = randn(32, B, 1, H, R), randn(33, B, 1, H, 64)
    buf = torch.full((8 + B * H * (R + 8) + 64,), -5.0, dtype=torch.bfloat16, device="cuda")
    out = buf[8:].as_strided((B, 1, H, R), (H * (R + 8), H * (R + 8), R + 8, 1))
    pda.paged_latent_attention(ql.cuda(), qr.cuda(), pg.cache, pg.dtable, pg.dlens, 0.07, out=out, status=pg.status)
    ref, tol = U.absorbed(ql, qr, pg.host, pg.table, lens, 0.07, R)
    U.check(out, ref, tol)
    out.fill_(-5.0)
    assert (buf == -5).all() and pg.status.item() == 0


def test_calls_captured_without_a_workspace_of_their_own():
    """Buffers that captured calls allocate are the graph's: replays between other calls give the same."""
    pg = U.Paged([3000, 70, 1], 64, 512, 64, 34)
    ql, qr = randn(35, 3, 1, 16, 512).cuda(), randn(36, 3, 1, 16, 64).cuda()
    want = pda.paged_latent_attention(ql, qr, pg.cache, pg.dtable, pg.dlens, 0.07).clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = pda.paged_latent_attention(ql, qr, pg.cache, pg.dtable, pg.dlens, 0.07)
    for _ in range(5):
        other = pda.paged_latent_attention(-ql, qr, pg.cache, pg.dtable, pg.dlens, 0.3)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    assert not torch.equal(other, want)


# ---- the longest sequences -------------------------------------------------------------------------

@pytest.mark.parametrize("T,H,short", [(1, 16, 1), (3, 8, 62), (1, 16, 0)])
def test_absorbed_longest_sequence(T, H, short):
    """Just below 2^31 tokens: the same page over and over, the last one its own. Every slot behind the end is NaN."""
    P, R, n = 1024, 128, 2 ** 21
    L = 2 ** 31 - 1 - short
    host = torch.stack([randn(1, P, R + 64), randn(2, P, R + 64)])
    host[1, P - 1 - short:] = float("nan")
    table = torch.zeros((1, n), dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    ql, qr, st = randn(3, 1, T, H, R), randn(4, 1, T, H, 64), ints([0])
    got = pda.paged_latent_attention(ql.cuda(), qr.cuda(), host.cuda(), table, ints([L]), 0.07, status=st)
    assert st.item() == 0
    # Each row of the first page stands there 2^21 - 1 times; the last page's share of 2^-21 is less than what the bound
    # allows for 1024 keys' roundings. A CTA adds up its 226719 tiles of 64 tokens in 32 bits: four products a tile into the
    # output sum, each off by at most a step of it (2^-23: whether the tensor core rounds or cuts off is not known), and one
    # addition a tile into a weights' sum, off by half a step.
    q = torch.cat([ql[0], qr[0]], dim=-1).reshape(T * H, -1)
    ref, tol = U.attend(q, host[0], host[0][:, :R], 0.07, torch.full((T * H,), P))
    A = U.attend(q, host[0], host[0][:, :R].abs(), 0.07, torch.full((T * H,), P))[0]
    U.check(got.reshape(T * H, R), ref, tol + 226719 * (4 * 2.0 ** -23 + 2.0 ** -24) * A)
