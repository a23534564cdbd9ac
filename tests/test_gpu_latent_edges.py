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
