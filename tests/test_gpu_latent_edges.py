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
