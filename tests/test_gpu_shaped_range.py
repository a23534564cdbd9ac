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
