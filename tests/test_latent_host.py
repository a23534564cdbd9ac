"""Host-side refusals of the latent-attention calls and the step tables: nothing is enqueued, no GPU needed."""
import ctypes as C

import pytest
import torch

from paper_2605_06068_b200 import binding as pda
from paper_2605_06068_b200 import build as pda_build

P = 0x10000


@pytest.fixture(scope="module")
def lib():
    pda_build.build()
    return pda.lib()


def desc(**kw):
    d = dict(page_stride=64 * 576, slot_stride=576, num_pages=10, page_size=64, latent_dim=512, rope_dim=64, dtype=0)
    d.update(kw)
    return C.byref(pda.LatentDesc(**d))


def attention(lib, d=None, ql=P, qls=(8192, 512), qr=P, qrs=(1024, 64), cache=P, bt=P, stride=4, sl=P, batch=1, heads=16, n=1,
              out=P, os_=(8192, 512), ws=P, wb=None, flags=0, status=None):
    if wb is None:
        wb = max(0, lib.pda_latent_workspace_bytes(1, max(heads, 1), max(n, 1), 512))
    return lib.paged_latent_attention(ql, *qls, qr, *qrs, cache, d or desc(), bt, stride, sl, batch, heads, n, 0.1, out, *os_, ws,
                                      wb, flags, status, None)


@pytest.mark.parametrize("want,kw", [
    (-1, dict(d=desc(page_size=0))), (-2, dict(d=desc(page_size=2048))), (-2, dict(d=desc(dtype=1))),
    (-2, dict(d=desc(latent_dim=516))), (-2, dict(d=desc(latent_dim=1032, slot_stride=1096))), (-2, dict(d=desc(rope_dim=264, slot_stride=776))),
    (-1, dict(d=desc(slot_stride=568))), (-3, dict(d=desc(slot_stride=580))), (-3, dict(d=desc(page_stride=64 * 576 + 4))),
    (-1, dict(d=desc(num_pages=-1))), (-1, dict(batch=-1)), (-1, dict(heads=0)), (-1, dict(n=0)), (-1, dict(n=4097)),
    (-4, dict(batch=40000, n=2)), (-4, dict(heads=70000)), (-1, dict(ql=None)), (-1, dict(qr=None)), (-1, dict(cache=None)),
    (-1, dict(bt=None)), (-1, dict(sl=None)), (-1, dict(out=None)), (-1, dict(ws=None)), (-1, dict(stride=0)),
    (-3, dict(ql=P + 8)), (-3, dict(out=P + 2)), (-3, dict(ws=P + 16)), (-3, dict(qls=(8192, 516))), (-1, dict(os_=(-8, 512))),
    (-1, dict(wb=100)), (-1, dict(flags=2)), (-3, dict(status=P + 2)), (0, dict(batch=0)),
])
def test_absorbed_refusals(lib, want, kw):
    assert attention(lib, **kw) == want


def test_workspace_size(lib):
    f = lib.pda_latent_workspace_bytes
    assert f(1, 0, 1, 512) == -1 and f(-1, 16, 1, 512) == -1 and f(1, 16, 0, 512) == -1 and f(1, 16, 1, 2000) == -1
    assert f(1, 16, 1, 512) < f(1, 32, 1, 512) < f(1, 128, 1, 512) == f(256, 128, 4, 512)


def append(lib, d=None, c=P, cs=576, r=P, rs=576, cache=P, w=None, eps=1e-6, slots=P, n=4):
    return lib.latent_append(c, cs, r, rs, cache, d or desc(), w, eps, slots, n, None, None)


@pytest.mark.parametrize("want,kw", [
    (-1, dict(c=None)), (-1, dict(r=None)), (-1, dict(cache=None)), (-1, dict(slots=None)), (-1, dict(n=-1)), (0, dict(n=0)),
    (-1, dict(eps=-1.0)), (-1, dict(eps=float("nan"))), (-1, dict(eps=float("inf"))), (-3, dict(cs=577)), (-3, dict(rs=4)),
    (-1, dict(cs=-8)), (-3, dict(c=P + 2)), (-3, dict(w=P + 4)), (-2, dict(d=desc(latent_dim=12))),
])
def test_append_refusals(lib, want, kw):
    assert append(lib, **kw) == want


def build_tables(lib, sl=P, nl=P, batch=2, page=16, free=P, cap_free=8, cnt=P, cnt_out=P, bt=P, stride=4, cu=P, slots=P, pos=None, cap=8):
    return lib.paged_build_tables(sl, nl, batch, page, free, cap_free, cnt, cnt_out, bt, stride, cu, slots, pos, cap, None, None)


@pytest.mark.parametrize("want,kw", [
    (-1, dict(sl=None)), (-1, dict(nl=None)), (-1, dict(batch=-1)), (-1, dict(page=0)), (-2, dict(page=2048)), (-1, dict(free=None)),
    (-1, dict(cap_free=-1)), (-1, dict(cnt=None)), (-1, dict(cnt_out=None)), (-1, dict(bt=None)), (-1, dict(stride=-1)),
    (-1, dict(cu=None)), (-1, dict(slots=None)), (-1, dict(cap=-1)), (-3, dict(pos=P + 1)),
])
def test_tables_refusals(lib, want, kw):
    assert build_tables(lib, **kw) == want


def prefill(lib, q=P, qs=(3200, 192), kn=P, kns=(4096, 256), kr=P, krs=64, v=P, vs=(4096, 256), cq=P, ck=P, batch=1, heads=16,
            dims=(128, 64, 128), max_q=4, tq=4, tk=4, out=P, os_=(2048, 128), flags=0):
    return lib.latent_prefill_attention(q, *qs, kn, *kns, kr, krs, v, *vs, cq, ck, batch, heads, *dims, max_q, tq, tk, 0.1, out,
                                        *os_, flags, None, None)


@pytest.mark.parametrize("want,kw", [
    (-1, dict(q=None)), (-1, dict(kn=None)), (-1, dict(kr=None)), (-1, dict(v=None)), (-1, dict(cq=None)), (-1, dict(ck=None)),
    (-1, dict(out=None)), (-1, dict(batch=-1)), (-4, dict(batch=70000)), (-1, dict(heads=0)), (-4, dict(heads=70000)),
    (-2, dict(dims=(132, 64, 128))), (-2, dict(dims=(128, 60, 128))), (-2, dict(dims=(128, 64, 520))), (-1, dict(dims=(0, 64, 128))),
    (-1, dict(max_q=-1)), (-1, dict(tq=-1)), (-1, dict(tk=-1)), (-3, dict(qs=(3201, 192))), (-1, dict(os_=(-8, 128))),
    (-3, dict(kn=P + 8)), (-1, dict(flags=8)), (0, dict(batch=0)), (0, dict(max_q=0)), (0, dict(tq=0)),
])
def test_prefill_refusals(lib, want, kw):
    assert prefill(lib, **kw) == want


def test_binding_refuses_what_it_can_see_without_a_gpu():
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        pda.latent_append(bf(2, 512), bf(2, 64), bf(3, 16, 576), i32(2))
    with pytest.raises(ValueError, match="one entry per token"):
        pda.latent_append(bf(2, 512), bf(2, 64), bf(3, 16, 576), i32(3))
    with pytest.raises(TypeError):
        pda.latent_append(torch.zeros(2, 512), bf(2, 64), bf(3, 16, 576), i32(2))
    with pytest.raises(ValueError, match="int32"):
        pda.paged_build_tables(i32(2).long(), i32(2), 16, i32(4), i32(1), i32(2, 4), i32(3), i32(8))
    with pytest.raises(ValueError, match="rows must follow"):
        pda.paged_build_tables(i32(2), i32(2), 16, i32(4), i32(1), i32(2, 8)[:, :4], i32(3), i32(8))
    with pytest.raises(ValueError, match="q_rope"):
        pda.paged_latent_attention(bf(2, 4, 512), bf(2, 4, 32), bf(3, 16, 576), i32(2, 4), i32(2), 0.1, workspace=i32(4))
    with pytest.raises(ValueError, match="evenly strided"):
        pda.paged_latent_attention(bf(2, 6, 4, 512)[:, :3], bf(2, 3, 4, 64), bf(3, 16, 576), i32(2, 4), i32(2), 0.1, workspace=i32(4))
    with pytest.raises(ValueError, match="k_rope"):
        pda.latent_prefill_attention(bf(4, 2, 192), bf(4, 2, 128), bf(3, 64), bf(4, 2, 128), i32(2), i32(2), 4, 0.1)
    with pytest.raises(ValueError, match="cu_q"):
        pda.latent_prefill_attention(bf(4, 2, 192), bf(4, 2, 128), bf(4, 64), bf(4, 2, 128), i32(2), i32(3), 4, 0.1)


def test_status_texts():
    assert "free pages" in pda.status_string(4) and "slot map" in pda.status_string(5)
    assert set(pda.DEV_STATUS) == {0, 1, 2, 3, 4, 5}
