"""Host-side refusals of the rotating cache append and of attention with shaped scores: nothing is enqueued, no GPU needed."""
import ctypes as C
import os
import re

import numpy as np
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
    d = dict(page_stride=8 * 16 * 128, head_stride=16 * 128, slot_stride=128, num_pages=10, page_size=16, num_kv_heads=8, head_dim=128, dtype=0)
    d.update(kw)
    return C.byref(pda.CacheDesc(**d))


def score(scale=0.1, softcap=0.0, slopes=None, window=0):
    return C.byref(pda.ScoreDesc(scale, softcap, slopes, window))


COMMON = [
    (-1, dict(d=desc(page_size=0))), (-2, dict(d=desc(page_size=32))), (-2, dict(d=desc(dtype=2))), (-2, dict(d=desc(head_dim=100))),
    (-2, dict(d=desc(head_dim=288, slot_stride=288))), (-1, dict(d=desc(slot_stride=64))), (-3, dict(d=desc(slot_stride=132))),
    (-1, dict(d=desc(num_pages=-1))), (-1, dict(d=desc(num_kv_heads=0))), (-1, dict(hq=0)), (-1, dict(q=None)), (-1, dict(k=None)),
    (-1, dict(v=None)), (-3, dict(q=P + 8)), (-3, dict(k=P + 4)), (-3, dict(v=P + 2)), (-1, dict(out=None)), (-3, dict(out=P + 2)),
    (-3, dict(status=P + 2)), (-1, dict(d=desc(dtype=1), ks=None)), (-1, dict(d=desc(dtype=1), vs=None)), (-3, dict(d=desc(dtype=1), ks=P + 2)),
]
SCORES = [(-1, dict(s=None)), (-1, dict(s=score(scale=float("nan")))), (-1, dict(s=score(scale=float("inf")))), (-1, dict(s=score(softcap=-1.0))),
          (-1, dict(s=score(softcap=float("nan")))), (-1, dict(s=score(softcap=float("inf")))), (-1, dict(s=score(softcap=1e-38, scale=10.0))),
          (-1, dict(s=score(window=-1))), (-3, dict(s=score(slopes=P + 2)))]


def prefill(lib, d=None, q=P, qs=(4096, 128), k=P, v=P, ks=P, vs=P, bt=P, stride=4, sl=P, cu=P, batch=1, hq=32, max_q=4, total=4, s=0,
            prefix=None, first=None, out=P, os_=(4096, 128), ws=None, wb=0, flags=0, status=None):
    return lib.paged_prefill_attention(q, *qs, k, v, d or desc(), ks, vs, bt, stride, sl, cu, batch, hq, max_q, total, score() if s == 0 else s,
                                       prefix, first, out, *os_, ws, wb, flags, status, None)


@pytest.mark.parametrize("want,kw", COMMON + SCORES + [
    (-1, dict(hq=30)), (-1, dict(batch=-1)), (-1, dict(max_q=-1)), (-1, dict(total=-1)), (-1, dict(stride=-1)), (-1, dict(stride=0)),
    (-1, dict(bt=None)), (-1, dict(sl=None)), (-1, dict(cu=None)), (-3, dict(cu=P + 2)), (-3, dict(bt=P + 1)), (-3, dict(sl=P + 2)),
    (-3, dict(prefix=P + 2)), (-3, dict(first=P + 2)), (-4, dict(batch=65536)), (-4, dict(hq=65536)),
    (-4, dict(max_q=1 << 27, total=1 << 27)), (-3, dict(qs=(4100, 128))), (-3, dict(qs=(4096, 4))), (-1, dict(qs=(-8, 128))),
    (-3, dict(os_=(4096, 130))), (-1, dict(os_=(4096, -8))), (-1, dict(flags=2)), (-3, dict(ws=P + 16, wb=1 << 30)), (-1, dict(ws=P, wb=16)),
    (0, dict(batch=0)), (0, dict(max_q=0)), (0, dict(total=0)),
])
def test_prefill_refusals(lib, want, kw):
    assert prefill(lib, **kw) == want


def decode(lib, d=None, q=P, k=P, v=P, ks=P, vs=P, bt=P, stride=4, sl=P, batch=1, hq=32, s=0, first=None, chunk=0, out=P, po=None, pl=None, mc=0,
           ws=None, flags=0, status=None):
    return lib.paged_biased_decode_attention(q, k, v, d or desc(), ks, vs, bt, stride, sl, batch, hq, score() if s == 0 else s, first, chunk, out, po,
                                             pl, mc, ws, flags, status, None)


@pytest.mark.parametrize("want,kw", COMMON + SCORES + [
    (-1, dict(hq=30)), (-1, dict(batch=-1)), (-4, dict(batch=65536)), (-1, dict(stride=0)), (-1, dict(bt=None)), (-1, dict(sl=None)),
    (-1, dict(chunk=24, po=P, pl=P, mc=4)), (-1, dict(chunk=-16)), (-1, dict(chunk=32)), (-1, dict(chunk=32, po=P, pl=P)),
    (-1, dict(chunk=32, po=P, pl=P, mc=4, out=None)), (-3, dict(chunk=32, po=P + 4, pl=P, mc=4)), (-3, dict(chunk=32, po=P, pl=P + 2, mc=4)),
    (-3, dict(chunk=32, po=P, pl=P, mc=4, ws=P + 2)), (-3, dict(first=P + 2)), (-1, dict(flags=4)), (0, dict(batch=0)),
])
def test_decode_refusals(lib, want, kw):
    assert decode(lib, **kw) == want


def append(lib, d=None, q=P, qs=(6144, 128), k=P, k_s=(6144, 128), v=P, v_s=(6144, 128), pos=P, ps=0, axes=1, axis=None, cs=P, table=100, rot=128,
           qn=None, kn=None, eps=1e-6, slots=P, n=4, hq=32, out=P, os_=(4096, 128), kc=P, vc=P, ks=P, vs=P, status=None):
    return lib.rope_kv_append(q, *qs, k, *k_s, v, *v_s, pos, ps, axes, axis, cs, table, rot, 0, qn, kn, eps, slots, n, hq, out, *os_, kc, vc,
                              d or desc(), ks, vs, status, None)


@pytest.mark.parametrize("want,kw", COMMON + [
    (-1, dict(n=-1)), (0, dict(n=0)), (-1, dict(rot=-16)), (-2, dict(rot=24)), (-1, dict(rot=144)), (-1, dict(table=-1)), (-1, dict(axes=0)),
    (-2, dict(axes=5, ps=4)), (-1, dict(axes=2, ps=3)), (-1, dict(axis=b"\1" * 64)), (-1, dict(axes=2, ps=4, axis=b"\2" * 64)),
    (-1, dict(eps=-1.0)), (-1, dict(eps=float("nan"))), (-1, dict(eps=float("inf"))), (-1, dict(pos=None)), (-1, dict(cs=None)),
    (-1, dict(slots=None)), (-1, dict(kc=None)), (-1, dict(vc=None)), (-3, dict(kc=P + 8)), (-3, dict(cs=P + 4)), (-3, dict(pos=P + 2)),
    (-3, dict(slots=P + 1)), (-3, dict(qn=P + 2)), (-3, dict(kn=P + 8)), (-3, dict(qs=(6145, 128))), (-1, dict(k_s=(-8, 128))),
    (-3, dict(v_s=(6144, 132))), (-3, dict(os_=(4096, 4))), (-4, dict(hq=65536)), (-4, dict(n=1 << 27)),
])
def test_append_refusals(lib, want, kw):
    assert append(lib, **kw) == want


def test_workspace_size(lib):
    f = lib.pda_prefill_workspace_bytes
    assert f(0, 128) == -1 and f(8, 0) == -1 and f(8, 100) == -1 and f(8, 288) == -1 and f(8, 128) > 0


def bf(*s):
    return torch.zeros(s, dtype=torch.bfloat16)


def i32(*s):
    return torch.zeros(s, dtype=torch.int32)


CACHE = dict(k_cache=bf(4, 2, 16, 64), v_cache=bf(4, 2, 16, 64))
BYTES = dict(k_cache=torch.zeros((4, 2, 16, 64), dtype=torch.uint8), v_cache=torch.zeros((4, 2, 16, 64), dtype=torch.uint8))


@pytest.mark.parametrize("kw,text", [
    (dict(v_cache=bf(4, 2, 16, 32)), "v_cache"), (dict(v_cache=BYTES["v_cache"]), "one type"), (dict(v_cache=bf(4, 16, 2, 64).transpose(1, 2)), "strides"),
    (BYTES, "k_scale"), (dict(BYTES, k_scale=torch.zeros(4, 2), v_scale=torch.zeros(4, 2, dtype=torch.float64)), "k_scale"),
    (dict(BYTES, k_scale=torch.zeros(4, 2), v_scale=torch.zeros(2, 4).T), "k_scale"),
    (dict(seq_lens=i32(2)), "cu_q"), (dict(cu_q=torch.zeros(4, dtype=torch.int64)), "int32"), (dict(block_table=i32(3, 8)[:, :4]), "block_table"),
    (dict(block_table=i32(2, 8)), "block_table"), (dict(slopes=torch.zeros(3)), "slopes"), (dict(slopes=torch.zeros(8)[::2]), "slopes"),
    (dict(prefix_lens=i32(2)), "prefix_lens"), (dict(first_keys=i32(3)), "first_keys"), (dict(out=bf(5, 2, 64)), "out"), (dict(out=bf(6, 4, 64)), "out"),
    (dict(q=bf(5, 4, 128)), "head_dim"), (dict(q=bf(5, 4, 128)[..., ::2]), "contiguous"), (dict(workspace=torch.zeros(1, dtype=torch.uint8).expand(1 << 28)), "workspace"),
    (dict(), "CUDA"),
])
def test_prefill_binding_refusals(kw, text):
    args = dict(dict(q=bf(5, 4, 64), block_table=i32(3, 8), seq_lens=i32(3), cu_q=i32(4), max_q=5, scale=0.1), **CACHE)
    args.update(kw)
    with pytest.raises(ValueError, match=text):
        pda.paged_prefill_attention(**args)


@pytest.mark.parametrize("kw,text", [
    (dict(q=bf(3, 4, 128)[..., ::2]), "q:"), (dict(q=bf(3, 8, 64)[:, ::2]), "q:"), (dict(seq_lens=i32(2)), "seq_lens"), (dict(first_keys=i32(4)), "first_keys"),
    (dict(chunk_tokens=64), "part_o"), (dict(chunk_tokens=64, part_o=torch.zeros(3, 4, 2, 64), part_lse=torch.zeros(3, 4, 3)), "part_o"),
    (dict(chunk_tokens=64, part_o=torch.zeros(3, 4, 2, 64), part_lse=torch.zeros(3, 4, 2).double()), "float32"),
    (dict(chunk_tokens=64, part_o=torch.zeros(3, 4, 2, 64), part_lse=torch.zeros(3, 4, 2), workspace=i32(7)), "workspace"),
    (dict(out=bf(3, 4, 32)), "out"), (dict(), "CUDA"),
])
def test_decode_binding_refusals(kw, text):
    args = dict(dict(q=bf(3, 4, 64), block_table=i32(3, 8), seq_lens=i32(3), scale=0.1), **CACHE)
    args.update(kw)
    with pytest.raises(ValueError, match=text):
        pda.paged_biased_decode_attention(**args)


@pytest.mark.parametrize("kw,text", [
    (dict(k=bf(5, 3, 64)), "heads"), (dict(v=bf(5, 1, 64)), "heads"), (dict(k=bf(4, 2, 64)), "k:"), (dict(out=bf(5, 3, 64)), "heads"),
    (dict(slot_map=i32(4)), "slot_map"), (dict(q_norm=bf(32)), "q_norm"), (dict(k_norm=bf(64, 2)[:, 0]), "k_norm"), (dict(k_norm=torch.zeros(64)), "k_norm"),
    (dict(cos_sin=torch.zeros(9, 64).double()), "cos_sin"), (dict(cos_sin=torch.zeros(9, 128)[:, ::2]), "cos_sin"), (dict(positions=i32(4)), "positions"),
    (dict(positions=i32(5).long()), "positions"), (dict(positions=i32(2, 5)), "freq_axis"), (dict(positions=i32(2, 5), freq_axis=[0] * 31), "freq_axis"),
    (dict(positions=i32(2, 5), freq_axis=[2] * 32), "freq_axis"), (dict(positions=i32(5, 2).T), "positions"), (dict(q=bf(5, 4, 32)), "head_dim"), (dict(), "CUDA"),
])
def test_append_binding_refusals(kw, text):
    args = dict(dict(q=bf(5, 4, 64), k=bf(5, 2, 64), v=bf(5, 2, 64), positions=i32(5), cos_sin=torch.zeros(9, 64), slot_map=i32(5)), **CACHE)
    args.update(kw)
    with pytest.raises(ValueError, match=text):
        pda.rope_kv_append(**args)


def source(name):
    return open(os.path.join(os.path.dirname(pda.__file__), "csrc", name)).read()


@pytest.mark.parametrize("name,reach,bound", [("c5", 0.5, 2.0 ** -17.4), ("c11", 1.25, 2.0 ** -18.6)])
def test_polynomials_of_the_cap_are_within_their_bounds(name, reach, bound):
    """The odd polynomials of the hyperbolic tangent, as they stand in the source, in 64 and in 32 bits (a rounding for each of
    their steps, of sums below 2)."""
    text = re.search(r"static const double %s\[\d+\] = \{([^}]*)\}" % name, source("prefill_tc.cu")).group(1)
    c = [float(x) for x in text.split(",")]
    x = np.linspace(-reach, reach, 400001)
    exact = np.tanh(x)
    assert np.abs(x * np.polyval(c[::-1], x * x) - exact).max() < bound
    f = x.astype(np.float32)
    t = f * f
    y = np.full(f.shape, c[-1], dtype=np.float32)
    for a in c[-2::-1]:
        y = y * t + np.float32(a)
    assert np.abs((f * y).astype(np.float64) - np.tanh(f.astype(np.float64))).max() < bound + (2 * len(c) + 2) * 2.0 ** -24 * reach


def test_polynomial_of_the_exponentials_is_within_its_bound():
    body = source("prefill_tc.cuh").split("void exp2_two", 1)[1].split("\n}", 1)[0]
    c = [float(x) for x in re.findall(r"both\((0\.\d+)f\)", body)]
    assert len(c) == 4
    f = np.linspace(-0.5, 0.5, 200001)
    assert np.abs(np.polyval(c, f) / np.exp2(f) - 1).max() < 7.6e-5      # (of the 2^-12 that the GPU tests' bounds allow)
