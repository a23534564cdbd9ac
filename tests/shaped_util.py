"""References in 64 bits for the rotating cache append and for attention with shaped scores over the paged cache, and what
the GPU results may be off by. Everything is computed on the CPU."""
from __future__ import annotations

import numpy as np
import torch

EPS = 2.0 ** -8          # half a step of bf16, relative
E4M3 = torch.float8_e4m3fn


def visible(lens, new, window=0, prefix=None, first=None):
    """Per sequence (lo, hi) of its query tokens; ``first`` is indexed by query token."""
    out, at = [], 0
    for b, (L, n) in enumerate(zip(lens, new)):
        p = torch.arange(n) + (L - n)
        hi = torch.where(p < 0, 0, torch.maximum(p + 1, torch.tensor(min(prefix[b], L) if prefix is not None else 0)))
        lo = torch.zeros_like(p)
        if first is not None:
            lo = torch.maximum(lo, torch.as_tensor(np.asarray(first[at:at + n])).long())
        if window:
            lo = torch.maximum(lo, p - window + 1)
        at += n
        out.append((lo, hi))
    return out


class Cache:
    """Random paged caches with permuted pages; everything that holds no live token is NaN. ``k``, ``v``: per sequence, the
    values that stand there, [L, Hkv, D] float64; ``vb``: largest |stored byte| of e4m3 values (1 for bf16)."""

    def __init__(self, lens, Hkv, D, fp8=False, seed=0, extra=3, spread=1.0, layout="head", shared=None):
        g = np.random.default_rng(seed)
        need = [-(-max(int(L), 0) // 16) for L in lens]
        n_pages = sum(need) + extra
        perm = g.permutation(n_pages)
        self.table = np.full((len(lens), max(max(need, default=0), 1) + 1), 2 ** 31 - 1, dtype=np.int32)
        self.lens, self.fp8, self.D = list(map(int, lens)), fp8, D
        gen = torch.Generator().manual_seed(seed)
        self.k, self.v, self.scales = [], [], []
        caches = []
        at = 0
        for b in range(len(lens)):
            self.table[b, :need[b]] = perm[at:at + need[b]]
            at += need[b]
        for which in range(2):
            host = torch.full((n_pages, Hkv, 16, D), float("nan"), dtype=torch.bfloat16)
            for b, L in enumerate(self.lens):
                for i in range(need[b]):
                    m = min(16, L - 16 * i)
                    host[int(self.table[b, i]), :, :m] = (torch.randn((Hkv, m, D), generator=gen) * spread).to(torch.bfloat16)
            scale = None
            if fp8:
                scale = torch.rand((n_pages, Hkv), generator=gen) * 0.01 + 0.005
                dead = host.isnan()
                host = (host.float() / scale[:, :, None, None]).clamp(-448, 448).to(E4M3)
                host.view(torch.uint8)[dead] = 0xFF
            rows = self.k if which == 0 else self.v
            for b, L in enumerate(self.lens):
                j = torch.arange(max(L, 0))
                pages = torch.as_tensor(self.table[b].astype(np.int64))[j // 16] if L > 0 else j
                x = host[pages, :, j % 16].double()
                if fp8:
                    x = x * scale[pages].double()[:, :, None]
                rows.append(x)
            if layout == "slot":     # [pages, slots, heads, D] storage
                dev = host.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3)
            else:
                dev = host.cuda()
            caches.append(dev)
            self.scales.append(scale)
        self.k_cache, self.v_cache = caches
        self.k_scale, self.v_scale = (None if s is None else s.cuda() for s in self.scales)
        self.byte = 1.0 / 0.005 * spread * 5 if fp8 else 0.0
        self.dev_table = torch.from_numpy(self.table).cuda()

    def args(self):
        return dict(k_scale=self.k_scale, v_scale=self.v_scale)


def attend(q, k, v, lo, hi, pos, scale, softcap=0.0, slope=0.0, decode_byte=0.0):
    """q [n,D] of one head, k, v [L,D] float64; row i stands at pos[i] and sees lo[i] <= j < hi[i]. Returns (out, tol), [n,D].

    ``tol`` bounds a kernel that holds scores, sums and outputs in 32 bits and rounds the weights and the output once to
    16 bits:
      output rounding            2^-8 |out|
      weights rounded to bf16    2 * 2^-8 A, A = sum_j w_j |v_j| (sum of the weights before or after the rounding)
      32-bit sums over keys      L 2^-24 A
      exponential                2^-12 A
      scores off by e_j          sum_j w_j e_j (|v_j| + |out|), doubled for the second order, where e_j adds up
                                 (D + 3) 2^-24 scale sum_d |q_d k_jd|      the product and its multiplications
                                 softcap 2^-17                             the hyperbolic tangent (relative to 1)
                                 2^-22 (slope |p - j| + |score|)           the bias and its addition
      decode, e4m3               2^-25 sum_j |byte_j|: weights times the value scale, held in fp16 (step 2^-24), next to
                                 the largest weight, which is 1"""
    q, n, L = q.double(), q.shape[0], k.shape[0]
    out = torch.zeros((n, v.shape[1]), dtype=torch.float64)
    tol = torch.zeros_like(out)
    if L == 0 or n == 0:
        return out, tol
    j = torch.arange(L)
    live = (j[None, :] >= lo[:, None]) & (j[None, :] < hi[:, None])
    some = live.any(1)
    if not some.any():
        return out, tol
    live, q, pos = live[some], q[some], pos[some]
    s = (q @ k.T) * scale
    e = (q.shape[1] + 3) * 2.0 ** -24 * abs(scale) * (q.abs() @ k.abs().T)
    if softcap > 0:
        s = softcap * torch.tanh(s / softcap)
        e = torch.minimum(e, torch.tensor(2 * softcap, dtype=torch.float64)) + softcap * 2.0 ** -17
    dist = (pos[:, None] - j[None, :]).abs().double()
    s = s - slope * dist
    e = e + 2.0 ** -22 * (abs(slope) * dist + s.abs())
    w = torch.softmax(torch.where(live, s, torch.tensor(float("-inf"), dtype=torch.float64)), dim=1)
    o = w @ v
    A = w @ v.abs()
    we = w * e
    t = EPS * o.abs() + (2 * EPS + L * 2.0 ** -24 + 2.0 ** -12) * A + 2 * (we @ v.abs() + we.sum(1, keepdim=True) * o.abs())
    t = t + 2.0 ** -25 * decode_byte * live.sum(1, keepdim=True)
    out[some], tol[some] = o, 1.01 * t
    return out, tol


def reference(c, q, new, scale, softcap=0.0, slopes=None, window=0, prefix=None, first=None, decode=False):
    """[T,Hq,D] (out, tol); ``q`` [T,Hq,D] CPU, ``c`` a Cache, ``new`` the query tokens of each sequence."""
    T, Hq, D = q.shape
    out = torch.zeros((T, Hq, D), dtype=torch.float64)
    tol = torch.zeros_like(out)
    see = visible(c.lens, new, window, prefix, first)
    at = 0
    for b, n in enumerate(new):
        L = max(c.lens[b], 0)
        Hkv = c.k[b].shape[1] if L else 1
        pos = torch.arange(n) + (L - n)
        for h in range(Hq):
            if L and n:
                g = h // (Hq // Hkv)
                out[at:at + n, h], tol[at:at + n, h] = attend(
                    q[at:at + n, h], c.k[b][:, g], c.v[b][:, g], *see[b], pos, scale, softcap, 0.0 if slopes is None else float(slopes[h]),
                    c.byte if decode and c.fp8 else 0.0)
        at += n
    return out, tol


def check(got, ref, tol, what=""):
    got = got.detach().cpu().double()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert torch.isfinite(got).all(), f"{what}: {int((~torch.isfinite(got)).sum())} non-finite values of {got.numel()}"
    over = (got - ref).abs() - tol
    assert float(over.max()) <= 0.0, f"{what}: off by {float((got - ref).abs().max()):.3e}, {int((over > 0).sum())} of {over.numel()} over the bound"


def rotate(x, weight, eps, cos, sin, rot, interleaved):
    """x [T,H,D] float64 -> (rotated rows, sizes that their 32-bit error is relative to); cos, sin [T, rot/2]."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    y, size = x.clone(), x.abs()
    half = rot // 2
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, half), slice(half, rot))
    c, s = cos[:, None, :].double(), sin[:, None, :].double()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    both = x[..., a].abs() + x[..., b].abs()
    size[..., a], size[..., b] = both, both
    return y, size
