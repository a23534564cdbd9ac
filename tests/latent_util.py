"""References in 64 bits for the latent-attention operators and the step tables, and what the GPU results may
be off by."""
from __future__ import annotations

import numpy as np
import torch

EPS = 2.0 ** -8          # half a step of bf16, relative


def attend(q, k, v, scale, n_keys):
    """q [N,D], k [L,D], v [L,Dv] (any float type, CPU or GPU), n_keys [N]: row i attends the first n_keys[i] keys.

    Returns (out, tol), both [N,Dv] float64. ``tol`` bounds the error of a kernel that holds scores, weights' sum
    and output sum in 32 bits and rounds the weights and the output once to bf16:
      output rounding          2^-8 |out|
      weights rounded to bf16  2^-8 A, A = sum_j w_j |v_j| (the weights' sum is taken before the rounding, or
                               after it: then the output moves by another 2^-8 |out|, which is below 2^-8 A)
      32-bit sums over keys    L 2^-24 A
      32-bit scores            a score off by e moves its weight by e relative, and the sum by as much: 2 E A with
                               E = (D + 1) 2^-24 scale max_j sum_d |q_d k_jd|
    (the exponential's and the reciprocal's few 2^-23 go under the 2^-12 A)."""
    q, k, v = q.double(), k.double(), v.double()
    L = k.shape[0]
    out = torch.zeros((q.shape[0], v.shape[1]), dtype=torch.float64, device=q.device)
    tol = torch.zeros_like(out)
    if L == 0 or q.shape[0] == 0:
        return out, tol
    live = torch.arange(L, device=q.device)[None, :] < n_keys.to(q.device)[:, None]
    some = live.any(1)
    s = torch.where(live, (q @ k.T) * scale, torch.tensor(float("-inf"), dtype=torch.float64, device=q.device))
    w = torch.softmax(s[some], dim=1)
    out[some] = w @ v
    A = w @ v.abs()
    E = (q.shape[1] + 1) * 2.0 ** -24 * scale * torch.where(live, q.abs() @ k.abs().T, torch.zeros((), dtype=torch.float64, device=q.device)).amax(1)
    tol[some] = 1.01 * (EPS * out[some].abs() + (2 * EPS + L * 2.0 ** -24 + 2.0 ** -12 + 2 * E[some][:, None]) * A)
    return out, tol


def check(got, ref, tol, what=""):
    got = got.detach().cpu().double()
    ref, tol = ref.cpu(), tol.cpu()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert torch.isfinite(got).all(), f"{what}: non-finite values"
    over = (got - ref).abs() - tol
    assert float(over.max()) <= 0.0, f"{what}: off by {float((got - ref).abs().max()):.3e}, {int((over > 0).sum())} of {over.numel()} over the bound"


def absorbed(q_latent, q_rope, cache, table, seq_lens, scale, R):
    """[B,T,H,R] reference of paged_latent_attention; ``table`` and ``seq_lens`` are host lists."""
    B, T, H, _ = q_latent.shape
    P = cache.shape[1]
    out = torch.zeros((B, T, H, R), dtype=torch.float64)
    tol = torch.zeros_like(out)
    for b in range(B):
        L = max(0, int(seq_lens[b]))
        j = np.arange(L)
        pages = torch.as_tensor(np.asarray(table[b])[j // P].astype(np.int64), device=cache.device)
        rows = cache[pages, torch.as_tensor(j % P, device=cache.device)]
        q = torch.cat([q_latent[b], q_rope[b]], dim=-1).reshape(T * H, -1)
        n_keys = (torch.arange(T) + (L - T + 1)).clamp(min=0).repeat_interleave(H)
        o, t = attend(q, rows, rows[:, :R], scale, n_keys)
        out[b], tol[b] = o.cpu().view(T, H, R), t.cpu().view(T, H, R)
    return out, tol


def expanded(q, k_nope, k_rope, v, cu_q, cu_k, scale):
    """[Tq,H,Dv] reference of latent_prefill_attention (rows outside all sequences are zero here)."""
    tq, H, _ = q.shape
    out = torch.zeros((tq, H, v.shape[2]), dtype=torch.float64)
    tol = torch.zeros_like(out)
    for b in range(len(cu_q) - 1):
        q0, q1, k0, k1 = cu_q[b], cu_q[b + 1], cu_k[b], cu_k[b + 1]
        n_keys = (torch.arange(q1 - q0) + (k1 - k0) - (q1 - q0) + 1).clamp(min=0)
        for h in range(H):
            k = torch.cat([k_nope[k0:k1, h], k_rope[k0:k1]], dim=1)
            o, t = attend(q[q0:q1, h], k, v[k0:k1, h], scale, n_keys)
            out[q0:q1, h], tol[q0:q1, h] = o.cpu(), t.cpu()
    return out, tol


def tables(seq_lens, new_lens, P, free_pages, count, table, capacity):
    """Reference of paged_build_tables for valid lengths: (table, cu, slots, positions, count)."""
    table = np.array(table)
    cu, slots, pos = [0], [], []
    for b, (L, n) in enumerate(zip(seq_lens, new_lens)):
        for i in range(-(-(L - n) // P), -(-L // P)):
            count -= 1
            table[b, i] = free_pages[count]
        cu.append(cu[-1] + n)
        pos += list(range(L - n, L))
        slots += [int(table[b, j // P]) * P + j % P for j in range(L - n, L)]
    pad = [-1] * (capacity - len(slots))
    return table, cu, slots + pad, pos + pad, count


class Paged:
    """A random latent cache with permuted pages; everything that holds no live token is NaN."""

    def __init__(self, lens, P, R, Dr, seed, pages_extra=3, slot_pad=0, page_pad=0, spread=1.0):
        g = np.random.default_rng(seed)
        need = [-(-max(int(L), 0) // P) for L in lens]
        n_pages = sum(need) + pages_extra
        perm = g.permutation(n_pages)
        self.table = np.full((len(lens), max(max(need), 1) + 1), 2 ** 31 - 1, dtype=np.int32)
        self.P, self.R, self.Dr, self.lens = P, R, Dr, list(lens)
        W, slot = R + Dr, R + Dr + slot_pad
        gen = torch.Generator().manual_seed(seed)
        flat = torch.full((n_pages * (P * slot + page_pad),), float("nan"), dtype=torch.bfloat16)
        cache = flat.as_strided((n_pages, P, W), (P * slot + page_pad, slot, 1))
        at = 0
        for b, L in enumerate(lens):
            self.table[b, :need[b]] = perm[at:at + need[b]]
            at += need[b]
            for i in range(need[b]):
                n = min(P, int(L) - i * P)
                cache[int(self.table[b, i]), :n] = (torch.randn((n, W), generator=gen) * spread).to(torch.bfloat16)
        dev = flat.cuda()
        self.cache = dev.as_strided(cache.shape, cache.stride())
        self.host = cache
        self.dtable = torch.from_numpy(self.table).cuda()
        self.dlens = torch.tensor(list(lens), dtype=torch.int32).cuda()
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
