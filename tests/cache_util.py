"""Plumbing of the 8-bit cache's tests: a context of one shape, its caches, and the definitions in 64 bits."""
from __future__ import annotations

import math

import numpy as np
import torch

from paper_2402_05109_amd import binding as hb

DEV = "cuda:0"
FMT = {"int8": hb.KV8_INT8, "e4m3": hb.KV8_E4M3}


def tree_parent(T, arity=3):
    return [-1] + [(n - 1) // arity for n in range(1, T)]


def ancestors(parent):
    m = torch.zeros(len(parent), len(parent), dtype=torch.bool)
    for n, p in enumerate(parent):
        if p >= 0:
            m[n] = m[p]
        m[n, n] = True
    return m


def context(H, Dh, B, T=1, NL=1, max_pos=256, arity=3, dtype=hb.HYDRA_BF16, parent=None):
    c = hb.Hydra(d=H * Dh, n_layers=NL, n_heads=H, head_dim=Dh, ffn=128, vocab=32, dtype=dtype, max_pos=max_pos, parent=parent or tree_parent(T, arity), max_batch=B)
    c.arena = torch.zeros(c.weights_bytes(), dtype=torch.uint8, device=DEV)
    c.bind_weights(c.arena)
    c.ws = torch.empty(c.workspace_bytes(B), dtype=torch.uint8, device=DEV)
    return c


def caches(H, Dh, B, NL, slots, fmt, seed=0, more=0):
    """An 8-bit cache with a full-length 16-bit tail, pages in random places; everything not written is NaN (codes that are NaN
    in e4m3).  more: so many unused pages in front of all others."""
    g = torch.Generator().manual_seed(seed)
    pages = (slots + 15) // 16
    n16 = more + B * pages + 2
    table16 = more + torch.randperm(B * pages + 2, generator=g)[:B * pages].reshape(B, pages)
    n8 = more + B * pages + 3
    table8 = more + torch.randperm(B * pages + 3, generator=g)[:B * pages].reshape(B, pages)
    block = H * 16 * Dh
    k, v = (torch.full((NL * n16 * block,), math.nan, dtype=torch.float16, device=DEV) for _ in range(2))
    tail = hb.KV(k, v, table16.to(torch.int32).to(DEV).contiguous(), n16)
    kc, vc = (torch.full((NL * n8 * block,), 0xFF, dtype=torch.uint8, device=DEV) for _ in range(2))
    scales = torch.full((NL, n8, H, 2), math.nan, device=DEV)
    return hb.KV8(tail, kc, vc, scales, table8.to(torch.int32).to(DEV).contiguous(), torch.zeros(B, dtype=torch.int32, device=DEV), n8, FMT[fmt])


def round11_up(a):
    """Smallest number of 11 significant bits >= a (float64, a > 0).  On the host: torch.ldexp multiplies by pow(2, e), which a GPU
    does not return exactly."""
    m, e = np.frexp(a.cpu().numpy())
    return torch.from_numpy(np.ldexp(np.ceil(m * 2048), e - 11)).to(a.device)


def exact_exp2(e):
    return torch.from_numpy(np.ldexp(1.0, e.cpu().numpy().astype(np.int64))).to(e.device)


def block_values(x, fmt):
    """x [..., 16, Dh] float64: one block in the last two dims.  (values that its codes stand for, scale [...]) by the definition."""
    x = x.double()
    top = x.abs().amax(dim=(-1, -2))
    safe = torch.where(top > 0, top, torch.ones_like(top))
    if fmt == "int8":
        s = torch.where(top > 0, round11_up(safe / 127), torch.ones_like(top))
        q = torch.round(x / s[..., None, None]).clamp(-127, 127)
        return q * s[..., None, None], s
    s = torch.where(top > 0, exact_exp2(torch.ceil(torch.log2(safe / 448))), torch.ones_like(top))
    y = x / s[..., None, None]
    step = exact_exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * s[..., None, None], s


def cache_values(kv, n_sealed, fmt):
    """kv [B, slots, 2, H, Dh] as written; rows' first n_sealed[b] pages as their 8-bit values.  Returns (values float64, scales of V per slot
    [B, slots, H], 1 in the tail)."""
    kv = kv.double().clone()
    B, S, _, H, Dh = kv.shape
    sv = torch.ones(B, S, H, dtype=torch.float64, device=kv.device)
    for b in range(B):
        n = int(n_sealed[b])
        if n:
            x = kv[b, :16 * n].reshape(n, 16, 2, H, Dh).permute(0, 2, 3, 1, 4)
            val, s = block_values(x, fmt)
            kv[b, :16 * n] = val.permute(0, 3, 1, 2, 4).reshape(16 * n, 2, H, Dh)
            sv[b, :16 * n] = s[:, 1].repeat_interleave(16, dim=0)
    return kv, sv


def attention_reference(q, values, sv, L, parent):
    """Result of tree attention in 64 bits, and how far the library's half may be from it.

    A weight w <= 1 is rounded to half (2^-11 of its value, or 2^-25 where it is subnormal), its exponent c s_K z carries the error of a
    sum of Dh products in 32 bits (rounded each by 2^-24 of the sum of magnitudes) and of a few further operations, and the result is
    rounded to half."""
    B, T, H, Dh = q.shape
    anc = ancestors(parent).to(q.device)
    out = torch.zeros(B, T, H, Dh, dtype=torch.float64, device=q.device)
    tol = torch.zeros_like(out)
    for b in range(B):
        n = int(L[b])
        keys = values[b, :n + T]
        seen = torch.cat([torch.ones(T, n, dtype=torch.bool, device=q.device), anc], dim=1)
        qb = q[b].double().permute(1, 0, 2).contiguous()                            # [H, T, Dh]
        k = keys[:, 0].permute(1, 2, 0).contiguous()                                # [H, Dh, S]
        v = keys[:, 1].permute(1, 0, 2).contiguous()
        s = torch.bmm(qb, k) / math.sqrt(Dh)
        size = torch.bmm(qb.abs(), k.abs()) / math.sqrt(Dh)
        s = torch.where(seen[None], s, torch.full_like(s, -math.inf))
        p = torch.softmax(s, dim=-1)
        o = torch.bmm(p, v)
        werr = 2 * (Dh + 8) * 2.0 ** -24 * torch.where(seen[None], size, torch.zeros_like(size)).amax(dim=-1, keepdim=True) + 2.0 ** -18
        pv = torch.bmm(p, v.abs())
        # w relative to the largest p s_V of the row; sub: what 2^-25 of it is in units of the result, per code of V
        sj = sv[b, :n + T].T[:, None, :]                                            # [H, 1, S]
        big = (p * sj).amax(dim=-1, keepdim=True)
        sub = 2.0 ** -25 * big * (v.abs() / sj.transpose(1, 2)).sum(dim=1, keepdim=True)
        out[b] = o.permute(1, 0, 2)
        tol[b] = ((2.0 ** -11 + werr) * pv + 2.0 ** -11 * o.abs() + sub + 2.0 ** -25).permute(1, 0, 2)
    return out, tol
