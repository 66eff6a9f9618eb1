"""Plumbing of the tests of part of a cache: a context, a cache in which everything unseen is NaN, and the definitions in 64 bits."""
from __future__ import annotations

import math

import torch

from paper_2402_05109_amd import binding as hb

DEV = "cuda:0"


def tree_parent(T, arity=3):
    return [-1] + [(n - 1) // arity for n in range(1, T)]


def depths(parent):
    d = [0] * len(parent)
    for n in range(1, len(parent)):
        d[n] = d[parent[n]] + 1
    return d


def context(H, Dh, B, parent=(-1,), NL=1, max_pos=256, f32=False, vocab=32):
    c = hb.Hydra(d=H * Dh, n_layers=NL, n_heads=H, head_dim=Dh, ffn=128, vocab=vocab, dtype=hb.HYDRA_F32 if f32 else hb.HYDRA_BF16, max_pos=max_pos,
                 parent=list(parent), max_batch=B)
    c.arena = torch.zeros(c.weights_bytes(), dtype=torch.uint8, device=DEV)
    c.bind_weights(c.arena)
    c.ws = torch.empty(c.workspace_bytes(B), dtype=torch.uint8, device=DEV)
    return c


def dtype_of(f32):
    return torch.float32 if f32 else torch.float16


def seen_by(parent, L, F, sinks, window):
    """For every node the list of slots that it sees (slots of the tree: L + node)."""
    d = depths(parent)
    out = []
    for n in range(len(parent)):
        p = L + d[n]
        held = [s for s in range(F, L) if window == 0 or s > p - window or s < F + sinks]
        a, tree = n, []
        while a >= 0:
            if window == 0 or d[a] > d[n] - window or L + d[a] < F + sinks or a == n:
                tree.append(L + a)
            a = parent[a]
        out.append(held + sorted(tree))
    return out


def masks(parent, lens, firsts, sinks, window, slots):
    m = torch.zeros(len(lens), len(parent), slots, dtype=torch.bool)
    for b, (L, F) in enumerate(zip(lens, firsts)):
        for n, see in enumerate(seen_by(parent, L, F, sinks, window)):
            m[b, n, torch.tensor(see)] = True
    return m


def cache(c, H, Dh, kv, mask, f32, seed=0, NL=1, spare=3):
    """A cache that holds kv [NL, B, slots, 2, H, Dh] where some node of the row sees the slot; all else is NaN, pages that no node sees have no
    entry (-1 or beyond the cache)."""
    _, B, slots = kv.shape[:3]
    pages = (slots + 15) // 16
    g = torch.Generator().manual_seed(seed)
    n = B * pages + spare
    full = torch.randperm(n, generator=g)[:B * pages].reshape(B, pages).to(torch.int32)
    store = [torch.full((NL * n * H * 16 * Dh,), math.nan, dtype=dtype_of(f32), device=DEV) for _ in range(2)]
    any_node = mask.any(dim=1)                                               # [B, slots]
    for b in range(B):
        row = hb.KV(*store, full[b:b + 1].to(DEV).contiguous(), n)
        at = any_node[b].nonzero()[:, 0].tolist()
        runs = []
        for s in at:
            if runs and runs[-1][1] == s:
                runs[-1][1] = s + 1
            else:
                runs.append([s, s + 1])
        for lo, hi in runs:
            for l in range(NL):
                c.kv_write(1, l, row, lo, hi - lo, kv[l, b:b + 1, lo:hi].float().contiguous().to(DEV))
    held = torch.nn.functional.pad(any_node, (0, pages * 16 - slots)).reshape(B, pages, 16).any(dim=2)
    hole = torch.where(torch.arange(pages) % 2 == 0, -1, n + 7).to(torch.int32)
    table = torch.where(held, full, hole[None, :]).to(DEV).contiguous()
    return hb.KV(*store, table, n)


def attention_reference(q, kv, mask, f32, n_scored):
    """(result, how far the library's may be from it, weights added per slot, how far those may be), in 64 bits.  q [B, T, H, Dh], kv [B, slots, 2, H, Dh], mask
    [B, T, slots].

    A score carries the error of a sum of Dh products in 32 bits (rounded each by 2^-24 of the sum of magnitudes), its exponent a few more roundings of its
    own size, the exponential 2^-21; so does the largest score.  16 bits: a weight w <= 1 is rounded to half (2^-11 of its value, or 2^-25 where it is
    subnormal) and the result too.  fp32: a sum over n slots rounds by n 2^-24 of its magnitudes."""
    q, kv = q.double().to(DEV), kv.double().to(DEV)
    mask = mask.to(DEV)
    B, T, H, Dh = q.shape
    k = kv[:, :, 0].permute(0, 2, 3, 1).contiguous()
    v = torch.where(mask.any(dim=1)[:, :, None, None], kv[:, :, 1], 0.0).permute(0, 2, 1, 3).contiguous()
    qh = q.permute(0, 2, 1, 3).contiguous()
    s = torch.matmul(qh, k) / math.sqrt(Dh)
    size = torch.matmul(qh.abs(), k.abs()) / math.sqrt(Dh)
    seen = mask[:, None]
    s = torch.where(seen, s, -math.inf)
    p = torch.softmax(s, dim=-1)
    o = torch.matmul(p, v)
    n = mask.shape[-1]
    werr = 2 * (Dh + 16) * 2.0 ** -24 * torch.where(seen, size, 0.0).amax(dim=-1, keepdim=True) + 2.0 ** -20 + (n + 16) * 2.0 ** -24
    pv = torch.matmul(p, v.abs())
    if f32:
        tol = werr * pv + 2.0 ** -23 * o.abs() + 1e-37
    else:
        big = p.amax(dim=-1, keepdim=True)
        sub = 2.0 ** -25 * big * v.abs().sum(dim=2, keepdim=True)
        tol = (2.0 ** -11 + werr) * pv + 2.0 ** -11 * o.abs() + sub + 2.0 ** -25
    add = p[:, :, :n_scored].sum(dim=2)
    add_tol = (p[:, :, :n_scored] * werr[:, :, :n_scored]).sum(dim=2) + (n_scored + 2) * 2.0 ** -24 * add + 1e-37
    return o.permute(0, 2, 1, 3), tol.permute(0, 2, 1, 3), add, add_tol


def keep_reference(score, lens, firsts, sinks, recent, keep, slack):
    """kept slots by the definition: nested lists [NL][B][H] (None where the row stays whole)."""
    NL, _, H, _ = score.shape
    x = score.double().cpu()
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x).tolist()
    out = []
    for l in range(NL):
        rows = []
        for b in range(len(lens)):
            L, F = lens[b], firsts[b]
            if L - F <= keep + slack:
                rows.append(None)
                continue
            heads = []
            for h in range(H):
                mid = list(range(F + sinks, L - recent))
                want = keep - sinks - recent
                best = sorted(mid, key=lambda s: (-x[l][b][h][s], s))[:want]
                heads.append(list(range(F, F + sinks)) + sorted(best) + list(range(L - recent, L)))
            rows.append(heads)
        out.append(rows)
    return out
