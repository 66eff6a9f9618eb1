"""The 8-bit KV cache and the management of cache pages, as cases that can be timed and compared.

A case is a dict of plain sizes; `listed()` names the ones that stand for real uses, `draw()` gives further ones of the same
ranges, `prepare()` makes what a decoding program holds before the call, `run()` is one pass, `work()` what a pass cannot do
without, `exact()` the values in 64 bits.  With `own` false `run()` computes the operators from elementary torch operations; with
`own` true it makes the library's calls.

attn      tree attention of T candidate nodes per row behind a cache whose whole pages are held in 8 bits (a scale for each page of 16
          tokens and head) and whose last, incomplete page and tree nodes are held in 16 bits
seal      the pages that a step or a prompt chunk has completed go into the 8-bit cache; the values they stand for are read back
turnover  rows that ended give their pages back, the others get the pages that their next step needs
fork      rows become copies of other rows: whole pages are shared, the last incomplete page is copied
compact   the pages in use move to the front of the pool, tables follow

An 8-bit block is one page of one layer and head.  int8: the scale is the smallest number of 11 significant bits that is no less than
the block's largest magnitude over 127, a code the nearest integer of value / scale (ties to even).  e4m3: the scale is the
smallest power of two that keeps the largest magnitude within 448.  A block of zeros has scale 1.
"""
from __future__ import annotations

import math
import zlib

import torch

own = False

DEV = "cuda:0"
PAGE = 16


# ---- cases -------------------------------------------------------------------------------------------------------
def listed():
    return [
        # plain autoregressive decoding of one request of the 7B shape, one node: latency
        dict(name="attn_7b_decode", kind="attn", H=32, Dh=128, B=1, T=1, ctx=701, ragged=0, fmt="int8", arity=1),
        # one request of the 7B shape, the 64-node tree, an odd length
        dict(name="attn_7b_tree", kind="attn", H=32, Dh=128, B=1, T=64, ctx=777, ragged=0, fmt="e4m3", arity=4),
        # a full serving batch: 16 requests of 64 nodes at different points, the longest at 2048 tokens
        dict(name="attn_7b_batch16", kind="attn", H=32, Dh=128, B=16, T=64, ctx=2048, ragged=37, fmt="int8", arity=4),
        # a long document behind the 13B shape, the smaller tree
        dict(name="attn_13b_long", kind="attn", H=40, Dh=128, B=1, T=32, ctx=32003, ragged=0, fmt="e4m3", arity=3),
        # the step of a batch in which every row has completed a page, 8 layers of the 7B shape
        dict(name="seal_7b_step", kind="seal", NL=8, H=32, Dh=128, B=16, before=40, new=1, fmt="int8"),
        # a prompt chunk of 128 tokens, 32 layers
        dict(name="seal_7b_chunk", kind="seal", NL=32, H=32, Dh=128, B=1, before=3, new=8, fmt="e4m3"),
        # a small server between two steps: 8 rows, a quarter of them ended
        dict(name="turnover_8", kind="turnover", B=8, rows=128, pool=1024, ctx=1500, extra=64, gone=4),
        # a large server: 64 rows of up to 32 k tokens on a pool of 64 k pages
        dict(name="turnover_64", kind="turnover", B=64, rows=2048, pool=65536, ctx=30000, extra=64, gone=8),
        # four beams of the 7B shape change places after a step: tables, and the last page of 32 layers
        dict(name="fork_7b_beams", kind="fork", NL=32, H=32, Dh=128, B=4, rows=64, pool=192, ctx=700, one=0),
        # one prompt shared by 32 rows, 8 layers
        dict(name="fork_7b_prompt32", kind="fork", NL=8, H=32, Dh=128, B=32, rows=96, pool=320, ctx=1205, one=1),
        # a pool that has become sparse, 16-bit pages, 16 layers of the 7B shape
        dict(name="compact_7b", kind="compact", NL=16, H=32, Dh=128, B=8, rows=64, pool=448, use=0.4, fmt="half"),
        # the same for the 8-bit pages of a smaller model
        dict(name="compact_small_int8", kind="compact", NL=4, H=16, Dh=64, B=4, rows=64, pool=300, use=0.3, fmt="int8"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(("attn", "seal", "turnover", "fork", "compact"), (6, 2, 2, 2, 2))[0]
    H, Dh = rng.choice(((16, 64), (32, 64), (16, 128), (24, 128), (32, 128), (40, 128), (52, 128)))
    fmt = rng.choice(("int8", "e4m3"))
    if kind == "attn":
        B, T = _log(rng, 1, 16), _log(rng, 1, 128)
        ctx = _log(rng, 1, 32000)
        while B * ctx > 32768 or B * T > 1024:
            B = max(1, B // 2)
            ctx = ctx * 3 // 4
        return dict(kind=kind, H=H, Dh=Dh, B=B, T=T, ctx=ctx, ragged=rng.randint(0, 50), fmt=fmt, arity=rng.randint(1, 6))
    if kind == "seal":
        B, new = _log(rng, 1, 16), _log(rng, 1, 8)
        while B * new > 16:
            B = max(1, B // 2)
        return dict(kind=kind, NL=rng.randint(1, 8), H=H, Dh=Dh, B=B, before=rng.randint(0, 60), new=new, fmt=fmt)
    if kind == "turnover":
        B, rows = _log(rng, 1, 64), _log(rng, 16, 2048)
        ctx = rng.randint(PAGE * rows // 4, PAGE * rows - 200)
        return dict(kind=kind, B=B, rows=rows, pool=max(64, int(B * rows * rng.uniform(0.4, 0.9))), ctx=ctx, extra=rng.randint(1, 128), gone=rng.randint(2, 9))
    if kind == "fork":
        B, rows = _log(rng, 2, 32), _log(rng, 16, 96)
        return dict(kind=kind, NL=rng.randint(1, 8), H=H, Dh=Dh, B=B, rows=rows, pool=B * 2 + rows * 3, ctx=rng.randint(1, PAGE * rows - 1), one=rng.randint(0, 1))
    return dict(kind=kind, NL=rng.randint(1, 8), H=H, Dh=Dh, B=rng.randint(1, 8), rows=64, pool=rng.randint(50, 400), use=rng.uniform(0.1, 0.9),
                fmt=rng.choice(("half", "int8", "e4m3")))


# ---- inputs ------------------------------------------------------------------------------------------------------
def _gen(seed, what):
    return torch.Generator(device=DEV).manual_seed((int(seed) * 1000003 + zlib.crc32(what.encode())) & 0x7FFFFFFFFFFFFFFF)


def _randn(seed, what, shape):
    return torch.randn(shape, generator=_gen(seed, what), device=DEV)


def _ints(seed, what, lo, hi, shape):
    return torch.randint(lo, hi, shape, generator=_gen(seed, what), device=DEV)


def _kv(seed, what, shape):
    """Keys and values [..., 2, H, Dh] as half: channels of a head differ in size (log-normal), keys more than values."""
    x = _randn(seed, what, shape)
    wide = torch.exp(_randn(seed, what + "/channels", shape[-3:]) * torch.tensor([0.6, 0.3], device=DEV)[:, None, None])
    return (x * wide).half()


def parents(T, arity):
    """A tree in breadth-first order in which every node has `arity` children until T nodes exist."""
    return [-1] + [(n - 1) // arity for n in range(1, T)]


def _ancestors(parent):
    m = torch.zeros(len(parent), len(parent), dtype=torch.bool)
    for n, p in enumerate(parent):
        if p >= 0:
            m[n] = m[p]
        m[n, n] = True
    return m


def _lengths(case):
    """Rows of a batch are at different points, the longest at ctx."""
    return [case["ctx"] - (b * case["ragged"]) % max(1, (case["ctx"] + 1) // 2) for b in range(case["B"])]


def _round11(a):
    """The smallest number of 11 significant bits >= a (a > 0, of the type of a)."""
    m, e = torch.frexp(a)
    return torch.ldexp(torch.ceil(m * 2048), e - 11)


def _quantise(x, fmt, t):
    """Codes and scales of x [pages, 16, H, Dh] (half), computed in type t; the scale is [pages, 1, H, 1]."""
    x = x.to(t)
    top = x.abs().amax(dim=(1, 3), keepdim=True)
    safe = torch.where(top > 0, top, torch.ones_like(top))
    if fmt == "int8":
        s = torch.where(top > 0, _round11(safe / 127), torch.ones_like(top))
        return torch.round(x / s).to(torch.int8), s
    m, e = torch.frexp(safe / 448)                  # in (2^(e-1), 2^e], an exact power of two having m = 0.5
    s = torch.where(top > 0, torch.ldexp(torch.ones_like(top), torch.where(m == 0.5, e - 1, e)), torch.ones_like(top))
    return (x / s).float().to(torch.float8_e4m3fn), s


def _context(case, T=1, arity=1, layers=None, max_pos=64, batch=None):
    """A library context of the case's shape with its arena bound; the products, which take no part, are small."""
    from paper_2402_05109_amd import binding as hb
    H, Dh = case.get("H", 16), case.get("Dh", 64)
    ctx = hb.Hydra(d=H * Dh, n_layers=layers or case.get("NL", 1), n_heads=H, head_dim=Dh, ffn=128, vocab=32, dtype=hb.HYDRA_BF16, max_pos=max_pos,
                   parent=parents(T, arity), max_batch=batch or case["B"])
    ctx.bind_weights(torch.empty(ctx.weights_bytes(), dtype=torch.uint8, device=DEV))
    return hb, ctx


def _caches(hb, case, NL, B, pages, slots):
    """An empty 16-bit cache of `slots` tokens per row and an empty 8-bit cache of `pages` pages per row."""
    H, Dh = case["H"], case["Dh"]
    tail_pages = (slots + PAGE - 1) // PAGE
    table = torch.arange(B * tail_pages, dtype=torch.int32, device=DEV).reshape(B, tail_pages)
    block = H * PAGE * Dh
    kp, vp = (torch.zeros(NL * B * tail_pages * block, dtype=torch.float16, device=DEV) for _ in range(2))
    tail = hb.KV(kp, vp, table, B * tail_pages)
    pages = max(1, pages)
    codes = [torch.zeros(NL * B * pages * block, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = torch.ones(NL, B * pages, H, 2, device=DEV)
    table8 = torch.arange(B * pages, dtype=torch.int32, device=DEV).reshape(B, pages)
    return hb.KV8(tail, codes[0], codes[1], scales, table8, torch.zeros(B, dtype=torch.int32, device=DEV), B * pages,
                  hb.KV8_INT8 if case["fmt"] == "int8" else hb.KV8_E4M3)


def prepare(case, seed):
    return {"attn": _prepare_attn, "seal": _prepare_seal, "turnover": _prepare_turnover, "fork": _prepare_fork, "compact": _prepare_compact}[case["kind"]](case, seed)


def _attn_inputs(case, seed):
    B, T, H, Dh = case["B"], case["T"], case["H"], case["Dh"]
    kv = _kv(seed, "kv", (B, case["ctx"] + T, 2, H, Dh))
    q = (_randn(seed, "q", (B, T, H, Dh)) * 1.5).half()
    return q, kv


def _prepare_attn(case, seed):
    B, T, H, Dh, ctx = (case[k] for k in ("B", "T", "H", "Dh", "ctx"))
    q, kv = _attn_inputs(case, seed)
    L = _lengths(case)
    whole = ctx // PAGE
    st = {"case": case, "q": q, "len": torch.tensor(L, dtype=torch.int32, device=DEV)}
    if own:
        hb, c = _context(case, T, case["arity"], 1, ctx + T + 1)
        kv8 = _caches(hb, case, 1, B, whole, ctx + T)
        c.kv_write(B, 0, kv8.tail, 0, ctx + T, kv.float())
        c.hydra_kv8_seal(B, st["len"], kv8)
        kv8.tail.seq_len_hint = ctx
        st |= {"c": c, "kv8": kv8, "ws": torch.empty(c.workspace_bytes(B), dtype=torch.uint8, device=DEV), "out": torch.empty_like(q)}
    else:
        # the codes and scales of the whole pages of every row, and the 16-bit values
        sealed = torch.tensor([n // PAGE for n in L], device=DEV)
        pages = kv[:, :whole * PAGE].reshape(B * whole, PAGE, 2 * H, Dh)
        if whole:
            codes, scale = _quantise(pages, case["fmt"], torch.float32)
            st |= {"codes": codes.reshape(B, whole, PAGE, 2, H, Dh), "scale": scale.reshape(B, whole, 1, 2, H, 1)}
        st |= {"kv": kv, "sealed": sealed, "anc": _ancestors(parents(T, case["arity"])).to(DEV)}
    return st


def _seal_inputs(case, seed):
    """The 16-bit values of the new pages [NL, B, new * 16, 2, H, Dh] and the rows' lengths."""
    kv = _kv(seed, "kv", (case["NL"], case["B"], case["new"] * PAGE, 2, case["H"], case["Dh"]))
    n = PAGE * (case["before"] + case["new"]) + _ints(seed, "len", 0, PAGE, (case["B"],))
    return kv, n.to(torch.int32)


def _prepare_seal(case, seed):
    NL, B, H, Dh, before, new = (case[k] for k in ("NL", "B", "H", "Dh", "before", "new"))
    kv, n = _seal_inputs(case, seed)
    st = {"case": case, "len": n}
    if own:
        hb, c = _context(case, min(128, PAGE * new), 1, NL, PAGE * (before + new + 2) + 128)
        kv8 = _caches(hb, case, NL, B, new, PAGE * (new + 1))
        # the pages in front of the new ones are never looked at: every row's tables name the new ones only
        ring = torch.zeros(B, before + new + 1, dtype=torch.int32, device=DEV)
        ring[:, before:] = kv8.tail.page_table
        table8 = torch.zeros(B, before + new, dtype=torch.int32, device=DEV)
        table8[:, before:] = kv8.page_table
        kv8.tail = hb.KV(kv8.tail.k_pages, kv8.tail.v_pages, ring, kv8.tail.n_pages)
        kv8.page_table, kv8.max_pages = table8, before + new
        for l in range(NL):
            c.kv_write(B, l, kv8.tail, before * PAGE, new * PAGE, kv[l].float())
        st |= {"c": c, "kv8": kv8, "start": torch.full((B,), before, dtype=torch.int32, device=DEV),
               "out": torch.empty(NL, B, new * PAGE, 2, H, Dh, device=DEV)}
    else:
        st["kv"] = kv
    return st


def _spread(seed, counts, B, rows, pool):
    """A page table in which row b holds counts[b] pages in front, of random pages of the pool, and the reference counts."""
    order = torch.randperm(pool, generator=_gen(seed, "pool"), device=DEV).to(torch.int32)
    at = torch.arange(rows, device=DEV)[None, :]
    n = torch.tensor(counts, device=DEV)
    first = (torch.cumsum(n, 0) - n)[:, None]
    held = at < n[:, None]
    table = torch.where(held, order[(first + at).clamp(max=pool - 1)], -1).to(torch.int32)
    ref = torch.zeros(pool, dtype=torch.int32, device=DEV)
    ref[order[:sum(counts)].long()] = 1
    return table, ref


def _pages(hb, st):
    st["pages"] = hb.Pages(st["table"], st["ref"])


def _prepare_turnover(case, seed):
    B, rows, pool, ctx = (case[k] for k in ("B", "rows", "pool", "ctx"))
    share = pool // B
    ctx = min(ctx, PAGE * share - case["extra"] - PAGE)      # what the pool can hold for all rows
    n = _ints(seed, "len", max(1, ctx // 2), max(2, ctx), (B,))
    counts = [min(rows, (int(v) + PAGE - 1) // PAGE) for v in n.tolist()]
    table, ref = _spread(seed, counts, B, rows, pool)
    gone = _ints(seed, "gone", 0, case["gone"], (B,)) == 0
    hi = torch.where(gone, 0, n).to(torch.int32)
    st = {"case": case, "table0": table, "ref0": ref, "hi": hi, "table": table.clone(), "ref": ref.clone()}
    if own:
        hb, c = _context(case)
        _pages(hb, st)
        st |= {"c": c, "ok": torch.zeros(B, dtype=torch.int32, device=DEV),
               "ws": torch.empty(hb.pages_workspace_bytes(B, pool, rows), dtype=torch.uint8, device=DEV)}
    return st


def _page_store(case, seed, what, pool):
    NL, H, Dh = case["NL"], case["H"], case["Dh"]
    dt, width = (torch.int16, 16) if case.get("fmt", "half") == "half" else (torch.uint8, 8)
    n = NL * pool * H * PAGE * Dh
    words = _ints(seed, what, -2 ** 62, 2 ** 62, (n * width // 64,))
    return words.view(dt).reshape(NL, pool, H * PAGE * Dh)


def _prepare_fork(case, seed):
    B, rows, pool, ctx = (case[k] for k in ("B", "rows", "pool", "ctx"))
    n = _ints(seed, "len", max(1, ctx * 3 // 4), ctx + 1, (B,))
    if case["one"]:
        n[1:] = 0                                            # row 0 holds the prompt, the others are empty
    src = torch.zeros(B, dtype=torch.int64, device=DEV) if case["one"] else _ints(seed, "src", 0, B, (B,))
    # the pool has room for the pages of a few rows: rows beyond those share the pages of row 0
    counts = [(int(v) + PAGE - 1) // PAGE for v in n.tolist()]
    own_rows = 1
    while own_rows < B and sum(counts[:own_rows + 1]) + B <= pool:
        own_rows += 1
    table, ref = _spread(seed, counts[:own_rows] + [0] * (B - own_rows), B, rows, pool)
    if own_rows < B and not case["one"]:
        n[own_rows:] = PAGE * (n[0] // PAGE)                 # whole pages of row 0
        whole = int(n[0]) // PAGE
        table[own_rows:, :whole] = table[0, :whole]
        ref[table[0, :whole].long()] += B - own_rows
    st = {"case": case, "table0": table, "ref0": ref, "table": table.clone(), "ref": ref.clone(), "len": n.to(torch.int32), "src": src.to(torch.int32),
          "k": _page_store(case, seed, "k", pool), "v": _page_store(case, seed, "v", pool)}
    if own:
        hb, c = _context(case)
        _pages(hb, st)
        st |= {"c": c, "kv": hb.KV(st["k"], st["v"], st["table"], pool), "ws": torch.empty(hb.pages_workspace_bytes(B, pool, rows), dtype=torch.uint8, device=DEV),
               "from": torch.zeros(B, dtype=torch.int32, device=DEV), "to": torch.zeros(B, dtype=torch.int32, device=DEV),
               "forked": torch.zeros(B, dtype=torch.int32, device=DEV)}
    return st


def _prepare_compact(case, seed):
    B, rows, pool = (case[k] for k in ("B", "rows", "pool"))
    used = min(int(pool * case["use"]), B * rows)
    counts = [used // B + (1 if b < used % B else 0) for b in range(B)]
    table, ref = _spread(seed, counts, B, rows, pool)
    st = {"case": case, "table0": table, "ref0": ref, "table": table.clone(), "ref": ref.clone(),
          "k": _page_store(case, seed, "k", pool), "v": _page_store(case, seed, "v", pool)}
    if case["fmt"] != "half":
        st["scales"] = torch.exp(_randn(seed, "scales", (case["NL"], pool, case["H"], 2)))
    if own:
        hb, c = _context(case)
        _pages(hb, st)
        st |= {"c": c, "ws": torch.empty(hb.pages_workspace_bytes(B, pool, rows), dtype=torch.uint8, device=DEV),
               "from": torch.zeros(pool, dtype=torch.int32, device=DEV), "to": torch.zeros(pool, dtype=torch.int32, device=DEV),
               "counts": torch.zeros(2, dtype=torch.int32, device=DEV)}
        if case["fmt"] == "half":
            st["kv"] = hb.KV(st["k"], st["v"], st["table"], pool)
        else:                                               # the 16-bit side takes no part in the move of sealed pages
            tail = hb.KV(st["k"], st["v"], torch.zeros(B, 1, dtype=torch.int32, device=DEV), 1)
            st["kv8"] = hb.KV8(tail, st["k"], st["v"], st["scales"], st["table"], torch.zeros(B, dtype=torch.int32, device=DEV), pool,
                               hb.KV8_INT8 if case["fmt"] == "int8" else hb.KV8_E4M3)
    return st


# ---- one pass ----------------------------------------------------------------------------------------------------
def run(st):
    return (_run_own if own else _run_plain)[st["case"]["kind"]](st)


def _own_attn(st):
    st["c"].tree_attention_kv8(st["case"]["B"], 0, st["ws"], st["q"], st["len"], st["kv8"], st["out"])
    return {"out": st["out"]}


def _own_seal(st):
    case, kv8 = st["case"], st["kv8"]
    kv8.n_sealed.copy_(st["start"])                          # the state of this step again: the call advances it
    st["c"].hydra_kv8_seal(case["B"], st["len"], kv8)
    st["c"].kv8_read(case["B"], -1, kv8, case["before"] * PAGE, case["new"] * PAGE, st["out"])
    return {"values": st["out"], "scales": kv8.scales, "n_sealed": kv8.n_sealed}


def _again(st):
    """The tables before the call again: the calls change them in place."""
    st["table"].copy_(st["table0"])
    st["ref"].copy_(st["ref0"])


def _own_turnover(st):
    case = st["case"]
    _again(st)
    st["c"].hydra_pages_release(case["B"], st["pages"], None, st["hi"])
    st["c"].hydra_pages_reserve(case["B"], st["ws"], st["pages"], None, st["hi"], case["extra"], st["ok"])
    return {"table": st["table"], "ref": st["ref"], "ok": st["ok"]}


def _own_fork(st):
    case = st["case"]
    _again(st)
    st["c"].hydra_pages_fork(case["B"], st["ws"], st["pages"], st["src"], st["len"], st["from"], st["to"], st["forked"])
    st["c"].hydra_kv_copy_pages(st["kv"], case["B"], st["from"], st["to"])
    return {"table": st["table"], "ref": st["ref"], "from": st["from"], "to": st["to"], "forked": st["forked"], "k": st["k"], "v": st["v"]}


def _own_compact(st):
    case = st["case"]
    _again(st)
    st["c"].hydra_pages_compact(case["B"], st["ws"], st["pages"], st["from"], st["to"], st["counts"])
    out = {"table": st["table"], "ref": st["ref"], "from": st["from"], "to": st["to"], "counts": st["counts"], "k": st["k"], "v": st["v"]}
    if case["fmt"] == "half":
        st["c"].hydra_kv_copy_pages(st["kv"], case["pool"], st["from"], st["to"], st["counts"])
        return out
    st["c"].hydra_kv8_copy_pages(st["kv8"], case["pool"], st["from"], st["to"], st["counts"])
    return {**out, "scales": st["scales"].view(torch.int32)}


def _plain_attn(st):
    case = st["case"]
    B, T, H, Dh, ctx = (case[k] for k in ("B", "T", "H", "Dh", "ctx"))
    kv = st["kv"].float()
    whole = ctx // PAGE
    at = torch.arange(ctx + T, device=DEV)[None, :]
    if whole:
        held = (st["codes"].float() * st["scale"].float()).reshape(B, whole * PAGE, 2, H, Dh)
        in8 = (at[:, :whole * PAGE] < PAGE * st["sealed"][:, None])[:, :, None, None, None]
        kv = torch.cat([torch.where(in8, held, kv[:, :whole * PAGE]), kv[:, whole * PAGE:]], dim=1)
    L = st["len"].long()[:, None]
    node = at - L                                            # tree node of a slot, negative: cached
    tree = st["anc"][:, node.clamp(0, T - 1)]                # [T, B, slots]
    seen = (node < 0)[None] | (tree & (node >= 0)[None] & (node < T)[None])
    k = kv[:, :, 0].permute(0, 2, 3, 1).contiguous()         # [B, H, Dh, slots]
    v = kv[:, :, 1].permute(0, 2, 1, 3).contiguous()
    s = torch.matmul(st["q"].float().permute(0, 2, 1, 3).contiguous(), k) / math.sqrt(Dh)
    s = torch.where(seen.permute(1, 0, 2)[:, None], s, -math.inf)
    p = torch.exp(s - s.amax(dim=-1, keepdim=True))
    o = torch.matmul(p, v) / p.sum(dim=-1, keepdim=True)
    return {"out": o.permute(0, 2, 1, 3).contiguous().half()}


def _plain_seal(st):
    case = st["case"]
    NL, B, H, Dh, before, new = (case[k] for k in ("NL", "B", "H", "Dh", "before", "new"))
    codes, s = _quantise(st["kv"].reshape(NL * B * new, PAGE, 2 * H, Dh), case["fmt"], torch.float32)
    values = (codes.float() * s).reshape(NL, B, new * PAGE, 2, H, Dh)
    scales = s.reshape(NL, B * new, 2, H).transpose(2, 3).contiguous()
    return {"values": values, "scales": scales, "n_sealed": torch.div(st["len"], PAGE, rounding_mode="floor").to(torch.int32)}


def _lowest_free(ref):
    """Free pages, lowest first (then the others), and how many are free."""
    return torch.sort((ref != 0).to(torch.int32), stable=True).indices.to(torch.int32), (ref == 0).sum()


def _counted(ref, pages, mask, by):
    """Reference counts with `by` added for every masked entry of `pages`."""
    add = torch.zeros_like(ref)
    add.scatter_add_(0, pages.reshape(-1).clamp(min=0).long(), (mask.reshape(-1).to(torch.int32) * by))
    return ref + add


def _plain_turnover(st):
    case = st["case"]
    table, ref = st["table0"], st["ref0"]
    at = torch.arange(case["rows"], device=DEV)[None, :]
    hi = st["hi"].long()[:, None]
    drop = (table >= 0) & (at >= torch.div(hi + PAGE - 1, PAGE, rounding_mode="floor"))
    ref = _counted(ref, table, drop, -1)
    table = torch.where(drop, -1, table)
    last = torch.div(hi + case["extra"] + PAGE - 1, PAGE, rounding_mode="floor")
    good = last <= case["rows"]
    want = (table < 0) & (at < last) & good
    need = want.sum(1)
    free, n_free = _lowest_free(ref)
    ok = good[:, 0] & ((need == 0) | (torch.cumsum(need, 0) <= n_free))
    want = want & ok[:, None]
    rank = (torch.cumsum(want.reshape(-1).to(torch.int64), 0) - 1).reshape(want.shape).clamp(min=0)
    table = torch.where(want, free[rank], table)
    return {"table": table, "ref": _counted(ref, table, want, 1), "ok": ok.to(torch.int32)}


def _plain_fork(st):
    case = st["case"]
    B = case["B"]
    t0, ref0, src, n = st["table0"], st["ref0"], st["src"].long(), st["len"].long()
    me = torch.arange(B, device=DEV)
    at = torch.arange(case["rows"], device=DEV)[None, :]
    take = t0[src]
    whole = torch.div(n[src], PAGE, rounding_mode="floor")
    part = torch.gather(take, 1, whole.clamp(max=case["rows"] - 1)[:, None])[:, 0]
    moved = src != me
    need = moved & (n[src] % PAGE != 0) & (part >= 0)
    free, n_free = _lowest_free(ref0)
    cum = torch.cumsum(need.to(torch.int64), 0)
    moved = moved & (~need | (cum <= n_free))
    need = need & moved
    fresh = free[(cum - 1).clamp(min=0)]
    shared = at < whole[:, None]
    new = torch.where(shared, take, torch.where(need[:, None] & (at == whole[:, None]), fresh[:, None], -1))
    table = torch.where(moved[:, None], new, t0)
    ref = _counted(ref0, t0, moved[:, None] & (t0 >= 0), -1)
    ref = _counted(ref, table, moved[:, None] & (table >= 0), 1)
    a, b = torch.where(need, part, -1), torch.where(need, fresh, -1)
    k, v = _moved(st["k"], a, b), _moved(st["v"], a, b)
    return {"table": table, "ref": ref, "from": a, "to": b, "forked": torch.where(moved, src, me).to(torch.int32), "k": k, "v": v}


def _moved(store, a, b):
    """`store` [layers, pages, ...] with page a[i] copied to page b[i], in place; entries of -1 copy nothing."""
    live = torch.nonzero(b >= 0)[:, 0]
    store.index_copy_(1, b[live].long(), store.index_select(1, a[live].long()))
    return store


def _plain_compact(st):
    case = st["case"]
    t0, ref0, pool = st["table0"], st["ref0"], case["pool"]
    used = ref0 > 0
    n_used = used.sum()
    at = torch.arange(pool, device=DEV)
    out_of = used & (at >= n_used)
    hole = ~used & (at < n_used)
    a = torch.sort((~out_of).to(torch.int32), stable=True).indices
    b = torch.sort((~hole).to(torch.int32), stable=True).indices
    n = out_of.sum()
    live = at < n
    to_new = at.clone()
    to_new = torch.where(out_of, torch.zeros_like(at).scatter(0, a, b), to_new)
    table = torch.where(t0 >= 0, to_new[t0.clamp(min=0).long()].to(torch.int32), t0)
    ref = torch.zeros_like(ref0).scatter_add(0, to_new, torch.where(used, ref0, 0))
    a, b = torch.where(live, a, -1).to(torch.int32), torch.where(live, b, -1).to(torch.int32)
    out = {"table": table, "ref": ref, "from": a, "to": b, "counts": torch.stack([n, n_used]).to(torch.int32), "k": _moved(st["k"], a, b), "v": _moved(st["v"], a, b)}
    return out if case["fmt"] == "half" else {**out, "scales": _moved(st["scales"], a, b).view(torch.int32)}


_run_own = {"attn": _own_attn, "seal": _own_seal, "turnover": _own_turnover, "fork": _own_fork, "compact": _own_compact}
_run_plain = {"attn": _plain_attn, "seal": _plain_seal, "turnover": _plain_turnover, "fork": _plain_fork, "compact": _plain_compact}


# ---- what a pass cannot do without ------------------------------------------------------------------------------
def work(case):
    kind, B = case["kind"], case["B"]
    if kind == "attn":
        T, H, Dh = case["T"], case["H"], case["Dh"]
        d, L = H * Dh, _lengths(case)
        held = sum(n // PAGE for n in L)
        tail = sum(n + T - n // PAGE * PAGE for n in L)
        return {"bytes": held * (PAGE * 2 * d + 8 * H) + tail * 4 * d + 4 * B * T * d, "flops": 4 * T * d * sum(n + T for n in L)}
    if kind == "seal":
        n = case["NL"] * B * case["new"]
        d = case["H"] * case["Dh"]
        # 16-bit values in, codes and scales out, codes in again, 32-bit values out
        return {"bytes": n * PAGE * 2 * d * (2 + 1 + 1 + 4) + n * case["H"] * 16, "flops": n * PAGE * 2 * d * 3}
    if kind == "turnover":
        return {"bytes": 4 * (2 * B * case["rows"] + 2 * case["pool"]), "flops": 0}
    page = case["NL"] * case["H"] * PAGE * case["Dh"] * (4 if case.get("fmt", "half") == "half" else 2)
    if kind == "fork":
        return {"bytes": 4 * (2 * B * case["rows"] + 2 * case["pool"]) + 2 * page * (B - 1), "flops": 0}
    used = min(int(case["pool"] * case["use"]), B * case["rows"])
    moves = used * (1 - used / case["pool"])                 # of the pages in use, those that lie behind the first `used` of the pool
    return {"bytes": int(4 * (2 * B * case["rows"] + 2 * case["pool"]) + 2 * page * moves), "flops": 0}


# ---- the same in 64 bits ----------------------------------------------------------------------------------------
def exact(case, seed):
    if case["kind"] == "seal":
        return _exact_seal(case, seed)
    if case["kind"] == "attn":
        return _exact_attn(case, seed)
    return None                                              # tables, counts and copied pages: whole numbers


def _exact_block(x, fmt):
    """The values that a block of 16 tokens [16, H, Dh] stands for in 8 bits, and its scales, in 64 bits."""
    x = x.double()
    out, scales = torch.zeros_like(x), torch.ones(x.shape[1], dtype=torch.float64, device=x.device)
    top = x.abs().amax(dim=(0, 2))
    some = top > 0
    if fmt == "int8":
        e = torch.floor(torch.log2(torch.where(some, top, 1.0) / 127)) - 10
        unit = torch.exp2(e)                                 # a unit of the 11th significant bit
        s = torch.ceil(torch.where(some, top, 1.0) / 127 / unit) * unit
        scales = torch.where(some, s, scales)
        out = torch.round(x / scales[None, :, None]) * scales[None, :, None]
    else:
        s = torch.exp2(torch.ceil(torch.log2(torch.where(some, top, 448.0) / 448)))
        scales = torch.where(some, s, scales)
        y = x / scales[None, :, None]
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        out = torch.round(y / step) * step * scales[None, :, None]
    return out, scales


def _exact_seal(case, seed):
    kv, n = _seal_inputs(case, seed)
    NL, B, H, Dh, new = (case[k] for k in ("NL", "B", "H", "Dh", "new"))
    values = torch.empty(kv.shape, dtype=torch.float64, device=DEV)
    scales = torch.empty(NL, B * new, H, 2, dtype=torch.float64, device=DEV)
    for l in range(NL):
        for b in range(B):
            for i in range(new):
                for j in range(2):
                    at = slice(i * PAGE, (i + 1) * PAGE)
                    values[l, b, at, j], scales[l, b * new + i, :, j] = _exact_block(kv[l, b, at, j], case["fmt"])
    return {"values": values, "scales": scales, "n_sealed": None}


def _exact_attn(case, seed):
    B, T, H, Dh = case["B"], case["T"], case["H"], case["Dh"]
    q, kv = _attn_inputs(case, seed)
    parent = parents(T, case["arity"])
    out = torch.zeros(B, T, H, Dh, dtype=torch.float64, device=DEV)
    for b, L in enumerate(_lengths(case)):
        row = kv[b, :L + T].double()
        for i in range(L // PAGE):
            at = slice(i * PAGE, (i + 1) * PAGE)
            for j in range(2):
                row[at, j] = _exact_block(kv[b, at, j], case["fmt"])[0]
        bias = torch.zeros(T, L + T, dtype=torch.float64)
        bias[:, L:] = -math.inf
        for n in range(T):
            a = n
            while a >= 0:
                bias[n, L + a] = 0.0
                a = parent[a]
        bias = bias.to(DEV)
        for h in range(H):
            s = q[b, :, h].double() @ row[:, 0, h].T.contiguous() / Dh ** 0.5 + bias
            out[b, :, h] = torch.softmax(s, dim=-1) @ row[:, 1, h].contiguous()
    return {"out": out}
