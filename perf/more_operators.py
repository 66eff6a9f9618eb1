"""Attention over part of a KV cache, eviction from a cache by accumulated attention weight, and log probabilities of given tokens, as
cases that can be timed and compared.

A case is a dict of plain sizes; `listed()` names the ones that stand for real uses, `draw()` gives further ones of the same
ranges, `prepare()` makes what a decoding program holds before the call, `run()` is one pass, `work()` what a pass cannot do
without, `exact()` the values in 64 bits.  With `own` false `run()` computes the operators from elementary torch operations; with
`own` true it makes the library's calls.

span      tree attention of T nodes per row in which a node at position p sees the slots behind p - window and a few first ones (sinks);
          what lies between may have no pages any more
score     the same behind a cache from which tokens were evicted, whose weights are also added up for every slot, layer and head
evict     rows that hold more than `keep` tokens are cut to that many: the sinks, the last `recent` ones and those of the largest
          accumulated weight, for each layer and head on its own (ties: the lower slot); they move to the row's last slots, in order
logprobs  for each row of logits: log probability and rank of a given token, entropy, and the k most likely tokens

Slots are positions: a row holds slots first .. len - 1, its nodes stand in slots len .. len + T - 1 at positions len + depth.
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
        # plain decoding of one request of the 7B shape far into a text, one node: latency
        dict(name="span_7b_decode", kind="span", H=32, Dh=128, B=1, T=1, ctx=8003, ragged=0, window=1024, sinks=4, cut=0, scored=0, dtype="bf16", arity=1),
        # one request of the 7B shape with the 64-node tree and a wide window
        dict(name="span_7b_tree", kind="span", H=32, Dh=128, B=1, T=64, ctx=29989, ragged=0, window=4096, sinks=16, cut=0, scored=0, dtype="bf16", arity=4),
        # a full serving batch: 16 requests of 64 nodes at different points
        dict(name="span_7b_batch16", kind="span", H=32, Dh=128, B=16, T=64, ctx=2048, ragged=37, window=1500, sinks=4, cut=0, scored=0, dtype="bf16", arity=4),
        # the tiny fp32 model with its 16-node tree
        dict(name="span_tiny_f32", kind="span", H=4, Dh=64, B=1, T=16, ctx=301, ragged=0, window=100, sinks=2, cut=0, scored=0, dtype="f32", arity=3),
        # a step of the 7B shape behind a cache held at about 2048 tokens: the root's weights are added up
        dict(name="score_7b_step", kind="score", H=32, Dh=128, B=1, T=64, ctx=12345, ragged=0, window=0, sinks=4, cut=10197, scored=1, dtype="bf16", arity=4),
        # a chunk of a long prompt behind the 13B shape: all its tokens count
        dict(name="score_13b_chunk", kind="score", H=40, Dh=128, B=1, T=128, ctx=16000, ragged=0, window=0, sinks=4, cut=0, scored=128, dtype="bf16", arity=1),
        # a long session of the 7B shape, 8 layers: the last 512 tokens push the lightest ones out
        dict(name="evict_7b_steps", kind="evict", NL=8, H=32, Dh=128, B=1, ctx=9000, ragged=0, cut=6440, keep=2048, recent=256, sinks=4, dtype="bf16", inplace=0),
        # a prompt of 16 k tokens behind the 13B shape, 4 layers, cut to 2048
        dict(name="evict_13b_prompt", kind="evict", NL=4, H=40, Dh=128, B=1, ctx=16003, ragged=0, cut=0, keep=2048, recent=512, sinks=4, dtype="bf16", inplace=0),
        # the tiny fp32 model, two rows, in place (the cache is set back in the pass)
        dict(name="evict_tiny_f32", kind="evict", NL=2, H=4, Dh=64, B=2, ctx=333, ragged=21, cut=0, keep=200, recent=50, sinks=2, dtype="f32", inplace=1),
        # one sampled token of one request, five alternatives: latency
        dict(name="logprobs_token", kind="logprobs", B=1, T=1, V=32000, k=5, tau=1.0),
        # a step of a full batch: all nodes of 16 trees
        dict(name="logprobs_batch16", kind="logprobs", B=16, T=64, V=32000, k=10, tau=0.7),
        # scoring of a prompt chunk with a large odd vocabulary, entropy and log probabilities alone
        dict(name="logprobs_chunk", kind="logprobs", B=1, T=128, V=100003, k=0, tau=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(("span", "score", "evict", "logprobs"), (4, 3, 3, 3))[0]
    if kind == "logprobs":
        B, T, V = _log(rng, 1, 16), _log(rng, 1, 128), _log(rng, 1000, 131072)
        while B * T * V > 16 * 64 * 32000:
            B, T = max(1, B // 2), max(1, T * 3 // 4)
        return dict(kind=kind, B=B, T=T, V=V, k=rng.choice((0, 1, 5, 20, 32)), tau=rng.choice((1.0, 0.7, 1.5)))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    H, Dh = rng.choice(((16, 64), (32, 64), (16, 128), (24, 128), (32, 128), (40, 128))) if dtype == "bf16" else rng.choice(((4, 64), (8, 64), (8, 128), (16, 128)))
    if kind == "evict":
        B, ctx = _log(rng, 1, 8), _log(rng, 40, 16000)
        NL = rng.randint(1, 6)
        while B * ctx * NL * H * Dh > 4 * 16003 * 40 * 128:
            B, ctx = max(1, B // 2), ctx * 3 // 4
        keep = max(8, int(ctx * rng.uniform(0.1, 0.95)))
        sinks = rng.randint(0, 4)
        return dict(kind=kind, NL=NL, H=H, Dh=Dh, B=B, ctx=ctx, ragged=rng.randint(0, 50), cut=rng.choice((0, 0, 7, 33)) if ctx > 100 else 0, keep=keep,
                    recent=rng.randint(0, keep - sinks), sinks=sinks, dtype=dtype, inplace=rng.randint(0, 1))
    B, T, ctx = _log(rng, 1, 16), _log(rng, 1, 128), _log(rng, 1, 32000)
    most = 32768 if dtype == "bf16" else 8192
    while B * ctx > most or B * T > (1024 if dtype == "bf16" else 256):
        B = max(1, B // 2)
        ctx, T = ctx * 3 // 4, max(1, T * 7 // 8)
    if kind == "span":
        return dict(kind=kind, H=H, Dh=Dh, B=B, T=T, ctx=ctx, ragged=rng.randint(0, 50), window=_log(rng, 1, 8192), sinks=rng.choice((0, 1, 4, 16, 33)), cut=0, scored=0,
                    dtype=dtype, arity=rng.randint(1, 6))
    window = rng.choice((0, 0, _log(rng, 8, 4096)))
    return dict(kind=kind, H=H, Dh=Dh, B=B, T=T, ctx=ctx, ragged=rng.randint(0, 50), window=window, sinks=rng.choice((0, 4)), cut=ctx * rng.choice((0, 1, 2)) // 3,
                scored=rng.choice((1, 1, T)), dtype=dtype, arity=rng.randint(1, 6))


# ---- inputs ------------------------------------------------------------------------------------------------------
def _gen(seed, what):
    return torch.Generator(device=DEV).manual_seed((int(seed) * 1000003 + zlib.crc32(what.encode())) & 0x7FFFFFFFFFFFFFFF)


def _randn(seed, what, shape):
    return torch.randn(shape, generator=_gen(seed, what), device=DEV)


def _rand(seed, what, shape):
    return torch.rand(shape, generator=_gen(seed, what), device=DEV)


def _ints(seed, what, lo, hi, shape):
    return torch.randint(lo, hi, shape, generator=_gen(seed, what), device=DEV)


def _type(case):
    return torch.float16 if case["dtype"] == "bf16" else torch.float32


def _kv(seed, case, shape):
    """Keys and values [..., 2, H, Dh]: channels of a head differ in size (log-normal), keys more than values."""
    x = _randn(seed, "kv", shape)
    x *= torch.exp(_randn(seed, "kv/channels", shape[-3:]) * torch.tensor([0.6, 0.3], device=DEV)[:, None, None])
    return x.to(_type(case))


def parents(T, arity):
    """A tree in breadth-first order in which every node has `arity` children until T nodes exist."""
    return [-1] + [(n - 1) // arity for n in range(1, T)]


def _tree(case):
    """Ancestors (a node is its own) [T, T] and depths [T]."""
    parent = parents(case["T"], case["arity"])
    anc, depth = torch.zeros(len(parent), len(parent), dtype=torch.bool), torch.zeros(len(parent), dtype=torch.int64)
    for n, p in enumerate(parent):
        if p >= 0:
            anc[n] = anc[p]
            depth[n] = depth[p] + 1
        anc[n, n] = True
    return anc.to(DEV), depth.to(DEV)


def _lengths(case):
    """Rows of a batch are at different points, the longest at ctx; what was evicted is the same number of slots in every row."""
    ctx, cut = case["ctx"], case["cut"]
    return torch.tensor([ctx - (b * case["ragged"]) % max(1, (ctx - cut + 1) // 2) for b in range(case["B"])], dtype=torch.int32, device=DEV)


def _context(case, NL, max_pos, T=1, arity=1, vocab=32):
    """A library context of the case's shape with its arena bound; the products, which take no part, are small."""
    from paper_2402_05109_amd import binding as hb
    H, Dh = case.get("H", 2), case.get("Dh", 64)
    ctx = hb.Hydra(d=H * Dh, n_layers=NL, n_heads=H, head_dim=Dh, ffn=128, vocab=vocab, dtype=hb.HYDRA_F32 if case.get("dtype") == "f32" else hb.HYDRA_BF16,
                   max_pos=max_pos, parent=parents(T, arity), max_batch=case["B"])
    ctx.bind_weights(torch.empty(ctx.weights_bytes(), dtype=torch.uint8, device=DEV))
    return hb, ctx


def _scores(seed, shape, scale=1.0):
    """Accumulated weights: heavy-tailed, a twentieth of the slots never looked at.  scale: small where few nodes have been counted yet."""
    x = scale * torch.exp(_randn(seed, "score", shape) * 2 - 3)
    return torch.where(_rand(seed, "score/none", shape) < 0.05, 0.0, x)


def prepare(case, seed):
    return {"span": _prepare_attn, "score": _prepare_attn, "evict": _prepare_evict, "logprobs": _prepare_logprobs}[case["kind"]](case, seed)


def _attn_inputs(case, seed):
    B, T, H, Dh = case["B"], case["T"], case["H"], case["Dh"]
    kv = _kv(seed, case, (B, case["ctx"] + T, 2, H, Dh))
    q = (_randn(seed, "q", (B, T, H, Dh)) * 1.5).to(_type(case))
    return q, kv


def _visible(case, L):
    """The slots [B, n] that some node of a row sees, sinks first (a slot behind the row's last node: none), and the first one of the window part.
    A node sees at least what is behind `low`; what is in both parts is named once."""
    cut, sinks, window, T = case["cut"], case["sinks"], case["window"], case["T"]
    low = (L + 1 - window).clamp(min=cut) if window else torch.full_like(L, cut)
    n_sinks = (low - cut).clamp(max=sinks)                   # per row: those in front of the window
    most = int((L + T - low).max())
    at = torch.arange(sinks + most, device=DEV)[None, :]
    j = at - n_sinks[:, None]
    slot = torch.where(j < 0, cut + at, low[:, None] + j)
    return slot, slot < (L + T)[:, None]


def _prepare_attn(case, seed):
    B, T, H, Dh, ctx = (case[k] for k in ("B", "T", "H", "Dh", "ctx"))
    q, kv = _attn_inputs(case, seed)
    L = _lengths(case)
    st = {"case": case, "q": q, "len": L}
    pages = (ctx + T + PAGE - 1) // PAGE
    if case["scored"]:
        st["score0"] = _scores(seed, (1, B, H, pages * PAGE), 0.01)
        st["score"] = st["score0"].clone()
    slot, live = _visible(case, L.long())
    if own:
        hb, c = _context(case, 1, ctx + T + 1, T, case["arity"])
        # pages in no order; what no node sees has none
        perm = torch.randperm(B * pages, generator=_gen(seed, "pages"), device=DEV).to(torch.int32).reshape(B, pages)
        store = [torch.zeros(B * pages * H * PAGE * Dh, dtype=_type(case), device=DEV) for _ in range(2)]
        full = hb.KV(store[0], store[1], perm, B * pages)
        c.kv_write(B, 0, full, 0, ctx + T, kv.float())
        seen = torch.zeros(B, pages, dtype=torch.bool, device=DEV)
        seen.scatter_(1, torch.where(live, slot, (L.long() + T - 1)[:, None]) // PAGE, True)
        table = torch.where(seen, perm, -1).to(torch.int32)
        span = hb.KVSpan(hb.KV(store[0], store[1], table, B * pages, seq_len_hint=ctx), first=torch.full((B,), case["cut"], dtype=torch.int32, device=DEV),
                         n_sinks=case["sinks"], window=case["window"], span_hint=ctx - case["cut"], score=st.get("score"), n_scored=case["scored"])
        st |= {"c": c, "span": span, "ws": torch.empty(c.workspace_bytes(B), dtype=torch.uint8, device=DEV), "out": torch.empty_like(q)}
    else:
        anc, depth = _tree(case)
        st |= {"kv": kv, "anc": anc, "depth": depth, "slot": slot, "live": live}
    return st


def _evict_inputs(case, seed):
    NL, B, H, Dh, ctx = (case[k] for k in ("NL", "B", "H", "Dh", "ctx"))
    kv = _kv(seed, case, (NL, B, ctx, 2, H, Dh))
    pages = (ctx + PAGE - 1) // PAGE + 1
    return kv, _scores(seed, (NL, B, H, pages * PAGE)), pages


def _tables(case, seed, pages, L):
    """Page tables [B, pages] of a row's slots and of the pages that its kept tokens are to go to (the same table where they stay in place), and
    how many pages each names."""
    B, keep = case["B"], case["keep"]
    src = torch.randperm(B * pages, generator=_gen(seed, "pages"), device=DEV).to(torch.int32).reshape(B, pages)
    if case["inplace"]:
        return src, src, B * pages, B * pages
    at = torch.arange(pages, device=DEV)[None, :]
    lo = ((L.long() - keep).clamp(min=0) // PAGE)[:, None]
    need = (at >= lo) & (at * PAGE < L[:, None])
    per = keep // PAGE + 2
    to = torch.randperm(B * per, generator=_gen(seed, "to"), device=DEV).to(torch.int32).reshape(B, per)
    dst = torch.where(need, to.gather(1, (at - lo).clamp(0, per - 1)), -1).to(torch.int32)
    return src, dst, B * pages, B * per


def _prepare_evict(case, seed):
    NL, B, H, Dh, ctx = (case[k] for k in ("NL", "B", "H", "Dh", "ctx"))
    kv, score0, pages = _evict_inputs(case, seed)
    L = _lengths(case)
    src, dst, n_src, n_dst = _tables(case, seed, pages, L)
    first0 = torch.full((B,), case["cut"], dtype=torch.int32, device=DEV)
    st = {"case": case, "len": L, "score0": score0, "first0": first0}
    if own:
        hb, c = _context(case, NL, ctx + 2)
        store = [torch.zeros(NL * n_src * H * PAGE * Dh, dtype=_type(case), device=DEV) for _ in range(2)]
        full = hb.KV(store[0], store[1], src, n_src)
        for l in range(NL):
            c.kv_write(B, l, full, 0, ctx, kv[l].float())
        # one pool: what the rows hold first, then what their kept tokens go to
        if case["inplace"]:
            st |= {"k0": store[0], "v0": store[1], "k": store[0].clone(), "v": store[1].clone()}
            table, target = src, None
        else:
            n = n_src + n_dst
            pool = [torch.zeros(NL, n, H * PAGE * Dh, dtype=_type(case), device=DEV) for _ in range(2)]
            for p, s in zip(pool, store):
                p[:, :n_src] = s.reshape(NL, n_src, -1)
            st |= {"k": pool[0], "v": pool[1], "n_src": n_src}
            table, target = src, torch.where(dst >= 0, dst + n_src, -1).to(torch.int32)
        kv_ = hb.KV(st["k"], st["v"], table, n_src if case["inplace"] else n_src + n_dst, seq_len_hint=0)
        st |= {"c": c, "target": target, "score": score0.clone(), "first": first0.clone(),
               "kept": torch.zeros(NL, B, H, case["keep"], dtype=torch.int32, device=DEV), "evicted": torch.zeros(B, dtype=torch.int32, device=DEV)}
        st["span"] = hb.KVSpan(kv_, first=st["first"], n_sinks=case["sinks"], window=0, span_hint=ctx - case["cut"], score=st["score"], n_scored=1)
    else:
        st |= {"kv": kv, "dst": dst, "n_dst": n_dst, "src": src}
    return st


def _logits(case, seed):
    """Logits as a model gives them: a wide bulk and a few tokens that stand out; the given tokens are mostly among those, some rows have none."""
    B, T, V = case["B"], case["T"], case["V"]
    x = _randn(seed, "logits", (B, T, V)) * 2.5
    top = _ints(seed, "top", 0, V, (B, T, 6))
    x.scatter_add_(2, top, _rand(seed, "peaks", (B, T, 6)) * 14)
    pick = _ints(seed, "pick", 0, 6, (B, T, 1))
    tok = torch.where(_rand(seed, "likely", (B, T)) < 0.8, top.gather(2, pick)[..., 0], _ints(seed, "any", 0, V, (B, T)))
    return x, torch.where(_rand(seed, "none", (B, T)) < 0.02, -1, tok).to(torch.int32)


def _prepare_logprobs(case, seed):
    B, T, V, k = (case[n] for n in ("B", "T", "V", "k"))
    x, tok = _logits(case, seed)
    st = {"case": case, "logits": x, "tokens": tok}
    if own:
        _, c = _context(case, 1, T + 1, T, 1, V)
        st |= {"c": c, "ws": torch.empty(c.workspace_bytes(B), dtype=torch.uint8, device=DEV), "logprob": torch.zeros(B, T, device=DEV),
               "rank": torch.zeros(B, T, dtype=torch.int32, device=DEV), "entropy": torch.zeros(B, T, device=DEV),
               "top_ids": torch.zeros(B, T, k, dtype=torch.int32, device=DEV) if k else None, "top_logprobs": torch.zeros(B, T, k, device=DEV) if k else None}
    return st


# ---- one pass ----------------------------------------------------------------------------------------------------
def run(st):
    kind = st["case"]["kind"]
    return (_run_own if own else _run_plain)["attn" if kind in ("span", "score") else kind](st)


def _own_attn(st):
    case = st["case"]
    out = {"out": st["out"]}
    if case["scored"]:
        st["score"].copy_(st["score0"])                      # the sums before the call again: the call adds to them
        out["score"] = st["score"]
    st["c"].tree_attention_span(case["B"], 0, st["ws"], st["q"], st["len"], st["span"], st["out"])
    return out


def _own_evict(st):
    case = st["case"]
    st["first"].copy_(st["first0"])                          # the state before the call again: the call changes it in place
    st["score"].copy_(st["score0"])
    if case["inplace"]:
        st["k"].copy_(st["k0"])
        st["v"].copy_(st["v0"])
    st["c"].hydra_kv_evict(case["B"], st["len"], st["span"], case["keep"], case["recent"], 0, st["kept"], st["evicted"], dst_table=st["target"])
    out = {"kept": st["kept"], "evicted": st["evicted"], "first": st["first"], "score": st["score"].view(torch.int32)}
    whole = torch.int16 if case["dtype"] == "bf16" else torch.int32
    for name in ("k", "v"):
        t = st[name] if case["inplace"] else st[name][:, st["n_src"]:]
        out[name] = t.view(whole).reshape(case["NL"], -1)
    return out


def _own_logprobs(st):
    case = st["case"]
    st["c"].hydra_token_logprobs(case["B"], st["ws"], st["logits"], st["tokens"], case["tau"], case["k"], st["logprob"], st["rank"], st["entropy"],
                                 st["top_ids"], st["top_logprobs"])
    out = {"logprob": st["logprob"], "rank": st["rank"], "entropy": st["entropy"]}
    return out | {"top_ids": st["top_ids"], "top_logprobs": st["top_logprobs"]} if case["k"] else out


def _seen(case, slot, live, L, anc, depth):
    """[B, T, n]: whether node t sees slot[b, n]."""
    cut, sinks, window, T = case["cut"], case["sinks"], case["window"], case["T"]
    node = slot - L[:, None]                                 # tree node of a slot, negative: cached
    mine = torch.where(node < 0, slot, L[:, None] + depth[node.clamp(0, T - 1)])                    # its position
    of = (node < 0)[:, None, :] | anc[:, node.clamp(0, T - 1)].permute(1, 0, 2)
    at = L[:, None] + depth[None, :]                         # positions of the nodes
    near = torch.ones_like(of) if not window else mine[:, None, :] > at[:, :, None] - window
    return of & live[:, None, :] & (near | (mine < cut + sinks)[:, None, :])


def _plain_attn(st):
    case = st["case"]
    B, T, H, Dh = (case[k] for k in ("B", "T", "H", "Dh"))
    L, slot, live = st["len"].long(), st["slot"], st["live"]
    seen = _seen(case, slot, live, L, st["anc"], st["depth"])
    rows = torch.arange(B, device=DEV)[:, None]
    kv = st["kv"][rows, torch.where(live, slot, 0)].float()                                         # [B, n, 2, H, Dh]
    k = kv[:, :, 0].permute(0, 2, 3, 1).contiguous()
    v = kv[:, :, 1].permute(0, 2, 1, 3).contiguous()
    s = torch.matmul(st["q"].float().permute(0, 2, 1, 3).contiguous(), k) / math.sqrt(Dh)
    s = torch.where(seen[:, None], s, -math.inf)
    p = torch.exp(s - s.amax(dim=-1, keepdim=True))
    p = p / p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p, v)
    out = {"out": o.permute(0, 2, 1, 3).contiguous().to(_type(case))}
    if case["scored"]:
        w = p[:, :, :case["scored"]].sum(dim=2)                                                     # [B, H, n]
        score = st["score0"].clone()
        tree = (slot >= L[:, None])[:, None, :]
        at = torch.where(live, slot, (L + T - 1)[:, None])[:, None, :].expand(B, H, -1)
        # a slot of the cache is added to, one of the tree starts anew
        held = torch.where(tree, 0.0, score[0].gather(2, at))
        new = torch.where(live[:, None, :], held + w, 0.0)
        base = score[0].scatter(2, at, 0.0)
        out["score"] = base.scatter_add_(2, at, new)[None]
    return out


def _keep_list(case, score, L):
    """kept slots [NL, B, H, keep] in order, and which rows are cut [B]."""
    keep, recent, sinks, cut = (case[k] for k in ("keep", "recent", "sinks", "cut"))
    at = torch.arange(score.shape[-1], device=score.device)
    n = L.long()[:, None]
    always = ((at < cut + sinks) | (at >= n - recent)) & (at >= cut) & (at < n)
    inside = (at >= cut) & (at < n)
    key = torch.where(always[None, :, None], math.inf, torch.where(inside[None, :, None], score, -math.inf))
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :keep]
    return torch.sort(order, dim=-1).values, L - cut > keep


def _plain_evict(st):
    case = st["case"]
    NL, B, H, Dh, keep, dt = case["NL"], case["B"], case["H"], case["Dh"], case["keep"], _type(case)
    L = st["len"].long()
    kept, cutrow = _keep_list(case, st["score0"], st["len"])
    to = (L[:, None] - keep) + torch.arange(keep, device=DEV)[None, :]                              # [B, keep]
    to = torch.where(cutrow[:, None], to, 0)
    score = st["score0"].scatter(3, to[None, :, None].expand(NL, B, H, keep), st["score0"].gather(3, kept))
    score = torch.where(cutrow[None, :, None, None], score, st["score0"])
    # contents: gather, then into pages as the cache places them (fp32: a token's dims in a row; 16 bits: K in runs of 8 dims, V by dim)
    l, b, h = torch.arange(NL, device=DEV)[:, None, None, None], torch.arange(B, device=DEV)[None, :, None, None], torch.arange(H, device=DEV)[None, None, :, None]
    n = st["n_dst"]
    fp32 = case["dtype"] == "f32"
    out = {"kept": torch.where(cutrow[None, :, None, None], kept, 0).to(torch.int32), "evicted": cutrow.to(torch.int32),
           "first": torch.where(cutrow, L - keep, st["first0"].long()).to(torch.int32), "score": score.view(torch.int32)}
    for i, name in enumerate(("k", "v")):
        store = torch.zeros((NL, n, H, PAGE, Dh) if fp32 else (NL, n, H, Dh // 8, PAGE, 8) if name == "k" else (NL, n, H, Dh, PAGE), dtype=dt, device=DEV)
        view = store if fp32 else store.permute(0, 1, 2, 4, 3, 5) if name == "k" else store.permute(0, 1, 2, 4, 3)          # [NL, n, H, token, ...]

        def place(slot, table):                              # page and place of slots [.., B, .., m]
            page = table[b, slot // PAGE].long()
            t = slot % PAGE
            if not fp32 and name == "v":
                t = ((t >> 2) & 1) * 8 + (t >> 3) * 4 + (t & 3)
            return page, t

        def put(values, slot, table, rows):
            page, t = place(slot, table)
            if not fp32 and name == "k":
                values = values.reshape(*values.shape[:-1], Dh // 8, 8)
            l_, b_, h_ = (x.expand(NL, B, H, slot.shape[-1]) for x in (l, b, h))
            m = rows[None, :, None, None].expand_as(l_) & (page >= 0)
            view[l_[m], page.expand_as(l_)[m], h_[m], t.expand_as(l_)[m]] = values[m]

        plane = st["kv"][:, :, :, i].permute(0, 1, 3, 2, 4)                                         # [NL, B, H, slots, Dh]
        if case["inplace"]:
            every = torch.arange(case["ctx"], device=DEV).expand(1, B, 1, case["ctx"])
            put(plane, every, st["src"], torch.ones_like(cutrow))
        put(plane[l, b, h, kept], to[None, :, None], st["dst"], cutrow)
        out[name] = store.view(torch.int32 if fp32 else torch.int16).reshape(NL, -1)
    return out


def _plain_logprobs(st):
    case, x, tok = st["case"], st["logits"] / st["case"]["tau"], st["tokens"].long()
    z = x - x.amax(dim=-1, keepdim=True)
    e = torch.exp(z)
    total = e.sum(dim=-1, keepdim=True)
    lp = z - torch.log(total)
    entropy = -(e / total * lp).sum(dim=-1)
    given = tok >= 0
    at = tok.clamp(min=0)[..., None]
    mine = st["logits"].gather(2, at)
    out = {"logprob": torch.where(given, lp.gather(2, at)[..., 0], 0.0),
           "rank": torch.where(given, (st["logits"] > mine).sum(dim=-1), -1).to(torch.int32), "entropy": entropy}
    if case["k"]:
        order = torch.sort(st["logits"], dim=-1, descending=True, stable=True).indices[..., :case["k"]]
        out |= {"top_ids": order.to(torch.int32), "top_logprobs": lp.gather(2, order)}
    return out


_run_own = {"attn": _own_attn, "evict": _own_evict, "logprobs": _own_logprobs}
_run_plain = {"attn": _plain_attn, "evict": _plain_evict, "logprobs": _plain_logprobs}


# ---- what a pass cannot do without -------------------------------------------------------------------------------
def work(case):
    if case["kind"] == "logprobs":
        rows, V, k = case["B"] * case["T"], case["V"], case["k"]
        return {"bytes": rows * (4 * V + 16 + 8 * k), "flops": 4 * rows * V}
    e, H, Dh, B = 2 if case["dtype"] == "bf16" else 4, case["H"], case["Dh"], case["B"]
    L = [case["ctx"] - (b * case["ragged"]) % max(1, (case["ctx"] - case["cut"] + 1) // 2) for b in range(B)]
    if case["kind"] == "evict":
        rows = sum(1 for n in L if n - case["cut"] > case["keep"])
        heads = case["NL"] * H
        read = sum(4 * heads * (n - case["cut"]) for n in L)
        return {"bytes": read + rows * heads * case["keep"] * (2 * 2 * Dh * e + 4 + 8), "flops": 0}
    T, total, pairs, sums = case["T"], 0, 0, 0
    for n in L:
        held = n - case["cut"]
        near = min(held, case["window"] - 1) if case["window"] else held
        slots = near + min(case["sinks"], held - near)
        total += slots + T
        pairs += T * slots
        sums += slots * 8 + T * 4
    nbytes = total * H * 2 * Dh * e + 2 * B * T * H * Dh * e
    if case["scored"]:
        nbytes += sums * H
    return {"bytes": nbytes, "flops": 4 * pairs * H * Dh}


# ---- the values in 64 bits ---------------------------------------------------------------------------------------
def exact(case, seed):
    return {"span": _exact_attn, "score": _exact_attn, "evict": _exact_evict, "logprobs": _exact_logprobs}[case["kind"]](case, seed)


def _exact_attn(case, seed):
    """Node by node from the definition: the list of what it sees, softmax, weighted sum."""
    B, T, H, Dh, cut, sinks, window = (case[k] for k in ("B", "T", "H", "Dh", "cut", "sinks", "window"))
    q, kv = _attn_inputs(case, seed)
    lens = _lengths(case).tolist()
    parent = parents(T, case["arity"])
    out = torch.zeros(B, T, H, Dh, dtype=torch.float64, device=DEV)
    pages = (case["ctx"] + T + PAGE - 1) // PAGE
    score = _scores(seed, (1, B, H, pages * PAGE), 0.01).double() if case["scored"] else None
    depth = [0] * T
    for t in range(1, T):
        depth[t] = depth[parent[t]] + 1
    for b, n in enumerate(lens):
        # everything that any node of the row may see, so that the row is converted once
        low = max(cut, n + 1 - window) if window else cut
        held = [s for s in range(cut, min(cut + sinks, low))] + list(range(low, n + T))
        index = torch.tensor(held, device=DEV)
        keys, vals = kv[b, index, 0].double(), kv[b, index, 1].double()                              # [m, H, Dh]
        where = {s: i for i, s in enumerate(held)}
        m = len(held)
        mask = torch.zeros(T, m, dtype=torch.bool)
        position = torch.tensor(held[:m - T])
        for t in range(T):
            p = n + depth[t]
            mask[t, :m - T] = (position < cut + sinks) | (position > p - window) if window else True
            a = t
            while a >= 0:
                if not window or depth[a] + window > depth[t] or n + depth[a] < cut + sinks:
                    mask[t, where[n + a]] = True
                a = parent[a]
        mask = mask.to(DEV)
        if case["scored"]:
            score[0, b, :, n:n + T] = 0.0
        for h in range(H):
            s = (q[b, :, h].double() @ keys[:, h].T.contiguous()) * Dh ** -0.5
            w = torch.softmax(s.masked_fill(~mask, -math.inf), dim=-1)
            out[b, :, h] = w @ vals[:, h].contiguous()
            if case["scored"]:
                score[0, b, h].index_add_(0, index, w[:case["scored"]].sum(dim=0))
    return {"out": out, "score": score} if case["scored"] else {"out": out}


def _exact_evict(case, seed):
    return None                                              # whole numbers: slots and bits


def _exact_logprobs(case, seed):
    x, tok = _logits(case, seed)
    x = x.double() / case["tau"]
    lp = torch.log_softmax(x, dim=-1)
    at = tok.long()
    out = {"logprob": torch.where(at < 0, 0.0, lp.gather(2, at.clamp(min=0)[..., None])[..., 0]), "rank": None,
           "entropy": -(lp.exp() * lp).sum(dim=-1)}
    if case["k"]:
        out |= {"top_ids": None, "top_logprobs": torch.topk(lp, case["k"], dim=-1).values}
    return out
