"""Accumulated weights as the forward passes and sessions take them: trees and prompt chunks that do not fill a query tile, workspaces that hold anything."""
from __future__ import annotations

import math

import pytest
import torch

from gpu_util import gpu_session, to_np
from helpers import make_weights
from paper_2402_05109_amd import binding as hb
from span_util import DEV, attention_reference, cache, context, dtype_of, masks, tree_parent
from synth import uniform_tokens
from test_gpu_span_session import F32, HALF, TREE, Decoder

pytestmark = pytest.mark.gpu


def off_by(cfg, dec):
    """How far a weight may be off, relative to itself.  16 bits: on its way to a score a vector is rounded at most ten times (norm, q or k, attention's weights and result, the norm
    and the product of the FFN, a layer before the last one's norm and q or k), each time by 2^-11 of its length, so a score q k / sqrt(Dh) by 2 * 10 * 2^-11 of |q| |k| / sqrt(Dh), its exponential
    by that and the sum that it is divided by as well.  |q| |k| / sqrt(Dh) is at most about 2 here: both have lengths of 0.02 sqrt(d Dh) = 3.6 and a quarter more.  fp32: the same
    with sums of up to 512 products for roundings, 2^-24 each."""
    size = (1.25 * 0.02) ** 2 * cfg.d * cfg.Dh / math.sqrt(cfg.Dh)
    return 2 * 2 * size * (10 * 2.0 ** -11 if cfg.dtype == "bf16" else 10 * 512 * 2.0 ** -24)


def check_scores(cfg, s, decs):
    """Each held slot's sum, and what a layer's head has given away in all."""
    for b, d in enumerate(decs):
        F, L = int(s.span.first[b]), int(s.seq_len[b])
        for l in range(cfg.NL):
            for h in range(cfg.H):
                mine = to_np(s.span.score[l, b, h, F:L])
                want = [e[3] for e in d.held[l][h]]
                assert len(want) == L - F
                for i, (a, w) in enumerate(zip(mine, want)):
                    assert abs(a - w) <= off_by(cfg, d) * w + 1e-6, f"row {b}, layer {l}, head {h}, slot {F + i}: {a}, not {w}"


@pytest.mark.parametrize("cfg", [HALF, F32])
@pytest.mark.parametrize("chunk", [False, True])
@pytest.mark.parametrize("T", [2, 5, 33, 36, 64, 100])
def test_whatever_the_workspace_held(T, chunk, cfg):
    """tree_verify_forward_span and hydra_prefill_chunk_span add up the weights of T nodes behind 96 tokens, whose tiles every node sees whole.  What the workspace holds before the call does not
    matter: each byte 0xff (as fp32 and as half not a number) leaves the very bits that zeros leave.  A node gives 1 in all, by weights that are each off by 2^-14 at most
    of themselves against the sum that they are divided by: two sums of 128 products whose magnitudes come to 2, 2 * 144 * 2 * 2^-24, an exponential, 2^-20, and a sum of 200 terms, 216 * 2^-24."""
    weights = make_weights(cfg)
    L, B = 96, 2
    toks = torch.stack([uniform_tokens(cfg.seed + b, 0, L + T, cfg.V) for b in range(B)]).to(torch.int32)
    s = gpu_session(cfg, TREE, B, 400, weights, budget=(380, 16, 0), prefill_chunk=32)
    s.prefill(toks[:, :L])
    name = f"chain{T}"
    c, o = s.ctx(name), s.out(name)
    o.tree_tokens.copy_(toks[:, L:])
    s._hint(T)
    s.span.n_scored = T
    before, got = s.span.score.clone(), []
    for fill in (0, 255):
        s.span.score.copy_(before)
        s.ws.fill_(fill)
        if chunk:
            c.hydra_prefill_chunk_span(B, s.ws, o.tree_tokens, s.seq_len, s.span)
        else:
            c.tree_verify_forward_span(B, s.ws, o.tree_tokens, s.seq_len, s.span, o.hidden, o.argmax, o.margin, o.logits)
        got.append(s.span.score.clone())
    assert torch.isfinite(got[1]).all()
    assert torch.equal(got[0], got[1])
    gave = (got[1] - before)[..., :L + T].double().sum(dim=-1)               # [NL, B, H]
    assert ((gave - T).abs() <= T * 2.0 ** -14 + 2.0 ** -24 * before.double().sum(dim=-1)).all()
    decs = [Decoder(cfg, weights) for _ in range(B)]
    for b, d in enumerate(decs):
        d.feed(toks[b].tolist(), L + T)
    s.seq_len.fill_(L + T)
    check_scores(cfg, s, decs)
    assert s.main.read_flags() == 0


@pytest.mark.parametrize("f32, key", [(False, False), (True, False), (True, True)])     # (what writes a 16-bit cache clamps infinities)
@pytest.mark.parametrize("T, n_scored", [(5, 3), (16, 15), (40, 33), (64, 50), (128, 96), (100, 70)])
def test_nodes_that_do_not_count_stay_out_of_the_sums(T, n_scored, key, f32):
    """Queries behind the counted ones that are no numbers; or (fp32) a K of -infinity, which gives the counted nodes' scores of -infinity, so weights of 0, and the others +infinity: every
    slot's sum is that of the counted nodes alone."""
    H, Dh, L, at, dim = 2, 64, 100, 40, 7
    parent = tree_parent(T)
    g = torch.Generator().manual_seed(T)
    c = context(H, Dh, 1, parent, max_pos=300, f32=f32)
    kv = torch.randn(1, 1, L + T, 2, H, Dh, generator=g).to(dtype_of(f32))
    q = torch.randn(1, T, H, Dh, generator=g).to(dtype_of(f32))
    m = masks(parent, [L], [0], 0, 0, L + T)
    seen = m.clone()
    if key:
        q[:, :n_scored, :, dim] = q[:, :n_scored, :, dim].abs() + 0.1
        q[:, n_scored:, :, dim] = -q[:, n_scored:, :, dim].abs() - 0.1
        kv[0, 0, at, 0, :, dim] = -math.inf
        seen[:, :, at] = False                                               # a weight of 0
    kvd = cache(c, H, Dh, kv, m, f32)
    given = q.clone()
    if not key:
        given[:, n_scored:] = math.nan
    score0 = torch.rand(1, 1, H, kvd.max_pages * 16, generator=g).to(DEV)
    score, out = score0.clone(), torch.empty(1, T, H, Dh, dtype=dtype_of(f32), device=DEV)
    c.tree_attention_span(1, 0, c.ws, given.to(DEV), torch.tensor([L], dtype=torch.int32, device=DEV), hb.KVSpan(kvd, score=score, n_scored=n_scored), out)
    plain = kv[0].clone()
    plain[:, at, 0, :, dim] = 0.0
    ref, tol, add, add_tol = attention_reference(q, plain if key else kv[0], seen, f32, n_scored)
    assert ((out.double() - ref).abs() <= tol)[:, :n_scored].all()
    want = torch.where(torch.arange(L + T, device=DEV) < L, score0[0, :, :, :L + T].double(), 0.0) + add
    assert ((score[0, :, :, :L + T].double() - want).abs() <= add_tol + 2.0 ** -24 * want).all()
    assert c.read_flags() == 0


def choose(score, first, L, sinks, recent, keep):
    """The slots that stay, by the definition, from the sums that the session itself had."""
    if L - first <= keep:
        return None
    mid = sorted(range(first + sinks, L - recent), key=lambda i: (-score[i], i))[:keep - sinks - recent]
    return list(range(first, first + sinks)) + sorted(mid) + list(range(L - recent, L))


@pytest.mark.parametrize("pool", [None, 60])
@pytest.mark.parametrize("keep, recent, sinks", [(48, 16, 4), (80, 0, 0), (70, 60, 4)])
def test_a_budget_in_16_bits_follows_the_definition(keep, recent, sinks, pool):
    """Chunks of 36 and a last one of 22, then trees of 16, slack 0, a workspace of 0xff bytes in front of every forward pass: after each chunk and step the sums of decoding in 64
    bits, and the tokens kept are the ones that the session's own sums say (the decoder follows these: two sums may be closer than 16 bits tell)."""
    cfg, L, chunk, B = HALF, 202, 36, 2
    weights = make_weights(cfg)
    p = torch.stack([uniform_tokens(cfg.seed + 5 + b, 0, L, cfg.V) for b in range(B)]).to(torch.int32)
    s = gpu_session(cfg, TREE, B, 400, weights, budget=(keep, recent, 0), sinks=sinks, prefill_chunk=chunk, want_logits=True, pool_pages=pool)
    decs = [Decoder(cfg, weights, 0, sinks) for _ in range(B)]
    forward, trim = s._forward, s._trim
    fed = []

    def dirty(*args, **kw):
        s.ws.fill_(255)
        forward(*args, **kw)

    def follow():
        for b, d in enumerate(decs):
            d.feed(fed[b][0], fed[b][1])
        check_scores(cfg, s, decs)
        score = to_np(s.span.score)
        state = [(int(s.span.first[b]), int(s.seq_len[b])) for b in range(B)]
        trim()
        for b, d in enumerate(decs):
            first, n = state[b]
            cut = n - first > keep
            assert int(s.span.first[b]) == (n - keep if cut else first)
            for l in range(cfg.NL):
                for h in range(cfg.H):
                    kept = choose(score[l, b, h], first, n, sinks, recent, keep)
                    if cut:
                        assert s._kept[l, b, h].tolist() == kept
                        d.held[l][h] = [d.held[l][h][i - first] for i in kept]
                        for j, e in enumerate(d.held[l][h]):
                            e[0] = n - keep + j
        check_scores(cfg, s, decs)

    s._forward, s._trim = dirty, follow

    def behind_chunk(name, pos, n):
        fed[:] = [(p[b, pos:pos + n].tolist(), n) for b in range(B)]

    s.prefill(p, behind_chunk)
    o = s.out()
    accept = s.accept

    def accepted(*args):
        accept(*args)
        fed[:] = [([int(o.tree_tokens[b, int(o.path[b, j])]) for j in range(int(o.n_acc[b]))], 1) for b in range(B)]

    s.accept = accepted
    for _ in range(10):
        s.step()
    assert s.main.read_flags() == 0
