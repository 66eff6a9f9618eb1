"""Sessions whose text is bounded by a window or a budget, and what the model thinks of tokens, against decoding in 64 bits that follows the definitions token
by token."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from gpu_util import gpu_session, max_rel, to_np
from helpers import make_weights, oracle_model
from oracle import hydra_oracle as O
from synth import CONFIGS, frozen_tree, uniform_tokens

pytestmark = pytest.mark.gpu

F32 = CONFIGS[1].with_(name="tiny", F=344, V=512)
HALF = CONFIGS[1].with_(name="tiny16bit", dtype="bf16", d=256, H=2, Dh=128, F=768, V=512, T=16)
TREE = frozen_tree("tiny16")


class Decoder:
    """Plain decoding in 64 bits of one row: every layer and head holds its own list of (slot, K, V, accumulated weight)."""

    def __init__(self, cfg, weights, window=0, sinks=0):
        self.m = oracle_model(cfg, weights)
        self.window, self.sinks = window, sinks
        self.held = [[[] for _ in range(self.m.H)] for _ in range(self.m.NL)]
        self.L = 0

    def feed(self, tokens, counted):
        """Tokens at positions L .. L + n - 1, the first `counted` of which add up their weights.  Returns (hidden, logits) of every token."""
        m = self.m
        x = [m.w("embed")[int(t)].copy() for t in tokens]
        for l in range(m.NL):
            p = f"layers.{l}."
            new = []
            for i, xi in enumerate(x):
                n1 = O.rmsnorm(xi, m.w(p + "attn_norm"), m.eps)
                q, k, v = ((m.w(p + w) @ n1).reshape(m.H, m.Dh) for w in ("wq", "wk", "wv"))
                new.append((O.rope(q, self.L + i, m.theta), O.rope(k, self.L + i, m.theta), v))
            att = np.zeros((len(x), m.H, m.Dh))
            for h in range(m.H):
                slots = self.held[l][h] + [[self.L + i, k[h], v[h], 0.0] for i, (_, k, v) in enumerate(new)]
                for i, (q, _, _) in enumerate(new):
                    p_ = self.L + i
                    first = slots[0][0]
                    see = [s for s in slots if s[0] <= p_ and (not self.window or s[0] > p_ - self.window or s[0] < first + self.sinks)]
                    w = O.softmax(np.array([s[1] @ q[h] for s in see]) / np.sqrt(m.Dh))
                    att[i, h] = sum(a * s[2] for a, s in zip(w, see))
                    if i < counted:
                        for a, s in zip(w, see):
                            s[3] += a
                self.held[l][h] = slots
            for i in range(len(x)):
                a = x[i] + m.w(p + "wo") @ att[i].reshape(m.d)
                n2 = O.rmsnorm(a, m.w(p + "ffn_norm"), m.eps)
                x[i] = a + m.w(p + "w_down") @ (O.silu(m.w(p + "w_gate") @ n2) * (m.w(p + "w_up") @ n2))
        self.L += len(x)
        hid = [O.rmsnorm(xi, m.w("final_norm"), m.eps) for xi in x]
        return hid, [m.w("lm_head") @ h for h in hid]

    def cut(self, keep, recent):
        for l in range(self.m.NL):
            for h in range(self.m.H):
                s = self.held[l][h]
                if len(s) <= keep:
                    continue
                mid = s[self.sinks:len(s) - recent]
                best = sorted(sorted(range(len(mid)), key=lambda i: (-mid[i][3], mid[i][0]))[:keep - self.sinks - recent])
                kept = s[:self.sinks] + [mid[i] for i in best] + s[len(s) - recent:]
                for j, e in enumerate(kept):
                    e[0] = self.L - keep + j                                  # they become the row's last slots
                self.held[l][h] = kept


def greedy(dec, prompt, n_new):
    _, lg = dec.feed(prompt, 0)
    out = [O.argmax_lowest(lg[-1])]
    while len(out) < n_new:
        _, lg = dec.feed(out[-1:], 0)
        out.append(O.argmax_lowest(lg[-1]))
    return out


@pytest.mark.parametrize("window, sinks, L", [(24, 0, 70), (40, 4, 130), (1, 2, 20), (200, 3, 60), (17, 20, 90)])
def test_windowed_generation_is_windowed_plain_decoding(window, sinks, L):
    """fp32, trees: token for token, in sessions of their own pages and of a small pool."""
    weights = make_weights(F32)
    prompt = uniform_tokens(F32.seed, 0, L, F32.V).to(torch.int32).reshape(1, L)
    want = greedy(Decoder(F32, weights, window, sinks), prompt[0].tolist(), 40)
    pages = (window + sinks + 64) // 16 + 5
    for kw in ({}, dict(pool_pages=pages)):
        s = gpu_session(F32, TREE, 1, 256, weights, window=window, sinks=sinks, prefill_chunk=32, **kw)
        s.prefill(prompt)
        got, accs = s.generate(40)
        assert got[0] == want and s.main.read_flags() == 0
        if kw:
            s._drop_scratch()
            seen = min(int(s.seq_len), window + sinks)
            assert int((s.page_table >= 0).sum()) <= seen // 16 + 3 and int((s.pages.ref > 0).sum()) == int((s.page_table >= 0).sum())


@pytest.mark.parametrize("pool", [None, 40])
def test_windowed_16_bit_sessions_follow_the_definition(pool):
    """Logits of a prompt and of verified trees' roots behind a window, 16 bits, ragged rows in one pool."""
    weights = make_weights(HALF)
    B, window, sinks = 2, 48, 5
    s = gpu_session(HALF, TREE, B, 256, weights, window=window, sinks=sinks, prefill_chunk=64, want_logits=True, pool_pages=pool)
    p = torch.stack([uniform_tokens(HALF.seed + i, 0, 150, HALF.V) for i in range(B)]).to(torch.int32)
    s.prefill(p)
    decs = [Decoder(HALF, weights, window, sinks) for _ in range(B)]
    last = [d.feed(p[b].tolist(), 0)[1][-1] for b, d in enumerate(decs)]
    n = 150 % 64
    assert max_rel(to_np(s.out(f"chain{n}").logits[:, n - 1]), np.stack(last)) < 2e-2
    for _ in range(4):
        before = s.seq_len.tolist()
        s.step()
        torch.cuda.synchronize()
        o = s.out()
        for b, d in enumerate(decs):
            toks = [int(o.tree_tokens[b, int(o.path[b, j])]) for j in range(int(o.n_acc[b]))]
            lg = d.feed(toks, 0)[1]
            for j in range(len(toks)):
                assert max_rel(to_np(o.logits[b, int(o.path[b, j])]), lg[j]) < 2e-2
            assert int(s.seq_len[b]) == before[b] + len(toks)
    assert s.main.read_flags() == 0


@pytest.mark.parametrize("pool", [None, 30])
@pytest.mark.parametrize("keep, recent, sinks", [(48, 16, 4), (40, 0, 0), (32, 28, 4), (300, 16, 4)])
def test_a_budget_follows_the_definition(keep, recent, sinks, pool):
    """fp32, slack 0: rows are cut behind every chunk and step.  Logits of every chunk and step against 64 bits with lists per head."""
    weights = make_weights(F32)
    L, chunk = 150, 32
    if pool and keep == 300:
        pool = 60
    s = gpu_session(F32, TREE, 1, 400, weights, budget=(keep, recent, 0), sinks=sinks, prefill_chunk=chunk, want_logits=True, pool_pages=pool)
    p = uniform_tokens(F32.seed + 1, 0, L, F32.V).to(torch.int32).reshape(1, L)
    got = []
    s.prefill(p, lambda name, pos, n: got.append(to_np(s.out(name).logits[0, :n])))
    d = Decoder(F32, weights, 0, sinks)
    for i, pos in enumerate(range(0, L, chunk)):
        toks = p[0, pos:pos + chunk].tolist()
        lg = d.feed(toks, len(toks))[1]
        d.cut(keep, recent)
        assert max_rel(got[i], np.stack(lg)) < 1e-4, f"chunk {i}"
    for step in range(12):
        s.step()
        torch.cuda.synchronize()
        o = s.out()
        toks = [int(o.tree_tokens[0, int(o.path[0, j])]) for j in range(int(o.n_acc[0]))]
        lg = d.feed(toks, 1)[1]
        d.cut(keep, recent)
        for j in range(len(toks)):
            assert max_rel(to_np(o.logits[0, int(o.path[0, j])]), lg[j]) < 1e-4, f"step {step}"
        held = int(s.seq_len[0]) - int(s.span.first[0])
        assert held == len(d.held[0][0]) <= keep
        for l in range(F32.NL):
            for h in range(F32.H):
                mine = to_np(s.span.score[l, 0, h, int(s.span.first[0]):int(s.seq_len[0])])
                assert np.allclose(mine, [e[3] for e in d.held[l][h]], rtol=1e-4, atol=1e-6)
    assert s.main.read_flags() == 0
    if pool:
        assert int((s.page_table >= 0).sum()) <= (min(keep, 300) + 64) // 16 + 2


@pytest.mark.parametrize("cfg", [F32, HALF])
def test_a_budget_that_is_never_reached_changes_nothing(cfg):
    weights = make_weights(cfg)
    p = uniform_tokens(cfg.seed, 0, 100, cfg.V).to(torch.int32).reshape(1, 100)
    a = gpu_session(cfg, TREE, 1, 256, weights)
    b = gpu_session(cfg, TREE, 1, 256, weights, budget=(250, 20, 0))
    for s in (a, b):
        s.prefill(p)
    assert a.generate(60)[0] == b.generate(60)[0] and b.span.first.tolist() == [0]


def test_rows_of_a_pool_under_a_budget():
    """A prompt shared by four rows that then go on by themselves, rows that are cut while they share pages, rows that end: the tokens of sessions that have each
    row for themselves."""
    cfg, keep, recent, slack, sinks = F32, 64, 24, 20, 3
    weights = make_weights(cfg)
    B, u = 4, torch.tensor([0.11, 0.37, 0.62, 0.93], device="cuda:0")
    p = uniform_tokens(cfg.seed + 3, 0, 90, cfg.V).to(torch.int32).reshape(1, 90)
    kw = dict(budget=(keep, recent, slack), sinks=sinks, prefill_chunk=32, want_logits=True)
    many = gpu_session(cfg, TREE, B, 400, weights, pool_pages=56, **kw)
    many.prefill(p)
    many.fork([0, 0, 0, 0])
    singles = []
    for b in range(B):
        s = gpu_session(cfg, TREE, 1, 400, weights, **kw)
        s.prefill(p)
        singles.append(s)
    texts = [[] for _ in range(B)]
    for step in range(25):
        many.step(typical=(0.8, 0.2, 0.4, (u + 0.29 * step) % 1.0))
        for b, s in enumerate(singles):
            s.step(typical=(0.8, 0.2, 0.4, ((u + 0.29 * step) % 1.0)[b:b + 1].contiguous()))
            o, t = s.out(), many.out()
            assert int(o.n_acc[0]) == int(t.n_acc[b]) and torch.equal(o.path[0], t.path[b])
            toks = [int(o.tree_tokens[0, int(o.path[0, j])]) for j in range(int(o.n_acc[0]))]
            assert toks == [int(t.tree_tokens[b, int(t.path[b, j])]) for j in range(int(t.n_acc[b]))]
            texts[b] += toks
        held = many.seq_len - many.span.first
        assert int(held.max()) <= keep + slack
    assert len({tuple(t) for t in texts}) == B and many.main.read_flags() == 0
    # contents of every row, layer and head, as the sessions of one row have them
    for b, s in enumerate(singles):
        n = int(s.seq_len[0]) - int(s.span.first[0])
        assert n == int(held[b]) and int(s.seq_len[0]) == int(many.seq_len[b])
        import paper_2402_05109_amd.binding as hb
        for l in range(cfg.NL):
            x, y = (torch.empty(1, n, 2, cfg.H, cfg.Dh, device="cuda:0") for _ in range(2))
            row = hb.KV(many.k_pages, many.v_pages, many.page_table[b:b + 1].contiguous(), many.n_pages)
            many.main.kv_read(1, l, row, int(s.span.first[0]), n, x)
            s.main.kv_read(1, l, s.kv, int(s.span.first[0]), n, y)
            assert (x - y).abs().max() <= 1e-4 * y.abs().max()
    ref = many.pages.ref.cpu()
    count = torch.zeros_like(ref)
    for e in many.page_table.cpu().flatten().tolist():
        if e >= 0:
            count[e] += 1
    assert torch.equal(ref, count)
    many.free_rows([1, 2])
    assert many.seq_len.tolist()[1:3] == [0, 0] and (many.span.score[:, 1:3] == 0).all() and many.span.first.tolist()[1:3] == [0, 0]
    many.defragment()
    many.step()
    many.reset()
    assert int(many.pages.ref.abs().sum()) == 0 and float(many.span.score.abs().sum()) == 0


def test_shared_rows_without_room_are_an_error():
    weights = make_weights(F32)
    s = gpu_session(F32, TREE, 4, 400, weights, budget=(64, 24, 0), prefill_chunk=32, pool_pages=17)
    s.prefill(uniform_tokens(F32.seed, 0, 64, F32.V).to(torch.int32).reshape(1, 64))
    s.fork([0, 0, 0, 0])
    with pytest.raises(RuntimeError, match="exhausted"):
        for _ in range(8):
            s.step()


@pytest.mark.parametrize("kw", [{}, dict(window=30, sinks=2), dict(budget=(40, 10, 8), sinks=2), dict(cache_format="int8")])
def test_log_probabilities_of_prompts(kw):
    """prompt_logprobs: what a bound or an 8-bit cache costs, from the logits that the session had."""
    cfg = HALF
    weights = make_weights(cfg)
    L, k = 100, 4
    s = gpu_session(cfg, TREE, 2, 256, weights, want_logits=True, prefill_chunk=32, **kw)
    p = torch.stack([uniform_tokens(cfg.seed + i, 0, L, cfg.V) for i in range(2)]).to(torch.int32)
    logits = []
    keep = s.logprobs
    s.logprobs = lambda t, tau, k, name, rows: (logits.append(s.out(name).logits[:, :t.shape[1]].clone()), keep(t, tau, k, name, rows))[1]
    got = s.prompt_logprobs(p, tau=0.9, k=k)
    x = torch.cat(logits, dim=1)
    assert x.shape == (2, L, cfg.V) and got["top_ids"].shape == (2, L, k)
    lp = torch.log_softmax(x.double() / 0.9, dim=-1)
    mine = lp[:, :-1].gather(2, p[:, 1:, None].long().cuda())[..., 0]
    assert ((got["logprob"][:, :-1].double() - mine).abs() <= 2e-5 * (1 + mine.abs())).all() and (got["logprob"][:, -1] == 0).all() and (got["rank"][:, -1] == -1).all()
    assert ((got["entropy"].double() + (lp.exp() * lp).sum(dim=-1)).abs() <= 1e-4).all()
    assert torch.equal(got["top_ids"].long(), torch.sort(x, dim=-1, descending=True, stable=True).indices[..., :k])
    assert s.main.read_flags() == 0


def test_log_probabilities_behind_a_step():
    weights = make_weights(HALF)
    s = gpu_session(HALF, TREE, 2, 256, weights, want_logits=True)
    s.prefill(torch.stack([uniform_tokens(HALF.seed + i, 0, 40, HALF.V) for i in range(2)]).to(torch.int32))
    s.step()
    o = s.out()
    got = s.logprobs(o.argmax, k=1)
    assert torch.equal(got["top_ids"][..., 0], o.argmax) and (got["rank"] == 0).all() and torch.equal(got["logprob"], got["top_logprobs"][..., 0])
    only = s.logprobs()
    assert set(only) == {"entropy"} and torch.equal(only["entropy"], got["entropy"])
    with pytest.raises(ValueError):
        s.logprobs(o.argmax[:, :3])
    plain = gpu_session(HALF, TREE, 1, 64, weights)
    with pytest.raises(ValueError):
        plain.logprobs()
    prompt = torch.ones(1, 8, dtype=torch.int32)
    with pytest.raises(ValueError):
        plain.prompt_logprobs(prompt)
    assert plain.seq_len.tolist() == [0]
    with pytest.raises(ValueError):
        s.prompt_logprobs(prompt.expand(2, 8)[:, :0])


@pytest.mark.parametrize("kw", [dict(window=0), dict(window=8, budget=(8, 2, 0)), dict(sinks=4), dict(window=8, sinks=-1), dict(budget=(0, 0, 0)), dict(budget=(8, 6, 0), sinks=3),
                                dict(budget=(8, 2)), dict(budget=(8, 2, -1)), dict(window=8, cache_format="int8"), dict(budget=(8, 2, 0), cache_format="e4m3")])
def test_refusals(kw):
    with pytest.raises(ValueError):
        gpu_session(HALF, TREE, 1, 64, make_weights(HALF), **kw)
    with pytest.raises(ValueError):
        gpu_session(HALF.with_(prefix=1), TREE, 1, 64, {}, window=8)


def test_a_prompt_that_is_broken_off_under_a_bound():
    """The state is that behind the last whole chunk, with and without a pool."""
    weights = make_weights(F32)
    p = uniform_tokens(F32.seed, 0, 96, F32.V).to(torch.int32).reshape(1, 96)
    for kw in (dict(window=20, sinks=2), dict(window=20, sinks=2, pool_pages=20), dict(budget=(30, 8, 4), pool_pages=20), dict(budget=(30, 8, 4))):
        s = gpu_session(F32, TREE, 1, 256, weights, prefill_chunk=32, want_logits=True, **kw)
        calls = []

        def hook(name, pos, n):
            calls.append(pos)
            if pos == 64:
                raise KeyboardInterrupt
        with pytest.raises(KeyboardInterrupt):
            s.prefill(p, hook)
        assert int(s.seq_len[0]) == 64
        t = gpu_session(F32, TREE, 1, 256, weights, prefill_chunk=32, want_logits=True, **kw)
        t.prefill(p[:, :64], lambda *a: None)
        assert torch.equal(s.h_last, t.h_last) and torch.equal(s.root, t.root)
        assert s.generate(12)[0] == t.generate(12)[0] and s.main.read_flags() == 0


@pytest.mark.parametrize("cfg", [F32, HALF])
def test_a_windowed_step_replays_from_a_graph(cfg):
    """Replay by replay the text of an eager session, with eager work between the replays.  The hint sizes grids, so sums may be taken in another order: in 16 bits a result of attention
    then rounds to its neighbour (2^-11 of it) in each of two layers, and what follows carries it on (twice that); in fp32 sums of up to 24 + 3 + 16 terms by 2^-24 each, twice."""
    weights = make_weights(cfg)
    p = torch.stack([uniform_tokens(cfg.seed + i, 0, 40, cfg.V) for i in range(2)]).to(torch.int32)
    a, b = (gpu_session(cfg, TREE, 2, 256, weights, window=24, sinks=3, want_logits=True) for _ in range(2))
    a.prefill(p)
    b.prefill(p)
    b.host_len += 120                                                        # frozen into the graph: a bound for every replay
    hint, state = b.host_len, [t.clone() for t in (b.seq_len, b.h_last, b.root)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.step()
    torch.cuda.current_stream().wait_stream(side)
    for t, s in zip((b.seq_len, b.h_last, b.root), state):
        t.copy_(s)
    b.host_len = hint
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step()
    for _ in range(6):
        graph.replay()
        a.step()
        assert torch.equal(a.seq_len, b.seq_len) and torch.equal(a.root, b.root) and torch.equal(a.out().n_acc, b.out().n_acc)
        assert max_rel(to_np(b.h_last), to_np(a.h_last)) <= (1e-5 if cfg is F32 else 2e-3)
        b.logprobs(k=2)
        torch.cuda.synchronize()
    assert a.main.read_flags() == 0 and b.main.read_flags() == 0
