"""Decoding sessions behind an 8-bit cache, and sessions whose rows share a pool of pages."""
from __future__ import annotations

import pytest
import torch

from gpu_util import gpu_session, max_rel, to_np
from helpers import make_weights
from synth import CONFIGS, frozen_tree, uniform_tokens

pytestmark = pytest.mark.gpu

BASE = CONFIGS[1].with_(name="tiny16bit", dtype="bf16", d=256, H=2, Dh=128, F=768, T=16)
TREE = frozen_tree("tiny16")


def prompts(cfg, n, L, first=0):
    return torch.stack([uniform_tokens(cfg.seed + first + i, 0, L, cfg.V) for i in range(n)]).to(torch.int32)


def rows_of(sess):
    """Every array that holds pages, as [layers, pages, ...], with the table that names them."""
    s = sess.shape
    block = s.H * 16 * s.Dh
    found = [(sess.k_pages.view(s.NL, -1, block), sess.kv.page_table), (sess.v_pages.view(s.NL, -1, block), sess.kv.page_table)]
    if sess.kv8 is not None:
        found += [(sess.k_codes.view(s.NL, -1, block), sess.page_table), (sess.v_codes.view(s.NL, -1, block), sess.page_table), (sess.kv8.scales, sess.page_table)]
    if sess.prefix:
        found += [(sess.pk_pages.view(1, -1, block), sess.page_table), (sess.pv_pages.view(1, -1, block), sess.page_table)]
    return found


def change_rows(sess, src):
    """What fork() means, by copying every page of a session whose rows have their own."""
    idx = torch.tensor(src, device=sess.dev)
    for pages, table in rows_of(sess):
        old = pages.clone()
        for b, s in enumerate(src):
            pages[:, table[b].long()] = old[:, table[s].long()]
    for t in [sess.seq_len, sess.h_last, sess.root] + ([sess.pseq_len] if sess.prefix else []) + ([sess.kv8.n_sealed] if sess.kv8 is not None else []):
        t.copy_(t[idx])


def state(sess):
    o = sess.out()
    return [t.clone() for t in (o.tree_tokens, o.hidden, o.argmax, o.logits, o.n_acc, o.path, sess.seq_len, sess.h_last, sess.root)]


def step_both(a, b, u):
    for s in (a, b):
        s.step(typical=(1.0, 0.05, 0.2, u))
    torch.cuda.synchronize()
    for x, y in zip(state(a), state(b)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("cache_format,prefix,shape", [(None, 0, BASE), ("int8", 0, BASE), ("e4m3", 0, BASE), ("int8", 1, BASE), (None, 1, BASE), (None, 0, CONFIGS[1])])
def test_rows_of_a_pool_decode_like_rows_of_their_own(cache_format, prefix, shape):
    """Prompts, forks, changes of places, rows that end, and a move of all pages: the same bits as rows that own copies."""
    B = 4
    cfg = shape.with_(prefix=prefix)
    W = make_weights(cfg)
    kw = dict(prefill_chunk=32, want_logits=True, cache_format=cache_format)
    pool = gpu_session(cfg, TREE, B, 260, W, pool_pages=60, **kw)
    own = gpu_session(cfg, TREE, B, 260, W, page_perm_seed=3, **kw)
    p = prompts(cfg, B, 75)
    pool.prefill(p)
    own.prefill(p)
    g = torch.Generator().manual_seed(1)

    def steps(n):
        for _ in range(n):
            step_both(pool, own, torch.rand(B, generator=g).to(own.dev))

    steps(2)
    pool.fork([0, 0, 2, 0])
    change_rows(own, [0, 0, 2, 0])
    shared = int((pool.pages.ref > 1).sum())
    assert shared >= 4                                    # the whole pages of row 0
    steps(6)
    pool.fork([3, 2, 1, -1])
    change_rows(own, [3, 2, 1, 3])
    steps(5)
    pool.free_rows([1])
    for t in [own.seq_len, own.h_last, own.root] + ([own.pseq_len] if prefix else []) + ([own.kv8.n_sealed] if cache_format else []):
        t[1] = 0
    steps(3)
    used = pool.defragment()
    assert used == int((pool.pages.ref > 0).sum()) and int((pool.pages.ref[used:] != 0).sum()) == 0
    assert used < 4 * 8
    steps(4)
    assert pool.main.read_flags() == 0 and own.main.read_flags() == 0
    named = torch.bincount(pool.page_table[pool.page_table >= 0].long(), minlength=pool.n_pages)
    assert torch.equal(named.to(torch.int32), pool.pages.ref)


@pytest.mark.parametrize("prefix", [0, 1])
def test_one_prompt_for_all_rows(prefix):
    """A prompt read once, by the first row alone, and shared: tokens as if every row had read it."""
    B, cfg = 3, BASE.with_(prefix=prefix)
    W = make_weights(cfg)
    p = prompts(cfg, 1, 90)
    pool = gpu_session(cfg, TREE, B, 200, W, prefill_chunk=32, want_logits=True, pool_pages=30)
    pool.prefill(p)
    assert pool.seq_len.tolist() == [90, 0, 0]
    pool.fork([0, 0, 0])
    assert pool.pages.ref[pool.page_table[0, :5].long()].tolist() == [3] * 5
    one = gpu_session(cfg, TREE, 1, 200, W, prefill_chunk=32, want_logits=True)
    one.prefill(p)
    for _ in range(6):
        pool.step()
        one.step()
    torch.cuda.synchronize()
    for b in range(B):
        assert max_rel(to_np(pool.out().hidden[b]), to_np(one.out().hidden[0])) < 2e-2
    assert torch.equal(pool.out().hidden[0], pool.out().hidden[1]) and torch.equal(pool.out().hidden[0], pool.out().hidden[2])
    toks, _ = pool.generate(20)
    assert len(toks) == B and toks[0] == toks[1] == toks[2]


@pytest.mark.parametrize("cache_format", ["int8", "e4m3"])
def test_every_step_behind_an_8_bit_cache_is_a_step_behind_its_values(cache_format):
    """At every step a 16-bit session whose cache holds the values that the 8-bit cache stands for (rounded to half: 2^-12 in int8, exact
    in e4m3) gives the same hidden states and logits; the text is long enough that every 16-bit page is taken several times."""
    B, cfg = 2, BASE
    W = make_weights(cfg)
    sess = gpu_session(cfg, TREE, B, 300, W, prefill_chunk=16, want_logits=True, cache_format=cache_format)
    ref = gpu_session(cfg, TREE, B, 300, W, prefill_chunk=16, want_logits=True)
    assert sess.n_tail == B * 2
    sess.prefill(prompts(cfg, B, 53))
    s, worst, g = cfg, 0.0, torch.Generator().manual_seed(5)
    for _ in range(25):
        L = int(sess.seq_len.max())
        plain = torch.empty(s.NL, B, L, 2, s.H, s.Dh, device=sess.dev)
        sess.main.kv8_read(B, -1, sess.kv8, 0, L, plain)
        for l in range(s.NL):
            ref.main.kv_write(B, l, ref.kv, 0, L, plain[l].contiguous())
        ref.seq_len.copy_(sess.seq_len)
        ref.host_len = L
        before = sess.seq_len.clone()
        sess.step(typical=(1.0, 0.05, 0.2, torch.rand(B, generator=g).to(sess.dev)))
        ref.out().tree_tokens.copy_(sess.out().tree_tokens)
        ref.verify()
        torch.cuda.synchronize()
        worst = max(worst, max_rel(to_np(sess.out().hidden), to_np(ref.out().hidden)), max_rel(to_np(sess.out().logits), to_np(ref.out().logits)))
        assert torch.equal(sess.kv8.n_sealed, sess.seq_len // 16) and bool((sess.seq_len > before).all())
    print(f"{cache_format}: largest difference {worst:.2e}")
    assert worst < 4e-3                                     # two layers of the 16-bit family: roundings of 2^-11 in a handful of places
    assert sess.main.read_flags() == 0


def test_a_pool_that_is_too_small_is_an_error():
    cfg = BASE
    W = make_weights(cfg)
    sess = gpu_session(cfg, TREE, 3, 200, W, prefill_chunk=32, pool_pages=14)
    sess.prefill(prompts(cfg, 2, 64))                       # 2 x 4 pages of text
    sess.free_rows([1])
    sess.fork([0, 0, 0])
    sess.step()                                             # 4 shared, 3 x (a page or two behind them)
    with pytest.raises(RuntimeError, match="exhausted"):
        for _ in range(60):
            sess.step()
    with pytest.raises(RuntimeError, match="exhausted"):
        sess.free_rows([0, 1, 2])
        sess.prefill(prompts(cfg, 3, 96))
    sess.reset()
    sess.prefill(prompts(cfg, 2, 64))
    sess.step()
    assert sess.main.read_flags() == 1                      # pools too small: the capacity bit of the calls above, nothing else


@pytest.mark.parametrize("cache_format", ["int8", "e4m3"])
def test_generation_behind_an_8_bit_cache(cache_format):
    """Session.generate takes the steps that a caller would, and leaves the same state."""
    B, cfg = 2, BASE
    W = make_weights(cfg)
    a, b = (gpu_session(cfg, TREE, B, 260, W, prefill_chunk=32, want_logits=True, cache_format=cache_format) for _ in range(2))
    for s in (a, b):
        s.prefill(prompts(cfg, B, 100))
    toks, accs = a.generate(40)
    got = [[] for _ in range(B)]
    for _ in accs:
        b.step()
        o = b.out()
        for r in range(B):
            n = int(o.n_acc[r])
            got[r] += [int(o.tree_tokens[r, int(o.path[r, j])]) for j in range(n)]
    assert [t[:40] for t in got] == toks
    assert torch.equal(a.seq_len, b.seq_len) and torch.equal(a.kv8.n_sealed, a.seq_len // 16) and torch.equal(a.h_last, b.h_last)
    assert a.main.read_flags() == 0


def test_refusals():
    cfg = BASE
    W = make_weights(cfg)
    with pytest.raises(ValueError):
        gpu_session(cfg, TREE, 1, 64, W, cache_format="int4")
    f32 = CONFIGS[1]
    with pytest.raises(ValueError):
        gpu_session(f32, TREE, 1, 64, make_weights(f32), cache_format="int8")
    sess = gpu_session(cfg, TREE, 2, 64, W, prefill_chunk=16, cache_format="int8")
    with pytest.raises(ValueError):
        sess.fork([0, 0])
    with pytest.raises(ValueError):
        sess.add_tree("wide", [-1] + [0] * 30)
    pool = gpu_session(cfg, TREE, 2, 64, W, prefill_chunk=16, pool_pages=8)
    with pytest.raises(ValueError):
        pool.fork([0])
    with pytest.raises(ValueError):
        pool.fork([0, 2])


@pytest.mark.parametrize("pool", [None, 40])
def test_text_behind_steps_stays_below_the_bound(pool):
    """The host's bound on the lengths comes from a copy that may be older than a later prompt."""
    cfg = BASE
    sess = gpu_session(cfg, TREE, 2, 256, make_weights(cfg), prefill_chunk=32, pool_pages=pool)
    sess.prefill(prompts(cfg, 2, 20))
    for _ in range(8):                                      # the last one asks for a copy of the lengths
        sess.step()
    assert sess._len_event is not None
    sess.prefill(prompts(cfg, 2, 90, 5))
    torch.cuda.synchronize()
    for _ in range(3):
        sess.step()
        assert sess.host_len >= int(sess.seq_len.max())
    assert sess.main.read_flags() == 0


@pytest.mark.parametrize("rows", [[2], [0, -1], [0.5], [10 ** 12]])
def test_rows_to_free_that_are_not_there(rows):
    cfg = BASE
    sess = gpu_session(cfg, TREE, 2, 64, make_weights(cfg), prefill_chunk=16, pool_pages=12)
    sess.prefill(prompts(cfg, 2, 20))
    with pytest.raises(ValueError, match="free_rows"):
        sess.free_rows(rows)
    sess.free_rows([])
    assert sess.seq_len.tolist() == [20, 20]
    sess.free_rows([1, 1])
    assert sess.seq_len.tolist() == [20, 0] and sess.main.read_flags() == 0


@pytest.mark.parametrize("cache_format", [None, "int8"])
def test_rows_that_end_make_room_for_the_next_text(cache_format):
    """Prompt after prompt in the same row, also while another row is nearly full: what counts is the lengths that the rows have."""
    cfg = BASE
    W = make_weights(cfg)
    sess = gpu_session(cfg, TREE, 2, 112, W, prefill_chunk=16, pool_pages=16, cache_format=cache_format, max_pos=144)
    alone = gpu_session(cfg, TREE, 1, 112, W, prefill_chunk=16, cache_format=cache_format, max_pos=144)
    for i in range(4):
        sess.free_rows([0])
        if i == 1:
            sess.free_rows([1])
            sess.prefill(prompts(cfg, 2, 96, 9))            # 96 of the 112: row 1 stays as long as that
            sess.free_rows([0])
        text = prompts(cfg, 1, 60, 20 + i)
        sess.prefill(text)
        alone.reset()
        alone.prefill(text)
        assert sess.seq_len.tolist() == [60, 0 if i == 0 else 96] and sess.host_len >= int(sess.seq_len.max())
        assert torch.equal(sess.h_last[0], alone.h_last[0]) and torch.equal(sess.root[:1], alone.root)
    sess.step()
    assert sess.main.read_flags() == 0
    with pytest.raises(Exception, match="capacity|CAPACITY|shorter|max_pos|exhausted"):
        sess.prefill(prompts(cfg, 1, 80, 3))                # 60 + 80 are more than the 128 slots of a row


def test_a_pool_that_a_larger_tree_has_used_up():
    """Pages behind the text that a wide tree needed are not there for a narrow one: an error, not a row without pages."""
    cfg = BASE
    sess = gpu_session(cfg, TREE, 3, 256, make_weights(cfg), prefill_chunk=16, pool_pages=16)
    sess.add_tree("wide", [-1] + [(n - 1) // 8 for n in range(1, 64)])
    sess.prefill(prompts(cfg, 3, 16))
    sess.free_rows([1, 2])
    sess.out("wide").tree_tokens.zero_()
    sess.verify("wide")                                     # 5 + 4 + 4 of the 16 pages
    sess.ctx("chain4")
    o = sess.out("chain4")
    o.tree_tokens.zero_(); o.path.copy_(torch.arange(4, dtype=torch.int32, device=sess.dev).expand(3, 4)); o.n_acc.fill_(4); o.last_node.fill_(3)
    with pytest.raises(RuntimeError, match="exhausted"):
        for _ in range(40):
            sess.verify("chain4")
            assert sess.main.read_flags() == 0
            sess.compact("chain4")
