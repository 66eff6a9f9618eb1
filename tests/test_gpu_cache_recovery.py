"""Sessions with a pool of pages or an 8-bit cache behind calls that were refused or broken off: they go on as if the call had not been made."""
from __future__ import annotations

import pytest
import torch

from gpu_util import gpu_session
from helpers import make_weights
from test_gpu_cache_session import BASE, TREE, prompts

pytestmark = pytest.mark.gpu


def same_steps(a, b, rows, n=3):
    for _ in range(n):
        for s in (a, b):
            s.step()
        torch.cuda.synchronize()
        for x, y in ((a.out().hidden, b.out().hidden), (a.out().argmax, b.out().argmax), (a.seq_len, b.seq_len), (a.h_last, b.h_last), (a.root, b.root)):
            assert torch.equal(x[:rows], y[:rows])


def pages_named(sess):
    """Every count is the number of entries that name the page."""
    for p in sess._pools():
        named = torch.bincount(p.page_table[p.page_table >= 0].long(), minlength=p.ref.numel())
        assert torch.equal(named.to(torch.int32), p.ref)


@pytest.mark.parametrize("cache_format", [None, "int8"])
@pytest.mark.parametrize("front", [0, 20])
def test_pages_of_a_prompt_that_the_pool_had_no_room_for(cache_format, front):
    """The prompt takes the whole pool and is broken off; what it took is free again, and the next prompt of all rows is read in pages of its own."""
    cfg = BASE
    W = make_weights(cfg)
    kw = dict(prefill_chunk=16, cache_format=cache_format)
    sess = gpu_session(cfg, TREE, 2, 400, W, pool_pages=14, **kw)
    fresh = gpu_session(cfg, TREE, 2, 400, W, pool_pages=14, **kw)
    for s in (sess, fresh):
        if front:
            s.prefill(prompts(cfg, 2, front))
    with pytest.raises(RuntimeError, match="exhausted"):
        sess.prefill(prompts(cfg, 1, 250, 7))
    assert sess.main.read_flags() == 1                      # the pool was too small, nothing else
    pages_named(sess)
    if cache_format is None:                                # the chunks in front of the last one leave no hidden states: back to the text in front
        assert sess.seq_len.tolist() == [front] * 2
        assert int((sess.pages.ref > 0).sum()) == 2 * ((front + 15) // 16)
    else:
        sess.free_rows([0])                                 # the other row keeps its text
        fresh.free_rows([0])
        if front:
            sess.free_rows([1])
            fresh.free_rows([1])
    for s in (sess, fresh):
        s.prefill(prompts(cfg, 2, 60, 3))
    assert sess.seq_len.tolist() == fresh.seq_len.tolist() and sess.main.read_flags() == 0
    assert torch.equal(sess.h_last, fresh.h_last) and torch.equal(sess.root, fresh.root)
    held = sess.page_table[:, :(60 + front + 15) // 16 if cache_format is None else 4]
    assert bool((held >= 0).all()) and held.unique().numel() == held.numel()
    same_steps(sess, fresh, 2)
    assert sess.main.read_flags() == 0


@pytest.mark.parametrize("pool", [None, 30])
def test_chains_that_the_16_bit_pages_cannot_hold(pool):
    """An 8-bit session keeps 16-bit pages for the trees that it was made for: a longer chain is refused, by name and by every call that would create it."""
    cfg = BASE
    W = make_weights(cfg)
    sess = gpu_session(cfg, TREE, 2, 200, W, prefill_chunk=24, cache_format="int8", pool_pages=pool)
    sess.prefill(prompts(cfg, 2, 40))
    for call in (sess.ctx, sess.draft, sess.verify, lambda name: sess.generate(1, name)):
        with pytest.raises(ValueError, match="16-bit pages"):
            call("chain25")
    assert "chain25" not in sess._ctx
    assert sess.ctx("chain24").T == 24 and sess.ctx("ar").T == 1
    wide = gpu_session(cfg, TREE, 2, 200, W, prefill_chunk=24, pool_pages=pool)
    assert wide.ctx("chain25").T == 25                       # a 16-bit cache has a page for every slot
    sess.step()
    assert sess.main.read_flags() == 0


@pytest.mark.parametrize("rows", [[0.5, 1], [0, 1.5], [float("nan"), 0], [0, float("inf")], [-1.5, 0], [0], [0, 2]])
def test_fork_of_rows_that_are_not_there(rows):
    cfg = BASE
    sess = gpu_session(cfg, TREE, 2, 64, make_weights(cfg), prefill_chunk=16, pool_pages=12)
    sess.prefill(prompts(cfg, 2, 20))
    before = [t.clone() for t in (sess.page_table, sess.pages.ref, sess.h_last, sess.root)]
    with pytest.raises(ValueError):
        sess.fork(rows)
    for t, w in zip((sess.page_table, sess.pages.ref, sess.h_last, sess.root), before):
        assert torch.equal(t, w)
    sess.fork([1, -1])
    assert torch.equal(sess.h_last[0], before[2][1]) and sess.main.read_flags() == 0


def test_a_pool_of_one_page():
    """The lists that the calls fill are as long as the calls need, also where the pool and the batch are smaller than a pair of counts."""
    cfg = BASE
    sess = gpu_session(cfg, [-1], 1, 16, make_weights(cfg), prefill_chunk=4, pool_pages=1)
    assert all(t.numel() >= 2 for t in sess._lists)          # the moves' counts are two
    sess.prefill(prompts(cfg, 1, 8))
    h = sess.h_last.clone()
    assert sess.defragment() == 1 and sess._lists[3].tolist() == [0] * sess._lists.shape[1]
    assert torch.equal(sess.h_last, h) and sess.page_table[0].tolist()[:1] == [0] and sess.main.read_flags() == 0
    sess.free_rows([0])
    assert sess.defragment() == 0
