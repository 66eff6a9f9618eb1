"""Sessions under a budget whose rows take pages from one pool: rows that are cut while others take a prompt, share pages or break off."""
from __future__ import annotations

import pytest
import torch

from gpu_util import gpu_session
from helpers import make_weights
from synth import uniform_tokens
from test_gpu_span_session import F32, TREE

pytestmark = pytest.mark.gpu


def text(seed, n):
    return uniform_tokens(F32.seed + seed, 0, n, F32.V).to(torch.int32)


def rows_and_counts_agree(s):
    """ref counts what the tables name."""
    table, ref = s.page_table.cpu().flatten(), s.pages.ref.cpu()
    return torch.equal(ref, torch.bincount(table[(table >= 0) & (table < s.n_pages)].long(), minlength=s.n_pages).to(torch.int32))


def test_a_prompt_beside_rows_that_are_cut():
    """Rows 1 to 3 hold 864 tokens each when row 0's new prompt makes them due to be cut to 64: what they held is there for the prompt, in a pool that has no room for both."""
    keep, recent, slack = 64, 16, 800
    weights = make_weights(F32)
    kw = dict(budget=(keep, recent, slack), prefill_chunk=32)
    s = gpu_session(F32, TREE, 4, 1200, weights, pool_pages=168, **kw)
    long = torch.stack([text(b, 864) for b in range(4)])
    for pos in range(0, 464, 16):
        s.free_rows([0])
        s.prefill(long[:, pos:pos + 16])
    s.free_rows([0])
    s.prefill(text(9, 32).reshape(1, 32))                                    # row 0 alone: the cut that is due finds no row over keep + slack / 2
    for pos in range(464, 864, 16):
        s.free_rows([0])
        s.prefill(long[:, pos:pos + 16])
    s.free_rows([0])
    assert s.seq_len.tolist() == [0, 864, 864, 864] and s.span.first.tolist() == [0, 0, 0, 0] and int((s.page_table >= 0).sum()) == 3 * 54
    prompt = text(10, 250).reshape(1, 250)
    s.prefill(prompt)
    assert s.span.first.tolist() == [0, 800, 800, 800] and s.seq_len.tolist() == [250, 864, 864, 864]
    assert s.main.read_flags() == 0 and rows_and_counts_agree(s)
    alone = gpu_session(F32, TREE, 1, 1200, weights, **kw)
    alone.prefill(prompt)
    assert torch.equal(s.root[0], alone.root[0]) and (s.h_last[0] - alone.h_last[0]).abs().max() <= 1e-4 * alone.h_last[0].abs().max()
    s._drop_scratch()
    assert [int((s.page_table[b] >= 0).sum()) for b in range(4)] == [16, 4, 4, 4]


def test_a_row_that_cannot_be_cut_gives_back_the_pages_reserved_for_it():
    """Rows that share pages are due to be cut; one has an entry that names no page: it stays whole and is flagged, and no page is left that no row names."""
    weights = make_weights(F32)
    s = gpu_session(F32, TREE, 4, 400, weights, budget=(64, 24, 0), prefill_chunk=32, pool_pages=80)
    s.prefill(text(0, 64).reshape(1, 64))
    s.fork([0, 0, 0, 0])
    for _ in range(2):
        s.step()
    assert s.main.read_flags() == 0
    s._drop_scratch()
    keep, s._trim = s._trim, lambda: None
    s.step()
    s._drop_scratch()
    lens = (s.seq_len - s.span.first).tolist()
    assert min(lens) > 64
    s.fork([0, 1, 2, 2])
    assert s.main.read_flags() == 0
    lens[3] = lens[2]
    bad = int(s.span.first[2]) // 16 + 1
    page = int(s.page_table[2, bad])
    s.page_table[2, bad] = s.n_pages + 3
    s.pages.ref[page] -= 1
    assert rows_and_counts_agree(s)
    keep()
    assert s.main.read_flags() == 64 and (s.seq_len - s.span.first).tolist() == [64, 64, lens[2], 64]
    assert rows_and_counts_agree(s)
    assert (s._dst.page_table == -1).all()


def test_rows_that_share_no_longer_are_cut_where_they_lie():
    """A fork whose other row ended: a pool of 12 pages holds two rows of 64 tokens and a tree each, and not what a cut to other pages takes besides."""
    weights = make_weights(F32)
    kw = dict(budget=(64, 24, 0), prefill_chunk=32)
    s = gpu_session(F32, TREE, 2, 400, weights, pool_pages=12, **kw)
    alone = gpu_session(F32, TREE, 1, 400, weights, **kw)
    prompt = text(0, 64).reshape(1, 64)
    s.prefill(prompt)
    alone.prefill(prompt)
    s.fork([0, 0])
    s.free_rows([1])
    for _ in range(60):
        s.step()
        alone.step()
        assert int(s.seq_len[0]) == int(alone.seq_len[0]) and int(s.root[0]) == int(alone.root[0])
    assert (s.seq_len - s.span.first).tolist() == [64, min(64, int(s.seq_len[1]))] and not s._shared
    assert s.main.read_flags() == 0 and rows_and_counts_agree(s)


def test_rows_that_share_pages_beside_rows_that_do_not():
    """Rows 0 and 1 are copies of one prompt, rows 2 and 3 have their own, in a pool without room for copies of all four: texts, lists of kept slots and sums of sessions of one row."""
    keep, recent, slack, B = 64, 24, 20, 4
    weights = make_weights(F32)
    kw = dict(budget=(keep, recent, slack), sinks=3, prefill_chunk=32, want_logits=True)
    prompts = torch.stack([text(b, 90) for b in (0, 0, 2, 3)])
    s = gpu_session(F32, TREE, B, 400, weights, pool_pages=44, **kw)
    s.prefill(prompts)
    s.fork([0, 0, 2, 3])
    singles = [gpu_session(F32, TREE, 1, 400, weights, **kw) for _ in range(B)]
    for b, one in enumerate(singles):
        one.prefill(prompts[b:b + 1])
    u = torch.tensor([0.11, 0.37, 0.62, 0.93], device="cuda:0")
    cuts = [0] * B
    for step in range(30):
        v = (u + 0.29 * step) % 1.0
        before = s.span.first.tolist()
        s.step(typical=(0.8, 0.2, 0.4, v))
        for b, one in enumerate(singles):
            one.step(typical=(0.8, 0.2, 0.4, v[b:b + 1].contiguous()))
            assert int(one.seq_len[0]) == int(s.seq_len[b]) and int(one.span.first[0]) == int(s.span.first[b]) and int(one.root[0]) == int(s.root[b])
            if int(s.span.first[b]) != before[b]:
                cuts[b] += 1
                assert torch.equal(s._kept[:, b], one._kept[:, 0])
            F, L = int(s.span.first[b]), int(s.seq_len[b])
            x, y = s.span.score[:, b, :, F:L], one.span.score[:, 0, :, F:L]
            assert ((x - y).abs() <= 1e-4 * y.abs() + 1e-6).all()
        assert rows_and_counts_agree(s)
    assert min(cuts) >= 2 and s.main.read_flags() == 0


@pytest.mark.parametrize("pool", [None, 40])
@pytest.mark.parametrize("behind", [True, False])
def test_a_chunk_that_is_broken_off_behind_its_compaction_counts(behind, pool):
    """An interrupt between the compaction of a chunk and the cut (or in front of both): what the row has taken is remembered, and it never holds more than keep + slack."""
    keep, slack = 64, 40
    weights = make_weights(F32)
    s = gpu_session(F32, TREE, 1, 600, weights, budget=(keep, 16, slack), prefill_chunk=32, pool_pages=pool)
    s.prefill(text(0, 96).reshape(1, 96))
    assert int(s.seq_len[0] - s.span.first[0]) <= keep + slack // 2
    compact = s._keep_accepted

    def broken(*args):
        if behind:
            compact(*args)
        raise KeyboardInterrupt

    for n in (17, 15):                                                       # slack - slack / 2 = 20 is reached with the second one
        s._keep_accepted = broken
        with pytest.raises(KeyboardInterrupt):
            s.prefill(text(1, n).reshape(1, n))
        s._keep_accepted = compact
    for _ in range(40):
        s.step()
        assert int(s.seq_len[0] - s.span.first[0]) <= min(keep + slack, s._most_held())
    assert s.main.read_flags() == 0
