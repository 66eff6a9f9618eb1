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
    assert s.main.read_flags() == 0 and s._shared
    s._drop_scratch()
    keep, s._trim = s._trim, lambda grown: None
    s.step()
    s._drop_scratch()
    lens = (s.seq_len - s.span.first).tolist()
    assert min(lens) > 64
    bad = int(s.span.first[2]) // 16 + 1
    page = int(s.page_table[2, bad])
    s.page_table[2, bad] = s.n_pages + 3
    s.pages.ref[page] -= 1
    s.fork([0, 1, 2, 0])                                                     # rows 0 and 3 share pages
    s.main.read_flags()
    assert rows_and_counts_agree(s)
    keep(1)
    assert s.main.read_flags() == 64 and (s.seq_len - s.span.first).tolist() == [64, 64, lens[2], 64]
    assert rows_and_counts_agree(s)
    assert (s._dst.page_table == -1).all()
