"""A budget session's step in a graph: each replay cuts the rows that need it."""
from __future__ import annotations

import pytest
import torch

from gpu_util import gpu_session, max_rel, to_np
from helpers import make_weights
from synth import uniform_tokens
from test_gpu_span_session import F32, HALF, TREE

pytestmark = pytest.mark.gpu


def captured(s):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.step()
    return graph


@pytest.mark.parametrize("cfg", [F32, HALF])
@pytest.mark.parametrize("slack", [0, 20])
@pytest.mark.parametrize("pool", [None, 60])
def test_a_step_under_a_budget_replays_from_a_graph(cfg, slack, pool):
    """Captured while no cut is due, replay by replay the text, the lists and the sums of a session that cuts each row over keep + slack / 2 behind every eager step; then eager steps again.
    Hints size grids, so sums may be taken in another order: the last step's outputs by as much as behind a window (16 bits: a result of attention rounds to its neighbour in each of two
    layers, 2^-11 of it, and what follows carries it on, twice that; fp32: sums of up to 60 terms, 2^-24 each, twice), the sums of weights, which those outputs change, by as much of themselves."""
    keep, recent, sinks, B = 48, 12, 3, 2
    weights = make_weights(cfg)
    p = torch.stack([uniform_tokens(cfg.seed + i, 0, 40, cfg.V) for i in range(B)]).to(torch.int32)
    a, b = (gpu_session(cfg, TREE, B, 400, weights, budget=(keep, recent, slack), sinks=sinks, want_logits=True, pool_pages=pool) for _ in range(2))
    a._trim = lambda: a.main.hydra_kv_evict(B, a.seq_len, a.span, keep, recent, slack // 2, a._kept, a._evicted)
    for s in (a, b):
        s.prefill(p)
        s.step()
    graph = captured(b)
    close = 1e-5 if cfg is F32 else 2e-3
    for i in range(30):
        graph.replay()
        a.step()
        assert torch.equal(a.seq_len, b.seq_len) and torch.equal(a.root, b.root) and torch.equal(a.span.first, b.span.first)
        held = b.seq_len - b.span.first
        assert int(held.max()) <= keep + slack // 2
        assert max_rel(to_np(b.h_last), to_np(a.h_last)) <= close
        for r in range(B):
            F, L = int(a.span.first[r]), int(a.seq_len[r])
            x, y = a.span.score[:, r, :, F:L], b.span.score[:, r, :, F:L]
            assert ((x - y).abs() <= close * x + 1e-6).all()
        b.logprobs(k=2)
        torch.cuda.synchronize()
    assert min(a.span.first.tolist()) > 0
    for _ in range(30):
        b.step()
        assert int((b.seq_len - b.span.first).max()) <= min(keep + slack, b._most_held())
    assert a.main.read_flags() == 0 and b.main.read_flags() == 0


def test_a_captured_step_of_rows_that_may_share_pages_is_refused():
    s = gpu_session(F32, TREE, 2, 400, make_weights(F32), budget=(48, 12, 0), pool_pages=80)
    s.prefill(uniform_tokens(F32.seed, 0, 40, F32.V).to(torch.int32).reshape(1, 40))
    s.fork([0, 0])
    n = s.seq_len.tolist()
    with pytest.raises(RuntimeError, match="share pages"):
        captured(s)
    torch.cuda.synchronize()
    assert s.seq_len.tolist() == n
    s.step()
    assert s.main.read_flags() == 0
