"""Attention over part of a cache and the weights that it adds up, against the definitions in 64 bits.  What no node sees is NaN or has no page."""
import itertools
import math

import pytest
import torch

from paper_2402_05109_amd import binding as hb
from span_util import DEV, attention_reference, cache, context, dtype_of, masks, tree_parent

pytestmark = pytest.mark.gpu


def chain(T):
    return [-1] + list(range(T - 1))


def run(parent, lens, firsts, sinks, window, H=2, Dh=64, f32=False, n_scored=None, seed=0, hint=True, scale=1.0):
    """One call and its check.  Returns (out, score) for further ones."""
    B, T = len(lens), len(parent)
    slots = max(lens) + T
    g = torch.Generator().manual_seed(seed)
    kv = torch.randn(1, B, slots, 2, H, Dh, generator=g).to(dtype_of(f32))
    q = (scale * torch.randn(B, T, H, Dh, generator=g)).to(dtype_of(f32)).to(DEV)
    c = context(H, Dh, B, parent, max_pos=slots + T + 1, f32=f32)
    m = masks(parent, lens, firsts, sinks, window, slots)
    kvd = cache(c, H, Dh, kv, m, f32, seed)
    pages = kvd.max_pages
    score = None
    if n_scored is not None:
        score0 = torch.rand(1, B + 1, H, pages * 16, generator=g).to(DEV)
        score = score0.clone()
    kvd.seq_len_hint = max(lens) if hint else 0
    span = hb.KVSpan(kvd, first=torch.tensor(firsts, dtype=torch.int32, device=DEV) if any(firsts) else None, n_sinks=sinks, window=window,
                     span_hint=max(l - f for l, f in zip(lens, firsts)) if hint else 0, score=score, n_scored=n_scored or 0)
    out = torch.full_like(q, math.nan)
    c.tree_attention_span(B, 0, c.ws, q, torch.tensor(lens, dtype=torch.int32, device=DEV), span, out)
    assert c.read_flags() == 0
    ref, tol, add, add_tol = attention_reference(q, kv[0], m, f32, n_scored or 0)
    far = ((out.double() - ref).abs() / tol).max().item()
    assert far <= 1, f"attention off by {far} times its tolerance"
    if score is not None:
        want, bound = score0.double().clone(), torch.zeros_like(score0, dtype=torch.float64)
        for b in range(B):
            L, see = lens[b], m[b].any(dim=0)
            for s in see.nonzero()[:, 0].tolist():
                base = want[0, b, :, s] if s < L else torch.zeros(H, dtype=torch.float64, device=DEV)
                want[0, b, :, s] = base + add[b, :, s]
                bound[0, b, :, s] = add_tol[b, :, s] + 2.0 ** -24 * want[0, b, :, s].abs()
        assert ((score.double() - want).abs() <= bound).all(), "accumulated weights"
    return out, score


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("T, L, first, sinks, window", [
    (1, 0, 0, 0, 0), (1, 0, 0, 4, 1), (1, 1, 0, 0, 1), (1, 1, 1, 2, 0), (1, 40, 0, 0, 1), (1, 300, 0, 4, 64), (1, 300, 299, 4, 0), (1, 300, 300, 4, 8),
    (5, 33, 0, 1, 2), (16, 100, 0, 2, 31), (16, 95, 17, 3, 20), (33, 250, 0, 16, 40), (64, 1000, 0, 33, 333), (64, 700, 123, 0, 0), (64, 500, 0, 10 ** 9, 5),
    (64, 400, 0, 3, 2 ** 31 - 1), (100, 90, 8, 5, 50), (128, 2, 0, 0, 3), (128, 260, 100, 7, 64),
])
def test_one_row(T, L, first, sinks, window, f32):
    run(tree_parent(T), [L], [first], sinks, window, f32=f32, seed=T + L)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("window", [1, 2, 3, 17, 64, 100])
@pytest.mark.parametrize("sinks", [0, 5, 40])
def test_windows_shorter_than_a_chain(window, sinks, f32):
    """Ancestors that are out of the window, sinks among the nodes themselves."""
    run(chain(96), [3, 33], [0, 2], sinks, window, f32=f32, n_scored=96, seed=window)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("n_scored", [0, 1, 7, 37])
def test_weights_of_ragged_rows(n_scored, f32):
    run(tree_parent(37), [0, 5, 64, 191, 320], [0, 5, 32, 100, 1], 3, 0, n_scored=n_scored, f32=f32, seed=n_scored)
    run(tree_parent(37), [0, 5, 64, 191, 320], [0, 0, 0, 0, 0], 6, 45, n_scored=n_scored, f32=f32, seed=n_scored + 1)


@pytest.mark.parametrize("H, Dh, B, T, L, window", [(2, 128, 3, 64, 2100, 900), (16, 64, 9, 64, 300, 0), (40, 128, 4, 40, 500, 333), (5, 128, 1, 1, 5000, 0),
                                                    (32, 128, 8, 128, 150, 70), (6, 64, 2, 20, 4000, 3000), (8, 128, 16, 33, 200, 0)])
@pytest.mark.parametrize("f32", [False, True])
def test_shapes_of_every_kernel(H, Dh, B, T, L, window, f32):
    """One and two query tiles to a wave, four and eight waves, keys of a head in one workgroup and in several, 64 and 128 dims."""
    if f32 and B * H * T * L > 2 ** 23:
        B = max(1, B // 4)
    run(tree_parent(T), [L - 13 * b for b in range(B)], [0] * B, 4, window, H=H, Dh=Dh, f32=f32, n_scored=min(T, 33), seed=L)


@pytest.mark.parametrize("f32", [False, True])
def test_results_do_not_depend_on_hints(f32):
    a, sa = run(tree_parent(20), [200, 90], [0, 10], 4, 64, f32=f32, n_scored=20, seed=3)
    b, sb = run(tree_parent(20), [200, 90], [0, 10], 4, 64, f32=f32, n_scored=20, seed=3, hint=False)
    assert (a.double() - b.double()).abs().max() <= 2.0 ** -9 * a.double().abs().max()      # two roundings of each side's tolerance; the grids differ


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("window, span_hint", [(0, 0), (0, 400), (300, 0)])
def test_the_roots_weights_of_more_slots_than_the_workspace_has_room_for(f32, window, span_hint):
    """max_pos sizes the workspace; this cache is longer."""
    H, Dh, T = 2, 128, 40
    parent, lens, firsts = tree_parent(T), [400, 30, 333], [0, 3, 150]
    c = context(H, Dh, 3, parent, max_pos=48, f32=f32)
    kv = torch.randn(1, 3, 400 + T, 2, H, Dh, generator=torch.Generator().manual_seed(1)).to(dtype_of(f32))
    m = masks(parent, lens, firsts, 4, window, 400 + T)
    kvd = cache(c, H, Dh, kv, m, f32)
    q = torch.randn(3, T, H, Dh, generator=torch.Generator().manual_seed(2)).to(dtype_of(f32)).to(DEV)
    out, score = torch.empty_like(q), torch.zeros(1, 3, H, kvd.max_pages * 16, device=DEV)
    span = hb.KVSpan(kvd, first=torch.tensor(firsts, dtype=torch.int32, device=DEV), n_sinks=4, window=window, span_hint=span_hint, score=score, n_scored=1)
    c.tree_attention_span(3, 0, c.ws, q, torch.tensor(lens, dtype=torch.int32, device=DEV), span, out)
    ref, tol, add, add_tol = attention_reference(q, kv[0], m, f32, 1)
    assert ((out.double() - ref).abs() <= tol).all() and c.read_flags() == 0
    seen = m.any(dim=1)[:, None].to(DEV)
    got = score[0, :, :, :400 + T].double()
    assert ((got - torch.where(seen, add, 0.0)).abs() <= add_tol).all()


@pytest.mark.parametrize("f32", [False, True])
def test_sharp_rows(f32):
    """Scores of deviation 30: nearly all weight on one slot."""
    run(tree_parent(30), [500], [0], 4, 200, f32=f32, n_scored=30, scale=30.0, seed=11)


@pytest.mark.parametrize("f32", [False, True])
def test_a_whole_cache_is_plain_tree_attention(f32):
    """No window, nothing evicted: what tree_attention computes."""
    H, Dh, T, L = 4, 64, 23, 210
    parent = tree_parent(T)
    c = context(H, Dh, 1, parent, max_pos=400, f32=f32)
    g = torch.Generator().manual_seed(5)
    kv = torch.randn(1, 1, L + T, 2, H, Dh, generator=g)
    m = masks(parent, [L], [0], 0, 0, L + T)
    kvd = cache(c, H, Dh, kv, m, f32)
    q = torch.randn(1, T, H, Dh, generator=g).to(dtype_of(f32)).to(DEV)
    n = torch.tensor([L], dtype=torch.int32, device=DEV)
    out, ref = torch.empty_like(q), torch.empty(1, T, H, Dh, device=DEV)
    c.tree_attention_span(1, 0, c.ws, q, n, hb.KVSpan(kvd), out)
    c.tree_attention(1, 0, c.ws, q.float(), n, kvd, ref)
    want, tol, _, _ = attention_reference(q, kv[0].to(dtype_of(f32)), m, f32, 0)
    assert ((out.double() - want).abs() <= tol).all() and ((out.double() - ref.double()).abs() <= 2 * tol).all()


def test_fp32_values_that_are_not_finite_reach_only_who_sees_them():
    """A node whose V is infinite, and a cached one at the edge of the window: their non-descendants and later nodes stay finite."""
    H, Dh, L, window = 2, 64, 70, 40
    parent = [-1, 0, 0, 1, 1, 2, 3]
    T = len(parent)
    c = context(H, Dh, 1, parent, max_pos=200, f32=True)
    kv = torch.randn(1, 1, L + T, 2, H, Dh, generator=torch.Generator().manual_seed(1))
    m = masks(parent, [L], [0], 0, window, L + T)
    edge = L + 1 - window                                                    # the root sees it, no other node
    assert m[0, 0, edge] and not m[0, 1:, edge].any()
    clean = kv.clone()
    kv[0, 0, L + 1, 1, 0, 3] = math.inf
    kv[0, 0, L + 2, 1, 1, 5] = math.nan
    kv[0, 0, edge, 1, 1, 9] = -math.inf
    kvd = cache(c, H, Dh, kv, m, True)
    q = torch.randn(1, T, H, Dh, generator=torch.Generator().manual_seed(2)).to(DEV)
    out = torch.empty_like(q)
    c.tree_attention_span(1, 0, c.ws, q, torch.tensor([L], dtype=torch.int32, device=DEV), hb.KVSpan(kvd, window=window), out)
    ref, tol, _, _ = attention_reference(q, clean[0], m, True, 0)
    bad = torch.zeros(1, T, H, Dh, dtype=torch.bool)
    bad[0, [1, 3, 4, 6], 0, 3] = True
    bad[0, [2, 5], 1, 5] = True
    bad[0, 0, 1, 9] = True
    bad = bad.to(DEV)
    assert torch.equal(~torch.isfinite(out), bad)
    assert ((out.double() - ref).abs() <= tol)[~bad].all()
    assert (out[0, [1, 3, 4, 6], 0, 3] == math.inf).all() and out[0, 0, 1, 9] == -math.inf and torch.isnan(out[0, [2, 5], 1, 5]).all()


@pytest.mark.parametrize("f32", [False, True])
def test_skipped_rows_and_bad_pages_are_flagged(f32):
    H, Dh, T = 2, 64, 6
    parent = tree_parent(T)
    B, L = 5, 50
    c = context(H, Dh, B, parent, max_pos=200, f32=f32)
    kv = torch.randn(1, B, L + T, 2, H, Dh, generator=torch.Generator().manual_seed(1)).to(dtype_of(f32))
    m = masks(parent, [L] * B, [0] * B, 2, 0, L + T)
    kvd = cache(c, H, Dh, kv, m, f32)
    q = torch.randn(B, T, H, Dh, generator=torch.Generator().manual_seed(2)).to(dtype_of(f32)).to(DEV)
    out = torch.full_like(q, 7.0)
    score = torch.zeros(1, B, H, kvd.max_pages * 16, device=DEV)
    room = kvd.max_pages * 16 - T
    lens = torch.tensor([L, -1, room + 1, L, L], dtype=torch.int32, device=DEV)
    first = torch.tensor([0, 0, 0, -1, L + 1], dtype=torch.int32, device=DEV)
    c.tree_attention_span(B, 0, c.ws, q, lens, hb.KVSpan(kvd, first=first, n_sinks=2, score=score, n_scored=T), out)
    assert c.read_flags() == 1
    assert (out[1:] == 7.0).all() and (score[0, 1:] == 0).all()
    ref, tol, _, _ = attention_reference(q, kv[0], m, f32, 0)
    assert ((out[:1].double() - ref[:1]).abs() <= tol[:1]).all()
    kvd.page_table[0, 1] = kvd.n_pages
    c.tree_attention_span(1, 0, c.ws, q[:1].contiguous(), lens[:1], hb.KVSpan(kvd, n_sinks=2, score=score, n_scored=T), out[:1])
    assert c.read_flags() == 64


@pytest.mark.parametrize("f32", [False, True])
def test_another_layer_another_stream_and_a_graph(f32):
    """A captured call with sums, replayed with eager calls of the same context between the replays."""
    H, Dh, T, L, NL = 2, 128, 40, 300, 3
    parent = tree_parent(T)
    c = context(H, Dh, 2, parent, NL=NL, max_pos=500, f32=f32)
    kv = torch.randn(NL, 2, L + T, 2, H, Dh, generator=torch.Generator().manual_seed(1)).to(dtype_of(f32))
    lens, firsts, sinks, window = [L, 111], [0, 0], 4, 100
    m = masks(parent, lens, firsts, sinks, window, L + T)
    kvd = cache(c, H, Dh, kv, m, f32, NL=NL)
    q = torch.randn(2, T, H, Dh, generator=torch.Generator().manual_seed(2)).to(dtype_of(f32)).to(DEV)
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    out, score = torch.empty_like(q), torch.zeros(NL, 2, H, kvd.max_pages * 16, device=DEV)
    span = hb.KVSpan(kvd, n_sinks=sinks, window=window, score=score, n_scored=T)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        c.tree_attention_span(2, 2, c.ws, q, n, span, out)
    st.synchronize()
    want_out, want = out.clone(), score.clone()
    ref, tol, _, _ = attention_reference(q, kv[2], m, f32, T)
    assert ((out.double() - ref).abs() <= tol).all() and (score[:2] == 0).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.tree_attention_span(2, 2, c.ws, q, n, span, out)
    for _ in range(4):
        score.zero_()
        out.fill_(math.nan)
        graph.replay()
        assert torch.equal(out, want_out) and torch.equal(score, want)
        other = torch.empty_like(q)
        c.tree_attention_span(2, 0, c.ws, q, n, hb.KVSpan(kvd, n_sinks=sinks, window=window), other)
        torch.cuda.synchronize()
    assert c.read_flags() == 0


@pytest.mark.parametrize("f32", [False, True])
def test_two_calls_at_once(f32):
    """Two streams, one context and cache, a workspace each: attention with scores beside attention without and log probabilities."""
    H, Dh, T, L, V = 4, 128, 40, 3000, 5000
    parent = tree_parent(T)
    c = context(H, Dh, 1, parent, max_pos=L + T + 1, f32=f32, vocab=V)
    g = torch.Generator().manual_seed(9)
    kv = torch.randn(1, 1, L + T, 2, H, Dh, generator=g).to(dtype_of(f32))
    kvd = cache(c, H, Dh, kv, masks(parent, [L], [0], 0, 0, L + T), f32)
    q = torch.randn(1, T, H, Dh, generator=g).to(dtype_of(f32)).to(DEV)
    n, x = torch.tensor([L], dtype=torch.int32, device=DEV), torch.randn(1, T, V, generator=g).to(DEV)
    ws = [torch.empty(c.workspace_bytes(1), dtype=torch.uint8, device=DEV) for _ in range(2)]
    span = [hb.KVSpan(kvd, n_sinks=3, window=1500), hb.KVSpan(kvd)]

    def first(out, score):
        span[0].score, span[0].n_scored = score, 7
        c.tree_attention_span(1, 0, ws[0], q, n, span[0], out)

    def second(out, lps, ids):
        c.tree_attention_span(1, 0, ws[1], q, n, span[1], out)
        c.hydra_token_logprobs(1, ws[1], x, None, 1.0, 3, top_ids=ids, top_logprobs=lps)

    def outputs():
        return (torch.empty_like(q), torch.zeros(1, 1, H, 16 * kvd.max_pages, device=DEV)), (torch.empty_like(q), torch.empty(1, T, 3, device=DEV), torch.empty(1, T, 3, dtype=torch.int32, device=DEV))
    want = outputs()
    first(*want[0]); second(*want[1])
    got = [outputs() for _ in range(5)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for a, b in got:
        with torch.cuda.stream(streams[0]):
            first(*a)
        with torch.cuda.stream(streams[1]):
            second(*b)
    torch.cuda.synchronize()
    for a, b in got:
        assert all(torch.equal(u, v) for u, v in zip(a + b, want[0] + want[1]))
    assert c.read_flags() == 0


@pytest.mark.parametrize("shape", [(1, 1, 2), (3, 1, 2), (2, 1, 1), (2, 1, 4), (2, 0, 2)])
def test_scores_of_another_model_are_refused(shape):
    c = context(2, 64, 1, [-1], NL=2, max_pos=64)
    kv = torch.zeros(2, 1, 33, 2, 2, 64, dtype=torch.float16)
    kvd = cache(c, 2, 64, kv, torch.ones(1, 1, 33, dtype=torch.bool), False, NL=2)
    score = torch.zeros(*shape, 16 * kvd.max_pages, device=DEV)
    n, q = torch.tensor([32], dtype=torch.int32, device=DEV), torch.zeros(1, 1, 2, 64, dtype=torch.float16, device=DEV)
    span = hb.KVSpan(kvd, first=torch.zeros_like(n), score=score, n_scored=1)
    ids = torch.zeros(1, 8, dtype=torch.int32, device=DEV)
    for call in (lambda: c.tree_attention_span(1, 0, c.ws, q, n, span, torch.empty_like(q)), lambda: c.hydra_score_compact(1, n, ids, n, span),
                 lambda: c.hydra_kv_evict(1, n, span, 8, 2, 0, torch.zeros(2, 1, 2, 8, dtype=torch.int32, device=DEV), ids[0])):
        with pytest.raises((ValueError, hb.HydraError)):
            call()
    assert (score == 0).all()


def test_slots_beyond_two_gigabytes_of_scores_and_pages():
    """Offsets that pass 32 bits: pages behind 4 GiB of others, scores of a late row."""
    H, Dh, T, L = 16, 128, 3, 70
    parent = tree_parent(T)
    c = context(H, Dh, 1, parent, max_pos=200)
    kv = torch.randn(1, 1, L + T, 2, H, Dh, generator=torch.Generator().manual_seed(1)).half()
    m = masks(parent, [L], [0], 0, 0, L + T)
    spare = 2 ** 32 // (H * 16 * Dh * 2) + 5
    small = cache(c, H, Dh, kv, m, False, spare=0)
    n = small.n_pages + spare
    store = []
    for t in (small.k_pages, small.v_pages):
        big = torch.empty(n * H * 16 * Dh, dtype=torch.float16, device=DEV)
        big[spare * H * 16 * Dh:] = t
        store.append(big)
    kvd = hb.KV(*store, (small.page_table + spare).contiguous(), n)
    q = torch.randn(1, T, H, Dh, generator=torch.Generator().manual_seed(2)).half().to(DEV)
    out = torch.empty_like(q)
    c.tree_attention_span(1, 0, c.ws, q, torch.tensor([L], dtype=torch.int32, device=DEV), hb.KVSpan(kvd), out)
    ref, tol, _, _ = attention_reference(q, kv[0], m, False, 0)
    assert ((out.double() - ref).abs() <= tol).all() and c.read_flags() == 0
