"""Eviction by accumulated weight, scores that follow accepted tokens, and the pages that nobody sees, against their definitions: whole numbers and bits."""
import math

import pytest
import torch

from paper_2402_05109_amd import binding as hb
from span_util import DEV, cache, context, dtype_of, keep_reference, masks, tree_parent

pytestmark = pytest.mark.gpu


def scores(kind, shape, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.exp(torch.randn(shape, generator=g) * 2 - 3)
    if kind == "ties":
        x = (x * 4).floor() / 4
    elif kind == "zeros":
        x = torch.zeros(shape)
    elif kind == "odd":                                                      # what nobody should pass, in every tenth place each
        r = torch.rand(shape, generator=g)
        for i, v in enumerate((math.nan, math.inf, -math.inf, -0.0, 0.0, -1.5, 1e-45, 3.4e38)):
            x = torch.where((r >= i / 10) & (r < (i + 1) / 10), torch.tensor(v), x)
    return x.to(DEV)


def setup(lens, firsts, NL, H, Dh, f32, seed=0):
    B, slots = len(lens), max(lens) + 1
    c = context(H, Dh, B, NL=NL, max_pos=slots + 2, f32=f32)
    kv = torch.randn(NL, B, slots, 2, H, Dh, generator=torch.Generator().manual_seed(seed)).to(dtype_of(f32))
    m = torch.zeros(B, 1, slots, dtype=torch.bool)
    for b, (L, F) in enumerate(zip(lens, firsts)):
        m[b, 0, F:L] = True
    kvd = cache(c, H, Dh, kv, m, f32, seed, NL=NL, spare=5)
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    return c, kv, kvd, n, torch.tensor(firsts, dtype=torch.int32, device=DEV)


def check(c, kv, kvd, lens, firsts, score0, score, first, kept, evicted, sinks, recent, keep, slack, f32, table=None):
    """kvd: the cache; table: where the kept tokens are (None: its own)."""
    NL, B, _, _, H, Dh = kv.shape
    want = keep_reference(score0, lens, firsts, sinks, recent, keep, slack)
    assert evicted.tolist() == [0 if want[0][b] is None else 1 for b in range(B)]
    assert first.tolist() == [firsts[b] if want[0][b] is None else lens[b] - keep for b in range(B)]
    expect = score0.cpu().clone()
    for b in range(B):
        lo, n = (firsts[b], lens[b] - firsts[b]) if want[0][b] is None else (lens[b] - keep, keep)
        if n == 0:
            continue
        row = hb.KV(kvd.k_pages, kvd.v_pages, (kvd.page_table if want[0][b] is None or table is None else table)[b:b + 1].contiguous(), kvd.n_pages)
        for l in range(NL):
            plain = torch.empty(1, n, 2, H, Dh, device=DEV)
            c.kv_read(1, l, row, lo, n, plain)
            for h in range(H):
                src = list(range(lo, lo + n)) if want[l][b] is None else want[l][b][h]
                if want[l][b] is not None:
                    assert kept[l, b, h].tolist() == src
                    expect[l, b, h, lo:lo + n] = score0[l, b, h].cpu()[torch.tensor(src)]
                assert torch.equal(plain[0, :, :, h].cpu(), kv[l, b, torch.tensor(src), :, h].float())
    assert torch.equal(score.cpu().view(torch.int32), expect.view(torch.int32))
    assert c.read_flags() == 0


CASES = [  # lens, firsts, NL, H, Dh, sinks, recent, keep, slack
    ([100], [0], 1, 2, 64, 0, 0, 10, 0), ([100], [0], 2, 4, 64, 4, 20, 50, 0), ([1], [0], 1, 2, 64, 0, 0, 1, 0), ([2], [0], 1, 2, 64, 0, 0, 1, 0), ([2], [0], 1, 1, 128, 0, 1, 1, 0),
    ([2], [0], 1, 1, 128, 1, 0, 1, 0), ([50], [13], 1, 2, 128, 2, 3, 5, 0), ([50, 60, 70], [0, 0, 0], 2, 2, 64, 1, 16, 48, 7), ([33, 0, 32, 31], [0, 0, 16, 31], 1, 2, 64, 0, 1, 15, 0),
    ([300, 299, 17], [5, 100, 2], 2, 4, 128, 4, 64, 128, 0), ([1000], [0], 1, 2, 64, 4, 0, 999, 0), ([1000], [0], 1, 2, 64, 0, 999, 999, 0), ([64], [0], 1, 2, 64, 0, 16, 32, 0),
    ([700], [300], 3, 2, 128, 3, 40, 200, 0), ([8300], [3], 1, 2, 64, 4, 50, 4000, 0), ([8194], [0], 1, 2, 64, 1, 0, 8000, 0), ([20000], [7], 1, 2, 64, 4, 100, 2048, 0),
]


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("kind", ["plain", "ties", "zeros", "odd"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_in_place(case, kind, f32):
    lens, firsts, NL, H, Dh, sinks, recent, keep, slack = CASES[case]
    if max(lens) > 5000 and kind in ("plain", "zeros") and f32:
        pytest.skip("the selection does not depend on the cache's type")
    c, kv, kvd, n, first = setup(lens, firsts, NL, H, Dh, f32, case)
    score0 = scores(kind, (NL, len(lens) + 1, H, kvd.max_pages * 16), case)
    score = score0.clone()
    kept = torch.full((NL, len(lens), H, keep), -7, dtype=torch.int32, device=DEV)
    evicted = torch.full((len(lens),), -7, dtype=torch.int32, device=DEV)
    c.hydra_kv_evict(len(lens), n, hb.KVSpan(kvd, first=first, n_sinks=sinks, score=score), keep, recent, slack, kept, evicted)
    check(c, kv, kvd, lens, firsts, score0, score, first, kept, evicted, sinks, recent, keep, slack, f32)


@pytest.mark.parametrize("kind", ["plain", "odd", "close", "wide", "two"])
@pytest.mark.parametrize("L, hint", [(40000, 0), (3000, 20), (6000, 1500), (9000, 5000), (1000, 0), (4000, 0)])
def test_choice_among_many(L, hint, kind):
    """More candidates than a workgroup holds in registers; scores that differ in their last bits, that fill the type's range, or that have two values."""
    NL, H, Dh, sinks, recent, keep = 1, 2, 64, 3, 20, L // 3
    c, kv, kvd, n, first = setup([L], [5], NL, H, Dh, False, 3)
    shape = (NL, 1, H, kvd.max_pages * 16)
    if kind == "close":
        score0 = scores("ties", shape, 5) * 0 + 1 + torch.randint(0, 300, shape, generator=torch.Generator().manual_seed(5)).to(DEV) * 2.0 ** -23
    elif kind == "wide":
        bits = torch.randint(-2 ** 31, 2 ** 31, shape, generator=torch.Generator().manual_seed(5)).to(torch.int32)
        score0 = bits.view(torch.float32).to(DEV)
    elif kind == "two":
        score0 = (scores("plain", shape, 5) > 0.05).float()
    else:
        score0 = scores(kind, shape, 5)
    score = score0.clone()
    kept = torch.full((NL, 1, H, keep), -7, dtype=torch.int32, device=DEV)
    evicted = torch.full((1,), -7, dtype=torch.int32, device=DEV)
    c.hydra_kv_evict(1, n, hb.KVSpan(kvd, first=first, n_sinks=sinks, score=score, span_hint=hint), keep, recent, 0, kept, evicted)
    check(c, kv, kvd, [L], [5], score0, score, first, kept, evicted, sinks, recent, keep, 0, False)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("case", [1, 3, 6, 7, 8, 9, 13])
def test_into_other_pages(case, f32):
    """The pages that the rows had keep their contents; a page shared by two rows is read by both."""
    lens, firsts, NL, H, Dh, sinks, recent, keep, slack = CASES[case]
    B = len(lens)
    c, kv, kvd, n, first = setup(lens, firsts, NL, H, Dh, f32, case)
    extra = B * (keep // 16 + 2)
    block = H * 16 * Dh
    pool = []
    for t in (kvd.k_pages, kvd.v_pages):
        big = torch.full((NL, kvd.n_pages + extra, block), math.nan, dtype=dtype_of(f32), device=DEV)
        big[:, :kvd.n_pages] = t.reshape(NL, kvd.n_pages, block)
        pool.append(big)
    before = [p.clone() for p in pool]
    table = torch.full_like(kvd.page_table, -1)
    at = kvd.n_pages
    for b, L in enumerate(lens):
        for lp in range(max(0, L - keep) // 16, (L + 15) // 16):
            if L - firsts[b] > keep + slack:
                table[b, lp] = at
                at += 1
    big = hb.KV(pool[0].reshape(-1), pool[1].reshape(-1), kvd.page_table, kvd.n_pages + extra)
    score0 = scores("ties", (NL, B, H, kvd.max_pages * 16), case)
    score = score0.clone()
    kept = torch.zeros(NL, B, H, keep, dtype=torch.int32, device=DEV)
    evicted = torch.zeros(B, dtype=torch.int32, device=DEV)
    ref = torch.full((kvd.n_pages + extra,), 2, dtype=torch.int32, device=DEV)     # shared pages do not matter here
    c.hydra_kv_evict(B, n, hb.KVSpan(big, first=first, n_sinks=sinks, score=score), keep, recent, slack, kept, evicted, dst_table=table, ref=ref)
    check(c, kv, big, lens, firsts, score0, score, first, kept, evicted, sinks, recent, keep, slack, f32, table)
    for p, q in zip(pool, before):
        assert torch.equal(p[:, :kvd.n_pages].nan_to_num(9.0), q[:, :kvd.n_pages].nan_to_num(9.0))


def test_again_and_again():
    """A row that grows and is cut several times, in place; every cut goes by the scores of the one before."""
    H, Dh, keep, recent, sinks = 2, 64, 64, 16, 4
    lens, firsts = [300], [0]
    c, kv, kvd, n, first = setup([300], [0], 1, H, Dh, False)
    score = scores("plain", (1, 1, H, kvd.max_pages * 16), 1)
    kept, evicted = torch.zeros(1, 1, H, keep, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    held = [[[s for s in range(0)] for _ in range(H)]]
    text = {h: [] for h in range(H)}                                          # original slots that a head holds
    for L in (100, 130, 131, 200, 300):
        n.fill_(L)
        F = int(first)
        for h in range(H):
            text[h] = text[h] + list(range(len(text[h]) + F, L)) if not text[h] else text[h] + list(range(F + len(text[h]), L))
        before = score.clone()
        c.hydra_kv_evict(1, n, hb.KVSpan(kvd, first=first, n_sinks=sinks, score=score), keep, recent, 0, kept, evicted)
        ref = keep_reference(before, [L], [F], sinks, recent, keep, 0)[0][0]
        for h in range(H):
            text[h] = [text[h][s - F] for s in ref[h]]
        assert int(first) == L - keep and evicted.tolist() == [1]
        plain = torch.empty(1, keep, 2, H, Dh, device=DEV)
        c.kv_read(1, 0, kvd, L - keep, keep, plain)
        for h in range(H):
            assert text[h][:sinks] == list(range(sinks)) and text[h][-recent:] == list(range(L - recent, L))
            assert torch.equal(plain[0, :, :, h].cpu(), kv[0, 0, torch.tensor(text[h]), :, h].float())
    assert c.read_flags() == 0


def test_rows_that_stay_whole():
    """Out of range, without pages, or with shared ones: nothing of such a row is touched, its neighbours are cut."""
    H, Dh, keep, recent, sinks = 2, 64, 32, 8, 2
    lens, firsts = [100] * 7, [0] * 7
    c, kv, kvd, n, first = setup(lens, firsts, 1, H, Dh, False)
    score0 = scores("plain", (1, 7, H, kvd.max_pages * 16), 1)
    score = score0.clone()
    n0, f0 = [100, -1, kvd.max_pages * 16 + 1, 100, 100, 100, 100], [0, 0, 0, 101, -1, 0, 0]
    n.copy_(torch.tensor(n0)); first.copy_(torch.tensor(f0))
    table = kvd.page_table
    shared = int(table[5, 2])
    table[6, 3] = -1
    ref = torch.ones(kvd.n_pages, dtype=torch.int32, device=DEV)
    ref[shared] = 2
    k0, v0 = kvd.k_pages.clone(), kvd.v_pages.clone()
    kept, evicted = torch.full((1, 7, H, keep), -7, dtype=torch.int32, device=DEV), torch.full((7,), -7, dtype=torch.int32, device=DEV)
    c.hydra_kv_evict(7, n, hb.KVSpan(kvd, first=first, n_sinks=sinks, score=score), keep, recent, 0, kept, evicted, ref=ref)
    assert c.read_flags() == 1 | 64
    assert evicted.tolist() == [1, 0, 0, 0, 0, 0, 0] and first.tolist() == [68] + f0[1:]
    assert torch.equal(score[:, 1:], score0[:, 1:]) and (kept[:, 1:] == -7).all()
    mine = set(table[0].tolist())
    block = H * 16 * Dh
    for t, t0 in ((kvd.k_pages, k0), (kvd.v_pages, v0)):
        a, b = t.reshape(-1, block), t0.reshape(-1, block)
        rest = [p for p in range(kvd.n_pages) if p not in mine]
        assert torch.equal(a[rest].nan_to_num(5.0), b[rest].nan_to_num(5.0))


def test_a_graph_of_an_eviction():
    H, Dh, keep, recent, sinks, NL = 4, 128, 100, 30, 4, 2
    c, kv, kvd, n, first = setup([250, 90], [0, 0], NL, H, Dh, False)
    score0 = scores("ties", (NL, 2, H, kvd.max_pages * 16), 3)
    score, k0, v0 = score0.clone(), kvd.k_pages.clone(), kvd.v_pages.clone()
    kept, evicted = torch.zeros(NL, 2, H, keep, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    span = hb.KVSpan(kvd, first=first, n_sinks=sinks, score=score)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.hydra_kv_evict(2, n, span, keep, recent, 0, kept, evicted)
    for _ in range(3):
        first.zero_(); score.copy_(score0); kvd.k_pages.copy_(k0); kvd.v_pages.copy_(v0); kept.zero_(); evicted.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        check(c, kv, kvd, [250, 90], [0, 0], score0, score, first, kept, evicted, sinks, recent, keep, 0, False)


@pytest.mark.parametrize("f32", [False, True])
def test_scores_follow_accepted_nodes(f32):
    parent = tree_parent(13, 3)
    H, NL, B = 4, 2, 5
    c = context(H, 64, B, parent, NL=NL, max_pos=200, f32=f32)
    kvd = hb.KV(torch.zeros(NL * 10 * H * 16 * 64, dtype=dtype_of(f32), device=DEV), torch.zeros(NL * 10 * H * 16 * 64, dtype=dtype_of(f32), device=DEV),
                torch.zeros(B, 5, dtype=torch.int32, device=DEV), 10)
    score0 = torch.rand(NL, B, H, 80, device=DEV)
    score = score0.clone()
    lens = [0, 20, 67, 68, 9]
    path = torch.tensor([[0, 1, 4], [0, 3, 12], [0, 2, -1], [0, 1, 5], [0, 2, 8]], dtype=torch.int32, device=DEV)
    n_acc = [3, 3, 2, 3, 1]
    c.hydra_score_compact(B, torch.tensor(n_acc, dtype=torch.int32, device=DEV), path, torch.tensor(lens, dtype=torch.int32, device=DEV), hb.KVSpan(kvd, score=score))
    want = score0.clone()
    for b in (0, 1, 2, 4):                                                    # row 3 does not fit its table: the attention has skipped it
        for j in range(n_acc[b]):
            want[:, b, :, lens[b] + j] = score0[:, b, :, lens[b] + int(path[b, j])]
    assert torch.equal(score, want) and c.read_flags() == 0
    c.hydra_score_compact(1, torch.tensor([3], dtype=torch.int32, device=DEV), torch.tensor([[0, 5, 4]], dtype=torch.int32, device=DEV),
                          torch.tensor([0], dtype=torch.int32, device=DEV), hb.KVSpan(kvd, score=score))
    want[:, 0, :, 1] = want[:, 0, :, 5]
    assert torch.equal(score, want) and c.read_flags() == 4


@pytest.mark.parametrize("sinks, window, use_first", [(0, 0, False), (4, 40, False), (17, 33, True), (0, 1, True), (10 ** 9, 5, False), (3, 2 ** 31 - 1, True)])
def test_pages_that_nobody_sees_go_back(sinks, window, use_first):
    B, pages, n_pages = 6, 12, 80
    c = context(2, 64, B, max_pos=400)
    lens = [0, 1, 16, 100, 191, 150]
    firsts = [0, 0, 16, 37, 90, 0] if use_first else [0] * B
    g = torch.Generator().manual_seed(1)
    table0 = torch.randperm(n_pages, generator=g)[:B * pages].reshape(B, pages).to(torch.int32)
    table0[5, 2] = table0[3, 1]                                               # a page that two rows share
    ref0 = torch.zeros(n_pages, dtype=torch.int32)
    for p in table0.flatten().tolist():
        ref0[p] += 1
    table, ref = table0.to(DEV), ref0.to(DEV)
    lo = torch.zeros(B, dtype=torch.int32, device=DEV)
    dummy = hb.KV(torch.zeros(8, dtype=torch.float16, device=DEV), torch.zeros(8, dtype=torch.float16, device=DEV), table, n_pages)
    span = hb.KVSpan(dummy, first=torch.tensor(firsts, dtype=torch.int32, device=DEV) if use_first else None, n_sinks=sinks, window=window)
    c.hydra_pages_release_span(B, hb.Pages(table, ref), torch.tensor(lens, dtype=torch.int32, device=DEV), span, lo)
    want, count = table0.clone(), ref0.clone()
    for b in range(B):
        L, F = lens[b], firsts[b]
        low = max(F, L + 1 - window) if window else F
        see = {s for s in range(F, L) if s >= low or s < F + sinks}
        assert int(lo[b]) == low
        for i in range(pages):
            if not any(i * 16 <= s < i * 16 + 16 for s in see):
                count[table0[b, i]] -= 1
                want[b, i] = -1
    assert torch.equal(table.cpu(), want) and torch.equal(ref.cpu(), count) and c.read_flags() == 0
