"""Pages of a pool: taking, giving back, sharing, moving, copying, against the same rules written out in Python."""
from __future__ import annotations

import random

import pytest
import torch

from cache_util import DEV, context
from paper_2402_05109_amd import binding as hb

pytestmark = pytest.mark.gpu


class Pool:
    """The rules, one entry at a time."""

    def __init__(self, B, rows, pool):
        self.t = [[-1] * rows for _ in range(B)]
        self.ref = [0] * pool
        self.rows = rows

    def free(self):
        return [p for p, n in enumerate(self.ref) if n == 0]

    def reserve(self, lo, hi, extra):
        free, ok, flags, out = self.free(), [], 0, False
        for b, row in enumerate(self.t):
            a, e = (lo[b] if lo else 0), hi[b] + extra
            if a < 0 or hi[b] < 0 or a > e or (e + 15) // 16 > self.rows:
                ok.append(0)
                flags |= 1
                continue
            want = [i for i in range(a // 16, (e + 15) // 16) if row[i] < 0]
            if want and (out or len(want) > len(free)):
                out = True
                ok.append(0)
                flags |= 1
                continue
            for i in want:
                row[i] = free.pop(0)
                self.ref[row[i]] = 1
            ok.append(1)
        return ok, flags

    def release(self, lo, hi):
        flags = 0
        for b, row in enumerate(self.t):
            a = lo[b] if lo else 0
            if a < 0 or hi[b] < 0:
                flags |= 1
                continue
            keep = range(a // 16, (hi[b] + 15) // 16) if hi[b] > a else range(0)
            for i, p in enumerate(row):
                if p >= 0 and i not in keep:
                    row[i] = -1
                    self.ref[p] -= 1
        return flags

    def fork(self, src, n):
        old, free, flags, out = [list(r) for r in self.t], self.free(), 0, False
        a, d, forked = [], [], []
        for b in range(len(self.t)):
            s = src[b]
            a.append(-1), d.append(-1), forked.append(b)
            if s < -1 or s >= len(self.t):
                flags |= 4
                continue
            if s in (-1, b):
                continue
            if n[s] < 0 or (n[s] + 15) // 16 > self.rows:
                flags |= 1
                continue
            whole, part = n[s] // 16, n[s] % 16
            new = old[s][:whole] + [-1] * (self.rows - whole)
            if part and old[s][whole] >= 0:
                if out or not free:
                    out, flags = True, flags | 1
                    continue
                a[b], d[b] = old[s][whole], free.pop(0)
                new[whole] = d[b]
            forked[b] = s
            for p in old[b]:
                if p >= 0:
                    self.ref[p] -= 1
            for p in new:
                if p >= 0:
                    self.ref[p] += 1
            self.t[b] = new
        return a, d, forked, flags

    def compact(self):
        used = [p for p, n in enumerate(self.ref) if n]
        U = len(used)
        src = [p for p in used if p >= U]
        dst = [p for p in range(U) if self.ref[p] == 0]
        to = dict(zip(src, dst))
        self.t = [[to.get(p, p) for p in r] for r in self.t]
        for a, d in to.items():
            self.ref[d], self.ref[a] = self.ref[a], 0
        return src, dst, U


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Both:
    """The library's pool and the rules' side by side."""

    def __init__(self, c, B, rows, pool):
        self.c, self.B, self.rules = c, B, Pool(B, rows, pool)
        self.pages = hb.Pages(torch.full((B, rows), -1, dtype=torch.int32, device=DEV), torch.zeros(pool, dtype=torch.int32, device=DEV))
        self.ws = torch.empty(hb.pages_workspace_bytes(B, pool, rows), dtype=torch.uint8, device=DEV)

    def same(self, flags=0):
        assert self.pages.page_table.tolist() == self.rules.t
        assert self.pages.ref.tolist() == self.rules.ref
        assert self.c.read_flags() == flags

    def reserve(self, lo, hi, extra):
        ok = torch.full((self.B,), 9, dtype=torch.int32, device=DEV)
        self.c.hydra_pages_reserve(self.B, self.ws, self.pages, None if lo is None else i32(lo), i32(hi), extra, ok)
        want, flags = self.rules.reserve(lo, hi, extra)
        assert ok.tolist() == want
        self.same(flags)
        return want

    def release(self, lo, hi):
        self.c.hydra_pages_release(self.B, self.pages, None if lo is None else i32(lo), i32(hi))
        self.same(self.rules.release(lo, hi))

    def fork(self, src, n):
        a, d, f = (torch.full((self.B,), 9, dtype=torch.int32, device=DEV) for _ in range(3))
        self.c.hydra_pages_fork(self.B, self.ws, self.pages, i32(src), i32(n), a, d, f)
        wa, wd, wf, flags = self.rules.fork(src, n)
        assert (a.tolist(), d.tolist(), f.tolist()) == (wa, wd, wf)
        self.same(flags)
        return wf

    def compact(self):
        pool = len(self.rules.ref)
        a, d, n = torch.full((pool,), 9, dtype=torch.int32, device=DEV), torch.full((pool,), 9, dtype=torch.int32, device=DEV), i32([9, 9])
        self.c.hydra_pages_compact(self.B, self.ws, self.pages, a, d, n)
        src, dst, U = self.rules.compact()
        assert n.tolist() == [len(src), U]
        assert a.tolist() == src + [-1] * (pool - len(src)) and d.tolist() == dst + [-1] * (pool - len(dst))
        self.same()


@pytest.mark.parametrize("B,rows,pool,seed", [(1, 1, 1, 0), (1, 5, 3, 1), (3, 8, 20, 2), (4, 70, 130, 3), (17, 9, 200, 4), (5, 300, 5000, 5), (70, 33, 1500, 6), (1100, 3, 2500, 7)])
def test_a_life_of_pages(B, rows, pool, seed):
    """Random calls, every table and count compared after each."""
    rng = random.Random(seed)
    both = Both(context(2, 64, B), B, rows, pool)
    n = [0] * B
    for step in range(24):
        kind = rng.choice(("reserve", "reserve", "release", "fork", "fork", "compact"))
        if kind == "reserve":
            hi = [min(16 * rows, x + rng.randint(0, 60)) if rng.random() < 0.7 else x for x in n]
            extra = rng.randint(0, 40)
            ok = both.reserve(None if rng.random() < 0.6 else [max(0, x - 40) for x in hi], hi, extra)
            n = [h if o else x for h, o, x in zip(hi, ok, n)]
        elif kind == "release":
            n = [0 if rng.random() < 0.3 else x for x in n]
            both.release(None if rng.random() < 0.6 else [max(0, x - 40) for x in n], n)
        elif kind == "fork":
            src = [rng.choice((-1, b, rng.randrange(B), rng.randrange(B))) for b in range(B)]
            forked = both.fork(src, n)
            n = [n[f] for f in forked]
        else:
            both.compact()


@pytest.mark.parametrize("B,rows,pool,seed", [(12, 2500, 30000, 1), (40, 300, 9000, 2), (3, 5000, 40000, 3)])
def test_long_rows_and_large_pools(B, rows, pool, seed):
    """Tables beyond what one workgroup holds, rows of thousands of entries, free pages far behind the first ones."""
    rng = random.Random(seed)
    both = Both(context(2, 64, B), B, rows, pool)
    n = [rng.randint(10 * rows, 16 * rows - 80) for _ in range(B)]
    ok = both.reserve(None, n, 0)
    n = [x if o else 0 for x, o in zip(n, ok)]
    both.reserve(None, n, 64)
    gone = rng.randrange(B)
    n[gone] = 0
    both.release(None, n)
    forked = both.fork([rng.choice((b, rng.randrange(B))) for b in range(B)], n)
    n = [n[f] for f in forked]
    both.reserve(None, n, 70)
    n = [x // 2 if rng.random() < 0.4 else x for x in n]
    both.release(None, n)
    both.compact()
    both.reserve(None, n, 33)
    both.fork([B - 1 - b for b in range(B)], n)


def test_rows_out_of_range():
    both = Both(context(2, 64, 6), 6, 4, 30)
    both.reserve([0, 0, -1, 40, 0, 0], [20, -1, 5, 20, 64, 65], 0)        # the last one needs a fifth page, row 3 ends before it begins
    both.reserve(None, [2 ** 31 - 1, 0, 0, 0, 0, 0], 2 ** 31 - 1)
    both.fork([0, 6, -2, 0, 0, 4], [20, 0, 0, 0, 65, 0])                  # sources outside the batch; a source longer than its table
    both.release([0, 0, -5, 0, 0, 0], [16, -1, 0, 0, 64, 0])


def test_pool_runs_out_in_the_middle_of_a_call():
    both = Both(context(2, 64, 5), 5, 8, 10)
    assert both.reserve(None, [40, 0, 100, 16, 0], 0) == [1, 1, 1, 0, 1]  # 3 + 7: nothing left for row 3, rows without a need are served
    both.release(None, [40, 0, 0, 0, 0])
    assert both.reserve(None, [40, 90, 60, 60, 0], 0) == [1, 1, 0, 0, 1]  # row 2 does not fit, so neither does row 3 that would
    both.fork([0, 1, 0, 0, 0], [40, 90, 0, 0, 0])                         # one page left for three copies


def test_entries_of_pages_that_are_not_there():
    c = context(2, 64, 2)
    both = Both(c, 2, 4, 6)
    both.reserve(None, [30, 30], 0)
    both.pages.page_table[0, 1] = 77
    both.pages.ref[2] = 0                                                  # row 1's first page: counted free although it is named
    c.hydra_pages_release(2, both.pages, None, i32([0, 0]))
    assert both.pages.page_table.tolist() == [[-1] * 4, [-1] * 4]
    assert both.pages.ref.tolist() == [0, 1, 0, 0, 0, 0] and c.read_flags() == 64


@pytest.mark.parametrize("dtype,NL,H,Dh", [(hb.HYDRA_BF16, 3, 2, 64), (hb.HYDRA_BF16, 2, 5, 128), (hb.HYDRA_F32, 2, 3, 64)])
def test_copies_of_pages(dtype, NL, H, Dh):
    n_pages = 70
    c = context(H, Dh, 2, 1, NL, dtype=dtype)
    t = torch.float16 if dtype == hb.HYDRA_BF16 else torch.float32
    k, v = (torch.randn(NL, n_pages, H * 16 * Dh, device=DEV).to(t) for _ in range(2))
    kv = hb.KV(k, v, i32([[0], [1]]), n_pages)
    src, dst = [3, -1, 5, 69, 8, 9, 200, 4, 11, 12] + list(range(20, 41)), [1, 2, -1, 0, 8, 10, 6, 70, 13, 14] + list(range(42, 63))
    wk, wv = k.clone(), v.clone()
    live = [(a, b) for a, b in zip(src, dst) if 0 <= a < n_pages and 0 <= b < n_pages]
    for a, b in live:
        wk[:, b], wv[:, b] = k[:, a], v[:, a]
    c.hydra_kv_copy_pages(kv, len(src), i32(src), i32(dst))
    assert torch.equal(k, wk) and torch.equal(v, wv) and c.read_flags() == 64
    # only the first entries, by a count on the device
    wk[:, 2], wv[:, 2] = k[:, 40], v[:, 40]
    c.hydra_kv_copy_pages(kv, 3, i32([40, 41, 42]), i32([2, 3, 4]), i32([1]))
    assert torch.equal(k, wk) and torch.equal(v, wv) and c.read_flags() == 0
    c.hydra_kv_copy_pages(kv, 0, i32([40]), i32([2]))
    c.hydra_kv_copy_pages(kv, 3, i32([40, 41, 42]), i32([2, 3, 4]), i32([-1]))
    assert torch.equal(k, wk) and torch.equal(v, wv)


@pytest.mark.parametrize("NL,H,Dh", [(2, 2, 64), (3, 5, 128)])
def test_copies_of_sealed_pages(NL, H, Dh):
    n_pages = 20
    c = context(H, Dh, 2, 1, NL)
    k, v = (torch.randint(0, 256, (NL, n_pages, H * 16 * Dh), device=DEV).to(torch.uint8) for _ in range(2))
    s = torch.rand(NL, n_pages, H, 2, device=DEV)
    tail = hb.KV(torch.zeros(8, device=DEV), torch.zeros(8, device=DEV), i32([[0]]), 1)
    kv8 = hb.KV8(tail, k, v, s, i32([[0], [1]]), i32([0, 0]), n_pages, hb.KV8_E4M3)
    want = [x.clone() for x in (k, v, s)]
    for x, w in zip((k, v, s), want):
        w[:, [1, 17, 0]] = x[:, [5, 6, 19]]
    c.hydra_kv8_copy_pages(kv8, 4, i32([5, 6, -1, 19]), i32([1, 17, 3, 0]))
    for x, w in zip((k, v, s), want):
        assert torch.equal(x, w)
    assert c.read_flags() == 0


def test_calls_in_a_graph():
    """reserve, fork, copy, compact and release of one pool, captured once and replayed on other tables."""
    B, rows, pool = 4, 12, 60
    c = context(2, 64, B)
    both = Both(c, B, rows, pool)
    k, v = (torch.randn(1, pool, 2 * 16 * 64, device=DEV).half() for _ in range(2))
    kv = hb.KV(k, v, both.pages.page_table, pool)
    n, src, gone = i32([0] * B), i32([0] * B), i32([0] * B)
    a, d, f, ok = (i32([0] * B) for _ in range(4))
    ma, md, counts = i32([0] * pool), i32([0] * pool), i32([0, 0])

    def calls():
        c.hydra_pages_reserve(B, both.ws, both.pages, None, n, 5, ok)
        c.hydra_pages_fork(B, both.ws, both.pages, src, n, a, d, f)
        c.hydra_kv_copy_pages(kv, B, a, d)
        c.hydra_pages_release(B, both.pages, None, gone)
        c.hydra_pages_compact(B, both.ws, both.pages, ma, md, counts)
        c.hydra_kv_copy_pages(kv, pool, ma, md, counts)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    rng = random.Random(1)
    for _ in range(5):
        both.pages.page_table.fill_(-1)
        both.pages.ref.zero_()
        both.rules = Pool(B, rows, pool)
        lens, srcs = [rng.randint(1, 150) for _ in range(B)], [rng.randrange(B) for _ in range(B)]
        n.copy_(i32(lens)), src.copy_(i32(srcs))
        keep = [lens[s] if rng.random() < 0.7 else 0 for s in srcs]
        gone.copy_(i32(keep))
        before = k.clone()
        graph.replay()
        torch.cuda.synchronize()
        both.rules.reserve(None, lens, 5)
        content = {p: before[0, p] for p in range(pool)}
        wa, wd, _, _ = both.rules.fork(srcs, lens)
        content.update({q: content[p] for p, q in zip(wa, wd) if p >= 0})
        both.rules.release(None, keep)
        s2, d2, _ = both.rules.compact()
        content.update({q: content[p] for p, q in zip(s2, d2)})
        both.same()
        assert all(torch.equal(k[0, p], content[p]) for p in range(pool))
