"""A life of a session with a pool: prompts, steps, forks, rows that end, moves of pages, and calls that the pool has no room for, at random.  A pool that is
often too small and one that never is go through the same calls: the same bits after each, except for what was refused."""
from __future__ import annotations

import random

import pytest
import torch

from gpu_util import gpu_session
from helpers import make_weights
from paper_2402_05109_amd import binding as hb
from test_gpu_cache_session import BASE, TREE, prompts

pytestmark = pytest.mark.gpu

WIDE = [-1] + [(n - 1) // 4 for n in range(1, 24)]


def state(s):
    return [s.seq_len, s.h_last, s.root] + ([s.kv8.n_sealed] if s.kv8 is not None else []) + ([s.pseq_len] if s.prefix else [])


def content(s):
    """What the base cache holds of every row's text; flags that reading rows without pages raises are cleared."""
    c, L, hint = s.shape, int(s.seq_len.max()), s.kv.seq_len_hint
    t = torch.zeros(c.NL, s.B, L, 2, c.H, c.Dh, device=s.dev)
    if L == 0:
        return t
    s.kv.seq_len_hint = 0
    if s.kv8 is not None:
        s.main.kv8_read(s.B, -1, s.kv8, 0, L, t)
    else:
        for l in range(c.NL):
            s.main.kv_read(s.B, l, s.kv, 0, L, t[l])
    s.kv.seq_len_hint = hint
    s.main.read_flags()
    behind = torch.arange(L, device=s.dev)[None] >= s.seq_len[:, None]
    return t.masked_fill(behind[None, :, :, None, None, None], 0.0)


def no_room(e):
    return "exhausted" in str(e) or (isinstance(e, hb.HydraError) and e.code == hb.E_CAPACITY)


@pytest.mark.parametrize("seed,cache_format,prefix,B,pages", [
    (1, None, 0, 3, 21), (2, "int8", 0, 4, 30), (3, "e4m3", 0, 2, 13), (4, None, 1, 2, 14), (5, "int8", 1, 3, 20), (6, "e4m3", 1, 5, 40), (7, "int8", 0, 1, 9), (8, None, 0, 5, 26),
])
def test_a_small_pool_and_a_large_one(seed, cache_format, prefix, B, pages):
    cfg = BASE.with_(prefix=prefix)
    W = make_weights(cfg)
    kw = dict(prefill_chunk=24, cache_format=cache_format, want_logits=True)
    small, large = gpu_session(cfg, TREE, B, 200, W, pool_pages=pages, **kw), gpu_session(cfg, TREE, B, 200, W, pool_pages=40 * B + 50, **kw)
    rng, g, refused = random.Random(seed), torch.Generator().manual_seed(seed), 0
    if not prefix:
        for s in (small, large):
            s.add_tree("wide", WIDE)
    for k in range(30):
        op = rng.choice(("prompt", "rows", "step", "step", "step", "wide", "fork", "fork", "free", "move"))
        print(k, op, small.seq_len.tolist(), flush=True)
        if op in ("prompt", "rows"):
            rows, text = (B if op == "prompt" else rng.randint(1, B)), rng.randint(1, 90)
            p, before, done = prompts(cfg, rows, text, 100 * seed + k), small.seq_len.tolist(), text
            try:
                small.prefill(p)
            except RuntimeError as e:
                assert no_room(e)
                grown = [a - b for a, b in zip(small.seq_len.tolist(), before)]
                assert len(set(grown[:rows])) == 1 and not any(grown[rows:])
                done, refused = grown[0], refused + 1
            if done:
                large.prefill(p[:, :done].contiguous())
        elif op in ("step", "wide"):
            name = "wide" if op == "wide" and not prefix else "main"
            for _ in range(rng.randint(1, 4)):
                u = torch.rand(B, generator=g).to(small.dev)
                try:
                    small.step(name, typical=(1.0, 0.05, 0.2, u))
                except RuntimeError as e:
                    assert no_room(e)
                    refused += 1
                    break
                large.step(name, typical=(1.0, 0.05, 0.2, u))
                a, b = small.out(name), large.out(name)
                assert torch.equal(a.hidden, b.hidden) and torch.equal(a.argmax, b.argmax) and torch.equal(a.logits, b.logits)
        elif op == "fork":
            src = [rng.choice((-1, b, rng.randrange(B))) for b in range(B)]
            try:
                small.fork(src)
            except RuntimeError as e:
                assert no_room(e)
                refused += 1
                src = [int(r) for r in small._lists[3][:B].tolist()]
            large.fork(src)
        elif op == "free":
            rows = [b for b in range(B) if rng.random() < 0.4]
            small.free_rows(rows), large.free_rows(rows)
        else:
            small.defragment(), large.defragment()
        assert small.main.read_flags() in (0, 1) and large.main.read_flags() == 0
        for a, b in zip(state(small), state(large)):
            assert torch.equal(a, b)
        assert torch.equal(content(small), content(large))
        for s in (small, large):
            assert s.host_len >= int(s.seq_len.max())
            for pool in s._pools():
                named = torch.bincount(pool.page_table[pool.page_table >= 0].long(), minlength=pool.ref.numel())
                assert torch.equal(named.to(torch.int32), pool.ref)
    assert refused > 0
