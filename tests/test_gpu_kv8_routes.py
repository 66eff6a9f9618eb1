"""Every kernel that attention behind an 8-bit cache can take: the rules by which it is chosen, written out, and cases that reach each one."""
from __future__ import annotations

import math
import os
import re

import pytest
import torch

from cache_util import DEV, attention_reference, cache_values, caches, context, tree_parent
from paper_2402_05109_amd.build import CSRC

LENGTHS = [700, 0, 333, 16, 15, 640, 1, 47, 95]
LONG = [2000, 31, 1203]
# H, Dh, T, lengths.  Dh of 64 and 128 and both formats of each
SHAPES = [
    (2, 5, LENGTHS[:3]),          # all keys in one workgroup, the head's dims in as many shares as there are
    (32, 20, LENGTHS[:3]),        # in two, (32, 40) in one
    (32, 40, LENGTHS[:3]),
    (32, 20, LENGTHS[:5]),
    (2, 64, LONG[:2]),            # keys split over workgroups, a query tile to a wave
    (2, 40, LONG),
    (2, 7, LONG),
    (32, 32, LENGTHS),            # more (row, head)s than compute units
    (32, 33, LENGTHS),            # two query tiles to a wave: a second one with one query in it, a whole one
    (32, 64, LENGTHS),
    (32, 65, LENGTHS),            # and one behind the last query
    (32, 97, LENGTHS),
    (32, 128, LENGTHS),
    (32, 64, LENGTHS[:8]),        # eight waves
    (32, 97, LENGTHS[:3]),
    (32, 65, LONG),
]


def route(H, Dh, B, T, longest):
    """What launch_kv8_attention chooses: ('short', Dh, shares) or ('attn', Dh, query tiles, waves, request policy)."""
    tiles, QT = math.ceil((longest + T) / 32) + 1, math.ceil(T / 32)
    if tiles <= (56 if QT > 1 else 36) and QT * H * B <= 256:
        shares = Dh // 32
        while shares > 1 and QT * H * B * shares > 256:
            shares //= 2
        return ("short", Dh, shares)
    qt = 2 if QT > 1 and H * B * QT > 256 else 1
    groups = math.ceil(QT / qt)
    waves = 4 if H * B * groups > 256 or (Dh == 128 and QT == 1) else 8
    return ("attn", Dh, qt, waves, 2 if groups == 1 else 0)


def test_the_cases_reach_every_kernel_that_is_built():
    src = open(os.path.join(CSRC, "kv8_attn.hip")).read()
    built = set()
    each = re.search(r"#define KV8_EACH_OF\(.*?\n", src).group()
    for qt, waves, policy in re.findall(r"X\(DHv, (\d), (\d), Fv, (\d)\)", each):
        built |= {("attn", Dh, int(qt), int(waves), int(policy)) for Dh in (64, 128)}
    more = re.search(r"#define KV8_EACH\(X\).*?\n\n|#define KV8_EACH\(X\).*?#define", src, re.S).group()
    built |= {("attn", int(a), int(b), int(c), int(d)) for a, b, c, d in re.findall(r"X\((\d+), (\d), (\d), KV8_\w+, (\d)\)", more)}
    short = re.search(r"#define KV8_SHORT_EACH\(X\).*?\n\n", src, re.S).group()
    built |= {("short", int(a), int(b)) for a, b in re.findall(r"X\((\d+), (\d), KV8_\w+\)", short)}
    assert len(built) == 18                                  # by two formats
    reached = {route(H, Dh, len(L), T, max(L)) for H, T, L in SHAPES for Dh in (64, 128)}
    assert reached == built


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("Dh", [64, 128])
@pytest.mark.parametrize("H,T,L", SHAPES)
def test_attention_of_every_kernel(fmt, Dh, H, T, L):
    B, slots = len(L), max(L) + T
    print("case", fmt, H, Dh, T, L, route(H, Dh, B, T, max(L)), flush=True)
    parent = tree_parent(T)
    c = context(H, Dh, B, T, 1, slots + 8)
    kv8 = caches(H, Dh, B, 1, slots, fmt, seed=T)
    g = torch.Generator(device=DEV).manual_seed(T + Dh)
    kv = (torch.randn(B, slots, 2, H, Dh, generator=g, device=DEV) * torch.exp(0.5 * torch.randn(2, H, Dh, generator=g, device=DEV))).half()
    q = (1.5 * torch.randn(B, T, H, Dh, generator=g, device=DEV)).half()
    c.kv_write(B, 0, kv8.tail, 0, slots, kv.float().contiguous())
    n = torch.tensor(L, dtype=torch.int32, device=DEV)
    c.hydra_kv8_seal(B, n, kv8)
    kv8.tail.seq_len_hint = max(L)
    out = torch.full_like(q, math.nan)
    c.tree_attention_kv8(B, 0, c.ws, q, n, kv8, out)
    values, sv = cache_values(kv, [x // 16 for x in L], fmt)
    ref, tol = attention_reference(q, values, sv, L, parent)
    assert c.read_flags() == 0
    worst = float(((out.double() - ref).abs() / tol).max())
    assert worst <= 1.0, f"{worst} times what the roundings allow"
    # the same bits whatever the workspace holds, and a row that is left out of the call is left alone
    c.ws.fill_(0xFF)
    again = torch.full_like(q, 7.0)
    c.tree_attention_kv8(B - 1, 0, c.ws, q, n, kv8, again)
    if route(H, Dh, B - 1, T, max(L)) == route(H, Dh, B, T, max(L)) and H * B > 256:
        assert torch.equal(again[:B - 1], out[:B - 1])
    assert bool((again[B - 1] == 7.0).all()) and c.read_flags() == 0
