"""Weights of the attention behind an 8-bit cache: what their rounding to 16 bits may cost, and what they may depend on."""
from __future__ import annotations

import math

import pytest
import torch

from cache_util import DEV, cache_values, caches, context, tree_parent
from gpu_util import gpu_session
from helpers import make_weights
from synth import CONFIGS, frozen_tree, uniform_tokens

pytestmark = pytest.mark.gpu


def fill(c, kv8, kv, L):
    B, slots = kv.shape[:2]
    c.kv_write(B, 0, kv8.tail, 0, slots, kv.float().contiguous())
    n = torch.full((B,), L, dtype=torch.int32, device=DEV)
    c.hydra_kv8_seal(B, n, kv8)
    return n


def attend(c, kv8, n, q):
    out = torch.full_like(q, math.nan)
    c.tree_attention_kv8(q.shape[0], 0, c.ws, q, n, kv8, out)
    assert c.read_flags() == 0
    return out


# few rows: all keys in one workgroup; more (row, head)s than compute units: four waves, one or two query tiles each
@pytest.mark.parametrize("fmt,v0", [("int8", 127.0), ("e4m3", 120.0)])
@pytest.mark.parametrize("H,Dh,B,T", [(2, 128, 1, 8), (2, 64, 2, 40), (32, 64, 9, 8), (32, 128, 9, 40)])
def test_the_largest_weight_is_not_rounded(fmt, v0, H, Dh, B, T):
    """Every key has the same V, so the result is that V whatever the weights are, but for their rounding.  One key has three quarters of the weight or
    more, behind keys whose scores are 5 to 9 powers of two below its own, one in each of the first 13 tiles of 32 keys.

    The one weight is a power of two, which is exact in 16 bits; the others, at most a quarter in all, are off by 2^-11 of theirs at most, the sum of a
    wave by a few 2^-24, the exponents by 2^-16.  So before it is rounded the result is within 0.25 * 2^-11 + 2^-15 = 2^-12.8 of V, and V
    (127 or 120, just below a power of two) is the nearest half up to 2^-11 * 64 / 127 = 2^-11.99."""
    L, parent = 700, tree_parent(T)
    g = torch.Generator(device=DEV).manual_seed(Dh + T)
    kv = torch.randn(B, L + T, 2, H, Dh, generator=g, device=DEV)
    sign = torch.randn(H, Dh, generator=g, device=DEV).sign()
    kv[:, :, 1] = v0 * sign
    way = torch.randn(H, Dh, generator=g, device=DEV)
    way *= math.sqrt(Dh) / way.norm(dim=-1, keepdim=True)
    kv[:, :, 0] -= (kv[:, :, 0] * way).sum(-1, keepdim=True) / Dh * way           # the others' keys have no part in the queries' direction
    # score of the key 4.3 sqrt(Dh) log2(e), in powers of two
    bits = 4.3 * math.sqrt(Dh) * math.log2(math.e)
    kv[:, 600, 0] = way
    kv[:, 5:13 * 32:32, 0] = way * (1 - 7.0 / bits)
    kv = kv.half()
    q = (way * torch.linspace(4.0, 4.6, T, device=DEV)[:, None, None]).expand(B, T, H, Dh).half().contiguous()
    c = context(H, Dh, B, T, 1, 1024)
    kv8 = caches(H, Dh, B, 1, L + T, fmt, seed=T)
    n = fill(c, kv8, kv, L)
    values, _ = cache_values(kv, [L // 16] * B, fmt)
    want = (v0 * sign).double()
    assert bool((values[:, :, 1] == want).all())                                 # the cache holds V exactly
    for b in (0, B - 1):                                                         # the weights are what they are meant to be
        s = torch.matmul(q[b].double().permute(1, 0, 2), values[b, :L, 0].permute(1, 2, 0).contiguous()) / math.sqrt(Dh) * math.log2(math.e)
        gap = s[:, :, 600] - s[:, :, 5:13 * 32:32].amax(-1)
        assert float(gap.min()) > 5.0 and float(gap.max()) < 9.0
        assert float(torch.softmax(s * math.log(2), -1)[:, :, 600].min()) > 0.75
    out = attend(c, kv8, n, q)
    off = (out.double() != want).sum()
    assert int(off) == 0, f"{int(off)} of {out.numel()} results are not V"


@pytest.mark.parametrize("cache_format", ["int8", "e4m3"])
@pytest.mark.parametrize("H,Dh,B,L", [(4, 64, 2, 75), (2, 128, 2, 1300), (16, 64, 17, 60)])
def test_results_do_not_depend_on_the_workspace(cache_format, H, Dh, B, L):
    """A tree whose nodes do not fill a tile of 32 queries: whatever the workspace holds in the other places, the same bits."""
    tree = frozen_tree("tiny16")
    cfg = CONFIGS[1].with_(name="tiny16bit", dtype="bf16", d=H * Dh, H=H, Dh=Dh, F=512, T=16)
    sess = gpu_session(cfg, tree, B, L + 60, make_weights(cfg), prefill_chunk=64, want_logits=True, cache_format=cache_format)
    sess.prefill(torch.stack([uniform_tokens(cfg.seed + i, 0, L, cfg.V) for i in range(B)]).to(torch.int32))
    sess.draft()
    seen = []
    for i in range(4):
        if i == 0:
            sess.ws.zero_()
        else:                                                # halves of every size
            sess.ws.copy_(torch.randint(0, 256, sess.ws.shape, generator=torch.Generator(device=DEV).manual_seed(i), device=DEV).to(torch.uint8))
        sess.verify()
        o = sess.out()
        seen.append([t.clone() for t in (o.hidden, o.argmax, o.margin, o.logits)])
    for other in seen[1:]:
        for a, b in zip(seen[0], other):
            assert torch.equal(a, b)
    assert sess.main.read_flags() == 0
