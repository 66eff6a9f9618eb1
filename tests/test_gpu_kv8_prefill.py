"""Prompts behind an 8-bit cache: chunks through the decoder layers alone, and prompts that are broken off."""
from __future__ import annotations

import pytest
import torch

from gpu_util import gpu_session
from helpers import make_weights
from test_gpu_cache_session import BASE, TREE, prompts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache_format", ["int8", "e4m3"])
@pytest.mark.parametrize("H,Dh,B,n,chunks", [(2, 128, 2, 16, 5), (4, 64, 3, 40, 3), (2, 128, 1, 128, 3), (4, 64, 17, 7, 4)])
def test_chunks_without_outputs(cache_format, H, Dh, B, n, chunks):
    """Chunks through the decoder layers alone leave the caches, and the last chunk's outputs, that whole forward passes leave."""
    cfg = BASE.with_(d=H * Dh, H=H, Dh=Dh, F=512)
    W = make_weights(cfg)
    front = 21
    a, b = (gpu_session(cfg, TREE, B, front + n * chunks, W, prefill_chunk=n, want_logits=True, cache_format=cache_format) for _ in range(2))
    text = prompts(cfg, B, n * chunks, 9).to(a.dev)
    for s in (a, b):
        s.prefill(prompts(cfg, B, front))
    c, o = (a.ctx(f"chain{n}"), b.ctx(f"chain{n}")), (a.out(f"chain{n}"), b.out(f"chain{n}"))
    for i in range(chunks):
        for k, s in enumerate((a, b)):
            o[k].tree_tokens.copy_(text[:, n * i:n * (i + 1)])
            o[k].n_acc.fill_(n), o[k].last_node.fill_(n - 1), o[k].next_root.zero_()
            o[k].path.copy_(torch.arange(n, dtype=torch.int32, device=s.dev).expand(B, n))
            s.kv.seq_len_hint = front + n * i if i % 2 else 0
        c[0].tree_verify_forward_kv8(B, a.ws, o[0].tree_tokens, a.seq_len, a.kv8, o[0].hidden, o[0].argmax, o[0].margin, o[0].logits)
        if i < chunks - 1:
            for t in (o[1].hidden, o[1].argmax, o[1].margin, o[1].logits):
                t.fill_(7)
            c[1].hydra_prefill_chunk_kv8(B, b.ws, o[1].tree_tokens, b.seq_len, b.kv8)
            assert all(bool((t == 7).all()) for t in (o[1].hidden, o[1].argmax, o[1].margin, o[1].logits))
        else:
            c[1].tree_verify_forward_kv8(B, b.ws, o[1].tree_tokens, b.seq_len, b.kv8, o[1].hidden, o[1].argmax, o[1].margin, o[1].logits)
        for k, s in enumerate((a, b)):
            c[k].kv_compact(B, o[k].n_acc, o[k].path, o[k].next_root, o[k].last_node, o[k].hidden, s.kv, s.seq_len, s.h_last, s.root, o[k].kv_index)
            c[k].hydra_kv8_seal(B, s.seq_len, s.kv8)
        for x, y in ((a.k_pages, b.k_pages), (a.v_pages, b.v_pages), (a.k_codes, b.k_codes), (a.v_codes, b.v_codes), (a.kv8.scales, b.kv8.scales),
                     (a.kv8.n_sealed, b.kv8.n_sealed), (a.seq_len, b.seq_len), (o[0].kv_index, o[1].kv_index)):
            assert torch.equal(x, y)
    for x, y in ((o[0].hidden, o[1].hidden), (o[0].argmax, o[1].argmax), (o[0].margin, o[1].margin), (o[0].logits, o[1].logits), (a.h_last, b.h_last)):
        assert torch.equal(x, y)
    assert a.seq_len.tolist() == [front + n * chunks] * B and a.main.read_flags() == 0 and b.main.read_flags() == 0
