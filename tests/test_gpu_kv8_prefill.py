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


class Stop(Exception):
    pass


def state(sess):
    o = sess.out()
    return [t.clone() for t in (o.tree_tokens, o.hidden, o.argmax, sess.seq_len, sess.h_last, sess.root, sess.kv8.n_sealed)]


@pytest.mark.parametrize("cache_format", ["int8", "e4m3"])
@pytest.mark.parametrize("pool", [None, 60])
@pytest.mark.parametrize("front", [0, 16, 37, 63])
@pytest.mark.parametrize("at,where", [(0, "_reserve"), (1, "_keep_accepted"), (5, "_reserve"), (6, "_keep_accepted")])
def test_a_prompt_that_is_broken_off(monkeypatch, cache_format, pool, front, at, where):
    """Where chunks without outputs have been computed, the text is again the one in front of the prompt, to the bit, and so is every step behind it.
    The 16-bit pages have been taken again by then."""
    cfg = BASE
    W = make_weights(cfg)
    sess, other = (gpu_session(cfg, TREE, 2, 260, W, prefill_chunk=16, cache_format=cache_format, pool_pages=pool) for _ in range(2))
    for s in (sess, other):
        if front:
            s.prefill(prompts(cfg, 2, front))
            if pool:
                s.fork([1, 0])
    calls, real = [0], getattr(sess, where)

    def broken(*args):
        calls[0] += 1
        if calls[0] > at:
            raise Stop
        return real(*args)

    monkeypatch.setattr(sess, where, broken)
    with pytest.raises(Stop):
        sess.prefill(prompts(cfg, 2, 16 * 8, 5))             # eight chunks of one length: seven without outputs
    monkeypatch.undo()
    assert sess.host_len >= front and sess.seq_len.tolist() == [front] * 2
    assert torch.equal(sess.kv8.n_sealed, sess.seq_len // 16)
    for s in (sess, other):
        s.prefill(prompts(cfg, 2, 40, 11))
        for _ in range(4):
            s.step()
    torch.cuda.synchronize()
    for x, y in zip(state(sess), state(other)):
        assert torch.equal(x, y)
    L = int(sess.seq_len.max())
    plain = [torch.zeros(cfg.NL, 2, L, 2, cfg.H, cfg.Dh, device=s.dev) for s in (sess, other)]
    for s, t in zip((sess, other), plain):
        s.main.kv8_read(2, -1, s.kv8, 0, L, t)
    assert torch.equal(*plain) and sess.main.read_flags() == 0 and other.main.read_flags() == 0


def test_a_prompt_for_which_the_pool_has_no_room(monkeypatch):
    """As above, with one row's prompt and the other row's text in the way: that row stays as it is too."""
    cfg = BASE
    W = make_weights(cfg)
    sess, other = (gpu_session(cfg, TREE, 2, 400, W, prefill_chunk=16, cache_format="int8", pool_pages=14) for _ in range(2))
    for s in (sess, other):
        s.prefill(prompts(cfg, 2, 37))
    with pytest.raises(RuntimeError, match="exhausted"):
        sess.prefill(prompts(cfg, 1, 250, 7))
    assert sess.main.read_flags() == 1 and sess.seq_len.tolist() == [37, 37]
    for s in (sess, other):
        for _ in range(4):
            s.step()
    torch.cuda.synchronize()
    for x, y in zip(state(sess), state(other)):
        assert torch.equal(x, y)
    assert sess.main.read_flags() == 0


@pytest.mark.parametrize("cache_format", ["int8", "e4m3"])
def test_chunks_whose_outputs_nobody_reads_take_the_decoder_layers_alone(monkeypatch, cache_format):
    from paper_2402_05109_amd import binding as hb
    cfg = BASE
    sess = gpu_session(cfg, TREE, 2, 260, make_weights(cfg), prefill_chunk=16, cache_format=cache_format)
    taken = []
    for name in ("hydra_prefill_chunk_kv8", "tree_verify_forward_kv8"):
        real = getattr(hb.Hydra, name)
        monkeypatch.setattr(hb.Hydra, name, lambda self, *a, _real=real, _name=name: (taken.append((_name, self.T)), _real(self, *a))[1])
    sess.prefill(prompts(cfg, 2, 16 * 5 + 7))
    assert taken == [("hydra_prefill_chunk_kv8", 16)] * 4 + [("tree_verify_forward_kv8", 16), ("tree_verify_forward_kv8", 7)]
    assert sess.seq_len.tolist() == [87, 87] and sess.main.read_flags() == 0


@pytest.mark.parametrize("chunks,at", [(8, 5), (8, 8), (1, 1)])
@pytest.mark.parametrize("pool", [None, 40])
def test_a_prompt_that_is_broken_off_before_its_pages_are_sealed(monkeypatch, chunks, at, pool):
    """Between the compaction of a chunk, which writes h_last and root where the chunk was computed whole, and the sealing of its pages: back to the text in
    front where chunks without outputs were computed, behind the chunk where it was the only one."""
    from paper_2402_05109_amd import binding as hb
    cfg = BASE
    W = make_weights(cfg)
    sess, other = (gpu_session(cfg, TREE, 2, 260, W, prefill_chunk=16, cache_format="int8", pool_pages=pool) for _ in range(2))
    for s in (sess, other):
        s.prefill(prompts(cfg, 2, 37))
    calls, real = [0], hb.Hydra.hydra_kv8_seal

    def broken(self, *args):
        calls[0] += 1
        if calls[0] == at:
            raise Stop
        return real(self, *args)

    text = prompts(cfg, 2, 16 * chunks, 5)
    monkeypatch.setattr(hb.Hydra, "hydra_kv8_seal", broken)
    with pytest.raises(Stop):
        sess.prefill(text)
    monkeypatch.undo()
    if chunks == 1:
        other.prefill(text)
    assert sess.seq_len.tolist() == other.seq_len.tolist() and sess.host_len == int(sess.seq_len.max())
    for s in (sess, other):
        for _ in range(4):
            s.step()
    torch.cuda.synchronize()
    for x, y in zip(state(sess), state(other)):
        assert torch.equal(x, y)
    assert sess.main.read_flags() == 0
