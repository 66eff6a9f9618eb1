"""Refusals of the 8-bit cache's and the page pool's calls, on the host, before anything is launched."""
import ctypes as C

import pytest

from paper_2402_05109_amd import binding as hb

SHAPE = dict(d=256, n_layers=2, n_heads=2, head_dim=128, ffn=256, vocab=32, max_batch=4, parent=[-1, 0, 0, 1])
MEM = C.create_string_buffer(4096)
P = (C.addressof(MEM) + 255) // 256 * 256                  # an aligned address that no call may come to use


def kv_desc(**kw):
    d = dict(k_pages=P, v_pages=P, page_table=P, n_pages=4, max_pages=8, seq_len_hint=0)
    d.update(kw)
    return hb.KVDesc(**d)


def kv8_desc(tail=None, **kw):
    d = dict(tail=tail or kv_desc(), k_codes=P, v_codes=P, scales=P, page_table=P, n_sealed=P, n_pages=4, max_pages=8, format=hb.KV8_INT8)
    d.update(kw)
    return hb.KV8Desc(**d)


def pages_desc(**kw):
    d = dict(page_table=P, ref=P, n_pages=4, max_pages=8)
    d.update(kw)
    return hb.PagesDesc(**d)


def calls(h, kv8, pages, kv, B=2, ws=P):
    """Every entry point once, with these descriptors."""
    lib = hb.lib()
    k8, pg, k = C.byref(kv8) if kv8 else None, C.byref(pages) if pages else None, C.byref(kv) if kv else None
    return {
        "tree_verify_forward_kv8": lambda: lib.tree_verify_forward_kv8(h, None, B, ws, P, P, k8, P, P, None, None),
        "hydra_prefill_chunk_kv8": lambda: lib.hydra_prefill_chunk_kv8(h, None, B, ws, P, P, k8),
        "tree_attention_kv8": lambda: lib.tree_attention_kv8(h, None, B, 0, ws, P, P, k8, P),
        "hydra_kv8_seal": lambda: lib.hydra_kv8_seal(h, None, B, P, k8),
        "hydra_kv8_read": lambda: lib.hydra_kv8_read(h, None, B, 0, k8, 0, 4, P),
        "hydra_pages_reserve": lambda: lib.hydra_pages_reserve(h, None, B, ws, pg, None, P, 1, None),
        "hydra_pages_release": lambda: lib.hydra_pages_release(h, None, B, pg, None, P),
        "hydra_pages_fork": lambda: lib.hydra_pages_fork(h, None, B, ws, pg, P, P, P, P, P),
        "hydra_pages_compact": lambda: lib.hydra_pages_compact(h, None, B, ws, pg, P, P, P),
        "hydra_kv_copy_pages": lambda: lib.hydra_kv_copy_pages(h, None, k, 2, P, P, None),
        "hydra_kv8_copy_pages": lambda: lib.hydra_kv8_copy_pages(h, None, k8, 2, P, P, None),
    }


NAMES = sorted(calls(None, None, None, None))


@pytest.mark.parametrize("name", NAMES)
def test_no_context_or_no_weights(name):
    assert calls(None, kv8_desc(), pages_desc(), kv_desc())[name]() == hb.E_INVALID_ARG
    h = hb.Hydra(**SHAPE, dtype=hb.HYDRA_BF16)
    assert calls(h._h, kv8_desc(), pages_desc(), kv_desc())[name]() == hb.E_STATE and hb.last_error()


@pytest.mark.parametrize("name", [n for n in NAMES if "copy" not in n])
@pytest.mark.parametrize("B", [0, -1, 5])
def test_batch_out_of_range(name, B):
    h = hb.Hydra(**SHAPE, dtype=hb.HYDRA_BF16)
    assert calls(h._h, kv8_desc(), pages_desc(), kv_desc(), B=B)[name]() == hb.E_CAPACITY


def test_pages_workspace():
    n = hb.pages_workspace_bytes
    assert n(0, 4, 4) == n(4, 0, 4) == n(4, 4, 0) == 0
    assert n(64, 65536, 2048) >= 4 * 64 * 2048 and n(1, 10 ** 6, 1) >= 4 * 10 ** 6 and n(3, 5, 7) % 256 == 0


def test_descriptors_have_the_headers_layout():
    assert C.sizeof(hb.KV8Desc) == 40 + 5 * 8 + 3 * 4 + 4 and hb.KV8Desc.k_codes.offset == 40 and hb.KV8Desc.format.offset == 88
    assert C.sizeof(hb.PagesDesc) == 24
