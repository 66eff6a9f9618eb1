"""Hints and tables at the ends of the integers: refused on the host, as smaller ones that do not fit are."""
import ctypes as C

import pytest

from cache_util import context
from paper_2402_05109_amd import binding as hb
from test_cache_abi import P, calls, kv8_desc, kv_desc

pytestmark = pytest.mark.gpu
KV8 = ["tree_verify_forward_kv8", "hydra_prefill_chunk_kv8", "tree_attention_kv8", "hydra_kv8_seal", "hydra_kv8_read"]


@pytest.fixture(scope="module")
def ctx():
    return context(2, 128, 4, 4, 2)


@pytest.mark.parametrize("hint", [2 ** 31 - 1, 2 ** 31 - 3])
def test_hints_that_end_behind_the_integers(ctx, hint):
    """seq_len_hint + T is 2^31 and more."""
    lib, h, kv = hb.lib(), ctx._h, C.byref(kv_desc(seq_len_hint=hint))
    for name in KV8:
        assert calls(h, kv8_desc(tail=kv_desc(seq_len_hint=hint)), None, None)[name]() == hb.E_CAPACITY and hb.last_error()
    assert lib.tree_verify_forward(h, None, 2, P, P, P, kv, P, P, None, None) == hb.E_CAPACITY
    assert lib.hydra_prefill_chunk(h, None, 2, P, P, P, kv) == hb.E_CAPACITY
    assert lib.tree_attention(h, None, 2, 0, P, P, P, kv, P) == hb.E_CAPACITY


@pytest.mark.parametrize("name", KV8)
def test_tables_whose_last_tile_ends_behind_the_integers(ctx, name):
    """A text of more than 2^31 - 32 slots has its last tile of 32 keys end at 2^31 or more, which came out negative."""
    pages = 2 ** 27 - 1
    assert calls(ctx._h, kv8_desc(max_pages=pages), None, None)[name]() == hb.E_CAPACITY and hb.last_error()
    assert calls(ctx._h, kv8_desc(tail=kv_desc(max_pages=pages)), None, None)[name]() == hb.E_CAPACITY
