"""Refusals that need a context with its weights bound: bad descriptors and arguments return an error and launch nothing."""
import ctypes as C

import pytest
import torch

from cache_util import context
from paper_2402_05109_amd import binding as hb
from test_cache_abi import P, calls, kv8_desc, kv_desc, pages_desc

pytestmark = pytest.mark.gpu
KV8 = ["tree_verify_forward_kv8", "hydra_prefill_chunk_kv8", "tree_attention_kv8", "hydra_kv8_seal", "hydra_kv8_read"]
POOL = ["hydra_pages_reserve", "hydra_pages_release", "hydra_pages_fork", "hydra_pages_compact"]


@pytest.fixture(scope="module")
def ctx():
    return context(2, 128, 4, 4, 2)


@pytest.mark.parametrize("name", KV8)
@pytest.mark.parametrize("bad,code", [
    (dict(tail=kv_desc(k_pages=0)), hb.E_INVALID_ARG), (dict(tail=kv_desc(n_pages=0)), hb.E_INVALID_ARG), (dict(tail=kv_desc(seq_len_hint=-1)), hb.E_INVALID_ARG),
    (dict(tail=kv_desc(seq_len_hint=125)), hb.E_CAPACITY), (dict(tail=kv_desc(v_pages=P + 8)), hb.E_INVALID_ARG),
    (dict(k_codes=0), hb.E_INVALID_ARG), (dict(v_codes=P + 8), hb.E_INVALID_ARG), (dict(scales=0), hb.E_INVALID_ARG), (dict(scales=P + 4), hb.E_INVALID_ARG),
    (dict(page_table=0), hb.E_INVALID_ARG), (dict(n_sealed=0), hb.E_INVALID_ARG), (dict(n_pages=0), hb.E_INVALID_ARG), (dict(max_pages=-1), hb.E_INVALID_ARG),
    (dict(format=2), hb.E_INVALID_ARG), (dict(format=-1), hb.E_INVALID_ARG),
])
def test_bad_8_bit_caches(ctx, name, bad, code):
    assert calls(ctx._h, kv8_desc(**bad), None, None)[name]() == code and hb.last_error()
    assert calls(ctx._h, None, None, None)[name]() == hb.E_INVALID_ARG


@pytest.mark.parametrize("name", KV8 + ["hydra_kv8_copy_pages"])
def test_fp32_contexts_have_no_8_bit_cache(name):
    c = context(2, 128, 4, 4, 2, dtype=hb.HYDRA_F32)
    assert calls(c._h, kv8_desc(), None, None)[name]() == hb.E_UNSUPPORTED


@pytest.mark.parametrize("name", POOL)
@pytest.mark.parametrize("bad", [dict(page_table=0), dict(ref=0), dict(n_pages=0), dict(max_pages=0)])
def test_bad_pools(ctx, name, bad):
    assert calls(ctx._h, None, pages_desc(**bad), None)[name]() == hb.E_INVALID_ARG
    assert calls(ctx._h, None, None, None)[name]() == hb.E_INVALID_ARG


@pytest.mark.parametrize("name", ["tree_verify_forward_kv8", "hydra_prefill_chunk_kv8", "tree_attention_kv8", "hydra_pages_reserve", "hydra_pages_fork", "hydra_pages_compact"])
@pytest.mark.parametrize("ws", [None, P + 64])
def test_bad_workspaces(ctx, name, ws):
    assert calls(ctx._h, kv8_desc(), pages_desc(), None, ws=ws)[name]() == hb.E_INVALID_ARG


def test_other_arguments(ctx):
    lib, h = hb.lib(), ctx._h
    k8, pg, kv = C.byref(kv8_desc()), C.byref(pages_desc()), C.byref(kv_desc())
    bad = hb.E_INVALID_ARG
    assert lib.tree_verify_forward_kv8(h, None, 1, P, None, P, k8, P, P, None, None) == bad
    assert lib.tree_verify_forward_kv8(h, None, 1, P, P, P, k8, P, None, None, None) == bad
    assert lib.hydra_prefill_chunk_kv8(h, None, 1, P, P, None, k8) == bad
    assert lib.tree_attention_kv8(h, None, 1, 2, P, P, P, k8, P) == bad and lib.tree_attention_kv8(h, None, 1, -1, P, P, P, k8, P) == bad
    assert lib.tree_attention_kv8(h, None, 1, 0, P, P + 8, P, k8, P) == bad and lib.tree_attention_kv8(h, None, 1, 0, P, P, P, k8, P + 2) == bad
    assert lib.tree_attention_kv8(h, None, 1, 0, P, None, P, k8, P) == bad
    assert lib.hydra_kv8_seal(h, None, 1, None, k8) == bad
    assert lib.hydra_kv8_read(h, None, 1, 2, k8, 0, 1, P) == bad and lib.hydra_kv8_read(h, None, 1, -2, k8, 0, 1, P) == bad
    assert lib.hydra_kv8_read(h, None, 1, 0, k8, 0, 1, P + 4) == bad and lib.hydra_kv8_read(h, None, 1, 0, k8, 0, 1, None) == bad
    assert lib.hydra_kv8_read(h, None, 1, 0, k8, 120, 9, P) == hb.E_CAPACITY and lib.hydra_kv8_read(h, None, 1, 0, k8, -1, 1, P) == hb.E_CAPACITY
    assert lib.hydra_kv8_read(h, None, 1, 0, k8, 2 ** 31 - 1, 2 ** 31 - 1, P) == hb.E_CAPACITY
    assert lib.hydra_kv8_read(h, None, 1, 0, k8, 5, 0, P) == hb.HYDRA_OK
    assert lib.hydra_pages_reserve(h, None, 1, P, pg, None, None, 1, None) == bad and lib.hydra_pages_reserve(h, None, 1, P, pg, None, P, -1, None) == bad
    assert lib.hydra_pages_release(h, None, 1, pg, None, None) == bad
    for i in range(5):
        a = [P] * 5
        a[i] = None
        assert lib.hydra_pages_fork(h, None, 1, P, pg, *a) == bad
    for i in range(3):
        a = [P] * 3
        a[i] = None
        assert lib.hydra_pages_compact(h, None, 1, P, pg, *a) == bad
    assert lib.hydra_kv_copy_pages(h, None, kv, -1, P, P, None) == bad and lib.hydra_kv_copy_pages(h, None, None, 1, P, P, None) == bad
    assert lib.hydra_kv_copy_pages(h, None, kv, 1, None, P, None) == bad and lib.hydra_kv_copy_pages(h, None, C.byref(kv_desc(v_pages=0)), 1, P, P, None) == bad
    assert lib.hydra_kv_copy_pages(h, None, C.byref(kv_desc(k_pages=P + 2)), 1, P, P, None) == bad
    assert lib.hydra_kv8_copy_pages(h, None, None, 1, P, P, None) == bad and lib.hydra_kv8_copy_pages(h, None, C.byref(kv8_desc(n_pages=0)), 1, P, P, None) == bad
    assert lib.hydra_kv_copy_pages(h, None, kv, 0, P, P, None) == hb.HYDRA_OK
    torch.cuda.synchronize()
    assert ctx.read_flags() == 0


@pytest.mark.parametrize("name", POOL)
@pytest.mark.parametrize("large", [dict(n_pages=2 ** 30 + 1), dict(max_pages=2 ** 27), dict(max_pages=2 ** 31 - 1)])
def test_pools_whose_numbers_would_not_fit(ctx, name, large):
    assert calls(ctx._h, None, pages_desc(**large), None)[name]() == hb.E_CAPACITY


def test_pools_with_too_many_entries_in_all_rows():
    c = context(1, 128, 16, 1, 1)
    assert calls(c._h, None, pages_desc(max_pages=2 ** 27 - 1), None, B=9)["hydra_pages_release"]() == hb.E_CAPACITY


@pytest.mark.parametrize("name", KV8)
@pytest.mark.parametrize("large", [dict(max_pages=2 ** 27), dict(tail=kv_desc(max_pages=2 ** 27))])
def test_tables_whose_slots_would_not_fit(ctx, name, large):
    assert calls(ctx._h, kv8_desc(**large), None, None)[name]() == hb.E_CAPACITY
