"""Refusals of the calls on part of a cache and of the log probabilities, on the host, before anything is launched."""
import ctypes as C
import math

import pytest
import torch

from paper_2402_05109_amd import binding as hb

SHAPE = dict(d=256, n_layers=2, n_heads=2, head_dim=128, ffn=256, vocab=32, max_batch=4, parent=[-1, 0, 0, 1])
MEM = C.create_string_buffer(4096)
P = (C.addressof(MEM) + 255) // 256 * 256                  # an aligned address that no call may come to use


def kv_desc(**kw):
    return hb.KVDesc(**(dict(k_pages=P, v_pages=P, page_table=P, n_pages=4, max_pages=8, seq_len_hint=0) | kw))


def span_desc(kv=None, **kw):
    return hb.KVSpanDesc(**(dict(kv=kv or kv_desc(), first=P, n_sinks=4, window=16, span_hint=0, n_scored=1, score=P, score_rows=4) | kw))


def calls(h, span, B=2, ws=P, pages=None, **kw):
    """Every entry point once; kw: other arguments."""
    lib = hb.lib()
    s = C.byref(span) if span else None
    pg = C.byref(pages or hb.PagesDesc(page_table=P, ref=P, n_pages=4, max_pages=8))
    a = dict(q=P, out=P, layer=0, keep=32, recent=8, slack=0, dst=None, kept=P, evicted=P, n=P, tau=1.0, k=2, tokens=P, logprob=P, rank=P, entropy=P, ids=P, lps=P, logits=P, path=P) | kw
    return {
        "tree_verify_forward_span": lambda: lib.tree_verify_forward_span(h, None, B, ws, P, a["n"], s, P, P, None, None),
        "hydra_prefill_chunk_span": lambda: lib.hydra_prefill_chunk_span(h, None, B, ws, P, a["n"], s),
        "tree_attention_span": lambda: lib.tree_attention_span(h, None, B, a["layer"], ws, a["q"], a["n"], s, a["out"]),
        "hydra_score_compact": lambda: lib.hydra_score_compact(h, None, B, P, a["path"], a["n"], s),
        "hydra_kv_evict": lambda: lib.hydra_kv_evict(h, None, B, a["n"], s, a["keep"], a["recent"], a["slack"], a["dst"], None, a["kept"], a["evicted"]),
        "hydra_pages_release_span": lambda: lib.hydra_pages_release_span(h, None, B, pg, a["n"], s, None),
        "hydra_token_logprobs": lambda: lib.hydra_token_logprobs(h, None, B, ws, a["logits"], a["tokens"], a["tau"], a["k"], a["logprob"], a["rank"], a["entropy"], a["ids"], a["lps"]),
    }


NAMES = sorted(calls(None, None))
SPANS = [n for n in NAMES if n != "hydra_token_logprobs"]


@pytest.fixture(params=[hb.HYDRA_BF16, hb.HYDRA_F32])
def bare(request):
    return hb.Hydra(**SHAPE, dtype=request.param)


@pytest.mark.parametrize("name", NAMES)
def test_no_context_or_no_weights(name, bare):
    assert calls(None, span_desc())[name]() == hb.E_INVALID_ARG
    assert calls(bare._h, span_desc())[name]() == hb.E_STATE and hb.last_error()


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("B", [0, -1, 5])
def test_batch_out_of_range(name, B, bare):
    assert calls(bare._h, span_desc(), B=B)[name]() == hb.E_CAPACITY


def test_descriptors_have_the_headers_layout():
    assert C.sizeof(hb.KVSpanDesc) == 40 + 8 + 16 + 8 + 8 and hb.KVSpanDesc.first.offset == 40 and hb.KVSpanDesc.n_sinks.offset == 48
    assert hb.KVSpanDesc.score.offset == 64 and hb.KVSpanDesc.score_rows.offset == 72


def test_span_checks_its_tensors():
    with pytest.raises(TypeError):
        hb.KVSpan(None, first=torch.zeros(2, dtype=torch.int32))              # not on a device


def test_workspace_has_room_for_records_and_statistics():
    h = hb.Hydra(**dict(SHAPE, vocab=100003, max_batch=16, parent=[-1] + list(range(127))), dtype=hb.HYDRA_BF16)
    assert h.workspace_bytes(16) >= 16 * 128 * 100003 * 4 + 16 * 2 * 128 * 8


@pytest.mark.parametrize("dtype", [hb.HYDRA_BF16, hb.HYDRA_F32])
@pytest.mark.parametrize("heads, T, vocab", [(2, 1, 64), (2, 59, 262147), (4, 16, 100003), (8, 128, 32000)])
def test_a_workspace_serves_fewer_rows(heads, T, vocab, dtype):
    """Plans differ by the number of rows; a session prefills some of its rows in the workspace of all."""
    h = hb.Hydra(d=64 * heads, n_layers=1, n_heads=heads, head_dim=64, ffn=128, vocab=vocab, max_pos=256, dtype=dtype, max_batch=200, parent=[-1] + list(range(T - 1)))
    sizes = [h.workspace_bytes(B) for B in range(1, 201)]
    assert sizes == sorted(sizes)


# ---- what is checked behind the weights: on a device, with a bare context, still before anything is launched
BAD_SPANS = [
    (dict(n_sinks=-1), hb.E_INVALID_ARG), (dict(window=-1), hb.E_INVALID_ARG), (dict(span_hint=-1), hb.E_INVALID_ARG), (dict(n_scored=-1), hb.E_INVALID_ARG),
    (dict(n_scored=5), hb.E_INVALID_ARG), (dict(score_rows=1), hb.E_CAPACITY), (dict(kv=kv_desc(k_pages=None)), hb.E_INVALID_ARG),
    (dict(kv=kv_desc(v_pages=P + 8)), hb.E_INVALID_ARG), (dict(kv=kv_desc(n_pages=0)), hb.E_INVALID_ARG), (dict(kv=kv_desc(max_pages=0)), hb.E_INVALID_ARG),
    (dict(kv=kv_desc(max_pages=2 ** 27)), hb.E_CAPACITY), (dict(kv=kv_desc(seq_len_hint=-1)), hb.E_INVALID_ARG), (dict(kv=kv_desc(seq_len_hint=125)), hb.E_CAPACITY),
]


@pytest.fixture(params=[hb.HYDRA_BF16, hb.HYDRA_F32])
def ready(request):
    h = hb.Hydra(**SHAPE, dtype=request.param)
    h.bind_weights(torch.zeros(h.weights_bytes(), dtype=torch.uint8, device="cuda:0"))
    return h


@pytest.mark.gpu
@pytest.mark.parametrize("name", [n for n in SPANS if n != "hydra_pages_release_span"])
@pytest.mark.parametrize("change, code", BAD_SPANS)
def test_bad_spans(name, change, code, ready):
    assert calls(ready._h, None)[name]() == hb.E_INVALID_ARG
    if name in ("hydra_kv_evict", "hydra_score_compact") and ("n_scored" in change or code == hb.E_CAPACITY and "kv" in change and change["kv"].seq_len_hint > 0):
        return                                              # of attention alone: these calls count no nodes, and put none behind the text
    assert calls(ready._h, span_desc(**change))[name]() == code and hb.last_error()


@pytest.mark.gpu
@pytest.mark.parametrize("name, change, code", [
    ("tree_verify_forward_span", dict(n=None), hb.E_INVALID_ARG), ("hydra_prefill_chunk_span", dict(n=None), hb.E_INVALID_ARG),
    ("tree_attention_span", dict(q=P + 8), hb.E_INVALID_ARG), ("tree_attention_span", dict(out=P + 2), hb.E_INVALID_ARG), ("tree_attention_span", dict(q=None), hb.E_INVALID_ARG),
    ("tree_attention_span", dict(out=None), hb.E_INVALID_ARG), ("tree_attention_span", dict(n=None), hb.E_INVALID_ARG), ("tree_attention_span", dict(layer=-1), hb.E_INVALID_ARG),
    ("tree_attention_span", dict(layer=2), hb.E_INVALID_ARG), ("tree_attention_span", dict(ws=None), hb.E_INVALID_ARG), ("tree_attention_span", dict(ws=P + 64), hb.E_INVALID_ARG),
    ("hydra_score_compact", dict(n=None), hb.E_INVALID_ARG), ("hydra_score_compact", dict(path=None), hb.E_INVALID_ARG), ("hydra_score_compact", dict(span=dict(score=None)), hb.E_INVALID_ARG),
    ("hydra_kv_evict", dict(keep=0), hb.E_INVALID_ARG), ("hydra_kv_evict", dict(recent=-1), hb.E_INVALID_ARG), ("hydra_kv_evict", dict(slack=-1), hb.E_INVALID_ARG),
    ("hydra_kv_evict", dict(keep=11), hb.E_SHAPE), ("hydra_kv_evict", dict(recent=2 ** 31 - 1), hb.E_SHAPE), ("hydra_kv_evict", dict(dst=P), hb.E_INVALID_ARG),
    ("hydra_kv_evict", dict(kept=None), hb.E_INVALID_ARG), ("hydra_kv_evict", dict(evicted=None), hb.E_INVALID_ARG), ("hydra_kv_evict", dict(n=None), hb.E_INVALID_ARG),
    ("hydra_kv_evict", dict(span=dict(first=None)), hb.E_INVALID_ARG), ("hydra_kv_evict", dict(span=dict(score=None)), hb.E_INVALID_ARG),
    ("hydra_pages_release_span", dict(n=None), hb.E_INVALID_ARG), ("hydra_pages_release_span", dict(span=dict(window=-1)), hb.E_INVALID_ARG),
    ("hydra_pages_release_span", dict(span=dict(n_sinks=-1)), hb.E_INVALID_ARG), ("hydra_pages_release_span", dict(pages=hb.PagesDesc(page_table=P, ref=None, n_pages=4, max_pages=8)), hb.E_INVALID_ARG),
    ("hydra_token_logprobs", dict(tau=0.0), hb.E_INVALID_ARG), ("hydra_token_logprobs", dict(tau=-1.0), hb.E_INVALID_ARG), ("hydra_token_logprobs", dict(tau=math.inf), hb.E_INVALID_ARG),
    ("hydra_token_logprobs", dict(tau=math.nan), hb.E_INVALID_ARG), ("hydra_token_logprobs", dict(tau=1e-44), hb.E_INVALID_ARG), ("hydra_token_logprobs", dict(k=-1), hb.E_UNSUPPORTED),
    ("hydra_token_logprobs", dict(k=33), hb.E_UNSUPPORTED), ("hydra_token_logprobs", dict(logits=None), hb.E_INVALID_ARG), ("hydra_token_logprobs", dict(tokens=None), hb.E_INVALID_ARG),
    ("hydra_token_logprobs", dict(ids=None), hb.E_INVALID_ARG), ("hydra_token_logprobs", dict(lps=None), hb.E_INVALID_ARG),
    ("hydra_token_logprobs", dict(k=0, logprob=None, rank=None, entropy=None), hb.E_INVALID_ARG), ("hydra_token_logprobs", dict(ws=None), hb.E_INVALID_ARG),
])
def test_bad_arguments(name, change, code, ready):
    change = dict(change)
    span = span_desc(**change.pop("span", {}))
    assert calls(ready._h, span, **change)[name]() == code and hb.last_error()


@pytest.mark.gpu
def test_more_alternatives_than_tokens():
    h = hb.Hydra(**dict(SHAPE, vocab=5), dtype=hb.HYDRA_F32)
    h.bind_weights(torch.zeros(h.weights_bytes(), dtype=torch.uint8, device="cuda:0"))
    assert calls(h._h, span_desc(), k=6)["hydra_token_logprobs"]() == hb.E_UNSUPPORTED


@pytest.mark.gpu
def test_tensors_of_the_wrong_kind():
    c = hb.Hydra(**SHAPE, dtype=hb.HYDRA_BF16)
    c.bind_weights(torch.zeros(c.weights_bytes(), dtype=torch.uint8, device="cuda:0"))
    kv = hb.KV(torch.zeros(2 * 4 * 2 * 16 * 128, dtype=torch.float16, device="cuda:0"), torch.zeros(2 * 4 * 2 * 16 * 128, dtype=torch.float16, device="cuda:0"),
               torch.zeros(1, 4, dtype=torch.int32, device="cuda:0"), 4)
    ws = torch.zeros(c.workspace_bytes(1), dtype=torch.uint8, device="cuda:0")
    n, q = torch.zeros(1, dtype=torch.int32, device="cuda:0"), torch.zeros(1, 4, 2, 128, dtype=torch.float16, device="cuda:0")
    for a, b in ((q.float(), q), (q, q.float()), (q.transpose(1, 2), q), (q.cpu(), q)):
        with pytest.raises(TypeError):
            c.tree_attention_span(1, 0, ws, a, n, hb.KVSpan(kv), b)
    with pytest.raises(ValueError):
        hb.KVSpan(kv, score=torch.zeros(2, 1, 2, 32, device="cuda:0"))
    with pytest.raises(TypeError):
        hb.KVSpan(kv, score=torch.zeros(2, 1, 2, 64, dtype=torch.float16, device="cuda:0"))
