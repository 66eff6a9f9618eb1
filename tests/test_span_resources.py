"""Compiler resource report of the kernels on part of a cache and of the log probabilities (no GPU needed): nothing of them may use scratch memory."""
from __future__ import annotations

import pytest

from test_kernel_resources import _resource_report


@pytest.mark.parametrize("source", ["span_attn.hip", "span_f32.hip", "span_evict.hip", "logprobs.hip"])
def test_kernels_keep_everything_in_registers(source):
    rep = _resource_report(source)
    assert len(rep) >= 4
    bad = {k: v for k, v in rep.items() if v["scratch"] != 0 or v["spill"] != 0}
    assert not bad, f"instantiations using scratch memory: {bad}"
