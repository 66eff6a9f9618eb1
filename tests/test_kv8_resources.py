"""Compiler resource report of the 8-bit cache's and the pages' kernels (no GPU needed): nothing of them may use scratch memory."""
from __future__ import annotations

import pytest

from test_kernel_resources import _resource_report


@pytest.mark.parametrize("source, families", [
    # (query tiles, waves, request policy) by dims and format; short: shares of the head's dims
    ("kv8_attn.hip", {"kv8_attn_kernel": 26, "kv8_short_kernel": 10, "kv8_merge_kernel": 1}),
    ("kv8_cache.hip", {"kv8_seal_kernel": 4, "kv8_sealed_kernel": 1, "kv8_read_kernel": 4}),
    ("pages.hip", {"pages_reserve_kernel": 1, "pages_release_kernel": 1, "pages_fork_small_kernel": 1, "pages_fork_plan_kernel": 1, "pages_fork_kernel": 1, "pages_compact_plan_kernel": 1,
                   "pages_remap_kernel": 1, "copy_pages_kernel": 1}),
])
def test_kernels_keep_everything_in_registers(source, families):
    rep = _resource_report(source)
    assert len(rep) == sum(families.values())
    for family, n in families.items():
        found = {k: v for k, v in rep.items() if family in k}
        assert len(found) == n, f"{family}: {sorted(found)}"
        bad = {k: v for k, v in found.items() if v["scratch"] != 0 or v["spill"] != 0}
        assert not bad, f"instantiations using scratch memory: {bad}"
