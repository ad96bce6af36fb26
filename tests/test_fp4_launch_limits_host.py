"""Attention over 4-bit pools of more work than one launch holds (CPU): refused before anything is enqueued, by its items and by the merge
of its split rows, which has more workgroups than the items."""
import ctypes

import pytest

import paper_2505_23970_amd as gc
from test_abi_host import HostBatch, geo


@pytest.mark.parametrize("name", ["gc_prefix_prefill_run_fp4", "gc_prefix_prefill_attention_fp4"])
@pytest.mark.parametrize("tiling,D,requests,unsupported", [
    (1, 128, 8193, True),    # 128-row tiles: 16 merging workgroups each, 2^24 of them and more
    (1, 128, 8191, False),   # just below
    (1, 64, 16385, True),    # rows of half the length: 8 each
    (1, 64, 16383, False),
    (1, 64, 32769, True),    # more items than a launch of such workgroups holds
])
def test_merges_of_too_many_rows(name, tiling, D, requests, unsupported):
    lib = gc.load_library()
    g = geo(Hq=128, Hkv=128, D=D, NB=1 << 20)
    b = HostBatch([0] * requests, [128] * requests)
    o = gc.PlanOptions()
    o.kv_split_tiles, o.tiling = 1, tiling
    # (a workspace that is far too small ends the calls that pass the limits)
    st = getattr(lib, name)(ctypes.byref(g), ctypes.byref(b.desc), ctypes.byref(o), 0x500000, 1 << 40, 1 << 41, 1 << 42, 0.1, 0x600000,
                            None, 0x400000, 4096, None)
    assert st == (-3 if unsupported else -5)
