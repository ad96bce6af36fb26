"""Batches without new tokens over pools of no blocks (CPU): every call over 4-bit pools returns before it looks at a pointer, as the
calls over the other pools do, and the binding's calls return empty results."""
import ctypes

import pytest

import paper_2505_23970_amd as gc
from test_abi_host import HostBatch, geo
from test_fp4_host import STATUS_CALLS, call


@pytest.fixture(scope="module")
def lib():
    return gc.load_library()


@pytest.mark.parametrize("name", STATUS_CALLS)
@pytest.mark.parametrize("lengths", [([4], [0]), ([], [])])
def test_no_tokens_no_pointers(lib, name, lengths):
    none = dict(k=None, v=None, s=None, k_new=None, v_new=None, q=None, out=None, ws=None, ws_bytes=0)
    for blocks in (64, 0):
        assert call(lib, name, geo(NB=blocks), HostBatch(*lengths), **none) == 0
    # (an invalid geometry is refused all the same)
    assert call(lib, name, geo(D=96), HostBatch(*lengths), **none) == -3


def test_plan_and_run_in_one_call(lib):
    for lengths, scales in ((([4], [0]), None), (([4], [3]), 0x100000)):
        b = HostBatch(*lengths)
        st = lib.gc_prefix_prefill_attention_fp4(ctypes.byref(geo()), ctypes.byref(b.desc), None, None, None, None, scales, 0.1, None,
                                                 None, None, 0, None)
        assert st == (0 if scales is None else -1)


@pytest.mark.gpu
def test_pools_of_no_blocks():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    pools = gc.alloc_pools_fp4(0, 2, 64)
    batch = gc.PagedBatch([0, 0], [0, 0], [[0], [0]])
    rows = lambda heads: torch.empty(0, heads, 64, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    table = torch.zeros(4, 32, 2, device="cuda")
    gc.kv_append_fp4(rows(2), rows(2), *pools, batch)
    assert gc.kv_append_rotary_fp4(rows(4), rows(2), rows(2), *pools, batch, table).shape == (0, 4, 64)
    assert all(t.shape == (0, 2, 64) for t in gc.kv_read_fp4(*pools, batch))
    assert gc.prefix_prefill_attention_fp4(rows(4), *pools, batch, 0.125).shape == (0, 4, 64)
