"""Which kind of pools a plan is made for: 8-bit value pools that were left untransposed are refused by name, 4-bit pools are taken."""
import types

import numpy as np
import pytest

import paper_2505_23970_amd as gc

HQ, HKV, NB = 16, 2, 40


def batch(device):
    return gc.PagedBatch([300, 20], [1, 1], np.arange(2 * 20).reshape(2, 20), device=device)


def pools(k_row, v_shape, device="cpu", dtype="uint8"):
    import torch
    k = torch.zeros(NB, HKV, 16, k_row, dtype=getattr(torch, dtype), device=device)
    return k, torch.zeros(NB, HKV, *v_shape, dtype=getattr(torch, dtype), device=device)


@pytest.mark.parametrize("dtype,D", [("uint8", 128), ("bfloat16", 64), ("bfloat16", 128)])
def test_untransposed_value_pools_are_refused(dtype, D):
    b = batch("cpu")
    for call in (gc.workspace_size, gc.alloc_workspace):
        with pytest.raises(ValueError, match="v_pool must be"):
            call(HQ, *pools(D, (16, D), dtype=dtype), b)


@pytest.mark.parametrize("D", [64, 128])
def test_every_kind_takes_the_same_workspace(D):
    b = batch("cpu")
    sizes = {gc.workspace_size(HQ, *p, b) for p in (pools(D, (D, 16), dtype="bfloat16"), pools(D, (D, 16)), pools(D // 2, (16, D // 2)))}
    assert len(sizes) == 1
    # only shapes are looked at for the pools that had them alone before
    shaped = [types.SimpleNamespace(shape=s) for s in ((NB, HKV, 16, D), (NB, HKV, D, 16))]
    assert sizes == {gc.workspace_size(HQ, *shaped, b)}


@pytest.mark.gpu
def test_plans_and_calls_refuse_them_too():
    """At D = 64 such 8-bit pools look like 4-bit pools of D = 128 to a plan; whatever reads or writes them refuses them."""
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    b = batch("cuda")
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError, match="v_pool must be"):
        gc.plan(HQ, *pools(128, (16, 128), "cuda"), b, ws)
    for D in (64, 128):
        p = pools(D, (16, D), "cuda")
        q, k, v = (torch.zeros(2, h, D, dtype=torch.bfloat16, device="cuda") for h in (HQ, HKV, HKV))
        for call in (lambda: gc.kv_append_fp8(k, v, *p, b, 1.0, 1.0), lambda: gc.prepare(k, v, *p, b, HQ, ws, k_scale=1.0, v_scale=1.0),
                     lambda: gc.run_fp8(q, *p, b, 0.1, 1.0, 1.0, ws), lambda: gc.prefix_prefill_attention_fp8(q, *p, b, 0.1, 1.0, 1.0),
                     lambda: gc.kv_read_fp8(*p, b, 1.0, 1.0)):
            with pytest.raises(ValueError, match="v_pool must be"):
                call()
