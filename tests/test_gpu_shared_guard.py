"""Runs of the shared-prefix attention on a workspace that holds another plan (GPU): they write nothing. The plan's
mark, 8 bytes at offset 128 of the workspace, is looked at before any such run is made."""
import numpy as np
import pytest

import gpu_helpers as H
import shared_helpers as SH

pytestmark = pytest.mark.gpu

MARK = slice(128, 136)


@pytest.fixture(scope="module", autouse=True)
def gpu_ready():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2505_23970_amd as gc
    gc.load_library()


def mark_of(ws):
    import torch
    torch.cuda.synchronize()
    return int(ws[MARK].cpu().numpy().view(np.uint64)[0])


def untouched(run, groups, w, ws):
    """A run of `groups` on what ws holds leaves out and lse alone."""
    import paper_2505_23970_amd as gc
    import torch
    out = torch.full_like(run.q, 7.0)
    lse = torch.full(run.q.shape[:2], 7.0, device="cuda")
    if run.k_pool.dtype == torch.uint8:
        gc.run_shared_fp8(run.q, run.k_pool, run.v_pool, groups, w.scale, run.ks, run.vs, ws, out=out, lse=lse)
    else:
        gc.run_shared(run.q, run.k_pool, run.v_pool, groups, w.scale, ws, out=out, lse=lse)
    torch.cuda.synchronize()
    assert bool((out == 7.0).all()) and bool((lse == 7.0).all())


def plain_call(call, run, w, ws):
    import paper_2505_23970_amd as gc
    Hq, fp8 = w.num_q_heads, hasattr(run, "ks")
    args = (run.q, run.k_pool, run.v_pool, run.batch, w.scale) + ((run.ks, run.vs) if fp8 else ())
    if call == "plan":
        gc.plan(Hq, run.k_pool, run.v_pool, run.batch, ws)
    elif call == "prepare":
        scales = dict(k_scale=run.ks, v_scale=run.vs) if fp8 else {}
        gc.prepare(run.k_new, run.v_new, run.k_pool, run.v_pool, run.batch, Hq, ws, **scales)
    elif call == "attention":
        (gc.prefix_prefill_attention_fp8 if fp8 else gc.prefix_prefill_attention)(*args, workspace=ws)
    else:   # the policy leaves the batch to the plain attention
        alone = gc.SharedPrefixes(run.batch, [1] * w.batch, [16] * w.batch)
        if call == "declined_plan":
            gc.plan_shared(Hq, run.k_pool, run.v_pool, alone, ws)
        else:
            (gc.shared_prefix_attention_fp8 if fp8 else gc.shared_prefix_attention)(
                run.q, run.k_pool, run.v_pool, alone, w.scale, *((run.ks, run.vs) if fp8 else ()), ws)


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
@pytest.mark.parametrize("call", ["plan", "prepare", "attention", "declined_plan", "declined_attention"])
def test_a_plain_plan_takes_a_shared_one_back(call, fp8):
    import paper_2505_23970_amd as gc
    import torch
    sizes, shared, beyond, new = SH.batches()["prompts"]
    w = SH.build(sizes, shared, beyond, new, 16, 2, 128, seed=3600, name="shared_taken_back")
    run = H.DeviceRunFp8(w, 0.02, 0.015) if fp8 else H.DeviceRun(w)
    run.append()
    groups = gc.SharedPrefixes(run.batch, sizes, shared, gc.SHARE_ALWAYS)
    ws = torch.zeros(1 << 26, dtype=torch.uint8, device="cuda")
    assert gc.shared_workspace_size(16, run.k_pool, run.v_pool, groups) <= ws.numel()
    gc.plan_shared(16, run.k_pool, run.v_pool, groups, ws)
    assert mark_of(ws) != 0
    plain_call(call, run, w, ws)
    assert mark_of(ws) == 0, "the run below would take the plain plan's items for its own"
    untouched(run, groups, w, ws)
    call = gc.shared_prefix_attention_fp8 if fp8 else gc.shared_prefix_attention
    args = (run.q, run.k_pool, run.v_pool, groups, w.scale) + ((run.ks, run.vs) if fp8 else ())
    again = call(*args, ws)
    assert torch.equal(again.view(torch.int16), call(*args).view(torch.int16))
