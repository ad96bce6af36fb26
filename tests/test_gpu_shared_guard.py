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


# (lengths past the shared ones, new tokens, group sizes, shared lengths) that make as many items, pieces and rows as
# the first, which is the plan in the workspace
def other_batches():
    n = 32
    base = dict(beyond=[5] * n, new=[1] * n, sizes=[n], shared=[512])
    a, b = [5] * n, [5] * n
    a[3], b[4] = 14, 14
    new_a, new_b = [1] * n, [1] * n
    new_a[3], new_b[4] = 0, 0
    two = dict(beyond=[5] * n, new=[1] * n, shared=[512, 512])
    return {
        "a_token_longer": (base, dict(base, beyond=[6] * n)),
        "lengths_exchanged": (dict(base, beyond=a), dict(base, beyond=b)),
        "new_tokens_exchanged": (dict(base, new=new_a), dict(base, new=new_b)),
        "another_group_border": (dict(two, sizes=[10, 22]), dict(two, sizes=[11, 21])),
        # 8 own tokens to the page that is shared no longer, and 8 back
        "shared_lengths_exchanged": (dict(two, sizes=[16, 16], beyond=[24] * 16 + [40] * 16, shared=[512, 496]),
                                     dict(two, sizes=[16, 16], beyond=[40] * 16 + [24] * 16, shared=[496, 512])),
    }


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
@pytest.mark.parametrize("case", sorted(other_batches()))
def test_another_batch_of_the_same_size_is_another_plan(case, fp8):
    """A decoding loop that leaves out a plan: the last step's work list would miss each row's newest key."""
    import paper_2505_23970_amd as gc
    import torch
    ws = torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")
    seen = []
    for k, x in enumerate(other_batches()[case]):
        w = SH.build(x["sizes"], x["shared"], x["beyond"], x["new"], 8, 1, 128, seed=3700, name=f"shared_{case}_{k}")
        run = H.DeviceRunFp8(w, 0.02, 0.015) if fp8 else H.DeviceRun(w)
        run.append()
        groups = gc.SharedPrefixes(run.batch, x["sizes"], x["shared"], gc.SHARE_ALWAYS)
        need = gc.shared_workspace_size(8, run.k_pool, run.v_pool, groups)
        assert need <= ws.numel()
        gc.plan_shared(8, run.k_pool, run.v_pool, groups, ws)
        assert gc.plan_status(ws) == 0
        seen.append((mark_of(ws), need, run, groups, w))
    (mark_a, need_a, run_a, groups_a, w_a), (mark_b, need_b, run_b, groups_b, w_b) = seen
    assert need_a == need_b
    assert mark_a != mark_b
    untouched(run_a, groups_a, w_a, ws)     # (the second batch's plan is there)
    gc.plan_shared(8, run_a.k_pool, run_a.v_pool, groups_a, ws)
    assert mark_of(ws) == mark_a
    untouched(run_b, groups_b, w_b, ws)


def test_plans_of_the_two_pool_kinds_differ():
    import paper_2505_23970_amd as gc
    import torch
    for name in ("prompts", "decode"):
        sizes, shared, beyond, new = SH.batches()[name]
        w = SH.build(sizes, shared, beyond, new, 16, 2, 128, seed=3300, name=f"shared_pool_kinds_{name}")
        ws = torch.zeros(1 << 26, dtype=torch.uint8, device="cuda")
        runs = [H.DeviceRun(w), H.DeviceRunFp8(w, 0.02, 0.015)]
        groups = gc.SharedPrefixes(runs[0].batch, sizes, shared, gc.SHARE_ALWAYS)
        for planned, other in (runs, runs[::-1]):
            gc.plan_shared(16, planned.k_pool, planned.v_pool, groups, ws)
            mark = mark_of(ws)
            gc.plan_shared(16, other.k_pool, other.v_pool, groups, ws)
            assert mark_of(ws) != mark
            untouched(planned, groups, w, ws)
