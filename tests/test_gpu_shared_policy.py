"""The default policy of the shared-prefix attention (GPU) against the float64 oracle, on batches that it takes, that it
takes some groups of, and that it leaves alone: up to and beyond 512 requests (the planner's LDS) and 512 groups (the
policy's choice of single ones), both pool kinds. Which of them a batch is, its workspace says before the call."""
import numpy as np
import pytest

import gpu_helpers as H
import shared_helpers as SH

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu_ready():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2505_23970_amd as gc
    gc.load_library()


# name -> (query heads, KV heads, head_dim, group sizes, shared tokens, cached tokens past them, new tokens, state)
def batches():
    rng = np.random.default_rng(11)
    past = lambda n, top=60: rng.integers(0, top, n).tolist()  # noqa: E731
    return {
        "taken": (64, 8, 128, [24], [2000], past(24), [1] * 24, "taken"),
        "taken_d64": (32, 8, 64, [40], [3200], past(40), [1] * 40, "taken"),
        # the second group gains; the first, of one request, and the third, of 16 tokens, do not; the last shares nothing
        "some_groups": (64, 8, 128, [1, 39, 3, 4], [1600, 1600, 16, 0], past(47), [1] * 47, "some"),
        "some_groups_last": (64, 8, 128, [3] * 60 + [40], [16] * 60 + [1600], past(220), [1] * 220, "some"),
        # few 128-row tiles: taken for the shorter chunks, beside a group that is too short
        "brief": (64, 8, 128, [2, 2], [512, 64], past(4), [3, 3, 3, 3], "some"),
        "some_512": (16, 2, 128, [1] * 256 + [256], [32] * 256 + [640], past(512, 30), [1] * 512, "some"),
        "some_513": (16, 2, 128, [1] * 257 + [256], [32] * 257 + [640], past(513, 30), rng.choice([0, 1, 1, 1], 513).tolist(), "some"),
        "many_groups_taken": (16, 2, 128, [200] + [1] * 520, [800] + [16] * 520, past(720, 30), [1] * 720, "taken"),
        "many_groups_left": (16, 2, 128, [1] * 520, [32] * 520, past(520, 30), [1] * 520, "left"),
        "left": (16, 2, 128, [2, 3], [64, 32], past(5), [1, 2, 1, 1, 5], "left"),
    }


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
@pytest.mark.parametrize("name", sorted(batches()))
def test_rows_of_the_default_policy(name, fp8):
    import paper_2505_23970_amd as gc
    import torch
    Hq, Hkv, D, sizes, shared, beyond, new, state = batches()[name]
    print(f"case {name} fp8={fp8}", flush=True)
    w = SH.build(sizes, shared, beyond, new, Hq, Hkv, D, seed=3800, name=f"shared_policy_{name}")
    run = H.DeviceRunFp8(w, 0.02, 0.015) if fp8 else H.DeviceRun(w)
    run.append()
    q, kp, vp = run.q, run.k_pool, run.v_pool
    groups = gc.SharedPrefixes(run.batch, sizes, shared)
    every = gc.SharedPrefixes(run.batch, sizes, shared, gc.SHARE_ALWAYS)
    need = gc.shared_workspace_size(Hq, kp, vp, groups)
    plain, all_of_them = gc.workspace_size(Hq, kp, vp, run.batch), gc.shared_workspace_size(Hq, kp, vp, every)
    assert plain != all_of_them
    assert ("left" if need == plain else "taken" if need == all_of_them else "some") == state, (need, plain, all_of_them)
    scales = (run.ks, run.vs) if fp8 else ()
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device="cuda")
    call = gc.shared_prefix_attention_fp8 if fp8 else gc.shared_prefix_attention
    call(q, kp, vp, groups, w.scale, *scales, ws, out=out, lse=lse)
    torch.cuda.synchronize()
    assert gc.plan_status(ws) == 0
    again = (gc.run_shared_fp8 if fp8 else gc.run_shared)(q, kp, vp, groups, w.scale, *scales, ws)
    assert torch.equal(again.view(torch.int16), out.view(torch.int16))
    if fp8:
        kp8, vp8 = H.oracle_pools_fp8(run)
        rows = H.sample_rows(w, heads_per_kv=1)
        ref, ref_lse = H.oracle_rows_fp8(run, kp8, vp8, rows=rows)
        vmax = max(H.e4m3_vmax(vp8[(vp8 & 0x7F) != 0x7F], run.vs), 1e-9)
    else:
        kp16, vp16 = H.oracle_pools(w)
        rows, vmax = H.sample_rows(w, heads_per_kv=1), None
        ref, ref_lse = H.oracle_rows(w, kp16, vp16, rows=rows)
    H.compare_attention(w, out, lse, ref, ref_lse, rows=rows, contract=False, vmax=vmax)
