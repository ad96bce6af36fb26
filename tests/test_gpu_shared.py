"""Attention of batches that share prefixes (GPU) against the float64 oracle over the same block tables:
every row within the bound of the plain attention, over shapes, groups, key splits and both pool kinds;
plans, refusals, bad pages, lengths that disagree, streams and captured graphs."""
import numpy as np
import pytest

import gpu_helpers as H
import oracle
import shared_helpers as SH
from paper_2505_23970_amd import workloads as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu_ready():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2505_23970_amd as gc
    gc.load_library()


class Run:
    def __init__(self, w, sizes, shared, fp8=False, policy=None):
        import paper_2505_23970_amd as gc
        self.w, self.fp8 = w, fp8
        self.run = H.DeviceRunFp8(w, 0.02, 0.015) if fp8 else H.DeviceRun(w)
        self.run.append()
        self.groups = gc.SharedPrefixes(self.run.batch, sizes, shared, gc.SHARE_ALWAYS if policy is None else policy)
        self.scales = (self.run.ks, self.run.vs) if fp8 else ()

    def attention(self, split=None, lse=True, **kw):
        import torch
        import paper_2505_23970_amd as gc
        q, kp, vp = self.run.q, self.run.k_pool, self.run.v_pool
        out = torch.full_like(q, float("nan"))
        got_lse = torch.full(q.shape[:2], float("nan"), dtype=torch.float32, device="cuda") if lse else None
        ws = gc.alloc_shared_workspace(q.shape[1], kp, vp, self.groups, split)
        ws.fill_(0xFF)   # nothing in it is read before it is written
        call = gc.shared_prefix_attention_fp8 if self.fp8 else gc.shared_prefix_attention
        call(q, kp, vp, self.groups, self.w.scale, *self.scales, ws, out=out, lse=got_lse, kv_split_tiles=split, **kw)
        torch.cuda.synchronize()
        assert gc.plan_status(ws) == 0
        return out, got_lse

    def reference(self):
        if self.fp8:
            kp, vp = H.oracle_pools_fp8(self.run)
            return (*H.oracle_rows_fp8(self.run, kp, vp), max(H.e4m3_vmax(vp[(vp & 0x7F) != 0x7F], self.run.vs), 1e-9))
        kp, vp = H.oracle_pools(self.w)
        return (*H.oracle_rows(self.w, kp, vp), None)

    def check(self, out, lse, ref):
        return H.compare_attention(self.w, out, lse, ref[0], ref[1], contract=False, vmax=ref[2])


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
@pytest.mark.parametrize("D,Hq,Hkv", [(128, 8, 1), (128, 8, 2), (64, 4, 4), (64, 16, 2), (128, 40, 2), (64, 128, 1)])
@pytest.mark.parametrize("batch", ["decode", "one_page", "groups", "no_own", "prompts", "many"])
def test_rows_against_the_oracle(batch, D, Hq, Hkv, fp8):
    sizes, shared, beyond, new = SH.batches()[batch]
    w = SH.build(sizes, shared, beyond, new, Hq, Hkv, D, seed=2000 + D + Hq, name=f"shared_{batch}_{Hq}_{Hkv}_d{D}")
    r = Run(w, sizes, shared, fp8)
    ref = r.reference()
    for split in (None, 1, -1):
        print(f"case {w.name} fp8={fp8} split={split}", flush=True)
        out, lse = r.attention(split)
        r.check(out, lse, ref)


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_long_prefixes_split_as_the_plan_does(fp8):
    """Enough keys that the plan cuts the shared and the own part into many chunks."""
    sizes, shared = [24, 8], [6000, 2000]
    rng = np.random.default_rng(9)
    beyond = rng.integers(0, 1500, 32)
    beyond[3] = 0
    new = rng.choice([1, 1, 2, 40], 32)
    w = SH.build(sizes, shared, beyond, new, 16, 2, 128, seed=2100, name="shared_long")
    r = Run(w, sizes, shared, fp8)
    out, lse = r.attention()
    r.check(out, lse, r.reference())


def test_policy_and_the_plain_attention():
    """A batch that the policy leaves alone gives the plain attention's bits; one that it takes, its rows."""
    import paper_2505_23970_amd as gc
    import torch
    w = SH.build([1, 1, 1], [64, 32, 0], [5, 40, 7], [1, 2, 1], 8, 2, 128, seed=2200, name="shared_none")
    r = Run(w, [1, 1, 1], [64, 32, 0], policy=gc.SHARE_AUTO)
    out, lse = r.attention()
    want = gc.prefix_prefill_attention(r.run.q, r.run.k_pool, r.run.v_pool, r.run.batch, w.scale)
    assert torch.equal(out.view(torch.int16), want.view(torch.int16))
    sizes, shared, beyond, new = SH.batches()["many"]
    w = SH.build(sizes, shared, beyond, new, 8, 1, 128, seed=2201, name="shared_auto")
    r = Run(w, sizes, shared, policy=gc.SHARE_AUTO)
    out, lse = r.attention()
    r.check(out, lse, r.reference())


def test_runs_are_deterministic_and_plans_serve_every_layer():
    import paper_2505_23970_amd as gc
    import torch
    sizes, shared, beyond, new = SH.batches()["prompts"]
    w = SH.build(sizes, shared, beyond, new, 16, 2, 128, seed=2300, name="shared_layers")
    r = Run(w, sizes, shared)
    out, _ = r.attention()
    q, kp, vp = r.run.q, r.run.k_pool, r.run.v_pool
    ws = gc.alloc_shared_workspace(16, kp, vp, r.groups)
    gc.plan_shared(16, kp, vp, r.groups, ws)
    for _ in range(3):
        again = gc.run_shared(q, kp, vp, r.groups, w.scale, ws)
        assert torch.equal(again.view(torch.int16), out.view(torch.int16))
    other = (-q).contiguous()   # another layer's queries on the same plan
    assert torch.equal(gc.run_shared(other, kp, vp, r.groups, w.scale, ws).view(torch.int16),
                       gc.shared_prefix_attention(other, kp, vp, r.groups, w.scale).view(torch.int16))


def test_stale_and_special_keys_and_values():
    """Whatever lies behind a sequence's end, or behind the shared keys in the same page run, never shows."""
    sizes, shared, beyond, new = [3], [80], [0, 5, 20], [1, 1, 2]
    w = SH.build(sizes, shared, beyond, new, 8, 2, 64, seed=2400, name="shared_stale")
    ref = Run(w, sizes, shared).reference()
    for stale in (0x7F80, 0xFF80, 0x7FC0, 0x7F7F):   # inf, -inf, NaN, the largest
        r = Run(w, sizes, shared)
        kp, vp = H.from_dev_bits(r.run.k_pool), H.from_dev_bits(r.run.v_pool)
        used = np.zeros((w.num_blocks, 16), bool)
        for i in range(3):
            for p in range(int(w.prefix_lens[i] + w.new_lens[i])):
                used[w.block_tables[i][p // 16], p % 16] = True
        kp[~np.broadcast_to(used[:, None, :, None], kp.shape)] = stale
        vp[~np.broadcast_to(used[:, None, None, :], vp.shape)] = stale
        r.run.k_pool.copy_(H.to_dev_bf16(kp))
        r.run.v_pool.copy_(H.to_dev_bf16(vp))
        for split in (None, 1):
            out, lse = r.attention(split)
            r.check(out, lse, ref)


def test_block_ids_outside_the_pool_reach_nothing_else():
    """A bad id makes the result of its group undefined; the other group's rows stay exact."""
    sizes, shared, beyond, new = [3, 2], [64, 32], [5, 40, 0, 3, 9], [1, 1, 2, 1, 1]
    w = SH.build(sizes, shared, beyond, new, 8, 2, 128, seed=2500, name="shared_bad_ids")
    ref = Run(w, sizes, shared).reference()
    w.block_tables[0:3, 1] = w.num_blocks + 7
    w.block_tables[1, 5] = -3
    r = Run(w, sizes, shared)
    out, _ = r.attention(lse=False)
    got = H.from_dev_f32(out).reshape(-1, 128)[4 * 8:]
    vmax = 4.0
    assert np.all(np.abs(got - ref[0][4 * 8:]) <= H.derived_bound(ref[0][4 * 8:], vmax))


@pytest.mark.parametrize("wrong", ["longer", "negative", "prefix_below_shared", "not_whole_pages", "group_bounds", "shared_longer"])
def test_device_lengths_that_disagree(wrong):
    """Nothing is written and the status says so."""
    import paper_2505_23970_amd as gc
    import torch
    sizes, shared, beyond, new = [3, 2], [64, 32], [5, 40, 0, 3, 9], [1, 1, 2, 1, 1]
    w = SH.build(sizes, shared, beyond, new, 8, 2, 128, seed=2600, name="shared_disagree")
    r = Run(w, sizes, shared)
    b, g = r.run.batch, r.groups
    if wrong == "longer":
        b.prefix_lens_dev[1] += 64 * 30
    elif wrong == "negative":
        b.prefix_lens_dev[1] = -5
    elif wrong == "prefix_below_shared":
        b.prefix_lens_dev[1] = 60
    elif wrong == "not_whole_pages":
        g.shared_lens_dev[0] = 60
    elif wrong == "group_bounds":
        g.group_first_dev[1] = 9
    else:
        g.shared_lens_dev[1] = 1 << 20
    q, kp, vp = r.run.q, r.run.k_pool, r.run.v_pool
    ws = gc.alloc_shared_workspace(8, kp, vp, g, 1)
    ws.fill_(0xFF)
    out = torch.full_like(q, 7.0)
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    gc.shared_prefix_attention(q, kp, vp, g, w.scale, ws, out=out, lse=lse, kv_split_tiles=1)
    assert gc.plan_status(ws) == gc.GC_ERR_LENGTHS
    assert bool((out == 7.0).all()) and bool((lse == 7.0).all())


def test_rows_of_no_request_are_left_alone():
    """Outputs behind the last new token, and the log-sum-exps, keep their contents."""
    import paper_2505_23970_amd as gc
    import torch
    sizes, shared, beyond, new = SH.batches()["groups"]
    w = SH.build(sizes, shared, beyond, new, 8, 2, 128, seed=2700, name="shared_tail")
    r = Run(w, sizes, shared)
    T = w.total_new
    big = torch.full((T + 40, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T + 40, 8), 7.0, device="cuda")
    gc.shared_prefix_attention(r.run.q, r.run.k_pool, r.run.v_pool, r.groups, w.scale, out=big[:T], lse=lse[:T])
    torch.cuda.synchronize()
    assert bool((big[T:] == 7.0).all()) and bool((lse[T:] == 7.0).all()) and bool((lse[:T] != 7.0).all())


@pytest.mark.parametrize("batch", [512, 513, 700])
def test_large_batches(batch):
    """On both sides of the planner's LDS limit; a request search of two steps in the merge."""
    rng = np.random.default_rng(batch)
    sizes = [batch // 2, 1, batch - batch // 2 - 1]
    shared, beyond, new = [48, 16, 32], rng.integers(0, 40, batch), rng.choice([0, 1, 1, 2], batch)
    w = SH.build(sizes, shared, beyond, new, 2, 1, 64, seed=2800 + batch, name=f"shared_batch_{batch}")
    r = Run(w, sizes, shared)
    ref = r.reference()
    for split in (None, 1):
        out, lse = r.attention(split)
        r.check(out, lse, ref)


def test_step_of_rotary_append_and_shared_attention():
    """A decoding step as a program makes it: projections in, rotated into pool and q_out, attention; in one
    captured graph, replayed over new projections, against the oracle on what the pools then hold."""
    import paper_2505_23970_amd as gc
    import torch
    sizes, shared, beyond, new = SH.batches()["decode"]
    w = SH.build(sizes, shared, beyond, new, 16, 2, 128, seed=2900, name="shared_step")
    run = H.DeviceRun(w)
    groups = gc.SharedPrefixes(run.batch, sizes, shared, gc.SHARE_ALWAYS)
    table = gc.rotary_table(400, 128)
    q_out, out = torch.empty_like(run.q), torch.empty_like(run.q)
    ws = gc.alloc_shared_workspace(16, run.k_pool, run.v_pool, groups)

    def step():
        gc.kv_append_rotary(run.q, run.k_new, run.v_new, run.k_pool, run.v_pool, run.batch, table, q_out=q_out)
        gc.plan_shared(16, run.k_pool, run.v_pool, groups, ws)
        gc.run_shared(q_out, run.k_pool, run.v_pool, groups, w.scale, ws, out=out)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for again in range(3):
        for t in (run.q, run.k_new, run.v_new):
            t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(again)).to(torch.bfloat16))
        out.fill_(float("nan"))
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        got, rotated = H.from_dev_f32(out), H.from_dev_bits(q_out)
        kp, vp = H.from_dev_bits(run.k_pool), H.from_dev_bits(run.v_pool)
        ref, _ = oracle.attention(w.prefix_lens, w.new_lens, w.block_tables, w.num_blocks, rotated, kp, vp, w.scale)
        vmax = float(np.nanmax(np.abs(W.bf16_bits_to_f32(vp))))
        assert np.all(np.abs(got.reshape(ref.shape) - ref) <= H.derived_bound(ref, vmax))
        step()
        torch.cuda.synchronize()
        assert np.array_equal(H.from_dev_f32(out), got)


def test_two_graphs_on_one_workspace_and_a_stream_of_its_own():
    """Two captured graphs that share a workspace, replayed in turn on one stream; and a call on another
    stream whose temporaries belong to that stream."""
    import paper_2505_23970_amd as gc
    import torch
    runs = []
    ws = None
    for k, name in enumerate(("decode", "groups")):
        sizes, shared, beyond, new = SH.batches()[name]
        w = SH.build(sizes, shared, beyond, new, 8, 2, 128, seed=3000 + k, name=f"shared_graph_{name}")
        r = Run(w, sizes, shared)
        need = gc.shared_workspace_size(8, r.run.k_pool, r.run.v_pool, r.groups)
        runs.append([r, r.attention()[0], torch.empty_like(r.run.q), None, need])
    ws = torch.empty(max(x[4] for x in runs), dtype=torch.uint8, device="cuda")
    for x in runs:
        r, graph = x[0], torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            gc.shared_prefix_attention(r.run.q, r.run.k_pool, r.run.v_pool, r.groups, r.w.scale, ws, out=x[2])
        x[3] = graph
    for _ in range(3):
        for x in runs:
            x[2].fill_(float("nan"))
            x[3].replay()
        torch.cuda.synchronize()
        for x in runs:
            assert torch.equal(x[1].view(torch.int16), x[2].view(torch.int16))
    side = torch.cuda.Stream()
    r, want = runs[0][:2]
    outs = [gc.shared_prefix_attention(r.run.q, r.run.k_pool, r.run.v_pool, r.groups, r.w.scale, stream=side) for _ in range(4)]
    side.synchronize()
    assert all(torch.equal(o.view(torch.int16), want.view(torch.int16)) for o in outs)


def test_refusals():
    import paper_2505_23970_amd as gc
    import torch
    sizes, shared, beyond, new = SH.batches()["groups"]
    w = SH.build(sizes, shared, beyond, new, 8, 2, 128, seed=3100, name="shared_refused")
    r = Run(w, sizes, shared)
    b, q, kp, vp = r.run.batch, r.run.q, r.run.k_pool, r.run.v_pool
    for sizes2, shared2 in (([3, 1, 4], [64, 48, 80]), ([3, 1, 4, 2, 0], [64, 48, 80, 0, 0]), ([10], [64, 0]), ([10], [64])):
        with pytest.raises(ValueError):   # sum, an empty group, lengths of lists, rows that differ
            gc.SharedPrefixes(b, sizes2, shared2)
    ws = gc.alloc_shared_workspace(8, kp, vp, r.groups)
    with pytest.raises(gc.GcError):
        gc.run_shared(q, kp, vp, r.groups, w.scale, ws[:-16].contiguous())
    with pytest.raises(gc.GcError):
        gc.run_shared(q, kp, vp, r.groups, -1.0, ws)
    with pytest.raises(TypeError):
        gc.run_shared_fp8(q, kp, vp, r.groups, w.scale, 0.1, 0.1, ws)
    with pytest.raises(ValueError):
        gc.run_shared(q[:-1].contiguous(), kp, vp, r.groups, w.scale, ws)
    off = torch.empty(q.numel() + 4, dtype=torch.bfloat16, device="cuda")[4:].view_as(q)
    with pytest.raises(gc.GcError):
        gc.run_shared(off, kp, vp, r.groups, w.scale, ws)


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_pools_beyond_4_gib(fp8):
    """Block ids whose byte offsets exceed 2^32, through the rotary append and the attention: bitwise what the
    unshifted run gives. The blocks that a wraparound of those offsets would reach hold NaN."""
    import paper_2505_23970_amd as gc
    import torch
    sizes, shared, beyond, new = SH.batches()["groups"]
    w = SH.build(sizes, shared, beyond, new, 16, 2, 128, seed=3200, name="shared_4gib")
    table = gc.rotary_table(400, 64)
    runs = [H.DeviceRunFp8(w, 0.02, 0.015) if fp8 else H.DeviceRun(w) for _ in range(2)]
    shift = (1 << 32) // (w.num_kv_heads * 16 * w.head_dim * (1 if fp8 else 2))
    for name in ("k_pool", "v_pool"):
        small = getattr(runs[1], name)
        big = torch.empty((shift + w.num_blocks,) + tuple(small.shape[1:]), dtype=small.dtype, device="cuda")
        (big[:w.num_blocks] if fp8 else big[:w.num_blocks].view(torch.int16)).fill_(0x7F if fp8 else int(W.BF16_NAN))
        big[shift:] = small
        setattr(runs[1], name, big)
    runs[1].batch = gc.PagedBatch(w.prefix_lens, w.new_lens, (w.block_tables + shift).astype(np.int32))
    got = []
    for run in runs:
        groups = gc.SharedPrefixes(run.batch, sizes, shared, gc.SHARE_ALWAYS)
        args = (run.q, run.k_new, run.v_new, run.k_pool, run.v_pool, run.batch, table)
        q = gc.kv_append_rotary_fp8(*args, run.ks, run.vs) if fp8 else gc.kv_append_rotary(*args)
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
        call = gc.shared_prefix_attention_fp8 if fp8 else gc.shared_prefix_attention
        out = call(q, run.k_pool, run.v_pool, groups, w.scale, *((run.ks, run.vs) if fp8 else ()), lse=lse, kv_split_tiles=1)
        got.append((out.view(torch.int16), lse, run.k_pool[-w.num_blocks:].view(torch.uint8), run.v_pool[-w.num_blocks:].view(torch.uint8)))
    assert not bool(got[0][0].view(torch.bfloat16).isnan().any())
    for a, b in zip(*got):
        assert torch.equal(a, b)
    del runs, got
    torch.cuda.empty_cache()


def test_runs_without_their_plan_write_nothing():
    """A cleared workspace, the plain attention's plan, the other pool kind's plan, another split's plan."""
    import paper_2505_23970_amd as gc
    import torch
    sizes, shared, beyond, new = SH.batches()["prompts"]
    w = SH.build(sizes, shared, beyond, new, 16, 2, 128, seed=3300, name="shared_no_plan")
    r = Run(w, sizes, shared)
    q, kp, vp = r.run.q, r.run.k_pool, r.run.v_pool
    ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    fp8 = H.DeviceRunFp8(w, 0.02, 0.015)

    def untouched(what):
        out = torch.full_like(q, 7.0)
        lse = torch.full(q.shape[:2], 7.0, device="cuda")
        gc.run_shared(q, kp, vp, r.groups, w.scale, ws, out=out, lse=lse)
        torch.cuda.synchronize()
        assert bool((out == 7.0).all()) and bool((lse == 7.0).all()), what

    for fill in (0, 0xFF, 0x01):
        ws.fill_(fill)
        untouched(f"filled with {fill}")
    gc.plan(16, kp, vp, r.run.batch, ws)
    untouched("plain plan")
    gc.plan_shared(16, fp8.k_pool, fp8.v_pool, r.groups, ws, kv_split_tiles=None)
    bf16_bytes = gc.shared_workspace_size(16, kp, vp, r.groups)
    if gc.shared_workspace_size(16, fp8.k_pool, fp8.v_pool, r.groups) != bf16_bytes:
        untouched("8-bit plan")
    gc.plan_shared(16, kp, vp, r.groups, ws, kv_split_tiles=1)
    untouched("another split")
    gc.plan_shared(16, kp, vp, r.groups, ws)
    out = gc.run_shared(q, kp, vp, r.groups, w.scale, ws)
    r.check(out, None, r.reference())


def test_masked_rows_of_a_request_see_only_their_keys():
    """Planted keys: one that would take over the softmax lies at the last shared key, at the first own one, at each
    new token. Row i must show it from there on, no earlier row and no other request anything of it."""
    import paper_2505_23970_amd as gc
    import torch
    sizes, shared, beyond, new = [3], [48], [0, 3, 20], [5, 5, 5]
    for where in ("last_shared", "first_own", "new_2"):
        w = SH.build(sizes, shared, beyond, new, 8, 2, 64, seed=3400, name=f"shared_planted_{where}")
        r = Run(w, sizes, shared)
        kp, vp = r.run.k_pool, r.run.v_pool
        req = 1
        pos = {"last_shared": 47, "first_own": 48, "new_2": int(w.prefix_lens[req]) + 2}[where]
        block, slot = int(w.block_tables[req][pos // 16]), pos % 16
        r.run.q.fill_(1.0)
        kp[block, :, slot, :] = 4.0     # score 4 * 64 / 8 = 32 above everything random here
        vp[block, :, :, slot] = 1000.0
        out = gc.shared_prefix_attention(r.run.q, kp, vp, r.groups, w.scale, kv_split_tiles=1)
        seen = (out.float().abs() > 500).all(dim=2).all(dim=1).cpu().numpy()
        none = (out.float().abs() < 500).all(dim=2).all(dim=1).cpu().numpy()
        want = np.zeros(15, bool)
        if where == "last_shared":
            want[:] = True
        else:
            want[5 + (0 if where == "first_own" else 2):10] = True
        assert np.array_equal(seen, want) and np.array_equal(none, ~want), where


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
@pytest.mark.parametrize("D,Hq", [(128, 8), (64, 16)])
def test_score_jumps_beyond_the_exponent_slack(D, Hq, fp8):
    """Keys that score 0, a later one that scores 100 and more above them, one that scores as much more again: the
    last takes all the weight (the others' are exp of at most -100, nothing in fp32), so each row is its value. In
    tiles of 128 rows the weights' sum passes fp32 at the jump, and the items run again with the exact maxima; the
    single tokens' small tiles take it as they go. The output: that value times its scale in fp32 (2^-24, two
    products), rounded to bf16 (2^-8)."""
    import paper_2505_23970_amd as gc
    import torch
    sizes, shared, beyond, new = [3, 2], [320, 0], [40, 0, 70, 200, 90], [20, 1, 30, 40, 1]
    w = SH.build(sizes, shared, beyond, new, Hq, 1, D, seed=3500, name=f"shared_jump_d{D}")
    r = Run(w, sizes, shared, fp8)
    kp, vp = r.run.k_pool, r.run.v_pool
    r.run.q.fill_(1.0)
    kp.zero_()
    # one key's element value x gives the score x * D * scale; e4m3 codes: 0x7E is 448, 0x76 is 224
    ks, vs = (r.run.ks, r.run.vs) if fp8 else (1.0, 1.0)
    scale = 120.0 / (D * (224 * ks if fp8 else 224.0))
    want = torch.empty(sum(new), D, device="cuda")
    at = 0
    for req, n in enumerate(new):
        table = w.block_tables[req]
        for pos, code in ((100 if req < 3 else 70, 0x76), (290 if req < 3 else 85, 0x7E)):
            kp[int(table[pos // 16]), 0, pos % 16] = code if fp8 else float(224 if code == 0x76 else 448)
        v = vp[int(table[pos // 16]), 0, :, pos % 16]
        want[at:at + n] = v.view(torch.float8_e4m3fn).float() * vs if fp8 else v.float()
        at += n
    for split in (None, 1, -1):
        args = (r.run.q, kp, vp, r.groups, scale) + ((ks, vs) if fp8 else ())
        lse = torch.empty(sum(new), Hq, device="cuda")
        out = (gc.shared_prefix_attention_fp8 if fp8 else gc.shared_prefix_attention)(*args, lse=lse, kv_split_tiles=split)
        err = (out.float() - want[:, None, :]).abs()
        assert bool((err <= want[:, None, :].abs() * (2.0 ** -8 + 2.0 ** -22)).all()), (split, float(err.max()))
        # the score itself: a sum of D equal products (exact), times scale, log2 e and ln 2 in fp32: five roundings
        assert bool(((lse - 240.0).abs() <= 240.0 * 2.0 ** -20).all()), split
