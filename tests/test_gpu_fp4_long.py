"""4-bit pools and reads of rows at sizes that change the path taken (GPU): many workgroups, rows past the last-level cache,
long rows that are not split, pages that lie past 32-bit offsets, and batches without work."""
import numpy as np
import pytest

import fp4_reference as R
import gpu_helpers as H
from paper_2505_23970_amd import workloads as W
from test_gpu_fp4 import Run4, appended, check, same_pools, wild
from test_gpu_read import expected, fresh, kinds, same_rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu_ready():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2505_23970_amd as gc
    gc.load_library()


def pages_of(P, n):
    return int(sum(-(-(p + m) // 16) - p // 16 for p, m in zip(P, n) if m))


# KV heads that do not fill the last workgroup of a page, at just enough pages for several heads a workgroup.
MANY = [(128, 5, 820), (128, 9, 456), (64, 3, 2050), (64, 9, 820)]


@pytest.mark.parametrize("D,Hkv,least", MANY)
def test_many_workgroups(D, Hkv, least):
    rng = np.random.default_rng(least)
    P, n = rng.integers(0, 18, least), rng.integers(1, 19, least)
    assert pages_of(P, n) * -(-Hkv // (2 if D == 64 else 1)) >= 4096
    w = wild(W.build(P, n, Hkv, Hkv, D, seed=4000 + Hkv, name=f"fp4_many_{Hkv}_d{D}"), Hkv)
    run = Run4(w)
    run.append()
    same_pools(run.images(), R.append(w, run.k4, run.v4, run.s4))
    w.block_tables[least // 2, 0] = w.num_blocks
    for name, call, images in kinds(w, Hkv):
        k, v = fresh(w)
        call(k_out=k, v_out=v)
        same_rows((k, v), expected(w, *images))


@pytest.mark.parametrize("D,Hkv", [(128, 7), (64, 12)])
def test_rows_past_the_cache(D, Hkv):
    """192 MB of rows in one append, against appends of a few requests each (which the tests above hold to the reference)."""
    import torch
    import paper_2505_23970_amd as gc
    batch = 40
    tokens = -(-(192 << 20) // (4 * Hkv * D)) // batch + 5
    rng = np.random.default_rng(D)
    P, n = rng.integers(0, 40, batch), tokens + rng.integers(0, 9, batch)
    slots = int(P.max() + n.max()) // 16 + 1
    tables = rng.permutation(batch * slots).reshape(batch, slots)
    g = torch.Generator(device="cuda").manual_seed(D)
    k, v = (torch.randn((int(n.sum()), Hkv, D), generator=g, device="cuda").bfloat16() for _ in range(2))
    assert 4 * k.numel() >= 192 << 20
    pools = [gc.alloc_pools_fp4(batch * slots, Hkv, D) for _ in range(2)]
    for t in pools[0] + pools[1]:
        t.fill_(0x5A)
    gc.kv_append_fp4(k, v, *pools[0], gc.PagedBatch(P, n, tables))
    cu = np.concatenate([[0], np.cumsum(n)])
    for r in range(0, batch, 3):
        some = slice(r, min(r + 3, batch))
        rows = slice(int(cu[some.start]), int(cu[some.stop]))
        gc.kv_append_fp4(k[rows], v[rows], *pools[1], gc.PagedBatch(P[some], n[some], tables[some]))
    for x, y in zip(*pools):
        assert torch.equal(x, y)


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 8, 1), (128, 20, 4)])
@pytest.mark.parametrize("tiling", [1, 2, 3], ids=["prefill", "small", "wide"])
def test_long_rows_in_one_piece(D, Hq, Hkv, tiling):
    """Rows of 2500 and 1100 keys (40 and 18 tiles), none split; then with scores that jump near the end, which takes the
    second pass over all of them."""
    for jump in (False, True):
        w = W.build([2460, 5], [40, 1100], Hq, Hkv, D, seed=4100 + D, values="unit" if jump else "peaked",
                    name=f"fp4_long_{Hq}_d{D}_{jump}")
        if jump:
            scaled = lambda x, f: W.f32_to_bf16_bits(W.bf16_bits_to_f32(x) * np.float32(f))  # noqa: E731
            w.k_prefix[:] = scaled(w.k_prefix, 0.01)
            w.k_new[:] = scaled(w.k_new, 0.01)
            w.k_prefix[2300:2330] = scaled(w.k_prefix[2300:2330], 9000.0)
            w.k_new[1040:1050] = scaled(w.k_new[1040:1050], 9000.0)
            w.finish()
        run, ref = appended(w)
        rows = H.sample_rows(w, tokens_per_request=6)
        check(w, *run.attention(split=-1, tiling=tiling), ref, rows)


def test_pages_past_32_bit_offsets():
    """Codes and scales from byte 2^31, 2^32 and more of their pools on: the same results as from a small pool."""
    import torch
    import paper_2505_23970_amd as gc
    Hq, Hkv, D = 16, 8, 128
    NB = (1 << 32) // (Hkv * 16 * D // 16) + 64           # scales: 1 KB a block, codes: 8 KB
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("needs 80 GB")
    w = W.build([130, 33, 900], [20, 1, 1], Hq, Hkv, D, seed=4200, values="peaked", name="fp4_far")
    run = Run4(w)
    far = gc.alloc_pools_fp4(NB, Hkv, D)
    rng = np.random.default_rng(3)
    borders = [b + i for b in (1 << 18, 1 << 19, 1 << 21, 1 << 22, NB - 8) for i in range(-8, 8) if b + i < NB]
    rest = np.unique(rng.integers(0, NB, 4 * w.num_blocks))
    ids = np.concatenate([borders, rng.permutation(np.setdiff1d(rest, borders))])[:w.num_blocks]
    ids = rng.permutation(ids)
    assert len(np.unique(ids)) == w.num_blocks
    to = torch.from_numpy(ids).cuda()
    for x, y in zip(far, run.dev):
        x[to] = y
    batch = gc.PagedBatch(w.prefix_lens, w.new_lens, ids[w.block_tables])
    table = torch.randn(1024, D // 2, 2, device="cuda")
    for rotary in (False, True):
        for pools, b in ((run.dev, run.batch), (far, batch)):
            if rotary:
                gc.kv_append_rotary_fp4(None, run.k_new, run.v_new, *pools, b, table)
            else:
                gc.kv_append_fp4(run.k_new, run.v_new, *pools, b)
        for x, y in zip(far, run.dev):
            assert torch.equal(x[to], y)
        for x, y in zip(gc.kv_read_fp4(*far, batch), gc.kv_read_fp4(*run.dev, run.batch)):
            assert torch.equal(x.view(torch.int16), y.view(torch.int16))
        for tiling in (None, 1, 2, 3):
            x = gc.prefix_prefill_attention_fp4(run.q, *far, batch, w.scale, tiling=tiling)
            y = gc.prefix_prefill_attention_fp4(run.q, *run.dev, run.batch, w.scale, tiling=tiling)
            assert bool(y.isfinite().all()) and torch.equal(x.view(torch.int16), y.view(torch.int16))
    del far, x, y
    torch.cuda.empty_cache()


def test_reads_past_32_bit_offsets():
    import torch
    import paper_2505_23970_amd as gc
    Hkv, D = 8, 128
    w = W.build([30, 5], [50, 17], Hkv, Hkv, D, seed=4300, name="read_far")
    for dtype, call in ((torch.bfloat16, gc.kv_read), (torch.uint8, lambda *a: gc.kv_read_fp8(*a, 0.5, 0.25))):
        NB = (1 << 32) // (Hkv * 16 * D * dtype.itemsize) + 40
        k, v = (torch.empty((NB, Hkv) + s, dtype=dtype, device="cuda") for s in ((16, D), (D, 16)))
        ids = np.arange(NB - w.num_blocks, NB)
        g = torch.Generator(device="cuda").manual_seed(5)
        small = [torch.randint(0, 100, (w.num_blocks,) + tuple(t.shape[1:]), generator=g, device="cuda").to(dtype) for t in (k, v)]
        for x, y in zip((k, v), small):
            x[-w.num_blocks:] = y
        got = call(k, v, gc.PagedBatch(w.prefix_lens, w.new_lens, ids[w.block_tables]))
        want = call(*small, gc.PagedBatch(w.prefix_lens, w.new_lens, w.block_tables))
        for x, y in zip(got, want):
            assert torch.equal(x.view(torch.int16), y.view(torch.int16))
        del k, v
    torch.cuda.empty_cache()


def test_batches_without_work():
    """Nothing new in any request: nothing is written. One token with nothing cached: its own value."""
    import torch
    import paper_2505_23970_amd as gc
    w = W.build([20, 0], [0, 0], 8, 2, 64, seed=4400, name="fp4_idle")
    run = Run4(w)
    out = gc.prefix_prefill_attention_fp4(run.q, *run.dev, run.batch, w.scale)
    assert tuple(out.shape) == (0, 8, 64)
    w = W.build([0], [1], 8, 2, 64, seed=4401, name="fp4_own_value")
    run, ref = appended(w)
    for tiling in (1, 2, 3):
        out, lse = run.attention(tiling=tiling)
        check(w, out, lse, ref)
        got = gc.kv_read_fp4(*run.dev, run.batch)[1]
        assert torch.equal(out, got.repeat_interleave(4, dim=1))


def test_calls_side_by_side_and_appends_in_a_graph():
    """Attention of three batches on three streams at once, each with its own workspace; an append captured and replayed."""
    import torch
    import paper_2505_23970_amd as gc
    cases = [W.build(P, n, 16, 2, 128, seed=4500 + i, values="peaked", name=f"fp4_beside_{i}")
             for i, (P, n) in enumerate((([3000, 500], [1, 1]), ([700, 0], [60, 90]), ([64] * 20, [130] * 20)))]
    runs = [appended(w)[0] for w in cases]
    want = [[t.clone() for t in r.attention()] for r in runs]
    streams = [torch.cuda.Stream() for _ in cases]
    plans = [gc.alloc_workspace(16, r.k, r.v, r.batch) for r in runs]
    outs = [torch.empty_like(r.q) for r in runs]
    torch.cuda.synchronize()
    for _ in range(5):
        for o in outs:
            o.fill_(float("nan"))
        torch.cuda.synchronize()
        for r, s, ws, o in zip(runs, streams, plans, outs):
            gc.prefix_prefill_attention_fp4(r.q, *r.dev, r.batch, r.w.scale, ws, out=o, stream=s)
        torch.cuda.synchronize()
        for o, (x, _) in zip(outs, want):
            assert torch.equal(o.view(torch.int16), x.view(torch.int16))
    r = runs[1]
    images = r.images()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.append()
    for _ in range(3):
        for t, image in zip(r.dev, (r.k4, r.v4, r.s4)):
            t.copy_(H.to_dev_u8(image))
        graph.replay()
        same_pools(r.images(), images)
