"""The append with rotary positions (GPU) against the rotation in float64: rotated keys and queries within
the rounding of fp32 arithmetic and of the type that holds them, values, unrotated elements and every other
pool byte bit for bit; both pairings, partial rotation, strided projections, in-place queries, 8-bit pools,
streams and captured graphs."""
import numpy as np
import pytest

import gpu_helpers as H
import oracle
import rotary_reference as RR
from paper_2505_23970_amd import workloads as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu_ready():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2505_23970_amd as gc
    gc.load_library()


def lengths(batch):
    rng = np.random.default_rng(batch)
    P = rng.integers(0, 50, batch)
    n = rng.choice([0, 1, 2, 3, 5, 9, 15, 16, 17, 33], batch)
    n[0] = 0 if batch > 1 else 5
    n[-1] = 0 if batch > 2 else 18
    n[batch // 2] = 40
    return P, n


def random_table(rows, rotary, seed):
    """Not on the unit circle, so that a cosine taken for a sine, or another row or pair, shows."""
    return np.random.default_rng(seed).uniform(-1.5, 1.5, (rows, rotary // 2, 2)).astype(np.float32)


def e4m3_values(codes):
    table = np.array([oracle.e4m3_value(c) for c in range(256)], np.float64)
    return table[codes]


def pool_rows(w, pool, values=False):
    """The new tokens' rows [T][Hkv][D] of a pool image."""
    rows, cu = np.empty((w.total_new, w.num_kv_heads, w.head_dim), pool.dtype), 0
    for r in range(w.batch):
        for i in range(int(w.new_lens[r])):
            p = int(w.prefix_lens[r]) + i
            page = pool[w.block_tables[r][p // 16]]
            rows[cu] = page[:, :, p % 16] if values else page[:, p % 16, :]
            cu += 1
    return rows


def fused(w, extra=0):
    """q, k_new, v_new as views of one [T][Hq + 2 Hkv + extra][D] buffer."""
    import torch
    Hq, Hkv = w.num_q_heads, w.num_kv_heads
    buf = torch.full((w.total_new, Hq + 2 * Hkv + extra, w.head_dim), float("nan"), dtype=torch.bfloat16, device="cuda")
    buf[:, :Hq] = H.to_dev_bf16(w.q)
    buf[:, Hq:Hq + Hkv] = H.to_dev_bf16(w.k_new)
    buf[:, Hq + Hkv:Hq + 2 * Hkv] = H.to_dev_bf16(w.v_new)
    return buf[:, :Hq], buf[:, Hq:Hq + Hkv], buf[:, Hq + Hkv:Hq + 2 * Hkv]


def call(run, table, fp8, q, k, v, **kw):
    import paper_2505_23970_amd as gc
    if fp8:
        return gc.kv_append_rotary_fp8(q, k, v, run.k_pool, run.v_pool, run.batch, table, run.ks, run.vs, **kw)
    return gc.kv_append_rotary(q, k, v, run.k_pool, run.v_pool, run.batch, table, **kw)


def check(w, run, table, fp8, interleaved, q_got, with_q=True):
    pos = RR.positions_of(w.prefix_lens, w.new_lens)
    R = 2 * table.shape[1]
    if with_q:
        y, mag = RR.rotate(W.bf16_bits_to_f32(w.q).astype(np.float64), pos, table, interleaved)
        err = np.abs(H.from_dev_f32(q_got) - y)
        assert np.all(err <= RR.bf16_bound(y, mag)), f"q off by {err.max()}"
        assert np.array_equal(H.from_dev_bits(q_got)[..., R:], w.q[..., R:]), "unrotated query elements"
    y, mag = RR.rotate(W.bf16_bits_to_f32(w.k_new).astype(np.float64), pos, table, interleaved)
    if fp8:
        kp, vp = run.pools()
        kp_ref, vp_ref = H.oracle_pools_fp8(run)
        ref, bound = RR.e4m3_bound(y, mag, oracle.inv_scale(run.ks))
        err = np.abs(e4m3_values(pool_rows(w, kp)) - ref)
    else:
        kp, vp = H.from_dev_bits(run.k_pool), H.from_dev_bits(run.v_pool)
        kp_ref, vp_ref = H.oracle_pools(w)
        bound = RR.bf16_bound(y, mag)
        err = np.abs(W.bf16_bits_to_f32(pool_rows(w, kp)).astype(np.float64) - y)
    assert np.all(err <= bound), f"k off by {err.max()}, at {np.argwhere(err > bound)[:4]}"
    assert np.array_equal(vp, vp_ref), f"v_pool differs at {np.argwhere(vp != vp_ref)[:5]}"
    # all but the rotated elements: the plain append's bytes
    assert np.array_equal(pool_rows(w, kp)[..., R:], pool_rows(w, kp_ref)[..., R:]), "unrotated key elements"
    cu = 0
    same = kp != kp_ref
    for r in range(w.batch):
        for i in range(int(w.new_lens[r])):
            p = int(w.prefix_lens[r]) + i
            same[w.block_tables[r][p // 16], :, p % 16, :R] = False
            cu += 1
    assert not same.any(), f"another slot changed: {np.argwhere(same)[:5]}"


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "interleaved"])
@pytest.mark.parametrize("D,Hq,Hkv,R", [(64, 1, 1, 64), (64, 6, 3, 16), (64, 34, 2, 48), (128, 8, 1, 128), (128, 64, 8, 64),
                                        (128, 21, 3, 48), (128, 3, 3, 16), (64, 32, 8, 32)])
def test_shapes_and_pairs(D, Hq, Hkv, R, interleaved, fp8):
    P, n = lengths(23)
    w = W.build(P, n, Hq, Hkv, D, seed=1000 + R + Hq, name=f"rotary_{Hq}_{Hkv}_{R}_d{D}", values="peaked")
    table = random_table(120, R, R)
    run = H.DeviceRunFp8(w, 0.02, 0.015) if fp8 else H.DeviceRun(w)
    print(f"case {w.name} fp8={fp8}", flush=True)
    q, k, v = fused(w, extra=R // 16 % 3) if R % 32 == 0 else (run.q, run.k_new, run.v_new)
    got = call(run, H_table(table), fp8, q, k, v, interleaved=interleaved)
    check(w, run, table, fp8, interleaved, got)


def H_table(table):
    import torch
    return torch.from_numpy(table).cuda()


@pytest.mark.parametrize("batch", [1, 2, 63, 64, 65, 66, 300])
def test_request_search(batch):
    P, n = lengths(batch)
    w = W.build(P, n, 6, 3, 64, seed=1100 + batch, name=f"rotary_batch_{batch}")
    table = random_table(100, 64, batch)
    run = H.DeviceRun(w)
    got = call(run, H_table(table), False, run.q, run.k_new, run.v_new)
    check(w, run, table, False, False, got)


def test_table_with_exactly_the_rows_needed():
    w = W.build([33, 0, 90], [7, 3, 1], 4, 2, 64, seed=1201, name="rotary_last_row")
    table = random_table(91, 64, 5)
    run = H.DeviceRun(w)
    check(w, run, table, False, False, call(run, H_table(table), False, run.q, run.k_new, run.v_new))


def test_queries_in_place_and_without_queries():
    import paper_2505_23970_amd as gc
    w = W.build([33, 0, 90], [7, 30, 1], 12, 2, 128, seed=1202, name="rotary_in_place")
    table = random_table(120, 128, 6)
    for interleaved in (False, True):
        run = H.DeviceRun(w)
        got = call(run, H_table(table), False, run.q, run.k_new, run.v_new, q_out=run.q, interleaved=interleaved)
        assert got is run.q
        check(w, run, table, False, interleaved, got)
        run = H.DeviceRun(w)
        assert gc.kv_append_rotary(None, run.k_new, run.v_new, run.k_pool, run.v_pool, run.batch, H_table(table),
                                   interleaved=interleaved) is None
        check(w, run, table, False, interleaved, None, with_q=False)


def test_far_positions_follow_the_angles_in_64_bits():
    """rotary_table at positions past 2^17: against the rotation by angles of 64 bits. The table's entries
    are off by half an fp32 step, 2^-25 of at most 1."""
    import paper_2505_23970_amd as gc
    w = W.build([140000, 131071], [3, 2], 4, 1, 64, seed=1203, name="rotary_far")
    run = H.DeviceRun(w)
    table = gc.rotary_table(140003, 64, base=500000.0)
    got = call(run, table, False, run.q, run.k_new, run.v_new)
    pos = RR.positions_of(w.prefix_lens, w.new_lens)
    inv = 500000.0 ** (-np.arange(0, 64, 2) / 64.0)
    angle = pos[:, None] * inv
    t64 = np.stack([np.cos(angle), np.sin(angle)], axis=-1)
    y, mag = RR.rotate(W.bf16_bits_to_f32(w.q).astype(np.float64), np.arange(len(pos)), t64, False)
    x = np.abs(W.bf16_bits_to_f32(w.q).astype(np.float64))
    assert np.all(np.abs(H.from_dev_f32(got) - y) <= RR.bf16_bound(y, mag) + 2.0 ** -24 * (x + np.roll(x, 32, axis=-1)))


@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "interleaved"])
def test_prompts_beyond_the_cache(interleaved):
    """Enough query bytes that they are read past the caches: 12300 tokens of 64 heads. Rows sampled."""
    import torch
    import paper_2505_23970_amd as gc
    P, n = [5, 700, 0], [6001, 3, 6296]
    T, Hq, D = sum(n), 64, 128
    assert T * Hq * D * 2 >= 192 << 20
    pages = [-(-(p + m) // 16) for p, m in zip(P, n)]
    tables = np.zeros((3, max(pages)), np.int32)
    order = np.random.default_rng(3).permutation(sum(pages)).astype(np.int32)
    for r, k in enumerate(pages):
        tables[r, :k], order = order[:k], order[k:]
    gen = torch.Generator(device="cuda").manual_seed(4)
    qkv = torch.randn((T, Hq + 2, D), generator=gen, device="cuda", dtype=torch.bfloat16)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + 1], qkv[:, Hq + 1:]
    kp = torch.zeros((sum(pages), 1, 16, D), dtype=torch.bfloat16, device="cuda")
    vp = torch.zeros((sum(pages), 1, D, 16), dtype=torch.bfloat16, device="cuda")
    table = random_table(6400, 96, 12)
    got = gc.kv_append_rotary(q, k, v, kp, vp, gc.PagedBatch(P, n, tables), H_table(table), interleaved=interleaved)
    pos = RR.positions_of(P, n)
    rows = np.unique(np.concatenate([np.arange(40), np.arange(5990, 6020), np.arange(T - 40, T),
                                     np.random.default_rng(5).integers(0, T, 300)]))
    dev = torch.from_numpy(rows).cuda()
    y, mag = RR.rotate(q[dev].double().cpu().numpy(), pos[rows], table, interleaved)
    assert np.all(np.abs(got[dev].double().cpu().numpy() - y) <= RR.bf16_bound(y, mag))
    y, mag = RR.rotate(k.double().cpu().numpy(), pos, table, interleaved)
    at = np.concatenate([tables[r][np.arange(P[r], P[r] + n[r]) // 16] for r in range(3)]).astype(np.int64)
    at, slot = torch.from_numpy(at).cuda(), torch.from_numpy(pos % 16).cuda()
    assert np.all(np.abs(kp[at, :, slot].double().cpu().numpy() - y) <= RR.bf16_bound(y, mag))
    assert torch.equal(vp[at, :, :, slot].view(torch.int16), v.contiguous().view(torch.int16))


def test_bad_pages_and_nothing_new():
    """Ids outside the pool: nothing is written for those pages, the queries are rotated all the same."""
    import torch
    import paper_2505_23970_amd as gc
    w = W.build([20, 5], [30, 9], 4, 2, 64, seed=1204, name="rotary_bad_page")
    table = random_table(64, 64, 8)
    w.block_tables[0][2] = w.num_blocks + 3
    w.block_tables[1][0] = -1
    run = H.DeviceRun(w)
    got = call(run, H_table(table), False, run.q, run.k_new, run.v_new)
    pos = RR.positions_of(w.prefix_lens, w.new_lens)
    y, mag = RR.rotate(W.bf16_bits_to_f32(w.q).astype(np.float64), pos, table, False)
    assert np.all(np.abs(H.from_dev_f32(got) - y) <= RR.bf16_bound(y, mag))
    good = W.build([20, 5], [30, 9], 4, 2, 64, seed=1204, name="rotary_good_page")
    changed = (H.from_dev_bits(run.k_pool) != w.k_pool).any(axis=(1, 2, 3))
    assert set(np.flatnonzero(changed)) == {int(good.block_tables[0][1]), int(good.block_tables[0][3])}
    none = W.build([20, 5], [0, 0], 4, 2, 64, seed=1205, name="rotary_nothing")
    run = H.DeviceRun(none)
    before = run.k_pool.view(torch.int16).clone()
    out = gc.kv_append_rotary(run.q, run.k_new, run.v_new, run.k_pool, run.v_pool, run.batch, H_table(table))
    assert tuple(out.shape) == (0, 4, 64) and torch.equal(before, run.k_pool.view(torch.int16))


def test_special_values_follow_the_formula():
    """Infinities and NaN reach only the elements of their own pair."""
    w = W.build([3], [4], 2, 1, 64, seed=1206, name="rotary_special")
    w.q[0, 0, 5], w.q[1, 1, 40], w.q[2, 0, 63] = 0x7F80, 0x7FC0, 0xFF80
    w.k_new[1, 0, 7] = 0x7FC0
    table = random_table(16, 64, 9)
    run = H.DeviceRun(w)
    got = H.from_dev_f32(call(run, H_table(table), False, run.q, run.k_new, run.v_new))
    pos = RR.positions_of(w.prefix_lens, w.new_lens)
    with np.errstate(invalid="ignore"):
        y, mag = RR.rotate(W.bf16_bits_to_f32(w.q).astype(np.float64), pos, table, False)
        fine = np.isfinite(y)
        assert np.array_equal(np.isnan(got), np.isnan(y)) and np.array_equal(got[np.isinf(y)], y[np.isinf(y)])
        assert np.all(np.abs(got - y)[fine] <= RR.bf16_bound(y, mag)[fine])
    assert (~fine).sum() == 6
    k = W.bf16_bits_to_f32(pool_rows(w, H.from_dev_bits(run.k_pool)))
    assert np.array_equal(np.argwhere(np.isnan(k)), [[1, 0, 7], [1, 0, 39]])


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_graph_replays_and_streams(fp8):
    """Captured once and replayed over changed inputs, with eager work between; and on a stream of its own."""
    import torch
    w = W.build([33, 100, 0], [1, 20, 5], 16, 2, 128, seed=1207, name="rotary_graph")
    table = random_table(128, 128, 10)
    dev_table = H_table(table)
    run = H.DeviceRunFp8(w, 0.02, 0.015) if fp8 else H.DeviceRun(w)
    q_out = torch.empty_like(run.q)
    call(run, dev_table, fp8, run.q, run.k_new, run.v_new, q_out=q_out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(run, dev_table, fp8, run.q, run.k_new, run.v_new, q_out=q_out)
    for again in range(3):
        other = W.build([33, 100, 0], [1, 20, 5], 16, 2, 128, seed=1300 + again, name="rotary_graph_again")
        other.block_tables[:], other.k_pool[:], other.v_pool[:] = w.block_tables, w.k_pool, w.v_pool
        fresh = H.DeviceRunFp8(other, 0.02, 0.015) if fp8 else H.DeviceRun(other)
        for name in ("q", "k_new", "v_new"):
            getattr(run, name).copy_(getattr(fresh, name))
        if fp8:
            fresh.k8_init, fresh.v8_init = run.k8_init, run.v8_init
        run.k_pool.copy_(H.to_dev_u8(run.k8_init) if fp8 else H.to_dev_bf16(w.k_pool))
        run.v_pool.copy_(H.to_dev_u8(run.v8_init) if fp8 else H.to_dev_bf16(w.v_pool))
        q_out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        fresh.k_pool, fresh.v_pool = run.k_pool, run.v_pool
        check(other, fresh, table, fp8, False, q_out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    run = H.DeviceRunFp8(w, 0.02, 0.015) if fp8 else H.DeviceRun(w)
    torch.cuda.synchronize()
    got = call(run, dev_table, fp8, run.q, run.k_new, run.v_new, stream=side)
    side.synchronize()
    check(w, run, table, fp8, False, got)


def test_refusals():
    import torch
    import paper_2505_23970_amd as gc
    w = W.build([33, 0], [7, 3], 4, 2, 64, seed=1208, name="rotary_refused")
    run = H.DeviceRun(w)
    table = H_table(random_table(64, 64, 11))
    k, v, kp, vp, b = run.k_new, run.v_new, run.k_pool, run.v_pool, run.batch
    for bad in (table.double(), table[:, :, :1], table[:, :, 0], table.cpu()):
        with pytest.raises((TypeError, ValueError)):
            gc.kv_append_rotary(run.q, k, v, kp, vp, b, bad)
    for bad in (table[:39], table[:, :4].contiguous(), table[:, :12].contiguous()):   # rows, 8 and 24 elements
        with pytest.raises(gc.GcError):
            gc.kv_append_rotary(run.q, k, v, kp, vp, b, bad)
    with pytest.raises(ValueError):
        gc.kv_append_rotary(run.q[:-1], k, v, kp, vp, b, table)
    with pytest.raises(ValueError):
        gc.kv_append_rotary(run.q.transpose(1, 2).contiguous().transpose(1, 2), k, v, kp, vp, b, table)
    with pytest.raises(ValueError):
        gc.kv_append_rotary(None, k, v, kp, vp, b, table, q_out=run.q)
    with pytest.raises(TypeError):
        gc.kv_append_rotary(run.q.half(), k, v, kp, vp, b, table)
    # q_out over a strided q, or over the keys
    q, k2, v2 = fused(w)
    buf = torch.as_strided(q, (10, 4, 64), (256, 64, 1))
    with pytest.raises(gc.GcError):
        gc.kv_append_rotary(q, k2, v2, kp, vp, b, table, q_out=buf)
    # an address off 16 bytes
    off = torch.empty(10 * 256 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(10, 4, 64)
    with pytest.raises(gc.GcError):
        gc.kv_append_rotary(off, k, v, kp, vp, b, table)
