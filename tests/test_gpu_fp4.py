"""4-bit pools (GPU): appended codes and scales bit for bit those of the reference in float64, plain and rotated; attention
over them against the float64 oracle on the same numbers, in every tiling; NaN in stale, masked and seen places; streams,
captured graphs, refusals; a whole step."""
import numpy as np
import pytest

import fp4_reference as R
import gpu_helpers as H
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


class Run4:
    """Device side of a workload over 4-bit pools (host images: k4, v4, s4)."""

    def __init__(self, w, pools=None):
        import paper_2505_23970_amd as gc
        self.w = w
        self.k4, self.v4, self.s4 = pools if pools is not None else R.pools(w)
        self.batch = gc.PagedBatch(w.prefix_lens, w.new_lens, w.block_tables)
        self.q, self.k_new, self.v_new = H.to_dev_bf16(w.q), H.to_dev_bf16(w.k_new), H.to_dev_bf16(w.v_new)
        self.k, self.v, self.s = H.to_dev_u8(self.k4), H.to_dev_u8(self.v4), H.to_dev_u8(self.s4)

    @property
    def dev(self):
        return self.k, self.v, self.s

    def images(self):
        return tuple(t.cpu().numpy() for t in self.dev)

    def append(self, **kw):
        import paper_2505_23970_amd as gc
        gc.kv_append_fp4(self.k_new, self.v_new, *self.dev, self.batch, **kw)

    def attention(self, split=None, tiling=None, **kw):
        import torch
        import paper_2505_23970_amd as gc
        T, Hq, D = self.w.q.shape
        lse = torch.full((T, Hq), float("nan"), dtype=torch.float32, device="cuda")
        out = torch.full((T, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        gc.prefix_prefill_attention_fp4(self.q, *self.dev, self.batch, self.w.scale, out=out, lse=lse, kv_split_tiles=split,
                                        tiling=tiling, **kw)
        torch.cuda.synchronize()
        return out, lse


def same_pools(got, want):
    for name, x, y in zip(("k", "v", "scales"), got, want):
        assert np.array_equal(x, y), f"{name} differs at {np.argwhere(x != y)[:5].tolist()}"


def lengths(batch, seed=None):
    rng = np.random.default_rng(batch if seed is None else seed)
    P = rng.integers(0, 50, batch)
    n = rng.choice([0, 1, 2, 3, 5, 9, 15, 16, 17, 33], batch)
    n[0] = 0 if batch > 1 else 5
    n[-1] = 0 if batch > 2 else 18
    n[batch // 2] = 40
    return P, n


def wild(w, seed):
    """Tokens of every magnitude, with zero blocks, infinities, NaN, subnormal numbers and borders among them."""
    rng = np.random.default_rng(seed)
    for x in (w.k_new, w.v_new):
        f = W.bf16_bits_to_f32(x)
        f = f * (2.0 ** rng.integers(-130, 120, f.shape[:2] + (1,))).astype(np.float32)
        at = rng.integers(0, 5, f.shape)
        f = np.where(at == 0, np.float32(1.75) * np.exp2(rng.integers(-4, 5, f.shape)).astype(np.float32), f)   # borders
        f = np.where(at == 1, np.float32(0.0), f)
        bits = W.f32_to_bf16_bits(f.astype(np.float32))
        bits[at == 2] ^= 0x8000
        flat = bits.reshape(-1, 32)
        pick = rng.permutation(len(flat))[:max(8, len(flat) // 8)]
        for i, kind in zip(pick, np.arange(len(pick)) % 6):
            if kind == 0:
                flat[i] = 0
            elif kind == 1:
                flat[i, 3] = 0x7FC0
            elif kind == 2:
                flat[i, 31] = 0xFF80
            elif kind == 3:
                flat[i] = rng.integers(0, 128, 32)   # subnormal
            elif kind == 4:
                flat[i, 0] = 0x7F7F                  # the largest
            else:
                flat[i, 9] = 0xFFFF                  # a NaN with its sign
    return w


SHAPES = [(64, 1, 1), (64, 6, 3), (64, 32, 8), (128, 8, 1), (128, 64, 8), (128, 21, 3)]


@pytest.mark.parametrize("D,Hq,Hkv", SHAPES)
def test_append_is_the_references(D, Hq, Hkv):
    P, n = lengths(23)
    w = wild(W.build(P, n, Hq, Hkv, D, seed=2000 + Hq, name=f"fp4_append_{Hq}_{Hkv}_d{D}"), Hq)
    run = Run4(w)
    run.append()
    same_pools(run.images(), R.append(w, run.k4, run.v4, run.s4))


@pytest.mark.parametrize("batch", [1, 2, 63, 64, 65, 66, 300])
def test_append_finds_its_request(batch):
    P, n = lengths(batch)
    w = W.build(P, n, 3, 3, 64, seed=2100 + batch, name=f"fp4_batch_{batch}")
    run = Run4(w)
    run.append()
    same_pools(run.images(), R.append(w, run.k4, run.v4, run.s4))


def random_table(rows, rotary, seed):
    return np.random.default_rng(seed).uniform(-1.5, 1.5, (rows, rotary // 2, 2)).astype(np.float32)


def rotated_keys(w, table, interleaved):
    """fl32 of the rotation (its two products are exact in float64, their sum is rounded to 53 bits first)."""
    pos = RR.positions_of(w.prefix_lens, w.new_lens)
    with np.errstate(all="ignore"):
        y, _ = RR.rotate(R.rows_of(w.k_new), pos, table, interleaved)
        return y.astype(np.float32).astype(np.float64)


def fused(w, extra=0):
    import torch
    Hq, Hkv = w.num_q_heads, w.num_kv_heads
    buf = torch.full((w.total_new, Hq + 2 * Hkv + extra, w.head_dim), float("nan"), dtype=torch.bfloat16, device="cuda")
    buf[:, :Hq] = H.to_dev_bf16(w.q)
    buf[:, Hq:Hq + Hkv] = H.to_dev_bf16(w.k_new)
    buf[:, Hq + Hkv:Hq + 2 * Hkv] = H.to_dev_bf16(w.v_new)
    return buf[:, :Hq], buf[:, Hq:Hq + Hkv], buf[:, Hq + Hkv:Hq + 2 * Hkv]


def check_q(w, table, interleaved, got):
    pos = RR.positions_of(w.prefix_lens, w.new_lens)
    y, mag = RR.rotate(R.rows_of(w.q), pos, table, interleaved)
    assert np.all(np.abs(H.from_dev_f32(got) - y) <= RR.bf16_bound(y, mag))


@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "interleaved"])
@pytest.mark.parametrize("D,Hq,Hkv,rotary", [(64, 1, 1, 64), (64, 6, 3, 16), (64, 34, 2, 48), (128, 8, 1, 128), (128, 64, 8, 64),
                                             (128, 21, 3, 48), (128, 3, 3, 16)])
def test_rotary_append_is_the_references(D, Hq, Hkv, rotary, interleaved):
    import torch
    import paper_2505_23970_amd as gc
    P, n = lengths(23)
    w = wild(W.build(P, n, Hq, Hkv, D, seed=2200 + rotary + Hq, name=f"fp4_rotary_{Hq}_{rotary}_d{D}"), Hq)
    table = random_table(120, rotary, rotary)
    run = Run4(w)
    q, k, v = fused(w, extra=rotary // 16 % 3) if rotary % 32 == 0 else (run.q, run.k_new, run.v_new)
    got = gc.kv_append_rotary_fp4(q, k, v, *run.dev, run.batch, torch.from_numpy(table).cuda(), interleaved=interleaved)
    check_q(w, table, interleaved, got)
    same_pools(run.images(), R.append(w, run.k4, run.v4, run.s4, keys=rotated_keys(w, table, interleaved)))
    run = Run4(w)
    assert gc.kv_append_rotary_fp4(None, k, v, *run.dev, run.batch, torch.from_numpy(table).cuda(), interleaved=interleaved) is None
    same_pools(run.images(), R.append(w, run.k4, run.v4, run.s4, keys=rotated_keys(w, table, interleaved)))


def test_append_from_pinned_memory_bad_pages_and_nothing():
    import torch
    w = W.build([20, 5, 0], [30, 9, 0], 4, 2, 64, seed=2300, name="fp4_bad_page")
    w.block_tables[0][2] = w.num_blocks + 3
    w.block_tables[1][0] = -1
    run = Run4(w)
    run.k_new, run.v_new = run.k_new.cpu().pin_memory(), run.v_new.cpu().pin_memory()
    run.append()
    torch.cuda.synchronize()
    same_pools(run.images(), R.append(w, run.k4, run.v4, run.s4))
    none = W.build([20, 5], [0, 0], 4, 2, 64, seed=2301, name="fp4_nothing")
    run = Run4(none)
    run.append()
    same_pools(run.images(), (run.k4, run.v4, run.s4))


# ------------------------------------------------------------------------------- attention

def appended(w):
    """Device pools after the append, and the oracle's bf16 pools of the same numbers."""
    run = Run4(w)
    run.append()
    images = R.append(w, run.k4, run.v4, run.s4)
    same_pools(run.images(), images)
    return run, R.as_bf16_pools(*images)


def check(w, out, lse, ref_pools, rows=None):
    ref, ref_lse = H.oracle_rows(w, *ref_pools, rows=rows)
    # (a value block's scale is at most 2 / 7 above its largest element's magnitude)
    vmax = 2 * float(np.abs(W.bf16_bits_to_f32(np.concatenate([w.v_new.ravel(), w.v_prefix.ravel()]))).max(initial=0.0))
    return H.compare_attention(w, out, lse, ref, ref_lse, rows=rows, contract=False, vmax=vmax)


BATCHES = {
    # single tokens: prefixes that end at, before and behind pages and tiles; nothing cached; nothing new
    "tokens": ([0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 127, 500, 40], [1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 0]),
    # a few tokens each
    "few": ([0, 14, 30, 100, 257, 5], [2, 2, 1, 2, 2, 0]),
    # prompts: none cached, tiles of 128 and 256 rows that end anywhere
    "prompts": ([0, 100, 0, 65, 7, 300], [17, 130, 0, 64, 1, 45]),
    # one long, split into chunks
    "long": ([3000], [3]),
    # rows far beyond a tile
    "deep": ([900, 0], [300, 411]),
}


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 4, 1), (64, 32, 8), (64, 8, 8), (128, 64, 8), (128, 8, 1), (128, 16, 2), (128, 3, 3),
                                      (64, 10, 2), (128, 40, 1)])
@pytest.mark.parametrize("name", list(BATCHES))
def test_attention(name, D, Hq, Hkv):
    P, n = BATCHES[name]
    w = W.build(P, n, Hq, Hkv, D, seed=2400 + Hq + D, values="peaked", name=f"fp4_{name}_{Hq}_{Hkv}_d{D}")
    run, ref = appended(w)
    rows = H.sample_rows(w, tokens_per_request=5) if name == "deep" else None
    check(w, *run.attention(), ref, rows)


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 8, 1), (128, 16, 2), (128, 20, 4), (64, 16, 1)])
@pytest.mark.parametrize("tiling", [1, 2, 3], ids=["prefill", "small", "wide"])
@pytest.mark.parametrize("split", [None, -1, 1, 3])
def test_tilings_and_splits(D, Hq, Hkv, tiling, split):
    w = W.build([0, 200, 61, 350, 0, 16], [70, 9, 1, 90, 0, 33], Hq, Hkv, D, seed=2500 + Hq, values="peaked",
                name=f"fp4_tiling_{Hq}_d{D}")
    run, ref = appended(w)
    check(w, *run.attention(split=split, tiling=tiling), ref)


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 34, 1), (128, 128, 1), (128, 51, 3), (64, 384, 3)])
def test_large_and_odd_groups(D, Hq, Hkv):
    """Groups of 17 to 128 query heads: no small tiles."""
    w = W.build([40, 3, 130], [1, 9, 4], Hq, Hkv, D, seed=2550 + Hq, values="peaked", name=f"fp4_group_{Hq}_{Hkv}")
    run, ref = appended(w)
    for tiling in (None, 1, 3):
        check(w, *run.attention(tiling=tiling), ref)


def test_queries_and_keys_of_every_magnitude():
    """Query elements from 2^-40 of the row's largest up, rows from 2^-60 to 2^60 and zero rows against keys that bring
    the scores back to 1: what h + l of a query loses does not show."""
    w = W.build([70, 33], [40, 1], 8, 2, 128, seed=2600, values="unit", name="fp4_magnitudes")
    rng = np.random.default_rng(7)
    q = W.bf16_bits_to_f32(w.q)
    q = q * (2.0 ** rng.integers(-40, 1, q.shape)).astype(np.float32)
    q[3] = 0
    w.q[:] = W.f32_to_bf16_bits(q)
    for e in (-60, 0, 60):
        v = W.build([70, 33], [40, 1], 8, 2, 128, seed=2600, values="unit", name="fp4_magnitudes")
        v.q[:] = W.f32_to_bf16_bits(q * np.float32(2.0 ** e))
        v.scale = w.scale * 2.0 ** -e * 4
        run, ref = appended(v)
        for tiling in (1, 2, 3):
            check(v, *run.attention(tiling=tiling), ref)


@pytest.mark.parametrize("tiling", [1, 2, 3], ids=["prefill", "small", "wide"])
def test_score_jumps_take_the_exact_pass(tiling):
    """Scores that grow by more than 2^100 in weight behind the first tile."""
    w = W.build([300, 130], [9, 70], 4, 2, 64, seed=2700, values="unit", name="fp4_jumps")
    w.k_prefix[:] = W.f32_to_bf16_bits(W.bf16_bits_to_f32(w.k_prefix) * np.float32(0.01))
    w.k_prefix[200:260] = W.f32_to_bf16_bits(W.bf16_bits_to_f32(w.k_prefix[200:260]) * np.float32(9000.0))
    w.finish()
    run, ref = appended(w)
    check(w, *run.attention(tiling=tiling), ref)


def numbers(t):
    return t.float().cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tiling", [1, 2, 3], ids=["prefill", "small", "wide"])
def test_nan_reaches_the_rows_that_see_it(tiling, D):
    """A NaN value among the new tokens: its block of elements in the rows from its token on, and nothing else. A NaN key:
    the whole rows from its token on. One in the cached tokens: all rows of its request."""
    Hq, Hkv = 4, 2
    for what, place in (("v", 5), ("v", 40), ("k", 21), ("cached v", 70), ("cached k", 3), ("last v", 49)):
        w = W.build([90, 20], [50, 6], Hq, Hkv, D, seed=2800 + D, values="peaked", name=f"fp4_nan_{what}_{place}")
        clean, _ = appended(w)
        base, base_lse = (t.clone() for t in clean.attention(tiling=tiling))
        if what.startswith("cached"):
            x = w.v_prefix if what.endswith("v") else w.k_prefix
            x[place, 1, 37] = 0x7FC0
            w.finish()
        else:
            (w.k_new if what == "k" else w.v_new)[place, 1, 37] = 0x7FC0
        run, _ = appended(w)
        out, lse = run.attention(tiling=tiling)
        got, want = numbers(out), numbers(base)
        nan = np.zeros(got.shape, bool)
        first = 0 if what.startswith("cached") else place
        nan[first:50, 2:4, slice(32, 64) if what.endswith("v") else slice(None)] = True   # (heads 2, 3: KV head 1)
        assert np.array_equal(np.isnan(got), nan), (what, place, np.argwhere(np.isnan(got) != nan)[:4])
        if what.endswith("v"):
            assert np.array_equal(got[~nan], want[~nan]) and np.array_equal(numbers(lse), numbers(base_lse))
        else:
            assert np.array_equal(got[~nan], want[~nan])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tiling", [1, 2, 3], ids=["prefill", "small", "wide"])
def test_queries_that_are_not_numbers(tiling, D):
    """NaN or an infinity in a head's query: that head's row is NaN, every other row what it was."""
    w = W.build([90, 20], [30, 6], 4, 2, D, seed=2850 + D, values="peaked", name="fp4_wild_queries")
    clean, _ = appended(w)
    base = numbers(clean.attention(tiling=tiling)[0])
    nan = np.zeros(base.shape, bool)
    for (token, head, el), bits in (((3, 1, 7), 0x7FC0), ((17, 2, D - 1), 0x7F80), ((33, 0, 0), 0xFF80)):
        w.q[token, head, el] = bits
        nan[token, head] = True
    run, _ = appended(w)
    got = numbers(run.attention(tiling=tiling)[0])
    assert np.array_equal(np.isnan(got), nan), np.argwhere(np.isnan(got) != nan)[:4]
    # (a NaN sum sends a whole tile through the second pass, whose offsets follow every tile: the other rows may round anew)
    assert np.allclose(got[~nan], base[~nan], rtol=0, atol=2.0 ** -6 * np.abs(base).max())


def test_pages_outside_the_pool_and_stale_blocks():
    """Ids outside the pool behind the last position are never followed; rows past a request's end keep their contents."""
    import torch
    import paper_2505_23970_amd as gc
    w = W.build([30, 60, 5], [10, 1, 3], 8, 2, 128, seed=2900, values="peaked", name="fp4_table_tail", extra_table_slots=3)
    for r in range(3):
        used = -(-int(w.prefix_lens[r] + w.new_lens[r]) // 16)
        w.block_tables[r, used:] = [1 << 30, -7, w.num_blocks][r]
    run, ref = appended(w)
    for tiling in (1, 2, 3):
        check(w, *run.attention(tiling=tiling), ref)
    # out and lse with rows behind the last sequence
    T = w.total_new
    out = torch.full((T + 5, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T + 5, 8), 7.0, device="cuda")
    gc.prefix_prefill_attention_fp4(run.q, *run.dev, run.batch, w.scale, out=out[:T], lse=lse[:T])
    torch.cuda.synchronize()
    check(w, out[:T], lse[:T], ref)
    assert bool((out[T:] == 7).all()) and bool((lse[T:] == 7).all())


def test_device_lengths_that_disagree_write_nothing():
    import torch
    import paper_2505_23970_amd as gc
    w = W.build([30, 60], [1, 1], 8, 2, 128, seed=2901, name="fp4_disagree")
    run, _ = appended(w)
    ws = gc.alloc_workspace(8, run.k, run.v, run.batch)
    run.batch.cu_new_lens_dev.copy_(torch.tensor([0, 1, 3], dtype=torch.int32))
    gc.plan(8, run.k, run.v, run.batch, ws)
    assert gc.plan_status(ws) == gc.GC_ERR_LENGTHS
    out = torch.full((2, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    gc.run_fp4(run.q, *run.dev, run.batch, w.scale, ws, out=out)
    torch.cuda.synchronize()
    assert bool((out == 7).all())


def test_one_plan_serves_every_kind_of_pool():
    """A plan made with bf16 pools of the same shape is run over 4-bit ones, and the other way round."""
    import torch
    import paper_2505_23970_amd as gc
    w = W.build([700, 20], [1, 1], 16, 2, 128, seed=2902, values="peaked", name="fp4_plans")
    run, ref = appended(w)
    kb, vb = H.to_dev_bf16(ref[0]), H.to_dev_bf16(ref[1])
    ws = gc.alloc_workspace(16, kb, vb, run.batch)
    assert ws.numel() == gc.alloc_workspace(16, run.k, run.v, run.batch).numel()
    gc.plan(16, kb, vb, run.batch, ws)
    a, lse = torch.empty_like(run.q), torch.empty((2, 16), device="cuda")
    gc.run_fp4(run.q, *run.dev, run.batch, w.scale, ws, out=a, lse=lse)
    check(w, a, lse, ref)
    gc.plan(16, run.k, run.v, run.batch, ws)
    b, lse_b = torch.empty_like(run.q), torch.empty((2, 16), device="cuda")
    gc.run(run.q, kb, vb, run.batch, w.scale, ws, out=b, lse=lse_b)
    check(w, b, lse_b, ref)


def test_resident_launch():
    """Wide tiles enough for two rounds of the compute units, which take them from queues."""
    import torch
    w = W.build([64] * 40, [130] * 40, 64, 8, 128, seed=2903, values="peaked", name="fp4_resident")
    run, ref = appended(w)
    out, lse = run.attention(tiling=3)
    check(w, out, lse, ref, H.sample_rows(w, tokens_per_request=3))
    again, lse2 = run.attention(tiling=3)   # the queues are left cleared
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and torch.equal(lse, lse2)


def test_same_bits_every_time():
    w = W.build([900, 37, 3], [1, 1, 1], 16, 2, 128, seed=2904, values="peaked", name="fp4_bits")
    run, _ = appended(w)
    first = [t.clone() for t in run.attention()]
    for _ in range(3):
        for x, y in zip(first, run.attention()):
            assert np.array_equal(numbers(x), numbers(y))


@pytest.mark.parametrize("D,prefix,new", [(128, [200, 33], [1, 1]), (64, [70, 0], [40, 25])], ids=["tokens", "prompts"])
def test_step_in_graphs_and_on_streams(D, prefix, new):
    """Rotary append, then plan and attention: captured once and replayed over changed inputs, with eager work between; two
    graphs that share a workspace; on a stream of its own."""
    import torch
    import paper_2505_23970_amd as gc
    build = lambda seed: W.build(prefix, new, 16, 2, D, seed=seed, values="peaked", name="fp4_graph")  # noqa: E731
    w = build(3000)
    table = random_table(256, D, 5)
    dev_table = torch.from_numpy(table).cuda()
    run = Run4(w)
    ws = gc.alloc_workspace(16, run.k, run.v, run.batch)
    q_out, out = torch.empty_like(run.q), torch.empty_like(run.q)
    lse = torch.empty(run.q.shape[:2], device="cuda")

    def step(**kw):
        gc.kv_append_rotary_fp4(run.q, run.k_new, run.v_new, *run.dev, run.batch, dev_table, q_out=q_out, **kw)
        gc.prefix_prefill_attention_fp4(q_out, *run.dev, run.batch, w.scale, ws, out=out, lse=lse, **kw)

    def load(seed):
        other = build(seed)
        other.block_tables[:], other.k_pool[:], other.v_pool[:] = w.block_tables, w.k_pool, w.v_pool
        for name in ("q", "k_new", "v_new"):
            getattr(run, name).copy_(H.to_dev_bf16(getattr(other, name)))
        for t, image in zip(run.dev, (run.k4, run.v4, run.s4)):
            t.copy_(H.to_dev_u8(image))
        out.fill_(float("nan"))
        lse.fill_(float("nan"))
        return other

    def verify(other):
        torch.cuda.synchronize()
        check_q(other, table, False, q_out)
        images = R.append(other, run.k4, run.v4, run.s4, keys=rotated_keys(other, table, False))
        same_pools(run.images(), images)
        turned = build(1)
        turned.q, turned.v_new, turned.v_prefix = H.from_dev_bits(q_out).reshape(w.q.shape), other.v_new, w.v_prefix
        turned.block_tables = w.block_tables
        check(turned, out, lse, R.as_bf16_pools(*images))

    step()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        graphs.append(g)
    for again in range(4):
        other = load(3100 + again)
        graphs[again % 2].replay()
        verify(other)
        other = load(3200 + again)
        step()
        verify(other)
    other = load(3300)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(stream=side)
    side.synchronize()
    verify(other)
    # workspace and outputs made by the call itself, on that stream
    with torch.cuda.stream(side):
        got = gc.prefix_prefill_attention_fp4(q_out, *run.dev, run.batch, w.scale)
    mine = gc.prefix_prefill_attention_fp4(q_out, *run.dev, run.batch, w.scale, stream=side)
    side.synchronize()
    assert torch.equal(got.view(torch.int16), out.view(torch.int16)) and torch.equal(mine.view(torch.int16), out.view(torch.int16))


def test_refusals():
    import torch
    import paper_2505_23970_amd as gc
    w = W.build([33, 0], [7, 3], 4, 2, 64, seed=3400, name="fp4_refused")
    run = Run4(w)
    k, v, s = run.dev
    kn, vn, b = run.k_new, run.v_new, run.batch
    for bad in ((k, v, s[..., :1].contiguous()), (k, v[..., :16].contiguous(), s), (k, v, s[:1]), (k.float(), v, s), (k, v, s.cpu()),
                (k[0], v[0], s[0]), (k.transpose(0, 1), v, s)):
        with pytest.raises((TypeError, ValueError)):
            gc.kv_append_fp4(kn, vn, *bad, b)
        with pytest.raises((TypeError, ValueError)):
            gc.prefix_prefill_attention_fp4(run.q, *bad, b, w.scale)
        with pytest.raises((TypeError, ValueError)):
            gc.kv_read_fp4(*bad, b)
    for bad in (kn[:-1], kn.float(), kn.cpu(), kn[:, :1], kn.transpose(0, 1).contiguous().transpose(0, 1), np.zeros(3)):
        with pytest.raises((TypeError, ValueError)):
            gc.kv_append_fp4(bad, vn, k, v, s, b)
    for bad in (run.q[:-1], run.q.float(), run.q[..., :32].contiguous()):
        with pytest.raises((TypeError, ValueError)):
            gc.prefix_prefill_attention_fp4(bad, k, v, s, b, w.scale)
    ws = gc.alloc_workspace(4, k, v, b)
    with pytest.raises(gc.GcError):
        gc.run_fp4(run.q, k, v, s, b, w.scale, ws[:64])
    with pytest.raises(gc.GcError):
        gc.run_fp4(run.q, k, v, s, b, float("nan"), ws)
    with pytest.raises(ValueError):
        gc.run_fp4(run.q, k, v, s, b, w.scale, ws, out=torch.empty_like(run.q[:-1]))
    with pytest.raises(ValueError):
        gc.run_fp4(run.q, k, v, s, b, w.scale, ws, lse=torch.empty(3, 4, device="cuda"))
    # 4-bit pools are not taken for the other kinds
    for call in (lambda: gc.kv_append_fp8(kn, vn, k, v, b, 1.0, 1.0), lambda: gc.kv_append(kn, vn, k, v, b),
                 lambda: gc.run_fp8(run.q, k, v, b, 0.1, 1.0, 1.0, ws), lambda: gc.kv_read_fp8(k, v, b, 1.0, 1.0),
                 lambda: gc.kv_read(k, v, b)):
        with pytest.raises((TypeError, ValueError)):
            call()


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 32, 8), (128, 8, 1), (128, 12, 4)])
@pytest.mark.parametrize("split", [None, -1, 2])
def test_tiles_that_are_not_full(D, Hq, Hkv, split):
    """128-row tiles of 1 to 128 rows: every number of 16-row blocks a wavefront, at its borders."""
    g = Hq // Hkv
    n = sorted({max(1, min(128 // g, (16 * b + d) // g)) for b in (0, 1, 3, 4, 5, 7, 8) for d in (-1, 0, 1, g)})
    P = np.arange(len(n)) * 37 % 200
    w = W.build(P, n, Hq, Hkv, D, seed=2580 + Hq + D, values="peaked", name=f"fp4_partial_{Hq}_{Hkv}_d{D}")
    run, ref = appended(w)
    check(w, *run.attention(split=split, tiling=1), ref)


def score_errors(w, images):
    """For every output row the most that one of its scores may be off by. The matrix products add the terms q k of eight
    neighbouring elements on a grid of 2^-13 of the largest one's power of two (of twice that where the key's code is 0.5), towards zero: each of
    the seven others loses less than 2^-12 of the largest. The split of a query adds 2^-22 of the row's largest per element, and its second part, at
    most 2^-4 of the first, as much of its own terms; fp32 sums, the scale and the offset round at 2^-24 of the sum of magnitudes, a few times."""
    T, Hq, D = w.q.shape
    q = np.abs(R.rows_of(w.q))
    out = np.zeros((T, Hq))
    k4 = np.abs(R.values(images[0], images[2][..., 0]))
    for r in range(w.batch):
        L = int(w.prefix_lens[r] + w.new_lens[r])
        pos = np.arange(L)
        k = k4[w.block_tables[r][pos // 16], :, pos % 16]             # [L][Hkv][D]
        for t in range(int(w.cu_new_lens[r]), int(w.cu_new_lens[r + 1])):
            seen = int(w.prefix_lens[r]) + t - int(w.cu_new_lens[r]) + 1
            for h in range(Hq):
                terms = q[t, h] * k[:seen, h // (Hq // w.num_kv_heads)]
                lost = 7 * 2.0 ** -12 * (1 + 2.0 ** -4) * terms.reshape(seen, D // 8, 8).max(axis=-1).sum(axis=-1)
                lost += 2.0 ** -22 * q[t, h].max() * k[:seen, h // (Hq // w.num_kv_heads)].sum(axis=-1) + 2.0 ** -21 * terms.sum(axis=-1)
                out[t, h] = w.scale * lost.max()
    return out.reshape(T * Hq)


def check_large_scores(w, out, lse, images):
    """The bounds of check, and what scores off by up to d do: weights change by factors within e^(+-2 d), so that an output moves by
    at most (e^(2 d) - 1) max |v|, and by no more than 2 max |v|; the log-sum-exp moves by d."""
    ref, ref_lse = H.oracle_rows(w, *R.as_bf16_pools(*images))
    T, Hq, D = w.q.shape
    vmax = 2 * float(np.abs(W.bf16_bits_to_f32(np.concatenate([w.v_new.ravel(), w.v_prefix.ravel()]))).max(initial=0.0))
    d = score_errors(w, images)
    got, got_lse = numbers(out).reshape(T * Hq, D), numbers(lse).reshape(T * Hq)
    more = vmax * np.minimum(np.expm1(np.minimum(2 * d, 1.0)), 2.0)
    more[2 * d > 1] = 2 * vmax
    assert np.all(np.abs(got - ref) <= H.derived_bound(ref, vmax) + more[:, None])
    assert np.all(np.abs(got_lse - ref_lse) <= 2.0 ** -8 + 1e-5 * np.abs(ref_lse) + d), np.abs(got_lse - ref_lse).max()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [35, 45, 61])
@pytest.mark.parametrize("jump", [9000.0, 900000.0])
def test_second_pass_of_tiles_that_are_not_full(jump, n, D):
    """Score jumps that only a few of a tile's 70 to 122 rows see, in their last blocks or in their first ones: the wavefronts of one and
    of two row blocks take the second pass together."""
    for last in (True, False):
        w = W.build([300], [n], 4, 2, D, seed=2750 + n, values="unit", name=f"fp4_jumps_{n}_{last}")
        w.k_prefix[:] = W.f32_to_bf16_bits(W.bf16_bits_to_f32(w.k_prefix) * np.float32(0.01))
        w.k_new[:] = W.f32_to_bf16_bits(W.bf16_bits_to_f32(w.k_new) * np.float32(0.01))
        if last:
            w.k_new[n - 3] = W.f32_to_bf16_bits(W.bf16_bits_to_f32(w.k_new[n - 3]) * np.float32(jump))
        else:
            w.k_prefix[290] = W.f32_to_bf16_bits(W.bf16_bits_to_f32(w.k_prefix[290]) * np.float32(jump))
            w.q[8:] = W.f32_to_bf16_bits(W.bf16_bits_to_f32(w.q[8:]) * np.float32(2.0 ** -14))
        w.finish()
        run, ref = appended(w)
        for split in (None, -1, 2):
            out, lse = run.attention(tiling=1, split=split)
            if jump < 10000:
                check(w, out, lse, ref)
            else:
                check_large_scores(w, out, lse, run.images())
