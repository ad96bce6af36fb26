"""Rows out of a pool (GPU): bf16 pools bit for bit, 8-bit pools to the bit of code value * scale, 4-bit pools exactly;
partial pages, strided batches, pinned host memory, and the way there and back."""
import numpy as np
import pytest

import fp4_reference as R
import gpu_helpers as H
import oracle
from paper_2505_23970_amd import workloads as W
from test_gpu_fp4 import Run4, lengths, same_pools, wild

pytestmark = pytest.mark.gpu
KS, VS = 0.0213, 0.0157


@pytest.fixture(scope="module", autouse=True)
def gpu_ready():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2505_23970_amd as gc
    gc.load_library()


def fresh(w):
    """Outputs whose untouched rows show."""
    import torch
    return [torch.full(w.k_new.shape, 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]


def expected(w, k_bits, v_bits):
    """Rows [T][Hkv][D] of bf16 pool images (values transposed), 7 where the page is outside the pool."""
    block, slot = R.slots(w)
    ok = (block >= 0) & (block < w.num_blocks)
    k, v = (np.full(w.k_new.shape, 0x40E0, np.uint16) for _ in range(2))
    k[ok], v[ok] = k_bits[block[ok], :, slot[ok]], v_bits[block[ok], :, :, slot[ok]]
    return k, v


def same_rows(got, want):
    for name, x, y in zip("kv", got, want):
        x = H.from_dev_bits(x)
        nan = (x & 0x7FFF) > 0x7F80
        assert np.array_equal(nan, (y & 0x7FFF) > 0x7F80), f"{name}: NaN elsewhere"
        assert np.array_equal(x[~nan], y[~nan]), f"{name} differs at {np.argwhere(~nan & (x != y))[:5].tolist()}"


def kinds(w, seed):
    """(name, call(k_out, v_out, stream), bf16 images of the pool's numbers) of every kind of pool, full of random codes."""
    import paper_2505_23970_amd as gc
    rng = np.random.default_rng(seed)
    batch = gc.PagedBatch(w.prefix_lens, w.new_lens, w.block_tables)
    NB, Hkv, D = w.num_blocks, w.num_kv_heads, w.head_dim
    kb, vb = rng.integers(0, 1 << 16, (NB, Hkv, 16, D)).astype(np.uint16), rng.integers(0, 1 << 16, (NB, Hkv, D, 16)).astype(np.uint16)
    dk, dv = H.to_dev_bf16(kb), H.to_dev_bf16(vb)
    yield "bf16", lambda **kw: gc.kv_read(dk, dv, batch, **kw), (kb, vb)
    k8, v8 = rng.integers(0, 256, kb.shape).astype(np.uint8), rng.integers(0, 256, vb.shape).astype(np.uint8)
    value = np.array([oracle.e4m3_value(c) for c in range(256)], np.float64)

    def image(codes, scale):
        x = value[codes].astype(np.float32) * np.float32(scale)   # (fl32, then bf16)
        return np.where(np.isnan(x), W.BF16_NAN, W.f32_to_bf16_bits(np.nan_to_num(x))).astype(np.uint16)
    d8 = H.to_dev_u8(k8), H.to_dev_u8(v8)
    yield "fp8", lambda **kw: gc.kv_read_fp8(*d8, batch, KS, VS, **kw), (image(k8, KS), image(v8, VS))
    k4, v4 = (rng.integers(0, 256, (NB, Hkv, 16, D // 2)).astype(np.uint8) for _ in range(2))
    s4 = rng.integers(3, 253, (NB, Hkv, 16, D // 32, 2)).astype(np.uint8)
    s4[rng.random(s4.shape) < 0.02] = 255
    d4 = [H.to_dev_u8(t) for t in (k4, v4, s4)]
    yield "fp4", lambda **kw: gc.kv_read_fp4(*d4, batch, **kw), R.as_bf16_pools(k4, v4, s4)


@pytest.mark.parametrize("D,Hkv", [(64, 1), (64, 3), (64, 8), (128, 1), (128, 3), (128, 8)])
def test_every_kind(D, Hkv):
    P, n = lengths(23)
    w = W.build(P, n, Hkv, Hkv, D, seed=3500 + Hkv, name=f"read_{Hkv}_d{D}")
    w.block_tables[11][:2] = [w.num_blocks, -3]   # (the request of 40 tokens)
    for name, call, images in kinds(w, Hkv):
        print(f"case {w.name} {name}", flush=True)
        k, v = fresh(w)
        got = call(k_out=k, v_out=v)
        assert got[0] is k and got[1] is v
        same_rows(got, expected(w, *images))


@pytest.mark.parametrize("batch", [1, 2, 64, 65, 300])
def test_batches(batch):
    P, n = lengths(batch)
    w = W.build(P, n, 2, 2, 64, seed=3600 + batch, name=f"read_batch_{batch}")
    for name, call, images in kinds(w, batch):
        same_rows(call(k_out=fresh(w)[0]), expected(w, *images))


def test_pinned_outputs_and_streams():
    import torch
    w = W.build([33, 0, 90], [7, 300, 1], 4, 2, 128, seed=3700, name="read_pinned")
    side = torch.cuda.Stream()
    for name, call, images in kinds(w, 1):
        pinned = [torch.empty(w.k_new.shape, dtype=torch.bfloat16, pin_memory=True) for _ in range(2)]
        torch.cuda.synchronize()
        call(k_out=pinned[0], v_out=pinned[1], stream=side)
        side.synchronize()
        same_rows(pinned, expected(w, *images))
        got = call(stream=side)
        side.synchronize()
        same_rows(got, expected(w, *images))
        k, v = fresh(w)
        call(k_out=k, v_out=v)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(k_out=k, v_out=v)
        for _ in range(3):
            k.fill_(7.0)
            v.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            same_rows((k, v), expected(w, *images))


def test_there_and_back():
    """Append, read, append what was read into other pages: the same codes and scales. Through bf16 pools: the same bits."""
    import torch
    import paper_2505_23970_amd as gc
    P, n = lengths(23)
    w = wild(W.build(P, n, 3, 3, 128, seed=3800, name="read_back"), 3)
    run = Run4(w)
    run.append()
    k, v = gc.kv_read_fp4(*run.dev, run.batch)
    torch.cuda.synchronize()
    images = R.append(w, run.k4, run.v4, run.s4)
    same_rows((k, v), expected(w, *R.as_bf16_pools(*images)))
    for t, image in zip(run.dev, (run.k4, run.v4, run.s4)):
        t.copy_(H.to_dev_u8(image))
    gc.kv_append_fp4(k, v, *run.dev, run.batch)
    same_pools(run.images(), images)
    plain = H.DeviceRun(W.build(P, n, 3, 3, 128, seed=3801, name="read_back_bf16"))
    plain.append()
    k, v = gc.kv_read(plain.k_pool, plain.v_pool, plain.batch)
    assert torch.equal(k.view(torch.int16), plain.k_new.view(torch.int16)) and torch.equal(v.view(torch.int16), plain.v_new.view(torch.int16))


def test_nothing_and_refusals():
    import torch
    import paper_2505_23970_amd as gc
    none = W.build([20, 5], [0, 0], 4, 2, 64, seed=3900, name="read_nothing")
    run = Run4(none)
    assert tuple(gc.kv_read_fp4(*run.dev, run.batch)[0].shape) == (0, 2, 64)
    w = W.build([33, 0], [7, 3], 4, 2, 64, seed=3901, name="read_refused")
    plain = H.DeviceRun(w)
    kp, vp, b = plain.k_pool, plain.v_pool, plain.batch
    good = torch.empty(w.k_new.shape, dtype=torch.bfloat16, device="cuda")
    for bad in (good[:-1], good.float(), good.cpu(), good.transpose(0, 1).contiguous().transpose(0, 1), np.zeros(3)):
        with pytest.raises((TypeError, ValueError)):
            gc.kv_read(kp, vp, b, k_out=bad)
        with pytest.raises((TypeError, ValueError)):
            gc.kv_read(kp, vp, b, v_out=bad)
    with pytest.raises(gc.GcError):
        gc.kv_read(kp, vp, b, k_out=good, v_out=good)
    with pytest.raises(gc.GcError):
        gc.kv_read(kp, vp, b, k_out=kp.view(-1)[:good.numel()].view(good.shape))
    with pytest.raises(gc.GcError):
        gc.kv_read_fp8(kp.view(torch.uint8).view(-1)[:kp.numel()].view(kp.shape), vp.view(torch.uint8).view(-1)[:vp.numel()].view(vp.shape),
                       b, float("inf"), 1.0)
    with pytest.raises(ValueError):
        gc.kv_read(kp, vp.transpose(2, 3).contiguous(), b)
