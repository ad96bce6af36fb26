"""4-bit pools and reading back on the CPU: the reference against hand-made blocks, and refusals before any HIP call."""
import ctypes

import numpy as np
import pytest

import fp4_reference as R
import paper_2505_23970_amd as gc
from paper_2505_23970_amd import workloads as W
from test_abi_host import HostBatch, geo


def block(*head):
    x = np.zeros(32)
    x[:len(head)] = head
    return x


def test_hand_made_blocks():
    # s = 1: every number, ties to the even code (0.25 -> 0, 0.75 -> 1, 1.25 -> 1, 1.75 -> 2, 2.5 -> 2, 3.5 -> 4, 5 -> 4)
    x = block(6, -4, 0.25, 0.75, -1.25, 1.75, 2.5, 3.5, 5.0, 5.001, -0.0, 0.26)
    code, s = R.quantise(x)
    assert s[0] == 127
    assert code[:12].tolist() == [7, 14, 0, 2, 10, 4, 4, 6, 6, 7, 8, 1]
    # just below 7 s stays and saturates, 7 s takes the next scale
    assert R.quantise(block(6.97))[1][0] == 127 and R.quantise(block(6.97))[0][0] == 7
    assert R.quantise(block(7.0))[1][0] == 128 and R.quantise(block(7.0))[0][0] == 6   # 3.5 -> 4
    # the ends of the range; zeros; infinities; NaN
    assert R.quantise(block(0.0))[1][0] == 3 and R.quantise(block(2.0 ** -130))[1][0] == 3
    assert R.quantise(block(3.3e38))[1][0] == 252 and R.quantise(block(3.3e38))[0][0] == 7
    assert R.quantise(block(np.inf, 1.0))[1][0] == 252 and R.quantise(block(-np.inf, 1.0))[0][:2].tolist() == [15, 0]
    code, s = R.quantise(block(1.0, np.nan))
    assert s[0] == 255 and not code.any() and np.isnan(R.values(R.pack(code), s)).all()


def test_scales_and_idempotence():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((400, 64)) * 2.0 ** rng.integers(-140, 127, (400, 1))
    x = W.bf16_bits_to_f32(W.f32_to_bf16_bits(x.astype(np.float32))).astype(np.float64)
    code, s = R.quantise(x)
    for row, c in zip(x.reshape(-1, 32), s.reshape(-1)):
        assert c == R.scale_code(np.abs(row).max())
    y = R.values(R.pack(code), s)
    again, t = R.quantise(y)
    assert np.array_equal(again, code) and np.array_equal(t, s)
    # off by at most half a step (s at the largest numbers), and what rounds there is near them
    step = np.repeat(2.0 ** (s.astype(np.float64) - 127), 32, axis=-1)
    ok = np.repeat(s < 252, 32, axis=-1)
    assert np.all(np.abs(y - x)[ok] <= np.maximum(step / 4, np.abs(x) / 4)[ok])


STATUS_CALLS = ("append", "rotary", "read", "read_fp8", "read_fp4", "run")


def call(lib, name, g, b, k=0x200000, v=0xA00000, s=0xC00000, k_new=0x10000, v_new=0x20000, scales=(0.5, 0.5),
         scale=0.1, ws=0x400000, ws_bytes=1 << 30, q=0x500000, out=0x600000):
    g, d = ctypes.byref(g), ctypes.byref(b.desc)
    if name == "append":
        return lib.gc_kv_append_fp4(g, d, k_new, v_new, k, v, s, None)
    if name == "rotary":
        rot = gc.Rotary(0x1000, 64, 64, 0)
        rows = gc.NewRows(None, k_new, v_new, 0, 256, 256)
        return lib.gc_kv_append_rotary_fp4(g, d, ctypes.byref(rot), ctypes.byref(rows), None, k, v, s, None)
    if name == "read":
        return lib.gc_kv_read(g, d, k, v, k_new, v_new, None)
    if name == "read_fp8":
        return lib.gc_kv_read_fp8(g, d, k, v, *scales, k_new, v_new, None)
    if name == "read_fp4":
        return lib.gc_kv_read_fp4(g, d, k, v, s, k_new, v_new, None)
    return lib.gc_prefix_prefill_run_fp4(g, d, None, q, k, v, s, scale, out, None, ws, ws_bytes, None)


@pytest.fixture(scope="module")
def lib():
    return gc.load_library()


# a workable call cannot be made here (it would launch): every case below changes one thing of it
@pytest.mark.parametrize("name", STATUS_CALLS)
def test_null_arguments_and_shapes(lib, name):
    g, b = geo(), HostBatch([4], [3])
    for missing in ("k", "v"):
        assert call(lib, name, g, b, **{missing: None}) == -1, missing
    if name in ("append", "rotary", "read_fp4", "run"):
        assert call(lib, name, g, b, s=None) == -1
    if name != "run":
        assert call(lib, name, g, b, k_new=None) == -1 and call(lib, name, g, b, v_new=None) == -1
    else:
        assert call(lib, name, g, b, q=None) == -1 and call(lib, name, g, b, out=None) == -1
        assert call(lib, name, g, b, ws=None) == -5 and call(lib, name, g, b, ws_bytes=16) == -5
        assert call(lib, name, g, b, ws=0x400008) == -5
        for bad in (0.0, -1.0, float("nan"), float("inf")):
            assert call(lib, name, g, b, scale=bad) == -2
        assert call(lib, name, g, b, q=0x500008) == -2 and call(lib, name, g, b, out=0x600002) == -2
    assert call(lib, name, g, HostBatch([4], [3], fake_dev=False)) == -1
    assert call(lib, name, geo(D=96), b) == -3 and call(lib, name, geo(S=32), b) == -3
    assert call(lib, name, geo(Hq=7), b) == -2 and call(lib, name, g, HostBatch([4], [-1])) == -2
    assert call(lib, name, g, HostBatch([4], [200])) == -4                    # past the table row
    assert call(lib, name, g, HostBatch([4], [0])) == 0 and call(lib, name, g, HostBatch([], [])) == 0


@pytest.mark.parametrize("name", STATUS_CALLS)
def test_alignment(lib, name):
    g, b = geo(), HostBatch([4], [3])
    for which in ("k", "v", "s"):
        if which == "s" and name in ("read", "read_fp8"):
            continue
        assert call(lib, name, g, b, **{which: 0x200008}) == -2, which
    if name != "run":
        assert call(lib, name, g, b, k_new=0x10008) == -2 and call(lib, name, g, b, v_new=0x20004) == -2


@pytest.mark.parametrize("name", ["read", "read_fp8", "read_fp4"])
def test_outputs_over_inputs_are_refused(lib, name):
    g, b = geo(), HostBatch([4], [3])
    assert call(lib, name, g, b, v_new=0x10000) == -2 and call(lib, name, g, b, v_new=0x10000 + 3 * 512 - 16) == -2
    assert call(lib, name, g, b, k_new=0x200000) == -2 and call(lib, name, g, b, v_new=0x200000 - 16) == -2
    pool = {"read": 2, "read_fp8": 1, "read_fp4": 0.5}[name] * 64 * 2 * 16 * 128
    assert call(lib, name, g, b, k_new=0x200000 + int(pool) - 16) == -2
    if name == "read_fp4":
        assert call(lib, name, g, b, s=0x10000) == -2


@pytest.mark.parametrize("name", ["append", "rotary"])
def test_written_pools_over_each_other_are_refused(lib, name):
    g, b = geo(), HostBatch([4], [3])
    pool, scales = 64 * 2 * 16 * 64, 64 * 2 * 16 * 8
    for over in (dict(v=0x200000), dict(v=0x200000 + pool - 16), dict(s=0x200000 + pool - 16), dict(s=0x200000 - scales + 16),
                 dict(s=0xA00000 + pool - 16), dict(s=0xA00000 - scales + 16)):
        assert call(lib, name, g, b, **over) == -2, over


@pytest.mark.parametrize("name", ["append", "rotary", "read", "read_fp8", "read_fp4"])
def test_more_work_than_a_launch_holds(lib, name):
    g = geo(Hkv=2, NB=1 << 28, maxb=1 << 26)
    b = HostBatch([0], [(1 << 30) - 64])
    status = call(lib, name, g, b, k=1 << 50, v=1 << 51, s=1 << 52, k_new=1 << 53, v_new=1 << 54)
    assert status == (-2 if name == "rotary" else -3)   # (its table has 64 rows)


def test_scales_of_8_bit_reads(lib):
    for ks, vs in ((0.0, 1.0), (1.0, float("nan")), (1e-39, 1.0)):
        assert call(lib, "read_fp8", geo(), HostBatch([4], [3]), scales=(ks, vs)) == -2


def test_rotated_queries_over_the_scales_are_refused(lib):
    g, b = geo(), HostBatch([4], [3])
    rot = gc.Rotary(0x1000, 64, 64, 0)
    rows = gc.NewRows(0x100000, 0x10000, 0x20000, 8 * 128, 256, 256)
    for q_out in (0x800000, 0x800000 + 64 * 2 * 16 * 8 - 16):
        assert lib.gc_kv_append_rotary_fp4(ctypes.byref(g), ctypes.byref(b.desc), ctypes.byref(rot), ctypes.byref(rows), q_out,
                                           0x200000, 0x400000, 0x800000, None) == -2


def test_allocated_pools_hold_zeros():
    k, v, s = gc.alloc_pools_fp4(3, 2, 64, device="cpu")
    assert k.shape == v.shape == (3, 2, 16, 32) and s.shape == (3, 2, 16, 2, 2)
    assert not R.values(k.numpy(), s.numpy()[..., 0]).any() and not R.values(v.numpy(), s.numpy()[..., 1]).any()
    with pytest.raises(ValueError):
        gc.alloc_pools_fp4(3, 2, 48, device="cpu")
