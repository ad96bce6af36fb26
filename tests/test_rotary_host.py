"""The rotary append on the CPU: refusals before any HIP call, the table, and the reference itself."""
import ctypes

import numpy as np
import pytest

import paper_2505_23970_amd as gc
import rotary_reference as RR
from test_abi_host import HostBatch, geo


@pytest.fixture(scope="module")
def lib():
    return gc.load_library()


def status(lib, g=None, b=None, rot=None, rows=None, q_out=0x900000, pools=(0x2000, 0x2000), **change):
    r = dict(table_dev=0x1000, num_positions=64, rotary_dim=64, pairs=0)
    n = dict(q=0x100000, k=0x200000, v=0x300000, q_stride=8 * 128, k_stride=256, v_stride=256)
    r.update({k: v for k, v in change.items() if k in r})
    n.update({k: v for k, v in change.items() if k in n})
    rot = gc.Rotary(**r) if rot is None else rot
    rows = gc.NewRows(**n) if rows is None else rows
    g = g or geo()
    b = b or HostBatch([4], [3])
    args = (ctypes.byref(g), ctypes.byref(b.desc), ctypes.byref(rot), ctypes.byref(rows), q_out)
    plain = lib.gc_kv_append_rotary(*args, *pools, None)
    assert lib.gc_kv_append_rotary_fp8(*args, 0.5, 0.5, *pools, None) == plain
    return plain


# a workable call cannot be made here (it would launch): every case below changes one thing of it
def test_null_arguments(lib):
    for name in ("table_dev", "k", "v", "q"):
        assert status(lib, **{name: None}) == -1, name
    assert status(lib, q_out=None) == -1
    assert status(lib, pools=(None, 0x2000)) == -1
    assert status(lib, pools=(0x2000, None)) == -1
    assert status(lib, b=HostBatch([4], [3], fake_dev=False)) == -1
    g, b = geo(), HostBatch([4], [3])
    assert lib.gc_kv_append_rotary(ctypes.byref(g), ctypes.byref(b.desc), None, ctypes.byref(gc.NewRows()), None, 0x2000, 0x2000, None) == -1
    assert lib.gc_kv_append_rotary(ctypes.byref(g), ctypes.byref(b.desc), ctypes.byref(gc.Rotary()), None, None, 0x2000, 0x2000, None) == -1


def test_shapes(lib):
    for R in (0, 8, 24, 72, 144, -16):
        assert status(lib, rotary_dim=R) == -2, R
    assert status(lib, pairs=2) == -2
    assert status(lib, num_positions=6) == -2          # positions 4 .. 6
    assert status(lib, b=HostBatch([4, 60], [3, 5])) == -2
    rot = gc.Rotary(0x1000, 64, 64, 0)
    rot.reserved[4] = 1
    assert status(lib, rot=rot) == -2
    assert status(lib, g=geo(D=96)) == -3
    assert status(lib, b=HostBatch([4], [-3])) == -2
    # more workgroups than a launch has threads for
    assert status(lib, g=geo(NB=1 << 30, maxb=1 << 26), b=HostBatch([0], [(1 << 30) - 64]), num_positions=1 << 30,
                  k=1 << 50, v=1 << 51, q=1 << 52, q_out=1 << 53) == -3


def test_strides_alignment_and_overlap(lib):
    assert status(lib, q_stride=8 * 128 - 8) == -2
    assert status(lib, k_stride=260) == -2
    assert status(lib, v_stride=248) == -2
    assert status(lib, v_stride=1 << 40) == -2
    for name in ("q", "k", "v", "table_dev"):
        assert status(lib, **{name: 0x100008}) == -2, name
    assert status(lib, q_out=0x900008) == -2
    assert status(lib, q_out=0x100010) == -2                       # over q
    assert status(lib, q_out=0x100000, q_stride=2048) == -2        # in place over strided rows
    assert status(lib, q_out=0x200000) == -2                       # over k
    assert status(lib, q_out=0x300200) == -2                       # over v
    assert status(lib, q_out=0x1100) == -2                         # over the table
    assert status(lib, q_out=0x20000) == -2                        # over the pools


def test_scales(lib):
    g, b = geo(), HostBatch([4], [3])
    rot, rows = gc.Rotary(0x1000, 64, 64, 0), gc.NewRows(None, 0x200000, 0x300000, 0, 256, 256)
    for ks, vs in ((0.0, 1.0), (1.0, float("nan")), (1e-39, 1.0)):
        assert lib.gc_kv_append_rotary_fp8(ctypes.byref(g), ctypes.byref(b.desc), ctypes.byref(rot), ctypes.byref(rows),
                                           None, ks, vs, 0x2000, 0x2000, None) == -2


def test_nothing_to_do(lib):
    assert status(lib, b=HostBatch([4], [0])) == 0
    assert status(lib, b=HostBatch([], [])) == 0


def test_table_holds_the_angles():
    t = gc.rotary_table(200001, 16, base=10000.0, device="cpu").numpy()
    assert t.shape == (200001, 8, 2) and t.dtype == np.float32
    for p in (0, 1, 77, 131072, 200000):
        for j in range(8):
            angle = p * 10000.0 ** (-2.0 * j / 16)
            assert abs(t[p, j, 0] - np.cos(angle)) <= 2.0 ** -24 and abs(t[p, j, 1] - np.sin(angle)) <= 2.0 ** -24
    own = gc.rotary_table(9, 16, inv_freq=np.arange(8) / 7.0, amplitude=1.25, device="cpu").numpy()
    assert np.allclose(own[5, :, 1], 1.25 * np.sin(5 * np.arange(8) / 7.0), rtol=0, atol=2.0 ** -23)
    for bad in (dict(rotary_dim=15), dict(rotary_dim=0), dict(positions=-1), dict(inv_freq=np.ones(7))):
        with pytest.raises(ValueError):
            gc.rotary_table(**{**dict(positions=4, rotary_dim=16, device="cpu"), **bad})


@pytest.mark.parametrize("interleaved", [False, True])
def test_reference_turns_as_complex_numbers_do(interleaved):
    """Pairs as complex numbers times exp(i angle), and the score of two rotated vectors goes by the
    difference of their positions alone."""
    rng = np.random.default_rng(3)
    table = gc.rotary_table(64, 32, device="cpu").numpy().astype(np.float64)
    x = rng.standard_normal((5, 2, 48))
    pos = np.array([0, 3, 9, 33, 63])
    y, mag = RR.rotate(x, pos, table, interleaved)
    pairs = (lambda v: v[..., 0:32:2] + 1j * v[..., 1:32:2]) if interleaved else (lambda v: v[..., :16] + 1j * v[..., 16:32])
    turn = (table[pos, :, 0] + 1j * table[pos, :, 1])[:, None, :]
    assert np.allclose(pairs(y), pairs(x) * turn, atol=1e-12)
    assert np.array_equal(y[..., 32:], x[..., 32:]) and not mag[..., 32:].any()
    a, b = rng.standard_normal((1, 1, 32)), rng.standard_normal((1, 1, 32))
    dot = lambda p, q: float((RR.rotate(a, np.array([p]), table, interleaved)[0] * RR.rotate(b, np.array([q]), table, interleaved)[0]).sum())  # noqa: E731
    assert abs(dot(40, 33) - dot(8, 1)) < 1e-5   # (the table is fp32)
