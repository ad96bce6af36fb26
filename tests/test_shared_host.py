"""Shared-prefix attention on the CPU: refusals before any HIP call, workspace sizes, what the policy takes."""
import ctypes

import numpy as np
import pytest

import paper_2505_23970_amd as gc
from test_abi_host import HostBatch, geo


@pytest.fixture(scope="module")
def lib():
    return gc.load_library()


class HostShared:
    def __init__(self, first, lens, policy=1, dev=0x1000, groups=None):
        self.first = np.ascontiguousarray(first, np.int32)
        self.lens = np.ascontiguousarray(lens, np.int32)
        p = ctypes.POINTER(ctypes.c_int32)
        self.desc = gc.Shared(len(self.lens) if groups is None else groups, self.first.ctypes.data_as(p),
                              self.lens.ctypes.data_as(p), dev, dev, policy)


def size(lib, g, b, s, opts=None, fp8=0):
    out = ctypes.c_size_t(0)
    st = lib.gc_shared_prefix_workspace_size(ctypes.byref(g), ctypes.byref(b.desc), ctypes.byref(s.desc),
                                             ctypes.byref(opts) if opts is not None else None, fp8, ctypes.byref(out))
    return st, out.value


def run(lib, g, b, s, opts=None, scale=0.1, ptrs=(0x2000, 0x2000, 0x2000, 0x2000), ws=0x3000, ws_bytes=1 << 40, scales=None):
    q, kp, vp, out = ptrs
    head = (ctypes.byref(g), ctypes.byref(b.desc), ctypes.byref(s.desc) if s is not None else None,
            ctypes.byref(opts) if opts is not None else None, q, kp, vp)
    if scales is None:
        got = {getattr(lib, f"gc_shared_prefix_{n}")(*head, scale, out, None, ws, ws_bytes, None) for n in ("run", "attention")}
    else:
        got = {getattr(lib, f"gc_shared_prefix_{n}_fp8")(*head, *scales, scale, out, None, ws, ws_bytes, None)
               for n in ("run", "attention")}
    assert len(got) == 1
    return got.pop()


B = lambda: HostBatch([40, 35, 33, 8], [1, 2, 1, 1])  # noqa: E731
GOOD = lambda **k: HostShared([0, 3, 4], [32, 0], **k)  # noqa: E731


def test_groups_and_shared_lengths(lib):
    assert size(lib, geo(), B(), GOOD())[0] == 0
    for first, lens in (([0, 3, 5], [32, 0]), ([0, 3, 3], [32, 0]), ([1, 3, 4], [32, 0]), ([0, 5, 4], [32, 0]),
                        ([0, 3, 4], [30, 0]), ([0, 3, 4], [-16, 0]), ([0, 3, 4], [48, 0]), ([0, 3, 4], [32, 16]),
                        ([0, 1, 2, 3, 4, 4], [0, 0, 0, 0, 0])):
        s = HostShared(first, lens)
        assert size(lib, geo(), B(), s)[0] == -2, (first, lens)
        assert run(lib, geo(), B(), s) == -2
    assert size(lib, geo(), B(), HostShared([0, 4], [8], groups=0))[0] == -2
    assert size(lib, geo(), B(), GOOD(policy=2))[0] == -2
    s = GOOD()
    s.desc.reserved[5] = 1
    assert size(lib, geo(), B(), s)[0] == -2
    # more rows than the merge's launch has threads for
    big = HostBatch([64], [1 << 28])
    assert size(lib, geo(NB=1 << 30, maxb=1 << 25), big, HostShared([0, 1], [64]))[0] == -2
    # the shared pages must lie in the table row, also of a group without new tokens
    assert size(lib, geo(maxb=3), HostBatch([80, 8], [0, 1]), HostShared([0, 1, 2], [80, 0]))[0] == -4


def test_null_arguments_and_pointers(lib):
    assert run(lib, geo(), B(), None) == -1
    assert run(lib, geo(), B(), GOOD(dev=None)) == -1
    for k in range(4):
        ptrs = [0x2000] * 4
        ptrs[k] = None
        assert run(lib, geo(), B(), GOOD(), ptrs=ptrs) == -1
        ptrs[k] = 0x2008
        assert run(lib, geo(), B(), GOOD(), ptrs=ptrs) == -2
    assert run(lib, geo(), B(), GOOD(), ws=None) == -5
    assert run(lib, geo(), B(), GOOD(), ws=0x3008) == -5
    need = size(lib, geo(), B(), GOOD())[1]
    assert run(lib, geo(), B(), GOOD(), ws_bytes=need - 1) == -5
    s = GOOD()
    assert lib.gc_shared_prefix_workspace_size(ctypes.byref(geo()), ctypes.byref(B().desc), ctypes.byref(s.desc), None, 0, None) == -1
    s.desc.group_first_host = None
    assert size(lib, geo(), B(), s)[0] == -1
    assert lib.gc_shared_prefix_plan(ctypes.byref(geo()), ctypes.byref(B().desc), ctypes.byref(GOOD().desc), None, 0, 0x3000, 100, None) == -5


def test_options_and_scales(lib):
    for tiling in (gc.TILES_PREFILL, gc.TILES_SMALL, gc.TILES_WIDE):
        assert run(lib, geo(), B(), GOOD(), opts=gc.PlanOptions(0, tiling)) == -3
    assert run(lib, geo(), B(), GOOD(), opts=gc.PlanOptions(0, 9)) == -2
    for scale in (0.0, float("inf"), float("nan")):
        assert run(lib, geo(), B(), GOOD(), scale=scale) == -2
    assert run(lib, geo(), B(), GOOD(), scales=(0.0, 1.0)) == -2
    assert run(lib, geo(D=96), B(), GOOD()) == -3


def test_nothing_to_do(lib):
    empty = HostShared([0], [])
    assert run(lib, geo(), HostBatch([], []), empty) == 0
    assert size(lib, geo(), HostBatch([], []), empty) == (0, 0)
    assert run(lib, geo(), HostBatch([40, 40], [0, 0]), HostShared([0, 2], [32])) == 0


def plain_size(lib, g, b):
    out = ctypes.c_size_t(0)
    assert lib.gc_prefix_prefill_workspace_size(ctypes.byref(g), ctypes.byref(b.desc), None, ctypes.byref(out)) == 0
    return out.value


@pytest.mark.parametrize("P,n,first,lens,taken", [
    ([6000] * 16, [1] * 16, [0, 16], [5600], True),                # answers on one document
    ([6000] * 16, [1] * 16, [0, 16], [48], False),                 # three pages
    ([6000] * 3, [1] * 3, [0, 3], [5600], False),                  # 24 rows of a 128-row tile
    ([6000, 6000], [1, 0], [0, 2], [5600], False),                 # one request alone
    ([6000] * 4, [160] * 4, [0, 4], [5600], False),                # whole query tiles each: nothing to save
    ([6000] * 48, [20] * 48, [0, 48], [5600], True),               # query tiles five eighths full
    ([6000] * 48, [20] * 48, [0, 48], [640], False),               # their partial rows cost more
    ([6000] * 4 + [50], [160] * 4 + [1], [0, 4, 5], [5600, 0], False),
    ([6000] * 40, [1] * 40, [0, 1, 40], [5600, 5600], True),       # the second group
])
def test_what_the_policy_takes(lib, P, n, first, lens, taken):
    """A batch that is left to the plain attention has its workspace."""
    g, b = geo(Hq=64, Hkv=8, NB=100000, maxb=400), HostBatch(P, n)
    st, auto = size(lib, g, b, HostShared(first, lens, policy=gc.SHARE_AUTO))
    assert st == 0
    assert (auto != plain_size(lib, g, b)) == taken
    st, always = size(lib, g, b, HostShared(first, lens, policy=gc.SHARE_ALWAYS))
    assert st == 0 and always != plain_size(lib, g, b)
    if taken and len(lens) == 1:
        assert auto == always


def test_groups_of_the_binding():
    batch = gc.PagedBatch([40, 40], [1, 1], np.zeros((2, 4), np.int32), device="cpu")
    gc.SharedPrefixes(batch, np.array([2]), np.array([32]))
    for sizes, lens in (([2], [[32]]), ([1], [32]), ([2, 0], [32, 0]), ([3, -1], [32, 0]), ([2], [32, 0]), ([2], [16.5]),
                        ([2], np.array([(1 << 32) + 32])), (np.array([(1 << 32) + 2]), [32])):
        with pytest.raises(ValueError):
            gc.SharedPrefixes(batch, sizes, lens)
    batch = gc.PagedBatch([40, 40], [1, 1], [[1, 2, 3, 4], [1, 5, 3, 4]], device="cpu")
    gc.SharedPrefixes(batch, [2], [16])
    with pytest.raises(ValueError):
        gc.SharedPrefixes(batch, [2], [32])


def test_runs_of_more_places_than_32_bits_hold(lib):
    """48 requests of 2^31 - 113 cached tokens at 32768 heads: equal runs of 2^37 places, whose low 32 bits are all 0.
    More work than a launch holds; no division by the truncated length."""
    g = geo(Hq=32768, Hkv=32768, NB=1 << 20, maxb=1 << 27)
    b = HostBatch([2 ** 31 - 113] * 48, [1] * 48)
    assert size(lib, g, b, HostShared([0, 48], [16], policy=gc.SHARE_ALWAYS))[0] == -2
    assert size(lib, g, b, HostShared([0, 48], [16], policy=gc.SHARE_AUTO)) == (0, plain_size(lib, g, b))


def test_more_merge_workgroups_than_a_launch_takes(lib):
    """20 million rows beside one of 312501 chunks: the merge deals a row's chunks to eight thread groups, a workgroup a
    row at d = 128. Refused before the plan and the items are on the stream; half the rows fit."""
    for requests, status in ((200000, -2), (100000, 0)):
        b = HostBatch([64] * requests + [20_000_000], [100] * requests + [1])
        g = geo(Hq=1, Hkv=1, NB=1 << 20, maxb=1 << 21)
        assert size(lib, g, b, HostShared([0, requests + 1], [16]), gc.PlanOptions(1, 0))[0] == status


@pytest.mark.parametrize("sizes,lens,n,taken", [
    ([1] * 513, [640] * 513, 1, False),                # requests alone: 304 us, taken 372
    ([2] * 520, [64] * 520, 1, False),                 # four pages of two requests each: 175, 219
    ([1] * 520, [512] * 520, 20, False),               # query tiles of one request: 477, 1204
    ([2] * 520, [1008] * 520, 20, False),              # 1441, 2330
    ([2] * 520 + [1] * 3000, [2000] * 520 + [2000] * 3000, [1] * 1040 + [0] * 3000, True),   # members without new tokens
    ([2] * 520, [2000] * 520, 1, True),                # 1504, 1019
    ([8] * 520, [1024] * 520, 1, True),                # 2648, 1217
    ([100] + [1] * 600, [8192] + [16] * 600, 1, True),   # one group gains more than the others lose: 229, 155
    ([20] + [1] * 600, [1024] + [512] * 600, 1, False),  # and less: 297, 368
])
def test_what_the_policy_takes_of_many_groups(lib, sizes, lens, n, taken):
    """More groups than the policy chooses from one by one: all or none (us at 64 and 8 heads, d = 128, bf16)."""
    P = np.repeat(lens, sizes) + 160
    g, b = geo(Hq=64, Hkv=8, NB=1000000, maxb=600), HostBatch(P, np.broadcast_to(n, P.shape))
    first = np.concatenate([[0], np.cumsum(sizes)])
    st, auto = size(lib, g, b, HostShared(first, lens, policy=gc.SHARE_AUTO))
    assert st == 0
    assert (auto != plain_size(lib, g, b)) == taken
    if taken:
        assert auto == size(lib, g, b, HostShared(first, lens, policy=gc.SHARE_ALWAYS))[1]


def test_a_batch_past_the_launch_limit_is_left_to_the_plain_attention(lib):
    """52500 questions of 20 tokens on one document: more rows than the merge's launch takes, which the plain attention
    does not have. The policy leaves it the batch; taken whatever it costs, it is refused."""
    g, b = geo(Hq=64, Hkv=8, NB=1 << 20, maxb=1 << 12), HostBatch([33000] * 52500, [20] * 52500)
    assert size(lib, g, b, HostShared([0, 52500], [32768], policy=gc.SHARE_AUTO)) == (0, plain_size(lib, g, b))
    assert size(lib, g, b, HostShared([0, 52500], [32768], policy=gc.SHARE_ALWAYS))[0] == -2
