"""Attention over 4-bit pools whose weights pass 2^100, or are no numbers, which takes a work item through a second pass (GPU): wide
tiles with rows in all eight wavefronts, items that end on every one of the three value buffers, in one piece and split, in plain and
in resident launches. Rows that the cause has nothing to do with are what they are without it."""
import numpy as np
import pytest

import fp4_bounds as B
from paper_2505_23970_amd import workloads as W
from test_gpu_fp4 import appended, numbers

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu_ready():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2505_23970_amd as gc
    gc.load_library()


# One element of the keys leads the rows of the later half of the tokens to the last 64 keys, another grows from tile to tile.
LAST, GROWS = 8, 17
GROWTH = (0, 1, 2, 3, 4, 6, 8, 12)


def build(tiles, D, Hq, Hkv, tokens, why, batch=1, seed=0):
    """Requests of `tokens` new tokens, one wide tile each, over tiles[r % len] tiles of 64 keys. The rows of the later half of the tokens
    have most of their weight on the last tile. why: "nan": NaN in one query of the first wavefront's rows; "jump": queries
    among the first quarter of the tokens, in one head, whose scores pass the tile before by more than 2^100 in weight; None:
    neither, with the same other queries."""
    tiles = [tiles[r % len(tiles)] for r in range(batch)]
    w = W.build([64 * t - tokens for t in tiles], [tokens] * batch, Hq, Hkv, D, seed=5000 + seed, values="unit",
                name=f"fp4_second_{D}_{Hq}_{Hkv}_{tiles[:6]}_{why}")
    g = Hq // Hkv
    q, kp, kn = (W.bf16_bits_to_f32(x).copy() for x in (w.q, w.k_prefix, w.k_new))
    q[..., LAST] = q[..., GROWS] = 0
    for r, t in enumerate(tiles):
        cu, P = int(w.cu_new_lens[r]), int(w.prefix_lens[r])
        q[cu + tokens // 2:cu + tokens, :, LAST] = 24.0
        k = np.concatenate([kp[int(w.cu_prefix_lens[r]):int(w.cu_prefix_lens[r]) + P], kn[cu:cu + tokens]])
        k[..., LAST] = k[..., GROWS] = 0
        k[64 * (t - 1):, :, LAST] = 4.0
        k[np.arange(t) * 64 + 3, :, GROWS] = np.array(GROWTH[:t], np.float32)[:, None]
        kp[int(w.cu_prefix_lens[r]):int(w.cu_prefix_lens[r]) + P], kn[cu:cu + tokens] = k[:P], k[P:]
        if why == "jump":
            q[cu:cu + tokens // 4, 0::g, GROWS] = 1024.0
        if why == "nan":
            q[cu + 1, 0::g, 5] = np.nan
    w.q[:], w.k_prefix[:], w.k_new[:] = W.f32_to_bf16_bits(np.nan_to_num(q)), W.f32_to_bf16_bits(kp), W.f32_to_bf16_bits(kn)
    w.q[np.isnan(q)] = W.BF16_NAN
    return w.finish()


def check(w, why, tiling, split, tokens, sampled=None):
    Hq, g = w.num_q_heads, w.num_q_heads // w.num_kv_heads
    run, _ = appended(w)
    out, lse = run.attention(tiling=tiling, split=split)
    moves = B.check_rows(w, out, lse, run.images(), tokens=sampled)
    # (what the bound allows the scores of ordinary rows is far below what other rows' values would change)
    ordinary = [m for i, m in moves.items() if i // Hq % tokens >= tokens // 2]
    assert max(ordinary) < 2.0 ** -5, max(ordinary)
    nan = np.zeros(out.shape[:2], bool)
    if why == "nan":
        nan.reshape(w.batch, tokens, Hq)[:, 1, 0::g] = True
    assert np.array_equal(np.isnan(numbers(out)), np.broadcast_to(nan[..., None], out.shape))


WIDE = [(64, 8, 2, 60), (128, 8, 2, 60), (128, 16, 1, 16), (64, 10, 2, 50)]   # D, Hq, Hkv, tokens: 240 to 256 rows


@pytest.mark.parametrize("D,Hq,Hkv,tokens", WIDE)
@pytest.mark.parametrize("why", ["nan", "jump"])
def test_wide_items_in_one_piece(why, D, Hq, Hkv, tokens):
    for tiles in range(1, 8):
        check(build([tiles], D, Hq, Hkv, tokens, why, seed=tiles), why, 3, -1, tokens)


@pytest.mark.parametrize("D,Hq,Hkv,tokens", WIDE)
@pytest.mark.parametrize("why", ["nan", "jump"])
def test_wide_items_of_split_rows(why, D, Hq, Hkv, tokens):
    for chunk in range(1, 5):
        check(build([2 * chunk], D, Hq, Hkv, tokens, why, seed=10 + chunk), why, 3, chunk, tokens)


@pytest.mark.parametrize("why", ["nan", "jump"])
def test_128_row_tiles(why):
    """The same with two 128-row tiles a request."""
    for tiles in (1, 2, 3, 4):
        check(build([tiles], 128, 8, 2, 60, why, seed=20 + tiles), why, 1, -1, 60)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("why", ["nan", "jump"])
def test_resident_launch(why, D):
    """Two rounds of wide items and more, from the queues: the next item's copies follow the second pass of the last."""
    import torch
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    w = build([1, 2, 3, 4, 5, 6, 7], D, 32, 8, 60, why, batch=-(-2 * cus // 8) + 5, seed=30)
    check(w, why, 3, -1, 60, sampled=(0, 1, 14, 33, 47, 59))


@pytest.mark.parametrize("D", [64, 128])
def test_rows_beside_a_nan_are_those_of_the_clean_run(D):
    """Rows 128 to 255 of an item with a NaN query among its first rows, against the same batch without it: off by the rounding of the
    weights, which the second pass takes relative to other offsets, and of the output."""
    import gpu_helpers as H
    for tiles in range(1, 7):
        clean, bad = (build([tiles], D, 8, 2, 60, why, seed=40 + tiles) for why in (None, "nan"))
        a, b = (numbers(appended(w)[0].attention(tiling=3, split=-1)[0])[32:] for w in (clean, bad))
        vmax = float(np.abs(W.bf16_bits_to_f32(np.concatenate([clean.v_new.ravel(), clean.v_prefix.ravel()]))).max()) * 2
        assert np.all(np.abs(a - b) <= 2 * H.derived_bound(a, vmax)), tiles
