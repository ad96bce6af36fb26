"""How exact the scores of the attention over 4-bit pools are (GPU): single scores against the bound that the header gives, and batches
with scores of tens of thousands, whose rows are held to what each row's own scores may be off by."""
import numpy as np
import pytest

import fp4_bounds as B
import fp4_reference as R
from paper_2505_23970_amd import workloads as W
from test_gpu_fp4 import Run4, appended, numbers

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu_ready():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2505_23970_amd as gc
    gc.load_library()


def one_key_each(D, seed):
    """Requests of one token on nothing: their log-sum-exps are single scores. Queries with full mantissas; in a third of the rows normal numbers, in
    a third one leading element in every group of eight and the others smaller by 2^5 to 2^14, in a third elements of any of 2^20
    magnitudes; keys of every code and several scales, in half of the rows with the query's signs, so that what is dropped adds up."""
    rng = np.random.default_rng(seed)
    w = W.build([0] * 120, [1] * 120, 16, 2, D, seed=5200 + seed, values="unit", name=f"fp4_scores_d{D}")
    shape = w.q.shape
    q = rng.uniform(1, 2, shape)
    lead = np.where(np.arange(D) % 8 == rng.integers(0, 8, shape[:2] + (1,)), 0, -rng.integers(5, 15, shape))
    kind = np.arange(120)[:, None, None] % 3
    q = np.where(kind == 0, rng.standard_normal(shape), np.where(kind == 1, q * 2.0 ** lead, q * 2.0 ** -rng.integers(0, 20, shape)))
    q = np.where(rng.random(shape) < 0.5, -q, q)
    k = R.MAGNITUDES[rng.integers(1, 8, (120, 2, D))] * 2.0 ** np.repeat(rng.integers(-3, 3, (120, 2, D // 32)), 32, axis=-1)
    k[..., ::32] = np.where(k[..., ::32] == 0, 1, k[..., ::32])
    sign = np.where(rng.random(k.shape) < 0.5, -1.0, 1.0)
    same = np.arange(120)[:, None, None] % 2 == 0   # (every head of the group then has the signs of its first)
    sign = np.where(same, np.sign(q[:, ::8]), sign)
    q = np.where(same, np.abs(q) * np.repeat(np.sign(q[:, ::8]), 8, axis=1), q)
    w.q[:], w.k_new[:] = W.f32_to_bf16_bits(q.astype(np.float32)), W.f32_to_bf16_bits((k * sign).astype(np.float32))
    return w


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tiling", [1, 2, 3], ids=["prefill", "small", "wide"])
def test_single_scores(tiling, D):
    w = one_key_each(D, D)
    run, _ = appended(w)
    out, lse = run.attention(tiling=tiling)
    images = run.images()
    k4, v4 = R.values(images[0], images[2][..., 0]), R.values(images[1], images[2][..., 1])
    blocks = w.block_tables[:, 0]
    q, got, o = R.rows_of(w.q), numbers(lse), numbers(out)
    for r in range(w.batch):
        for h in range(16):
            k = k4[blocks[r], h // 8, 0]
            s = w.scale * float(k @ q[r, h])
            e = float(B.score_errors_of(q[r, h], k[None], w.scale)[0])
            assert abs(got[r, h] - s) <= e + 2.0 ** -22 * abs(s), (r, h, got[r, h], s, e)
            assert np.array_equal(o[r, h], v4[blocks[r], h // 8, 0])   # (a weight of 1)


def jumps(n, D, last):
    """Score jumps to tens of thousands, up or down, that few rows see in their last keys, or many in earlier ones."""
    w = W.build([300], [n], 4, 2, D, seed=2750 + n, values="unit", name=f"fp4_far_jumps_{n}_{last}")
    scaled = lambda x, f: W.f32_to_bf16_bits(W.bf16_bits_to_f32(x) * np.float32(f))  # noqa: E731
    w.k_prefix[:], w.k_new[:] = scaled(w.k_prefix, 0.01), scaled(w.k_new, 0.01)
    if last:
        w.k_new[n - 3] = scaled(w.k_new[n - 3], 900000.0)
    else:
        w.k_prefix[290] = scaled(w.k_prefix[290], 900000.0)
    return w.finish()


def check_jumps(w, out, lse, images, first):
    """Every row within its own bound; of the rows that see the jump (tokens from `first` on) nearly all have it lead or trail
    by far, so that their bounds are those of ordinary rows."""
    moves = B.check_rows(w, out, lse, images)
    see = [m for i, m in moves.items() if i // w.num_q_heads >= first]
    assert np.mean(np.array(see) < 2.0 ** -7) >= 0.75


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [35, 45, 61, 110])
@pytest.mark.parametrize("tiling", [1, 2, 3], ids=["prefill", "small", "wide"])
def test_far_jumps(tiling, n, D):
    for last in (True, False):
        w = jumps(n, D, last)
        run, _ = appended(w)
        for split in (None, -1, 2):
            out, lse = run.attention(tiling=tiling, split=split)
            check_jumps(w, out, lse, run.images(), n - 3 if last else 0)
