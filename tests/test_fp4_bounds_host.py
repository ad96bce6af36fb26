"""The bounds that attention over 4-bit pools is held to (CPU): scores moved by what the bound allows stay inside it, and what wrong
values, keys or buffers would give does not."""
import numpy as np
import pytest

import fp4_bounds as B
import fp4_reference as R


def inputs(seed, L=70, D=64, jump=0.0):
    rng = np.random.default_rng(seed)
    q = rng.standard_normal(D)
    k, v = (R.values(*map(np.asarray, _packed(rng.standard_normal((L, D))))) for _ in range(2))
    if jump:
        k = k * 0.015625
        k[L // 3] *= jump
    return q, k, v


def _packed(x):
    code, s = R.quantise(x)
    return R.pack(code), s


def attention(s, v):
    p = np.exp(s - s.max())
    return (p / p.sum()) @ v, s.max() + np.log(p.sum())


@pytest.mark.parametrize("jump", [0.0, 2.0 ** 12, 2.0 ** 20])
def test_moved_scores_stay_inside(jump):
    rng = np.random.default_rng(9)
    for seed in range(20):
        q, k, v = inputs(seed, jump=jump)
        o, lse, move, lse_move = B.row(q, k, v, 0.125)
        e = B.score_errors_of(q, k, 0.125)
        s = 0.125 * (k @ q)
        for i in range(20):
            d = e * (rng.choice([-1.0, 1.0], len(e)) if i % 2 else rng.uniform(-1, 1, len(e)))
            o2, lse2 = attention(s + d, v)
            assert np.all(np.abs(o2 - o) <= move + 1e-9) and abs(lse2 - lse) <= lse_move + 1e-9


def test_a_key_far_from_the_others_leaves_no_room():
    """The errors of its score are tens, but its weight is 1 or 0: the bound is far below what another key's value, a zero row or the
    mean of the values would give."""
    for seed in range(20):
        q, k, v = inputs(seed, jump=2.0 ** 20)
        assert B.score_errors_of(q, k, 0.125).max() > 1
        o, _, move, _ = B.row(q, k, v, 0.125)
        s = 0.125 * (k @ q)
        if abs(s[23]) < 100:   # (neither leads nor trails)
            continue
        assert move.max() < 1e-2
        wrong = v.mean(axis=0) if s[23] > 0 else v[23]
        assert np.any(np.abs(wrong - o) > 0.5 + move)
        if s[23] > 0:
            assert np.array_equal(o, v[23]) and np.any(np.abs(o) > 0.5 + move)


def test_values_replaced_by_other_rows_show():
    """What a tile's last values would be if other rows' outputs lay over them: most elements leave the bounds of the wide tiles' tests."""
    import test_gpu_fp4_second_pass as T
    for tiles in (1, 4):
        w = T.build([tiles], 128, 8, 2, 60, "jump")
        images = R.append(w, *R.pools(w))
        rows = {i: r[0] for i, r, _ in B.rows_of(w, images)}
        k4, v4 = R.values(images[0], images[2][..., 0]), R.values(images[1], images[2][..., 1])
        pos = np.arange(64 * tiles)
        k, v = (x[w.block_tables[0][pos // 16], 0, pos % 16] for x in (k4, v4))
        v = v.copy()
        v[-64:] = [rows[t * 8 + h] for t in range(16) for h in range(4)]
        for t in (40, 59):
            o, _, move, _ = B.row(R.rows_of(w.q)[t, 0], k[:64 * tiles - 59 + t], v[:64 * tiles - 59 + t], w.scale)
            bound = 2.0 ** -7 * (np.abs(v4[np.isfinite(v4)]).max() + np.abs(rows[t * 8])) + move
            assert np.mean(np.abs(o - rows[t * 8]) > bound) > 0.5
