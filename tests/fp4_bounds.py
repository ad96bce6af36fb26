"""Attention over 4-bit pools in float64, row by row, with how far the scores' own errors may move each output.

A score of the kernels is off by at most e (score_errors_of). With p the exact weights and o the exact output, scores off by d_k,
|d_k| <= e_k, give
    o' - o = sum_k p_k (exp(d_k - d) - 1) (v_k - o) / sum_k p_k exp(d_k - d)
for any d, as adding one number to all scores changes nothing. With d = 0, and with d = d_c for the key c of the largest weight
(whose term is then 0, the others' exponents at most e_k + e_c), |o' - o| is bounded, and the smaller of the two bounds holds. A key
that leads or trails all others by more than the errors leaves next to nothing of the bound, however large its own error is."""
from __future__ import annotations

import numpy as np

import fp4_reference as R
import gpu_helpers as H


def score_errors_of(q, k, scale):
    """Most that the scores of a query row q [D] with keys k [L][D] may be off by. The products q k of eight neighbouring elements are
    added on a grid of 2^-13 of the largest one's power of two (of twice that where that key's code is 0.5), towards zero: each of the seven
    others loses less than 2^-12 of the largest. The query's second part, at most 2^-4 of the first, loses as much of its own
    terms. Splitting the query adds 2^-22 of the row's largest per element. fp32 sums, the scale and the offset round at 2^-24 of the sum
    of magnitudes, a few times."""
    terms = np.abs(q * k)
    group = terms.reshape(len(k), -1, 8).max(axis=-1).sum(axis=-1)
    return scale * (7 * 2.0 ** -12 * (1 + 2.0 ** -4) * group + 2.0 ** -22 * np.abs(q).max() * np.abs(k).sum(axis=-1)
                    + 2.0 ** -21 * terms.sum(axis=-1))


def moved(p, e, v, o):
    """Bound on |o' - o| [D] by scores off by up to e [L] (weights p [L], values v [L][D])."""
    best = None
    away = np.abs(v - o)
    for c in (None, int(np.argmax(p))):
        x = e if c is None else np.where(np.arange(len(p)) == c, 0.0, e + e[c])
        with np.errstate(over="ignore"):
            b = (p * np.expm1(x)) @ away / (p * np.exp(-x)).sum()
        best = b if best is None else np.minimum(best, b)
    return best


def row(q, k, v, scale):
    """(output [D], log-sum-exp, bound on the output's move [D], bound on the log-sum-exp's) of one query row."""
    s = scale * (k @ q)
    e = score_errors_of(q, k, scale)
    top = s.max()
    p = np.exp(s - top)
    total = p.sum()
    p /= total
    o = p @ v
    i = int(np.argmax(s + e))
    up = s[i] + e[i] + np.log(np.exp(s + e - s[i] - e[i]).sum())
    j = int(np.argmax(s - e))
    down = s[j] - e[j] + np.log(np.exp(s - e - s[j] + e[j]).sum())
    lse = top + np.log(total)
    return o, lse, moved(p, e, v, o), max(up - lse, lse - down)


def rows_of(w, images, tokens=None, heads=None):
    """For every (request, token of the request, head) asked for: (index into [T * Hq], row(..), largest value magnitude)."""
    k4, v4 = R.values(images[0], images[2][..., 0]), R.values(images[1], images[2][..., 1])
    g = w.num_q_heads // w.num_kv_heads
    q = R.rows_of(w.q)
    for r in range(w.batch):
        P, n, cu = int(w.prefix_lens[r]), int(w.new_lens[r]), int(w.cu_new_lens[r])
        pos = np.arange(P + n)
        k = k4[w.block_tables[r][pos // 16], :, pos % 16].transpose(1, 0, 2)      # [Hkv][L][D]
        v = v4[w.block_tables[r][pos // 16], :, pos % 16].transpose(1, 0, 2)
        for t in range(n) if tokens is None else tokens:
            seen = P + t + 1
            for h in range(w.num_q_heads) if heads is None else heads:
                if np.isnan(q[cu + t, h]).any():
                    continue
                yield (cu + t) * w.num_q_heads + h, row(q[cu + t, h], k[h // g, :seen], v[h // g, :seen], w.scale), np.abs(v[h // g, :seen]).max()


def check_rows(w, out, lse, images, tokens=None, heads=None):
    """Every row asked for (all; rows of NaN queries left out) within derived_bound and what its scores' errors may move; the log-sum-exps
    likewise. Returns the outputs' moves, largest element of each row over the largest value, by row index."""
    T, Hq, D = w.q.shape
    got, got_lse = H.from_dev_f32(out).reshape(T * Hq, D), H.from_dev_f32(lse).reshape(T * Hq)
    moves = {}
    for i, (o, ref_lse, move, lse_move), vmax in rows_of(w, images, tokens, heads):
        bad = ~(np.abs(got[i] - o) <= H.derived_bound(o, vmax) + move)
        assert not bad.any(), f"token {i // Hq} head {i % Hq}: {got[i][bad][:4]}, expected {o[bad][:4]} +- {move[bad][:4]}"
        assert abs(got_lse[i] - ref_lse) <= 2.0 ** -8 + 1e-5 * abs(ref_lse) + lse_move, (i // Hq, i % Hq, got_lse[i], ref_lse, lse_move)
        moves[i] = float(move.max() / vmax)
    return moves
