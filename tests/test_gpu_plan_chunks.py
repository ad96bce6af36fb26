"""The plan of query tiles cut into many chunks (GPU): their items, one for every chunk of every query tile, whatever wrote
them: a tile's chunks cover its key tiles once, in order, with consecutive partial slots, longest items first."""
import numpy as np
import pytest

from paper_2505_23970_amd import workloads as W

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("P,n,split", [([6000], [1], 1), ([6000, 40, 2500, 1056], [1, 1, 1, 1], 2), ([1024], [1], 1),
                                       ([3000, 5], [300, 7], 1), ([992 + i for i in range(70)], [1] * 70, 1),
                                       ([20000, 19000, 18011], [1, 1, 1], 3)])
def test_chunks_cover_every_tile(P, n, split):
    import torch
    import paper_2505_23970_amd as gc
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Hq, Hkv, D = 4, 1, 64
    pages = [-(-(p + m) // 16) for p, m in zip(P, n)]
    tables = np.zeros((len(P), max(pages)), np.int32)
    batch = gc.PagedBatch(P, n, tables)
    pool = torch.zeros(1, Hkv, 16, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, Hkv, D, 16, dtype=torch.bfloat16, device="cuda")
    ws = gc.alloc_workspace(Hq, *pool, batch, kv_split_tiles=split)
    ws.fill_(0xAA)
    gc.plan(Hq, *pool, batch, ws, kv_split_tiles=split)
    assert gc.plan_status(ws) == gc.GC_OK
    small = all(m * Hq <= 16 for m in n)
    tq, keys = (4, 32) if small else (32, 64)
    expected = []   # (request, first token, key tiles)
    for r, (p, m) in enumerate(zip(P, n)):
        for q0 in range(0, m, tq):
            expected.append((r, q0, -(-(p + min(q0 + tq, m)) // keys)))
    total = sum(-(-kt // split) for _, _, kt in expected)
    items = ws.cpu().numpy()[256:256 + 32 * total].view(np.int32).reshape(total, 8)
    cost = items[:, 3] - items[:, 2]
    if len(expected) <= 4:
        assert np.all(np.diff(cost) <= 0)      # (no grouping by request in so short a list of tiles)
    cu = np.concatenate([[0], np.cumsum(n)])
    parts = []
    for r, q0, kt in expected:
        mine = items[(items[:, 0] == r) & (items[:, 1] == q0)]
        ns = -(-kt // split)
        mine = mine[np.argsort(mine[:, 2])]
        assert len(mine) == ns and mine[0, 2] == 0 and mine[-1, 3] == kt
        assert np.array_equal(mine[1:, 2], mine[:-1, 3])
        assert np.array_equal(mine[:, 2], np.arange(ns) * kt // ns)
        if ns > 1:
            assert np.array_equal(mine[:, 4], mine[0, 4] + np.arange(ns))
            parts += mine[:, 4].tolist()
        else:
            assert mine[0, 4] == -1
        assert (mine[:, 5] == P[r]).all() and (mine[:, 6] == cu[r]).all() and (mine[:, 7] == n[r]).all()
    assert sorted(parts) == list(range(len(parts)))
