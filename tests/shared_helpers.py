"""Batches whose requests share the head of their prefix: a workload of the generator with the groups'
block-table rows pointed at the first request's pages (the oracle reads through the same tables)."""
from __future__ import annotations

import numpy as np

from paper_2505_23970_amd import workloads as W


def build(sizes, shared, beyond, new, Hq, Hkv, D, *, seed, values="peaked", name="shared"):
    """sizes, shared: requests and shared tokens of each group; beyond[r]: cached tokens past the shared
    ones; new[r]: new tokens."""
    first = np.concatenate([[0], np.cumsum(sizes)])
    P = np.concatenate([np.asarray(beyond[first[g]:first[g + 1]]) + shared[g] for g in range(len(sizes))]).astype(np.int64)
    w = W.build(P, new, Hq, Hkv, D, seed=seed, values=values, name=name)
    for g, S in enumerate(shared):
        w.block_tables[first[g]:first[g + 1], :S // 16] = w.block_tables[first[g], :S // 16]
    return w


# name -> (group sizes, shared tokens, cached tokens past them, new tokens)
def batches():
    rng = np.random.default_rng(5)
    return {
        # one token each; prefixes that end at, before and behind pages and tiles, and at the shared end
        "decode": ([7], [192], [0, 5, 16, 31, 32, 100, 63], [1] * 7),
        # one request, one shared page
        "one_page": ([1], [16], [3], [1]),
        # shared lengths around the 64-key tiles; a group of one; a group that shares nothing; empty requests
        "groups": ([3, 1, 4, 2], [64, 48, 80, 0], [1, 0, 40, 17, 5, 0, 0, 130, 9, 0], [1, 0, 2, 1, 0, 3, 1, 1, 5, 1]),
        # nothing of one's own cached, requests without new tokens first and last, a group without any
        "no_own": ([3, 2, 3], [112, 32, 128], [0] * 8, [0, 1, 1, 0, 0, 2, 1, 0]),
        # prompts: several 128-row tiles a request beside single tokens
        "prompts": ([4, 3], [176, 64], [20, 0, 77, 3, 0, 50, 8], [45, 1, 130, 17, 64, 2, 33]),
        # many requests: more query tiles in a group than one
        "many": ([70, 30], [96, 144], rng.integers(0, 60, 100).tolist(), rng.choice([0, 1, 1, 1, 2], 100).tolist()),
    }

