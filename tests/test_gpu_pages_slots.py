"""Slots of new tokens behind last blocks that name no block of the pool, in one launch and in three, up to the cache store."""
import numpy as np
import pytest

import page_reference as P
from test_gpu_pages import G, dev, host, resize  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hint", [0, 1 << 20])
def test_last_blocks_that_are_none(G, hint):  # noqa: F811
    """Rows that grow behind an entry below 0, at the pool's end, far beyond it, and a good one; one that is cut and one that ends there."""
    import torch
    NB, bs, M = 30, 16, 4
    bad = [-4, NB, 1 << 28, 7, 2 ** 31 - 1, -1]
    tables = np.array([[b, x, -7, -7] for b, x in enumerate(bad)], np.int32)
    lens, new = np.array([20, 31, 17, 20, 20, 20], np.int32), np.array([37, 33, 18, 25, 18, 0], np.int32)
    refs = np.zeros(NB, np.int32)
    refs[[0, 1, 2, 3, 4, 5, 7]] = 1
    cu = np.concatenate([[0], np.cumsum(np.maximum(new - lens, 0))])
    t, n, r, slots, pairs, lacking = resize(G, tables, lens, refs, new, cu, int(cu[-1]), bs, hint)
    want = P.resize(tables.astype(np.int64), lens, refs, new, cu, int(cu[-1]), bs)
    blocks = np.array([want[0][b, p // bs] for b in range(4) for p in range(lens[b], new[b])])
    assert (t == want[0]).all() and (n == want[1]).all() and (r == want[2]).all() and not pairs and lacking == 0
    assert (slots == np.where((blocks >= 0) & (blocks < NB), want[3], -1)).all() and (slots == -1).sum() == 12 + 1 + 1
    # the store: those rows alone, nothing beside the caches
    Hkv, D = 2, 64
    around = torch.full((NB + 4, Hkv, bs, D), 3.0, dtype=torch.float16, device="cuda")
    k, v = around[2:-2], torch.full((NB, Hkv, bs, D), 3.0, dtype=torch.float16, device="cuda")
    rows = torch.randn(len(slots), Hkv, D, device="cuda").half()
    G.reshape_and_cache(rows, -rows, k, v, dev(slots, np.int64))
    expect = torch.full_like(around, 3.0)
    for i, slot in enumerate(slots):
        if slot >= 0:
            expect[2 + slot // bs, :, slot % bs] = rows[i]
    assert torch.equal(around, expect) and int((v != 3.0).any(dim=3).any(dim=1).sum()) == int((slots >= 0).sum())
