"""CPU: where the workgroups of the common prefix's part of a launch find their work, over the card's eight XCDs."""
import ctypes

import numpy as np
import pytest

import common_prefix_plan as P


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return P.build(tmp_path_factory.mktemp("rules"))


def places(lib, kv_heads, ranges, tiles):
    out = np.zeros((lib.common_prefix_places(kv_heads, ranges, tiles, None), 3), np.int32)
    lib.common_prefix_places(kv_heads, ranges, tiles, ctypes.c_void_p(out.ctypes.data))
    return out


def check(lib, kv_heads, ranges, tiles):
    """Every (KV head, range, tile) once; no XCD has more than an eighth of them, rounded up, or reads more ranges' keys than it must."""
    all_of = places(lib, kv_heads, ranges, tiles)
    work = all_of[all_of[:, 0] >= 0]
    items = kv_heads * ranges * tiles
    assert len(work) == items and len(np.unique(work, axis=0)) == items
    assert (work >= 0).all() and (work < [kv_heads, ranges, tiles]).all()
    for x in range(8):
        mine = all_of[x::8]
        mine = mine[mine[:, 0] >= 0]
        assert len(mine) <= -(-items // 8)
        assert len(np.unique(mine[:, :2], axis=0)) <= -(-items // 8 // tiles) + 1


@pytest.mark.parametrize("tokens,seqs,heads,kv_heads,prefix", [
    (576, 64, 32, 4, 4096),             # 64 sequences of 9 new tokens: 4 (KV head, range) units of 36 row tiles
    (2048, 1, 32, 4, 4096),             # a chunk: 4 of 128
    (2048, 1, 8, 1, 4096),              # a single KV head
    (576, 64, 16, 4, 4096),             # 12 of 18
    (64, 64, 32, 4, 4096), (64, 64, 32, 8, 32768), (88, 16, 64, 8, 8192), (4, 4, 8, 2, 256), (1, 1, 8, 1, 64)])
def test_all_xcds_have_as_much_to_do(lib, tokens, seqs, heads, kv_heads, prefix):
    p = P.plan(lib, tokens, seqs, heads, kv_heads, prefix, prefix + 512, -(-tokens // seqs))
    check(lib, kv_heads, p.ranges, p.row_tiles)


def test_any_counts(lib):
    rng = np.random.default_rng(1)
    for kv_heads, ranges, tiles in np.exp(rng.uniform(0, np.log(33), (300, 3))).astype(int):
        check(lib, int(kv_heads), int(ranges), int(tiles))
    assert len(places(lib, 8, 0, 1)) == 0                        # no prefix
