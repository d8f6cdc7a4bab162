"""CPU: masks of trees, sizes, and what the calls for trees refuse before any launch."""
import ctypes
import os

import numpy as np
import pytest


@pytest.fixture(scope="module")
def G():
    import paper_2505_02351_amd as G
    if not os.path.exists(G.LIB_PATH):
        from paper_2505_02351_amd import build
        build.build()
    G.load_library()
    return G


ONE, ODD = ctypes.c_void_p(16), ctypes.c_void_p(18)      # never dereferenced: every call below fails first or has nothing to do


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 64, 100])
def test_masks_of_a_tree(G, n):
    rng = np.random.RandomState(n)
    parents = [int(rng.randint(-1, i)) if rng.rand() < 0.9 else -5 for i in range(n)]
    masks, depths = G.tree_masks(parents, -(-n // 32) + n % 2)
    words = masks.numpy().view(np.uint32)
    for i in range(n):
        line, j = [], i
        while j >= 0:
            line.append(j)
            j = parents[j]
        assert depths[i] == len(line) - 1
        assert {c for c in range(32 * words.shape[1]) if words[i, c // 32] >> np.uint32(c % 32) & 1} == set(line)
    assert G.tree_masks(parents)[0].shape == (n, -(-n // 32))


def test_masks_refuse(G):
    assert G.tree_masks([])[0].shape == (0, 1)
    for parents, words, status in (([0], None, -6), ([-1, 1], None, -6), ([-1, 0, 5], None, -6), ([-1] * 33, 1, -2), ([-1], 0, -2)):
        with pytest.raises(G.OptGqaError) as e:
            G.tree_masks(parents, words)
        assert e.value.status == status
    f = G.load_library().optgqa_tree_masks_host
    assert f(None, ONE, ONE, 1, 1) == -1 and f(ONE, None, ONE, 1, 1) == -1 and f(ONE, ONE, None, 1, 1) == -1 and f(None, None, None, 0, 1) == 0
    assert f(ONE, ONE, ONE, -1, 1) == -2


def test_trees_refuse_before_any_launch(G):
    lib = G.load_library()
    need = G.tree_workspace_bytes(8, 4, 8, 2, 64, 16, 2, 64, 3)
    assert need > 0

    def c(call=lib.optgqa_paged_attention_tree, scales=(), out=ONE, q=ONE, kc=ONE, vc=ONE, pt=ONE, bt=ONE, cl=ONE, cu=ONE, masks=ONE, pos=ONE, sl=ONE,
          scale=0.1, words=1, T=8, B=4, Hq=8, Hkv=2, D=64, bs=16, NP=2, MB=4, most=64, n=3, ws=ONE, ws_bytes=None, dt=0):
        return call(out, q, kc, vc, pt, bt, cl, cu, masks, pos, sl, scale, *scales, words, T, B, Hq, Hkv, D, bs, NP, MB, most, n, ws,
                    need if ws_bytes is None else ws_bytes, dt, None)

    heads = dict(call=lib.optgqa_paged_attention_tree_fp8_heads, scales=(ONE, ONE))
    tensor = dict(call=lib.optgqa_paged_attention_tree_fp8, scales=(0.1, 0.1))
    for kw in ({}, heads, tensor):
        def a(**more):
            return c(**{**kw, **more})
        assert a(T=-1) == -2 and a(B=-1) == -2 and a(Hq=0) == -2 and a(Hkv=3) == -2 and a(NP=-1) == -2 and a(most=-1) == -2 and a(n=-1) == -2
        assert a(scale=float("nan")) == -2 and a(D=96) == -3 and a(bs=8) == -3 and a(dt=2) == -3
        assert a(words=0) == -2 and a(words=-1) == -2 and a(n=33) == -2 and a(n=65, words=2) == -2
        assert a(most=65) == -2 and a(B=0) == -2 and a(n=0) == -2 and a(cu=None) == -2
        for name in ("out", "q", "kc", "vc", "pt", "bt", "cl", "masks", "pos"):
            assert a(**{name: None}) == -1, name
        for name in ("out", "q", "kc", "vc", "masks", "pos"):
            assert a(**{name: ODD}) == -3, name
        assert a(ws=None) == -4 and a(ws_bytes=need - 1) == -4 and a(ws=ctypes.c_void_p(24)) == -4
        assert a(T=0, masks=None, q=None) == 0
    assert c(call=lib.optgqa_paged_attention_tree_fp8_heads, scales=(None, ONE)) == -1 and c(call=lib.optgqa_paged_attention_tree_fp8_heads, scales=(ONE, None)) == -1
    assert c(call=lib.optgqa_paged_attention_tree_fp8, scales=(0.0, 1.0)) == -2 and c(call=lib.optgqa_paged_attention_tree_fp8, scales=(1.0, float("inf"))) == -2


def test_a_workspace_covers_every_smaller_call(G):
    rng = np.random.RandomState(0)
    for _ in range(400):
        Hkv = int(rng.choice([1, 2, 8, 16]))
        Hq, D, bs = Hkv * int(rng.choice([1, 4, 8])), int(rng.choice([64, 128])), int(rng.choice([16, 32, 64]))
        B, n, NP = int(rng.randint(1, 100)), int(rng.randint(1, 70)), int(rng.choice([0, rng.randint(1, 600)]))
        T, most = B * n, NP * bs + int(rng.randint(0, 9000))
        need = G.tree_workspace_bytes(T, B, Hq, Hkv, D, bs, NP, most, n)
        assert need > 0 and need >= G.common_prefix_workspace_bytes(T, B, Hq, Hkv, D, bs, NP, most, n)
        for _ in range(6):
            b, k, p = int(rng.randint(1, B + 1)), int(rng.randint(1, n + 1)), int(rng.randint(0, NP + 1))
            assert G.tree_workspace_bytes(int(rng.randint(1, b * k + 1)), b, Hq, Hkv, D, bs, p, int(rng.randint(0, most + 1)), k) <= need


def test_the_binding_refuses(G):
    import torch
    q, cache, i32 = torch.zeros(4, 8, 64, dtype=torch.float16), torch.zeros(3, 2, 16, 64, dtype=torch.float16), torch.int32
    table, lens, cu, none = torch.zeros(2, 3, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(3, dtype=i32), torch.zeros(0, dtype=i32)
    masks, pos = torch.zeros(4, 1, dtype=i32), torch.zeros(4, dtype=i32)
    with pytest.raises(TypeError, match="tree_masks"):
        G.paged_attention_tree(q, q, cache, cache, none, table, lens, cu, masks.long(), pos, None, 0.1, 48, 2)
    with pytest.raises(TypeError, match="positions"):
        G.paged_attention_tree(q, q, cache, cache, none, table, lens, cu, masks, pos.long(), None, 0.1, 48, 2)
    with pytest.raises(TypeError, match="tree_masks"):
        G.paged_attention_tree(q, q, cache, cache, none, table, lens, cu, None, pos, None, 0.1, 48, 2)
    with pytest.raises(ValueError, match="GPU memory"):
        G.paged_attention_tree(q, q, cache, cache, none, table, lens, cu, masks, None, None, 0.1, 48, 2)
