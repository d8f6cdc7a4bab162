"""Host-only checks of the operators around a step's attention: frequencies, sizes, and what is refused before any launch."""
import ctypes
import math
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


ONE = ctypes.c_void_p(16)       # non-null, aligned, never dereferenced: every call below fails first or has nothing to do


def test_rotary_frequencies(G):
    f, m = G.rotary_frequencies(128, 10000.0)
    assert m == 1.0 and np.allclose(f.numpy(), 10000.0 ** (-np.arange(0, 128, 2) / 128), rtol=1e-14, atol=0)
    g, m = G.rotary_frequencies(128, 10000.0, G.ROTARY_LINEAR, 4.0)
    assert m == 1.0 and np.allclose(g, f / 4, rtol=1e-14, atol=0)
    g, m = G.rotary_frequencies(128, 10000.0, G.ROTARY_BASE, 4.0)     # the slowest pair is slowed by the factor, the fastest not at all
    assert m == 1.0 and g[0] == 1.0 and math.isclose(g[63], f[63] / 4, rel_tol=1e-12) and (g[1:] < f[1:]).all()
    g, m = G.rotary_frequencies(64, 10000.0, G.ROTARY_YARN, 16.0, 4096.0)
    f, _ = G.rotary_frequencies(64, 10000.0)
    turns = 4096.0 * f / (2 * math.pi)
    assert math.isclose(m, 0.1 * math.log(16.0) + 1.0, rel_tol=1e-6)
    assert (g[turns > 64] == f[turns > 64]).all() and np.allclose(g[turns < 0.5], f[turns < 0.5] / 16, rtol=1e-12, atol=0)
    assert (g <= f).all() and (g >= f / 16.001).all() and (g[1:] < g[:-1]).all()
    g, m = G.rotary_frequencies(64, 10000.0, G.ROTARY_WAVELENGTH, 8.0, 4096.0)
    assert m == 1.0 and (g[turns >= 4] == f[turns >= 4]).all() and np.allclose(g[turns <= 1], f[turns <= 1] / 8, rtol=1e-12, atol=0)
    mid = (turns > 1) & (turns < 4)
    s = (turns[mid] - 1) / 3
    assert mid.any() and np.allclose(g[mid], f[mid] * s + f[mid] / 8 * (1 - s), rtol=1e-12, atol=0)


def test_rotary_frequencies_refuse(G):
    for kw in (dict(rotary_dim=0), dict(rotary_dim=7), dict(rotary_dim=-2), dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")),
               dict(scaling=G.ROTARY_LINEAR, factor=0.5), dict(scaling=G.ROTARY_LINEAR, factor=float("nan")), dict(scaling=G.ROTARY_BASE, rotary_dim=2, factor=2.0),
               dict(scaling=G.ROTARY_YARN, factor=2.0), dict(scaling=G.ROTARY_YARN, factor=2.0, original_len=100.0, a=1.0, b=2.0),
               dict(scaling=G.ROTARY_WAVELENGTH, factor=2.0, original_len=100.0, a=4.0, b=1.0)):
        with pytest.raises(G.OptGqaError) as e:
            G.rotary_frequencies(**{"rotary_dim": 64, **kw})
        assert e.value.status == -2, kw
    for scaling in (5, -1):
        with pytest.raises(G.OptGqaError) as e:
            G.rotary_frequencies(64, scaling=scaling)
        assert e.value.status == -3
    f = G.load_library().optgqa_rotary_frequencies_host
    assert f(None, ONE, 64, 10000.0, 0, 1.0, 0.0, 0.0, 0.0) == -1 and f(ONE, None, 64, 10000.0, 0, 1.0, 0.0, 0.0, 0.0) == -1


def test_rotary_refuses_before_any_launch(G):
    lib = G.load_library()

    def rows(q_out=ONE, q=ONE, k_out=ONE, k=ONE, pos=ONE, f=ONE, T=3, Hq=4, Hkv=2, D=64, rot=64, m=1.0, s=(256, 256, 128, 128), dt=0):
        return lib.optgqa_rotary_embedding(q_out, q, k_out, k, pos, f, T, Hq, Hkv, D, rot, 0, m, 0, *s, dt, None)

    assert rows(T=-1) == -2 and rows(Hq=-1) == -2 and rows(Hq=0, Hkv=0) == -2 and rows(Hq=70000) == -2
    assert rows(D=96) == -3 and rows(dt=2) == -3
    assert rows(rot=0) == -2 and rows(rot=66) == -2 and rows(rot=63) == -2
    assert rows(m=float("nan")) == -2 and rows(m=float("inf")) == -2
    assert rows(s=(255, 256, 128, 128)) == -2 and rows(s=(256, 255, 128, 128)) == -2 and rows(s=(256, 256, 127, 128)) == -2 and rows(s=(256, 256, 128, 127)) == -2
    for name in ("q_out", "q", "k_out", "k", "pos", "f"):
        assert rows(**{name: None}) == -1, name
    odd = ctypes.c_void_p(17)
    for name in ("q_out", "q", "k_out", "k", "pos", "f"):
        assert rows(**{name: odd}) == -3, name
    assert rows(T=0, q=None, k=None) == 0

    def append(call=lib.optgqa_rotary_and_cache, scales=(), q_out=ONE, q=ONE, k=ONE, v=ONE, kc=ONE, vc=ONE, slots=ONE, pos=ONE, f=ONE, T=3,
               Hq=4, Hkv=2, D=64, rot=64, m=1.0, bs=16, s=(256, 256, 128, 128), dt=1):
        return call(q_out, q, k, v, kc, vc, slots, pos, f, T, Hq, Hkv, D, rot, 0, m, bs, *s, *scales, dt, None)

    one, heads = lib.optgqa_rotary_and_cache_fp8, lib.optgqa_rotary_and_cache_fp8_heads
    for call, scales in ((lib.optgqa_rotary_and_cache, ()), (one, (1.0, 1.0)), (heads, (ONE, ONE))):
        def a(**kw):
            return append(call, scales, **kw)
        assert a(T=-1) == -2 and a(Hq=0) == -2 and a(Hkv=0) == -2 and a(bs=8) == -3 and a(D=32) == -3 and a(dt=9) == -3
        assert a(rot=65) == -2 and a(m=float("nan")) == -2 and a(s=(256, 256, 128, 100)) == -2 and a(s=(256, 256, 100, 128)) == -2
        for name in ("q_out", "q", "k", "v", "kc", "vc", "slots", "pos", "f"):
            assert a(**{name: None}) == -1, name
        assert a(v=ctypes.c_void_p(17)) == -3
        assert a(T=0, q=None) == 0
    assert append(kc=ctypes.c_void_p(17)) == -3
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        assert append(one, (bad, 1.0)) == -2 and append(one, (1.0, bad)) == -2
    assert append(heads, (None, ONE)) == -1 and append(heads, (ONE, None)) == -1


def test_the_binding_refuses_what_the_library_cannot_see(G):
    import torch
    q, k = torch.zeros(3, 4, 64, dtype=torch.float16), torch.zeros(3, 2, 64, dtype=torch.float16)
    pos, f = torch.zeros(3, dtype=torch.int32), torch.zeros(32, dtype=torch.float64)
    with pytest.raises(TypeError):
        G.rotary_embedding(q, q, k, k, pos.long(), f)
    with pytest.raises(TypeError):
        G.rotary_embedding(q, q, k, k, pos, f.float())
    with pytest.raises(TypeError):
        G.rotary_embedding(q, q, k, k.bfloat16(), pos, f)
    with pytest.raises(ValueError):
        G.rotary_embedding(q, q, k, None, pos, f)
    with pytest.raises(ValueError):
        G.rotary_embedding(q, q, k, k, pos, f)                   # not on a GPU


def test_rows_that_are_not_dense_are_refused(G):
    import torch
    from paper_2505_02351_amd.operators import _rows
    assert _rows(torch.zeros(3, 2, 64), "q", 3, 64) == (2, 128) and _rows(torch.zeros(3, 200)[:, 8:136].view(3, 2, 64), "q", 3, 64) == (2, 200)
    assert _rows(torch.zeros(5, 64, 1, dtype=torch.float16).transpose(1, 2)[:1], "q", 1, 64) == (1, 64)
    for T, H in ((1, 1), (1, 2), (3, 1), (3, 2)):
        for t in (torch.zeros(T, H, 128)[:, :, ::2], torch.zeros(T, 64, max(H, 2)).transpose(1, 2)[:, :H]):
            with pytest.raises(ValueError):
                _rows(t, "q", T, 64)


def test_verification_refuses_before_any_launch(G):
    lib = G.load_library()
    need = G.verify_drafts_workspace_bytes(3, 32000)
    assert need > 0 and G.verify_drafts_workspace_bytes(0, 5) == 0 and G.verify_drafts_workspace_bytes(5, 0) == 0

    def v(tokens=ONE, n=ONE, p=ONE, q=ONE, ids=ONE, cu=ONE, a=ONE, s=ONE, B=3, V=32000, most=4, ps=32000, qs=32000, ws=ONE, wsb=None, dt=2):
        return lib.optgqa_verify_drafts(tokens, n, p, q, ids, cu, a, s, B, V, most, ps, qs, ws, need if wsb is None else wsb, dt, None)

    assert v(B=-1) == -2 and v(V=0) == -2 and v(most=-1) == -2 and v(ps=31999) == -2 and v(qs=31999) == -2 and v(V=2**30, ps=2**30, qs=2**30) == -2
    assert v(dt=3) == -3 and v(dt=-1) == -3
    for name in ("tokens", "n", "p", "cu", "s"):
        assert v(**{name: None}) == -1, name
    for name, at in (("tokens", 20), ("n", 18), ("p", 18), ("q", 18), ("ids", 20), ("cu", 18), ("a", 18), ("s", 18)):
        assert v(**{name: ctypes.c_void_p(at)}) == -3, name
    assert v(ws=None) == -4 and v(wsb=need - 1) == -4 and v(ws=ctypes.c_void_p(8)) == -4
    assert v(B=0, tokens=None) == 0


def test_common_prefix_refuses_before_any_launch(G):
    lib = G.load_library()
    need = G.common_prefix_workspace_bytes(8, 4, 8, 2, 64, 16, 16, 320, 3)
    assert need > 0
    for kw in (dict(T=0), dict(B=0), dict(Hq=7), dict(D=96), dict(bs=8), dict(NP=-1), dict(Lmax=-1), dict(n=0)):
        a = {**dict(T=8, B=4, Hq=8, Hkv=2, D=64, bs=16, NP=16, Lmax=320, n=3), **kw}
        assert G.common_prefix_workspace_bytes(a["T"], a["B"], a["Hq"], a["Hkv"], a["D"], a["bs"], a["NP"], a["Lmax"], a["n"]) == 0, kw

    def c(call=lib.optgqa_paged_attention_common, scales=(), out=ONE, q=ONE, kc=ONE, vc=ONE, pt=ONE, bt=ONE, cl=ONE, cu=ONE, scale=0.1, T=8, B=4,
          Hq=8, Hkv=2, D=64, bs=16, NP=16, MB=20, Lmax=320, n=3, ws=ONE, wsb=None, dt=0):
        return call(out, q, kc, vc, pt, bt, cl, cu, None, scale, *scales, T, B, Hq, Hkv, D, bs, NP, MB, Lmax, n, ws, need if wsb is None else wsb, dt, None)

    one, heads = lib.optgqa_paged_attention_common_fp8, lib.optgqa_paged_attention_common_fp8_heads
    for call, scales in ((lib.optgqa_paged_attention_common, ()), (one, (1.0, 1.0)), (heads, (ONE, ONE))):
        def a(**kw):
            return c(call, scales, **kw)
        assert a(T=-1) == -2 and a(B=-1) == -2 and a(Hq=7) == -2 and a(Hq=0) == -2 and a(Hkv=0) == -2 and a(NP=-1) == -2 and a(Lmax=-1) == -2
        assert a(n=-1) == -2 and a(n=0) == -2 and a(B=0) == -2 and a(MB=19) == -2 and a(Hq=70000, Hkv=70000) == -2
        assert a(scale=float("nan")) == -2 and a(scale=float("inf")) == -2
        assert a(D=96) == -3 and a(bs=8) == -3 and a(dt=2) == -3 and a(dt=-1) == -3
        for name in ("out", "q", "kc", "vc", "pt", "bt", "cl"):
            assert a(**{name: None}) == -1, name
        for name in ("out", "q", "kc", "vc"):
            assert a(**{name: ctypes.c_void_p(8)}) == -3, name
        assert a(cu=None) == -2                                  # 8 tokens of 4 sequences
        assert a(ws=None) == -4 and a(wsb=need - 1) == -4 and a(ws=ctypes.c_void_p(8)) == -4
        assert a(T=0, q=None) == 0
        assert a(T=2**30, Hq=64, Hkv=2) == -2                    # 2^35 rows
        assert a(NP=2**27, Lmax=100) == -2
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        assert c(one, (bad, 1.0)) == -2 and c(one, (1.0, bad)) == -2
    assert c(heads, (None, ONE)) == -1 and c(heads, (ONE, None)) == -1


def test_common_prefix_workspace_covers_every_smaller_call(G):
    """Sized by bounds: a call with one new token a sequence fits what its drafts' bound asks for."""
    for T, B, Hq, Hkv, D, NP, Lmax, n in ((9, 9, 32, 8, 128, 100, 5000, 9), (64, 64, 32, 4, 128, 0, 4000, 5), (600, 64, 8, 8, 64, 1000, 20000, 100)):
        big = G.common_prefix_workspace_bytes(T, B, Hq, Hkv, D, 16, NP, Lmax, n)
        assert big >= G.common_prefix_workspace_bytes(T, B, Hq, Hkv, D, 16, NP, Lmax, 1)


def test_common_prefix_sizes_at_their_ends(G):
    """Chunks of long contexts fit where the bound on one sequence's tokens, taken for all of them, would not."""
    def need(T, B, Lmax, n, Hq=64, Hkv=8):
        return G.common_prefix_workspace_bytes(T, B, Hq, Hkv, 128, 16, 0, Lmax, n)
    assert need(8192 + 63, 64, 1 << 20, 8192) > 0
    assert need(1, 1, 1 << 25, 1) > 0 and need(1, 1, (1 << 25) + 1, 1, 128, 1) == 0
    assert need(128, 1, 1 << 25, 128, 1, 1) > 0 and need(128, 1, (1 << 25) + 1, 128, 1, 1) == 0


def test_types_are_refused_before_places(G):
    """CPU tensors throughout: a wrong type is a TypeError, right types a ValueError."""
    import torch
    i32, i64 = torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)
    h, c = torch.zeros(3, 4, 64, dtype=torch.float16), torch.zeros(2, 2, 16, 64, dtype=torch.float16)
    kv, f = torch.zeros(3, 2, 64, dtype=torch.float16), torch.zeros(32, dtype=torch.float64)
    bt, ws = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(64, dtype=torch.uint8)
    good = {G.rotary_and_cache: [h, h, kv, kv, c, c, i64, i32, f], G.paged_attention_common: [h, h, c, c, i32, bt, i32, None, None, 0.1, 100, 1, ws],
            G.rotary_and_cache_fp8: [h, h, kv, kv, c.byte(), c.byte(), i64, i32, f, 1.0, 1.0],
            G.paged_attention_common_fp8: [h, h, c.byte(), c.byte(), i32, bt, i32, None, torch.zeros(4), 0.1, 1.0, 1.0, 100, 1, ws],
            G.verify_drafts: [torch.zeros(3, 3, dtype=torch.int64), i32, torch.zeros(6, 50), torch.zeros(3, 50), i64, torch.zeros(4, dtype=torch.int32),
                              torch.zeros(3), torch.zeros(3), ws]}
    for call, args in good.items():
        with pytest.raises(ValueError):
            call(*args)
        for i, x in enumerate(args):
            if not isinstance(x, torch.Tensor) or x is ws:
                continue
            with pytest.raises(TypeError):
                call(*args[:i], x.to(torch.complex64), *args[i + 1:])
            with pytest.raises((TypeError, AttributeError)):
                call(*args[:i], np.zeros(3), *args[i + 1:])
