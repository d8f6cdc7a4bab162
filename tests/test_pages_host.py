"""CPU: what the page calls refuse before any launch, and the plain versions that the GPU tests compare with."""
import ctypes
import os

import numpy as np
import pytest

import page_reference as P


@pytest.fixture(scope="module")
def G():
    import paper_2505_02351_amd as G
    if not os.path.exists(G.LIB_PATH):
        from paper_2505_02351_amd import build
        build.build()
    G.load_library()
    return G


ONE, ODD = ctypes.c_void_p(16), ctypes.c_void_p(18)      # never dereferenced: every call below fails first or has nothing to do
FAR = ctypes.c_void_p(1 << 40)


def test_resize_refuses(G):
    lib = G.load_library()

    def call(tables=ONE, lens=ONE, refs=ONE, new=ONE, slots=ONE, cu=ONE, copies=ONE, counts=ONE, S=3, M=4, NB=10, bs=16, n=5, most=1, ws=ONE,
             ws_bytes=1 << 20):
        return lib.optgqa_resize_sequences(tables, lens, refs, new, slots, cu, copies, counts, S, M, NB, bs, n, most, ws, ws_bytes, None)

    assert call(S=-1) == -2 and call(M=0) == -2 and call(NB=0) == -2 and call(n=-1) == -2 and call(most=-1) == -2 and call(S=1 << 24) == -2
    assert call(bs=8) == -3 and call(bs=48) == -3
    for name in ("tables", "lens", "refs", "new", "cu", "copies", "counts"):
        assert call(**{name: None}) == -1, name
        assert call(**{name: ODD}) == -3, name
    assert call(slots=ctypes.c_void_p(20)) == -3
    need = G.resize_workspace_bytes(3, 4, 10)
    assert need >= 4 * (3 * 3 + 10)
    assert call(ws=None) == -4 and call(ws_bytes=need - 1) == -4 and call(ws=ctypes.c_void_p(24)) == -4
    assert G.resize_workspace_bytes(0, 4, 10) == 0 and G.resize_workspace_bytes(3, 0, 10) == 0 and G.resize_workspace_bytes(3, 4, 0) == 0
    assert G.resize_workspace_bytes(1 << 10, (1 << 21) - 2, 1 << 30) == 4 * (3 * (1 << 10) + (1 << 30))
    # blocks that all rows could ask for, counted in 32 bits
    assert G.resize_workspace_bytes(1 << 10, (1 << 21) - 1, 1 << 30) == 0 and call(S=1 << 10, M=(1 << 21) - 1, ws_bytes=1 << 40) == -2


def test_fork_refuses(G):
    lib = G.load_library()

    def call(out=FAR, lens_out=FAR, tables=ONE, lens=ONE, refs=ONE, parents=ONE, N=2, S=3, M=4, NB=10, bs=16):
        return lib.optgqa_fork_sequences(out, lens_out, tables, lens, refs, parents, N, S, M, NB, bs, None)

    assert call(S=-1) == -2 and call(N=-1) == -2 and call(M=0) == -2 and call(NB=-3) == -2 and call(bs=17) == -3
    for name in ("out", "lens_out", "tables", "lens", "refs", "parents"):
        assert call(**{name: None}) == -1, name
        assert call(**{name: ODD}) == -3, name
    # rows of the new tables are written while the old ones are read
    assert call(out=ONE) == -2 and call(out=ctypes.c_void_p(16 + 4 * 11)) == -2 and call(lens_out=ctypes.c_void_p(16 + 8)) == -2
    assert call(N=0, S=0, out=None, lens_out=None, tables=None, lens=None, refs=None, parents=None) == 0


def test_compact_refuses(G):
    lib = G.load_library()

    def call(tables=ONE, lens=ONE, refs=ONE, copies=ONE, counts=ONE, S=3, M=4, NB=10, bs=16, most=5, ws=ONE, ws_bytes=1 << 20):
        return lib.optgqa_compact_blocks(tables, lens, refs, copies, counts, S, M, NB, bs, most, ws, ws_bytes, None)

    assert call(S=-1) == -2 and call(M=0) == -2 and call(NB=0) == -2 and call(most=-1) == -2 and call(bs=128) == -3
    for name in ("tables", "lens", "refs", "copies", "counts"):
        assert call(**{name: None}) == -1, name
        assert call(**{name: ODD}) == -3, name
    assert call(ws=None) == -4 and call(ws_bytes=G.compact_workspace_bytes(10) - 1) == -4 and G.compact_workspace_bytes(0) == 0


def test_copy_and_keep_refuse(G):
    lib = G.load_library()

    def copy(caches=ONE, n=2, copies=ONE, count=ONE, most=3, NB=10, size=64):
        return lib.optgqa_copy_blocks(caches, n, copies, count, most, NB, size, None)

    assert copy(n=-1) == -2 and copy(most=-1) == -2 and copy(NB=0) == -2 and copy(size=0) == -2 and copy(size=24) == -3
    assert copy(caches=None) == -1 and copy(copies=None) == -1 and copy(count=None) == -1
    assert copy(caches=ctypes.c_void_p(20)) == -3 and copy(copies=ODD) == -3 and copy(count=ODD) == -3
    assert copy(n=0, caches=None) == 0 and copy(most=0, copies=None) == 0

    def keep(caches=ONE, n=2, tables=ONE, start=ONE, paths=ONE, path_lens=ONE, S=3, P=4, M=5, NB=10, Hkv=2, D=64, bs=16, size=2):
        return lib.optgqa_keep_tokens(caches, n, tables, start, paths, path_lens, S, P, M, NB, Hkv, D, bs, size, None)

    assert keep(n=-1) == -2 and keep(S=-1) == -2 and keep(S=65536) == -2 and keep(P=-1) == -2 and keep(M=0) == -2 and keep(NB=0) == -2 and keep(Hkv=0) == -2
    assert keep(D=96) == -3 and keep(bs=8) == -3 and keep(size=4) == -3
    for name in ("caches", "tables", "start", "paths", "path_lens"):
        assert keep(**{name: None}) == -1, name
        assert keep(**{name: ODD}) == -3, name
    assert keep(n=0, caches=None) == 0 and keep(S=0, tables=None) == 0 and keep(P=0, paths=None) == 0


def test_binding_refuses(G):
    import torch
    i32 = dict(dtype=torch.int32)
    tables, lens, refs, counts = torch.zeros(2, 3, **i32), torch.zeros(2, **i32), torch.zeros(9, **i32), torch.zeros(2, **i32)
    with pytest.raises(TypeError):
        G.resize_sequences(tables.long(), lens, refs, lens, None, None, torch.zeros(2, 2, **i32), counts, 16, 1, None)
    with pytest.raises(ValueError, match="GPU memory"):
        G.resize_sequences(tables, lens, refs, lens, None, None, torch.zeros(2, 2, **i32), counts, 16, 1, None)
    with pytest.raises(TypeError):
        G.fork_sequences(tables, lens, tables, lens, refs.float(), lens, 16)
    with pytest.raises(ValueError, match="GPU memory"):
        G.compact_blocks(tables, lens, refs, torch.zeros(4, 2, **i32), counts, 16, None)
    with pytest.raises(TypeError, match="CacheSet"):
        G.copy_blocks([torch.zeros(9, 1, 16, 64)], torch.zeros(4, 2, **i32), counts)
    with pytest.raises(TypeError, match="CacheSet"):
        G.keep_tokens(None, tables, lens, tables, lens)
    half = torch.zeros(3, 1, 16, 64, dtype=torch.float16)
    for bad, error in (([], ValueError), ([half.float()], TypeError), ([half, half.bfloat16()], TypeError), ([half, half[:2]], ValueError),
                       ([half.transpose(0, 1)], ValueError), ([half[0]], ValueError), ([half], ValueError), (["x"], TypeError)):
        with pytest.raises(error):
            G.CacheSet(bad)


def count(tables, lens, NB, bs):
    refs = np.zeros(NB, np.int64)
    for row, n in zip(tables, lens):
        np.add.at(refs, row[:P.have(n, bs)], 1)
    return refs


@pytest.mark.parametrize("seed", range(6))
def test_plain_versions_keep_counts_and_tables_in_step(seed):
    """Whatever is done, a block's count is the number of entries that hold it, and no sequence's rows change but for the asked ones."""
    rng = np.random.RandomState(seed)
    B, M, bs = rng.randint(1, 12), rng.randint(1, 9), 16
    tables, lens, refs = P.pool(rng, B, M, bs, rng.randint(0, 6), 0.5)
    for _ in range(6):
        new = np.clip(lens + rng.randint(-40, 41, B), 0, M * bs) * (rng.rand(B) < 0.9)
        cu = np.concatenate([[0], np.cumsum(np.maximum(new - lens, 0))])
        before, grown = tables, new > lens
        tables, lens, refs, slots, pairs, lacking = P.resize(tables, lens, refs, new, cu, cu[-1], bs)
        assert (refs == count(tables, lens, len(refs), bs)).all() and (lacking or (lens == new).all())
        assert len({b for _, b in pairs}) == len(pairs) and all(refs[b] == 1 for _, b in pairs)
        if not lacking:                                      # nobody else holds what is about to be written
            assert all(refs[s // bs] == 1 for s in slots) and len(set(slots)) == len(slots) and grown.sum() >= len(pairs)
        else:
            assert (slots == -1).all() and (tables == before).all()
        parents = rng.randint(-1, B + 1, B)
        rows, lens, refs = P.fork(tables, lens, refs, parents, bs)
        tables = np.full_like(tables, -7)
        for i, row in enumerate(rows):
            tables[i, :len(row)] = row
        assert (refs == count(tables, lens, len(refs), bs)).all()
        tables, refs, pairs, used = P.compact(tables, lens, refs, len(refs), bs)
        assert (refs[:used] > 0).all() and (refs[used:] == 0).all() and (refs == count(tables, lens, len(refs), bs)).all()
