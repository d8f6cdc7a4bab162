"""The page calls against their plain versions, every entry of every table; and runs of them over caches whose rows say whose they are."""
import numpy as np
import pytest

import page_reference as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    import paper_2505_02351_amd as G
    return G


def dev(x, dtype=np.int32):
    import torch
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, dtype))).cuda()


def host(t):
    return t.cpu().numpy()


def resize(G, tables, lens, refs, new, cu, num_slots, bs, hint=None, stream=None):
    """What the call makes of its arguments, as page_reference.resize gives it."""
    import torch
    B, M = tables.shape
    t, n, r = dev(tables), dev(lens), dev(refs)
    copies, counts = torch.full((B, 2), -5, dtype=torch.int32, device="cuda"), torch.full((2,), -5, dtype=torch.int32, device="cuda")
    slots = None if num_slots is None else torch.full((num_slots,), -2, dtype=torch.int64, device="cuda")
    ws = torch.full((G.resize_workspace_bytes(B, M, len(refs)),), 0xa5, dtype=torch.uint8, device="cuda")
    if hint is None:
        hint = int(np.abs(P.clamped(new, M, bs) - P.clamped(lens, M, bs)).max()) if B else 0
    new_d, cu_d = dev(new), None if num_slots is None else dev(cu)
    G.resize_sequences(t, n, r, new_d, slots, cu_d, copies, counts, bs, hint, ws)
    torch.cuda.synchronize()
    made, lacking = host(counts).tolist()
    pairs = host(copies)
    assert (pairs[made:] == -5).all()
    return host(t), host(n), host(r), None if slots is None else host(slots), [tuple(x) for x in pairs[:made].tolist()], lacking


def same(got, want):
    for a, b, what in zip(got, want, ("tables", "lens", "refs", "slots", "pairs", "lacking")):
        if what == "pairs":
            assert a == [tuple(int(y) for y in x) for x in b], what
        elif a is not None:
            assert (np.asarray(a) == np.asarray(b)).all(), what


SHAPES = [(1, 1, 16, 0), (1, 40, 16, 3), (7, 5, 32, 2), (64, 9, 16, 11), (65, 33, 64, 0), (1025, 3, 16, 7), (2100, 2, 16, 100)]


@pytest.mark.parametrize("B,M,bs,spare", SHAPES)
@pytest.mark.parametrize("change", [1, 17, 300])
def test_resize(G, B, M, bs, spare, change):
    rng = np.random.RandomState(B * 31 + M + change)
    tables, lens, refs = P.pool(rng, B, M, bs, spare, 0.4)
    step = rng.randint(-change, change + 1, B)
    if change == 1:
        step = np.abs(step)
    new = np.where(rng.rand(B) < 0.1, 0, np.clip(lens + step, 0, M * bs))
    cu = np.concatenate([[0], np.cumsum(np.maximum(new - lens, 0))])
    want = P.resize(tables, lens, refs, new, cu, int(cu[-1]) + 3, bs)
    # in one launch and in three (what the bound says; neither depends on it for its result)
    for hint in (0, 1 << 20):
        same(resize(G, tables, lens, refs, new, cu, int(cu[-1]) + 3, bs, hint), want)
    same(resize(G, tables, lens, refs, new, cu, None, bs), want)


@pytest.mark.parametrize("hint", [0, 1 << 20])
@pytest.mark.parametrize("holders,writers", [(1, 1), (2, 1), (2, 2), (5, 3), (5, 5), (70, 70), (1100, 1100), (1100, 1099)])
def test_a_shared_last_block_is_replaced(G, holders, writers, hint):
    """Of those who hold a block, `writers` go on: all get a block of their own, but the last one where nobody is left."""
    bs, M = 16, 2
    rng = np.random.RandomState(holders + writers)
    tables, lens, refs = np.full((holders, M), -7, np.int32), np.full(holders, 5, np.int32), np.zeros(holders + 9, np.int32)
    tables[:, 0], refs[4] = 4, holders
    new = lens.copy()
    new[rng.permutation(holders)[:writers]] += rng.randint(1, 20, writers)
    cu = np.concatenate([[0], np.cumsum(new - lens)])
    want = P.resize(tables, lens, refs, new, cu, int(cu[-1]), bs)
    assert want[5] > 0 or len(want[4]) == (writers - 1 if writers == holders else writers)
    same(resize(G, tables, lens, refs, new, cu, int(cu[-1]), bs, hint), want)


@pytest.mark.parametrize("hint", [0, 1 << 20])
@pytest.mark.parametrize("short", [0, 1, 7])
def test_blocks_run_out(G, hint, short):
    """One block too few and no sequence grows: lengths, tables and counts as before but for what is cut, slots -1."""
    bs, M, B = 16, 6, 9
    rng = np.random.RandomState(5)
    tables, lens, refs = P.pool(rng, B, M, bs, 0, 0.5, 0.4)
    new = np.minimum(lens + 40, M * bs)
    new[2], new[5] = 0, lens[5] // 2
    cu = np.concatenate([[0], np.cumsum(np.maximum(new - lens, 0))])
    free = np.flatnonzero(P.resize(tables, lens, refs, np.minimum(new, lens), cu * 0, 0, bs)[2] == 0)
    wanted = len(free) - (P.resize(tables, lens, refs, new, cu, 0, bs)[2] == 0).sum()
    refs[free[max(wanted - short, 0):]] = 1                  # held by somebody else
    want = P.resize(tables, lens, refs, new, cu, int(cu[-1]), bs)
    assert want[5] == short
    same(resize(G, tables, lens, refs, new, cu, int(cu[-1]), bs, hint), want)


@pytest.mark.parametrize("hint", [0, 1 << 20])
def test_odd_contents(G, hint):
    """Lengths outside a row, entries that name no block, prefix sums that leave more or less room than the tokens take, and beyond
    the slots that there are."""
    bs, M = 16, 4
    tables = np.array([[3, 99, -4, 0], [5, 6, -7, -7], [1, 2, 4, 8], [-7, -7, -7, -7]], np.int32)
    lens, new = np.array([50, 20, 1000, -3], np.int32), np.array([-9, 33, 5, 99], np.int32)
    refs = np.zeros(30, np.int32)
    refs[[3, 0, 5, 6, 1, 2, 4, 8]] = 1
    for cu in ([0, 0, 13, 13, 77], [0, 2, 40, 41, 200], [0, 0, 5, 5, 9]):
        want = P.resize(tables, lens, refs, new, cu, 100, bs)
        same(resize(G, tables, lens, refs, new, cu, 100, bs, hint), want)


@pytest.mark.parametrize("NB", [1, 4095, 4096, 4097, 20000])
def test_the_lowest_free_blocks_of_a_large_pool(G, NB):
    rng = np.random.RandomState(NB)
    refs = (rng.rand(NB) < 0.99).astype(np.int32)
    refs[-1] = 0
    free = int((refs == 0).sum())
    M = max(free, 1)
    tables, lens, new = np.full((1, M), -7, np.int32), np.zeros(1, np.int32), np.array([free * 16 - 3])
    same(resize(G, tables, lens, refs, new, [0, 0], 0, 16), P.resize(tables, lens, refs, new, [0, 0], 0, 16))


@pytest.mark.parametrize("hint", [0, 1 << 20])
def test_thousands_of_new_blocks(G, hint):
    """More new blocks than a plan holds in LDS, given to few rows; some of them shared, some lacking none."""
    bs, M = 16, 1500
    rng = np.random.RandomState(7)
    tables, lens, refs = P.pool(rng, 6, M, bs, 50, 0.5)
    lens, refs = np.minimum(lens, 1000).astype(np.int32), np.zeros_like(refs)
    for row, n in zip(tables, lens):
        np.add.at(refs, row[:P.have(n, bs)], 1)
    new = np.full(6, M * bs - 5)
    cu = np.concatenate([[0], np.cumsum(new - lens)])
    want = P.resize(tables, lens, refs, new, cu, int(cu[-1]), bs)
    assert want[5] == 0 and len(np.flatnonzero(want[2] != refs)) > 4096
    same(resize(G, tables, lens, refs, new, cu, int(cu[-1]), bs, hint), want)


@pytest.mark.parametrize("B,N,M,bs", [(1, 1, 1, 16), (3, 8, 5, 16), (64, 40, 9, 32), (300, 300, 3, 64), (2, 3, 2500, 16)])
def test_fork(G, B, N, M, bs):
    import torch
    rng = np.random.RandomState(B + N + M)
    tables, lens, refs = P.pool(rng, B, M, bs, 3, 0.4)
    lens[rng.randint(0, B)] = 0 if B > 2 else lens[0]
    for kind in ("mixed", "one", "stay", "none"):
        parents = {"mixed": rng.randint(-1, B + 1, N), "one": np.full(N, B - 1), "stay": np.arange(N), "none": np.full(N, 1 << 30)}[kind]
        rows, new, counts = P.fork(tables, lens, refs, parents, bs)
        out, out_lens, r = torch.full((N, M), -9, dtype=torch.int32, device="cuda"), torch.full((N,), -9, dtype=torch.int32, device="cuda"), dev(refs)
        t, n = dev(tables), dev(lens)
        G.fork_sequences(out, out_lens, t, n, r, dev(parents), bs)
        out, out_lens = host(out), host(out_lens)
        assert (out_lens == new).all() and (host(r) == counts).all() and (host(t) == tables).all() and (host(n) == lens).all()
        for i in range(N):
            assert (out[i, :len(rows[i])] == rows[i]).all() and (out[i, len(rows[i]):] == -9).all()


@pytest.mark.parametrize("B,M,bs,spare", [(1, 1, 16, 0), (5, 7, 16, 40), (64, 30, 32, 3), (1030, 3, 16, 500), (3, 2000, 64, 9)])
@pytest.mark.parametrize("most", [0, 1, 5, None])
def test_compact(G, B, M, bs, spare, most):
    import torch
    rng = np.random.RandomState(B + M)
    tables, lens, refs = P.pool(rng, B, M, bs, spare, 0.3)
    most = len(refs) if most is None else most
    want_tables, want_refs, pairs, used = P.compact(tables, lens, refs, most, bs)
    t, n, r = dev(tables), dev(lens), dev(refs)
    copies, counts = torch.full((most, 2), -5, dtype=torch.int32, device="cuda"), torch.full((2,), -5, dtype=torch.int32, device="cuda")
    ws = torch.full((G.compact_workspace_bytes(len(refs)),), 0xa5, dtype=torch.uint8, device="cuda")
    G.compact_blocks(t, n, r, copies, counts, bs, ws)
    assert host(counts).tolist() == [len(pairs), used]
    got = host(copies)
    assert [tuple(x) for x in got[:len(pairs)].tolist()] == [tuple(int(y) for y in x) for x in pairs] and (got[len(pairs):] == -5).all()
    assert (host(t) == want_tables).all() and (host(r) == want_refs).all()


@pytest.mark.parametrize("NB,full", [(9, True), (5000, True), (5000, False)])
def test_compact_full_and_empty(G, NB, full):
    import torch
    refs = np.full(NB, 1 if full else 0, np.int32)
    tables, lens = (np.arange(NB, dtype=np.int32)[None], np.array([NB * 16], np.int32)) if full else (np.full((1, 4), -7, np.int32), np.zeros(1, np.int32))
    t, r, copies, counts = dev(tables), dev(refs), dev(np.full((NB, 2), -5)), dev([-5, -5])
    ws = torch.empty(G.compact_workspace_bytes(NB), dtype=torch.uint8, device="cuda")
    G.compact_blocks(t, dev(lens), r, copies, counts, 16, ws)
    assert host(counts).tolist() == [0, NB if full else 0] and (host(t) == tables).all() and (host(r) == refs).all() and (host(copies) == -5).all()


def caches(G, n, shape, dtype, seed):
    import torch
    gen = torch.Generator("cuda").manual_seed(seed)
    bits = [torch.randint(0, 256, (*shape[:3], shape[3] * (1 if dtype == torch.uint8 else 2)), generator=gen, device="cuda", dtype=torch.uint8)
            for _ in range(n)]
    made = [b if dtype == torch.uint8 else b.view(dtype) for b in bits]
    return G.CacheSet(made), [host(b).copy() for b in bits]          # (all bit patterns: NaN and infinities among them)


def bits_of(t):
    import torch
    return host(t.view(torch.uint8))


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "uint8"])
@pytest.mark.parametrize("n,shape,most,made", [(1, (2, 1, 16, 64), 1, 1), (4, (40, 2, 16, 64), 20, 20), (3, (40, 3, 64, 128), 20, 13), (70, (9, 1, 16, 64), 4, 4),
                                               (2, (40, 2, 16, 64), 8, 0), (2, (40, 2, 16, 64), 8, 100), (2, (40, 2, 16, 64), 8, -1)])
def test_copy_blocks(G, dtype, n, shape, most, made):
    import torch
    s, want = caches(G, n, shape, getattr(torch, dtype), 3)
    rng = np.random.RandomState(most)
    pairs = rng.permutation(shape[0])[:2 * most].reshape(most, 2)
    G.copy_blocks(s, dev(pairs), dev([made]))
    for w, t in zip(want, s.caches):
        for a, b in pairs[:max(min(made, most), 0)]:
            w[b] = w[a]
        assert (bits_of(t) == w).all()


def test_copy_blocks_passes_over_what_is_no_block(G):
    import torch
    s, want = caches(G, 2, (6, 2, 16, 64), torch.uint8, 3)
    G.copy_blocks(s, dev([[0, 6], [-1, 1], [1 << 30, 2], [3, -7], [4, 5]]), dev([5]))
    for w, t in zip(want, s.caches):
        w[5] = w[4]
        assert (bits_of(t) == w).all()


@pytest.mark.parametrize("dtype", ["float16", "uint8"])
@pytest.mark.parametrize("n,Hkv,bs,D,B,nodes,longest", [(1, 1, 16, 64, 1, 1, 1), (3, 2, 16, 64, 5, 20, 20), (2, 8, 32, 128, 33, 64, 9), (5, 3, 64, 128, 4, 100, 40)])
def test_keep_tokens(G, dtype, n, Hkv, bs, D, B, nodes, longest):
    """Branches that begin in the middle of a block and cross several, rows that are read for one place and written for another."""
    import torch
    rng = np.random.RandomState(nodes + B)
    M = -(-(70 + nodes) // bs)
    NB = B * M + 2
    tables = rng.permutation(NB)[:B * M].reshape(B, M)
    start = rng.randint(0, 71, B)
    counts = rng.randint(0, longest + 1, B)
    counts[0] = longest
    paths = np.full((B, longest), 1 << 20, np.int64)
    for b in range(B):
        paths[b, :counts[b]] = np.sort(rng.permutation(nodes)[:counts[b]])
    s, want = caches(G, n, (NB, Hkv, bs, D), getattr(torch, dtype), 5)
    G.keep_tokens(s, dev(tables), dev(start), dev(paths), dev(counts))
    for w, t in zip(want, s.caches):
        for b in range(B):
            at = start[b] + paths[b, :counts[b]]
            rows = w[tables[b, at // bs], :, at % bs].copy()
            at = start[b] + np.arange(counts[b])
            w[tables[b, at // bs], :, at % bs] = rows
        assert (bits_of(t) == w).all()


def test_rows_beyond_4_gib(G):
    """A cache of more than 2^32 bytes: blocks are copied and rows moved at both of its ends."""
    import torch
    NB, Hkv, bs, D = 70000, 4, 64, 128
    cache = torch.empty(NB, Hkv, bs, D, dtype=torch.float16, device="cuda")
    assert cache.numel() * 2 > 1 << 32
    gen = torch.Generator("cuda").manual_seed(1)
    used = [0, 1, NB - 1, NB - 2, 33000]
    for b in used:
        cache[b] = torch.randn(Hkv, bs, D, generator=gen, device="cuda").half()
    before = {b: cache[b].clone() for b in used}
    s = G.CacheSet([cache])
    G.copy_blocks(s, dev([[0, NB - 1], [NB - 2, 1]]), dev([2]))
    assert torch.equal(cache[NB - 1], before[0]) and torch.equal(cache[1], before[NB - 2]) and torch.equal(cache[33000], before[33000])
    # rows 60 and 66 of a sequence whose blocks lie at either end
    first, last = cache[NB - 1].clone(), cache[33000].clone()
    G.keep_tokens(s, dev([[NB - 1, 33000]]), dev([10]), dev([[0, 50, 56]]), dev([3]))
    want = first.clone()
    want[:, 11], want[:, 12] = first[:, 60], last[:, 2]
    assert torch.equal(cache[NB - 1], want) and torch.equal(cache[33000], last) and torch.equal(cache[0], before[0])


def test_keep_tokens_passes_over_what_is_nowhere(G):
    import torch
    tables = np.array([[0, 1], [7, 2], [3, 99]])
    s, want = caches(G, 2, (5, 1, 16, 64), torch.float16, 5)
    # behind the table; a block that is none; a place before its own; more places than there are; lengths below 0
    paths = np.array([[2, 40, 1 << 30], [17, 18, 19], [1, -3, 1]])
    G.keep_tokens(s, dev(tables), dev([0, -5, 3]), dev(paths), dev([3, 2, 50]))
    for w, t in zip(want, s.caches):
        w[0, :, 0] = w[0, :, 2]
        w[3, :, 3] = w[3, :, 4]
        assert (bits_of(t) == w).all()
    G.keep_tokens(s, dev(tables), dev([0, 0, 0]), dev(paths), dev([0, -1, -50]))
    for w, t in zip(want, s.caches):
        assert (bits_of(t) == w).all()


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("spare", [0, 30, -1])
def test_a_run_of_calls_keeps_every_sequence_its_tokens(G, seed, spare):
    """Random steps of everything together: each sequence's rows, read through its table, are the tokens that were appended to it or
    to those it came from."""
    import torch
    rng = np.random.RandomState(seed)
    B, M, bs, Hkv, D = int(rng.randint(2, 20)), int(rng.randint(2, 8)), 16, 2, 64
    NB = B * M // 2 if spare == 0 else B * M + spare if spare > 0 else max(B * M // 6, 2)
    pools = [torch.zeros(NB, Hkv, bs, D, dtype=torch.float16, device="cuda") for _ in range(2)]
    s = G.CacheSet(pools)
    tables, lens, refs = dev(np.full((B, M), -7)), dev(np.zeros(B)), dev(np.zeros(NB))
    other, other_lens = dev(np.full((B, M), -7)), dev(np.zeros(B))
    copies, pairs, counts = dev(np.zeros((B, 2))), dev(np.zeros((NB, 2))), dev([0, 0])
    ws = torch.empty(max(G.resize_workspace_bytes(B, M, NB), G.compact_workspace_bytes(NB)), dtype=torch.uint8, device="cuda")
    mine, token, lacked = [[] for _ in range(B)], 0, 0
    for step in range(25):
        new = np.clip([len(x) for x in mine] + rng.randint(-20, 25, B), 0, M * bs) * (rng.rand(B) < 0.9)
        grown = np.maximum(new - [len(x) for x in mine], 0)
        cu = np.concatenate([[0], np.cumsum(grown)])
        slots = torch.zeros(int(cu[-1]), dtype=torch.int64, device="cuda")
        G.resize_sequences(tables, lens, refs, dev(new), slots, dev(cu), copies, counts, bs, int(rng.choice([0, 5000])), ws)
        G.copy_blocks(s, copies, counts)
        ids = np.arange(token, token + cu[-1]) % 2000 + 1
        token += cu[-1]
        rows = dev(np.broadcast_to(ids[:, None, None], (len(ids), Hkv, D)), np.float16)
        G.reshape_and_cache(rows, -rows, *pools, slots)
        lacking = int(counts[1])
        lacked += lacking > 0
        for b in range(B):
            if new[b] <= len(mine[b]):
                mine[b] = mine[b][:int(new[b])]
            elif not lacking:
                mine[b] = mine[b] + ids[cu[b]:cu[b + 1]].tolist()
        if rng.rand() < 0.4:                                 # a branch of the last tokens of each sequence is kept
            count = np.array([rng.randint(0, min(len(x), 9) + 1) for x in mine])
            chosen = [np.sort(rng.permutation(min(len(x), 9))[:c]) for x, c in zip(mine, count)]
            shared = host(refs)                              # (not where others hold the blocks as well)
            t = host(tables)
            paths = np.zeros((B, 9), np.int64)
            for b in range(B):
                start = len(mine[b]) - min(len(mine[b]), 9)
                if any(shared[t[b, (start + i) // bs]] > 1 for i in range(min(len(mine[b]), 9))):
                    chosen[b], count[b] = np.arange(count[b]), count[b]
                paths[b, :count[b]] = chosen[b]
            start = np.array([len(x) - min(len(x), 9) for x in mine])
            G.keep_tokens(s, tables, dev(start), dev(paths), dev(count))
            mine = [x[:a] + [x[a + i] for i in c] for x, a, c in zip(mine, start, chosen)]
            G.resize_sequences(tables, lens, refs, dev([len(x) for x in mine]), None, None, copies, counts, bs, 9, ws)
        if rng.rand() < 0.4:
            parents = np.where(rng.rand(B) < 0.5, np.arange(B), rng.randint(-1, B, B))
            G.fork_sequences(other, other_lens, tables, lens, refs, dev(parents), bs)
            tables, other, lens, other_lens = other, tables, other_lens, lens
            mine = [list(mine[p]) if p >= 0 else [] for p in parents]
        if rng.rand() < 0.3:
            G.compact_blocks(tables, lens, refs, pairs, counts, bs, ws)
            G.copy_blocks(s, pairs, counts)
        t, r = host(tables), host(refs)
        assert host(lens).tolist() == [len(x) for x in mine]
        held = np.zeros(NB, np.int64)
        keys, values = host(pools[0]), host(pools[1])
        for b in range(B):
            n = P.have(len(mine[b]), bs)
            np.add.at(held, t[b, :n], 1)
            at = np.arange(len(mine[b]))
            got = keys[t[b, at // bs], :, at % bs]
            assert (got == np.array(mine[b]).reshape(-1, 1, 1)).all() and (values[t[b, at // bs], :, at % bs] == -got).all(), (step, b)
        assert (held == r).all()
    assert spare >= 0 or lacked                              # (a sixth of a pool: it has run out at times)


def test_captured_and_on_other_streams(G):
    """A step's calls recorded once and replayed, with the pool's own changes between the replays; two graphs share a workspace; the
    same calls on a stream of their own."""
    import torch
    rng = np.random.RandomState(1)
    B, M, bs = 33, 6, 16
    s, want = caches(G, 3, (B * M + 9, 2, bs, 64), torch.float16, 7)
    first = P.pool(rng, B, M, bs, 9, 0.4)
    tables, lens, refs = (dev(x) for x in first)
    out, out_lens = dev(np.full((B, M), -9)), dev(np.zeros(B))
    new, cu, slots = dev(np.zeros(B)), dev(np.zeros(B + 1)), torch.zeros(B * 20, dtype=torch.int64, device="cuda")
    copies, pairs, counts, parents = dev(np.zeros((B, 2))), dev(np.zeros((B * M, 2))), dev([0, 0]), dev(np.zeros(B))
    ws = torch.empty(max(G.resize_workspace_bytes(B, M, B * M + 9), G.compact_workspace_bytes(B * M + 9)), dtype=torch.uint8, device="cuda")

    def grow(most):
        G.resize_sequences(tables, lens, refs, new, slots, cu, copies, counts, bs, most, ws)
        G.copy_blocks(s, copies, counts)

    def tidy():
        G.fork_sequences(out, out_lens, tables, lens, refs, parents, bs)
        tables.copy_(out)
        lens.copy_(out_lens)
        G.compact_blocks(tables, lens, refs, pairs, counts, bs, ws)
        G.copy_blocks(s, pairs, counts)

    for work in (lambda: grow(20), lambda: grow(1 << 20), tidy):         # (first calls outside of a capture)
        new.copy_(lens)
        work()
    torch.cuda.synchronize()
    graphs = []
    for work in (lambda: grow(20), lambda: grow(1 << 20), tidy):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            work()
        graphs.append(g)
    side = torch.cuda.Stream()
    t0, n0, r0 = (host(x).copy() for x in (tables, lens, refs))
    out.fill_(-9)
    bits = [bits_of(c).copy() for c in s.caches]
    for step in range(12):
        what = np.clip(n0 + rng.randint(-20, 21, B), 0, M * bs)
        c = np.concatenate([[0], np.cumsum(np.maximum(what - n0, 0))])
        p = np.where(rng.rand(B) < 0.7, np.arange(B), rng.randint(0, B, B))
        new.copy_(dev(what)), cu.copy_(dev(c)), parents.copy_(dev(p))
        torch.cuda.synchronize()
        if step % 3 == 2:
            with torch.cuda.stream(side):
                grow(20)
                tidy()
        else:
            graphs[step % 3].replay()
            graphs[2].replay()
        torch.cuda.synchronize()
        t0, n0, r0, _, moved, lacking = P.resize(t0, n0, r0, what, c, 0, bs)
        for w in bits:
            for a, b in moved:
                w[b] = w[a]
        rows, n0, r0 = P.fork(t0, n0, r0, p, bs)
        for i, row in enumerate(rows):
            t0[i, :len(row)] = row
        t0, r0, moved, used = P.compact(t0, n0, r0, B * M, bs)
        for w in bits:
            for a, b in moved:
                w[b] = w[a]
        assert (host(lens) == n0).all() and (host(refs) == r0).all() and host(counts).tolist() == [len(moved), used]
        got = host(tables)
        for i in range(B):
            assert (got[i, :P.have(n0[i], bs)] == t0[i, :P.have(n0[i], bs)]).all()
        for w, x in zip(bits, s.caches):
            assert (bits_of(x) == w).all()
