"""The operators of several continuations of one sequence over a paged cache, as cases that can be timed: attention of a
tree of drafted tokens, the rows of the accepted branch moved to the front, and the pages themselves - sequences that
fork, grow (copy on write), shrink and are freed, a pool that is compacted, blocks that are copied.

``run`` computes them in plain torch operations (floating point in 32 bits), or, with ``own``, through the package's entry
points.  Head counts, head sizes, block sizes, batches and lengths are those of the configured workloads (workloads.py)
and odd ones of the same ranges.

Calls that change page tables or reference counts in place begin a pass with a fresh copy of them: one copy of one
buffer, on both sides.
"""
import math
import random

import numpy as np
import torch

own = False

KV_SCALE = 0.0125           # E4M3 caches of N(0, 1) data: +-448 codes cover +-5.6 sigma
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.uint8}


def _tree(name, dtype, batch, heads, kv_heads, dim, block, prefix, mine, nodes, alibi=False, e4m3=False):
    """prefix: common blocks; mine: range of a sequence's own cached tokens behind them; nodes: range of its tree's tokens."""
    return {"name": name, "kind": "tree", "dtype": dtype, "batch": batch, "heads": heads, "kv_heads": kv_heads, "dim": dim, "block": block,
            "prefix": prefix, "own_lo": mine[0], "own_hi": mine[1], "nodes_lo": nodes[0], "nodes_hi": nodes[1], "alibi": alibi, "e4m3": e4m3}


def _keep(name, dtype, batch, caches, kv_heads, dim, block, most, nodes, path):
    """most: cached tokens of a sequence; nodes: of a tree; path: accepted ones at most."""
    return {"name": name, "kind": "keep", "dtype": dtype, "batch": batch, "caches": caches, "kv_heads": kv_heads, "dim": dim, "block": block,
            "most": most, "nodes": nodes, "path": path}


def _pages(name, kind, batch, block, blocks, forked, change):
    """blocks: entries of a table's row; forked: share of the rows that came from another one; change: tokens by which a row's
    length changes at most."""
    return {"name": name, "kind": kind, "batch": batch, "block": block, "blocks": blocks, "forked": forked, "change": change}


def _compact(name, dtype, batch, caches, kv_heads, dim, block, pool, used):
    return {"name": name, "kind": "compact", "dtype": dtype, "batch": batch, "caches": caches, "kv_heads": kv_heads, "dim": dim, "block": block,
            "pool": pool, "used": used}


def listed():
    return [
        # a tree of eight drafts behind a short prompt of a small model: two launches are all there is
        _tree("tree_one", "f16", 1, 8, 2, 64, 16, 0, (100, 100), (8, 8)),
        # a full batch, each sequence with a tree of 12 to 24 drafts, slopes
        _tree("tree_batch64", "bf16", 64, 32, 8, 128, 32, 0, (511, 2047), (12, 24), alibi=True),
        # two long documents, trees of 64
        _tree("tree_long", "bf16", 2, 64, 8, 128, 16, 0, (32000, 32703), (64, 64)),
        # requests behind a common prompt of 8192 tokens, trees of 20 to 60, 8-bit caches
        _tree("tree_prompt_e4m3", "f16", 16, 32, 4, 128, 32, 256, (63, 511), (20, 60), e4m3=True),
        # the accepted branch of one small tree, two layers
        _keep("keep_one", "f16", 1, 4, 2, 64, 16, 130, 8, 3),
        # a full batch's branches in all caches of 16 layers
        _keep("keep_batch64", "bf16", 64, 32, 8, 128, 16, 500, 61, 9),
        # four beams that go on from two of them
        _pages("fork_beams", "fork", 4, 16, 33, 0.5, 0),
        # a large batch with long tables, a third of it forked or ended
        _pages("fork_batch", "fork", 256, 16, 2048, 0.4, 0),
        # a decode step of a full batch, some rows just forked: one token each
        _pages("resize_step", "resize", 64, 16, 256, 0.4, 1),
        # admission and eviction: rows that end, are cut back, grow by chunks
        _pages("resize_mixed", "resize", 500, 16, 1024, 0.3, 2048),
        # a small pool, two layers
        _compact("compact_small", "f16", 5, 4, 2, 64, 16, 61, 0.5),
        # a pool of 4000 blocks, three quarters in use, 16 layers
        _compact("compact_pool", "bf16", 64, 32, 8, 128, 16, 4000, 0.75),
    ]


def _log(rng, lo, hi):
    """A whole number, spread over the logarithm of lo .. hi."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    case = _draw(rng)
    del case["name"]
    return case


def _draw(rng):
    kind = rng.choice(["tree", "tree", "tree", "tree_e4m3", "keep", "fork", "resize", "resize", "compact"])
    heads, kv_heads = rng.choice([(8, 2), (16, 4), (32, 8), (32, 4), (64, 8), (40, 8), (16, 16)])
    dim, block, dtype = rng.choice([64, 128, 128]), rng.choice([16, 32, 64]), rng.choice(["f16", "bf16"])
    if kind in ("tree", "tree_e4m3"):
        batch, nodes, hi = _log(rng, 1, 64), _log(rng, 1, 64), _log(rng, 1, 32703)
        prefix = _log(rng, 16, 16384) if rng.random() < 0.4 else 0
        while batch * nodes * heads * (prefix + hi) * dim > 3.4e10 or batch * (prefix + hi) * kv_heads * dim > 2.2e8:
            prefix, hi = prefix * 2 // 3, max(hi * 2 // 3, 1)
        return _tree("", dtype, batch, heads, kv_heads, dim, block, -(-prefix // block), (hi // 4, hi), (max(1, nodes // 2), nodes),
                     rng.random() < 0.4, kind == "tree_e4m3")
    if kind == "fork" or kind == "resize":
        batch, blocks = _log(rng, 1, 256 if kind == "fork" else 500), _log(rng, 4, 2048)
        while batch * blocks > 524288:
            blocks = blocks * 2 // 3
        return _pages("", kind, batch, block, blocks, rng.choice([0.0, 0.2, 0.6]), 0 if kind == "fork" else rng.choice([1, 9, 64, 2048]))
    caches, dtype = 2 * _log(rng, 1, 16), rng.choice(["f16", "bf16", "e4m3"])
    if kind == "keep":
        nodes, batch, most = _log(rng, 2, 64), _log(rng, 1, 64), _log(rng, 8, 500)
        return _keep("", dtype, batch, caches, kv_heads if kv_heads < 16 else 8, dim, block, most, nodes, rng.randint(1, min(nodes, 9)))
    pool = _log(rng, 16, 4000 * 16 // block)
    return _compact("", dtype, _log(rng, 1, 64), caches, kv_heads if kv_heads < 16 else 8, dim, block, pool, rng.choice([0.1, 0.3, 0.6, 0.9]))


def _lengths(case):
    """(own cached tokens, tree tokens) of each sequence: the case's own, whatever the seed."""
    rng = random.Random("%(batch)d %(own_lo)d %(own_hi)d %(nodes_lo)d %(nodes_hi)d" % case)
    mine = [rng.randint(case["own_lo"], case["own_hi"]) for _ in range(case["batch"])]
    return mine, [rng.randint(case["nodes_lo"], case["nodes_hi"]) for _ in range(case["batch"])]


def _starts(counts):
    return torch.tensor([0] + np.cumsum(counts).tolist(), dtype=torch.int32)


def prepare(case, seed):
    return {"tree": _prepare_tree, "keep": _prepare_keep, "fork": _prepare_pages, "resize": _prepare_pages,
            "compact": _prepare_compact}[case["kind"]](case, seed)


def _prepare_tree(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    rng = np.random.RandomState(seed % (1 << 32))
    dt, (mine, nodes) = DTYPES[case["dtype"]], _lengths(case)
    B, Hq, Hkv, D, bs, NP = case["batch"], case["heads"], case["kv_heads"], case["dim"], case["block"], case["prefix"]
    lens = [NP * bs + m + n for m, n in zip(mine, nodes)]
    need = [-(-n // bs) for n in lens]
    pool = NP + sum(n - NP for n in need) + 16
    order = torch.from_numpy(rng.permutation(pool).astype(np.int32))
    table = torch.zeros(B, max(need), dtype=torch.int32)
    at = NP
    for b in range(B):
        table[b, :NP] = order[:NP]
        table[b, NP:need[b]] = order[at:at + need[b] - NP]
        at += need[b] - NP
    # trees: each token's parent is one of the eight before it, the first one is the root; a token sees itself and its ancestors
    words = -(-max(nodes) // 32)
    masks, positions = np.zeros((sum(nodes), words), np.uint32), np.zeros(sum(nodes), np.int32)
    t = 0
    for b in range(B):
        for i in range(nodes[b]):
            if i:
                parent = t - rng.randint(1, min(i, 8) + 1)
                masks[t], positions[t] = masks[parent], positions[parent] + 1
            else:
                positions[t] = lens[b] - nodes[b]
            masks[t, i // 32] |= np.uint32(1 << i % 32)
            t += 1

    def cache():
        x = torch.randn((pool, Hkv, bs, D), generator=gen, device="cuda")
        return (x * (1.0 / KV_SCALE)).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) if case["e4m3"] else x.to(dt)

    h = torch.arange(1, Hq + 1, dtype=torch.float64)
    q = torch.randn(sum(nodes), Hq, D, generator=gen, device="cuda").to(dt)
    return {"case": case, "q": q, "out": torch.empty_like(q), "k_cache": cache(), "v_cache": cache(), "table": table.cuda(),
            "prefix": order[:NP].cuda(), "lens": torch.tensor(lens, dtype=torch.int32).cuda(), "cu": _starts(nodes).cuda(),
            "masks": torch.from_numpy(masks.view(np.int32)).cuda(), "positions": torch.from_numpy(positions).cuda(),
            "slopes": torch.exp2(-8.0 * h / Hq).float().cuda() if case["alibi"] else None, "scale": 1.0 / math.sqrt(D),
            "max_len": max(lens), "max_nodes": max(nodes)}


def _caches(case, pool, seed):
    """All layers' caches, one tensor: [caches, blocks, kv heads, block, dim]."""
    gen = torch.Generator("cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    c = torch.empty((case["caches"], pool, case["kv_heads"], case["block"], case["dim"]), dtype=dt, device="cuda")
    for x in c:
        y = torch.randn(x.shape, generator=gen, device="cuda")
        x.copy_((y * (1.0 / KV_SCALE)).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) if dt == torch.uint8 else y)
    return c


def _bits(caches):
    """What a copied or moved row is compared as: its bits."""
    return caches if caches.dtype == torch.uint8 else caches.view(torch.int16)


def _prepare_keep(case, seed):
    rng = np.random.RandomState(seed % (1 << 32))
    B, bs, n = case["batch"], case["block"], case["nodes"]
    start = rng.randint(case["most"] // 4, case["most"] + 1, B)
    need, width = -(-(start + n) // bs), -(-(case["most"] + n) // bs)
    pool = B * width + 3
    order, table, at = rng.permutation(pool), np.zeros((B, width), np.int32), 0
    paths, path_lens = np.full((B, case["path"]), -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
        # trees level by level: a branch begins at the root, may go on along the first tokens, and then lies behind all of its own places
        length = rng.randint(1, case["path"] + 1)
        stay = rng.randint(1, min(length, 2) + 1)
        far = np.sort(rng.permutation(np.arange(length, n))[:length - stay])
        path = np.concatenate([np.arange(stay), far])
        paths[b, :len(path)], path_lens[b] = path, len(path)
    caches = _caches(case, pool, seed)
    return {"case": case, "caches": caches, "table": torch.from_numpy(table).cuda(), "start": torch.from_numpy(start.astype(np.int32)).cuda(),
            "paths": torch.from_numpy(paths).cuda(), "path_lens": torch.from_numpy(path_lens).cuda()}


def _buffer(parts):
    """int32 arrays side by side in one device buffer, each on 16 bytes -> (fresh, working copy, the working copy's views)."""
    places, at = {}, 0
    for name, x in parts.items():
        places[name] = (at, x.shape)
        at += (x.size + 3) // 4 * 4
    flat = np.zeros(at, np.int32)
    for name, x in parts.items():
        flat[places[name][0]:places[name][0] + x.size] = x.reshape(-1)
    fresh = torch.from_numpy(flat).cuda()
    work = torch.empty_like(fresh)
    return fresh, work, {name: work[a:a + math.prod(shape)].view(*shape) for name, (a, shape) in places.items()}


def _rows(rng, B, M, bs, forked, slack):
    """Tables of B rows of up to M blocks, some of them forked from the row before: (tables, lens, reference counts)."""
    lens, tables, refs = np.zeros(B, np.int64), np.zeros((B, M), np.int32), []
    pool = B * M + slack
    order, at = rng.permutation(pool).astype(np.int32), 0
    refs = np.zeros(pool, np.int32)
    for b in range(B):
        lens[b], shared = rng.randint(1, M * bs + 1), 0
        if b and rng.rand() < forked:
            if rng.rand() < 0.5:                             # just forked: all of it, the last block too
                lens[b] = lens[b - 1]
                shared = -(-lens[b] // bs)
            else:                                            # some time ago: whole blocks
                shared = int(rng.randint(0, min(lens[b], lens[b - 1]) // bs + 1))
        have = -(-lens[b] // bs)
        tables[b, :shared] = tables[b - 1, :shared]
        tables[b, shared:have] = order[at:at + have - shared]
        at += have - shared
        refs[tables[b, :have]] += 1
    return tables, lens.astype(np.int32), refs


def _prepare_pages(case, seed):
    rng = np.random.RandomState(seed % (1 << 32))
    B, M, bs = case["batch"], case["blocks"], case["block"]
    tables, lens, refs = _rows(rng, B, M, bs, case["forked"], 5)
    parts = {"tables": tables, "lens": lens, "refs": refs}
    s = {"case": case}
    if case["kind"] == "fork":
        # beams: most rows go on, some twice or more, some not at all, a few places stay empty
        parents = np.where(rng.rand(B) < 0.6, np.arange(B), rng.randint(0, B, B))
        parents = np.where(rng.rand(B) < 0.05, -1, parents)
        s.update(parents=torch.from_numpy(parents.astype(np.int32)).cuda(),
                 tables_out=torch.zeros(B, M, dtype=torch.int32, device="cuda"), lens_out=torch.zeros(B, dtype=torch.int32, device="cuda"))
    else:
        c = case["change"]
        step = rng.randint(0, c + 1, B) if c > 1 else np.ones(B, np.int64)
        if c >= 64:                                          # chunks in, rows cut back, rows that end
            what = rng.rand(B)
            step = np.where(what < 0.25, -step, step)
            step = np.where(what > 0.9, -lens, step)
        new = np.clip(lens + step, 0, M * bs)
        grown = np.maximum(new - lens, 0)
        parts.update(copies=np.full((B, 2), -1, np.int32), counts=np.zeros(2, np.int32))
        s.update(new=torch.from_numpy(new.astype(np.int32)).cuda(), cu=_starts(grown).cuda(), most=int(np.abs(new - lens).max()),
                 slots=torch.zeros(B * c, dtype=torch.int64, device="cuda"))
    s["fresh"], s["work"], views = _buffer(parts)
    return {**s, **views}


def _prepare_compact(case, seed):
    rng = np.random.RandomState(seed % (1 << 32))
    B, bs, pool = case["batch"], case["block"], case["pool"]
    used = max(1, int(pool * case["used"]))
    B = min(B, used)
    blocks = rng.permutation(pool)[:used].astype(np.int32)
    cuts = np.sort(np.random.RandomState(pool).permutation(np.arange(1, used))[:B - 1]) if used > 1 else np.zeros(0, np.int64)
    rows = np.split(blocks, cuts)
    tables, lens, refs = np.zeros((B, max(len(r) for r in rows) + 1), np.int32), np.zeros(B, np.int32), np.zeros(pool, np.int32)
    for b, r in enumerate(rows):
        if b and b % 4 == 0:                                 # begins with the row before's first block
            r = np.concatenate([rows[b - 1][:1], r])
        tables[b, :len(r)] = r
        lens[b] = len(r) * bs - rng.randint(0, bs)
        refs[r] += 1
    s = {"case": case, "caches": _caches(case, pool, seed)}
    s["fresh"], s["work"], views = _buffer({"tables": tables, "lens": lens, "refs": refs, "copies": np.full((max(pool // 2, 1), 2), -1, np.int32),
                                            "counts": np.zeros(2, np.int32)})
    return {**s, **views}


def run(s):
    kind = s["case"]["kind"]
    if kind in ("fork", "resize", "compact"):
        s["work"].copy_(s["fresh"])
    return {"tree": _run_tree, "keep": _run_keep, "fork": _run_fork, "resize": _run_resize, "compact": _run_compact}[kind](s)


def _run_tree(s):
    case = s["case"]
    if not own:
        return {"out": _plain_tree(s)}
    import paper_2505_02351_amd as G
    B, Hq, Hkv, D, bs = case["batch"], case["heads"], case["kv_heads"], case["dim"], case["block"]
    if "ws" not in s:
        n = G.tree_workspace_bytes(s["q"].shape[0], B, Hq, Hkv, D, bs, case["prefix"], s["max_len"], s["max_nodes"])
        s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    args = (s["out"], s["q"], s["k_cache"], s["v_cache"], s["prefix"], s["table"], s["lens"], s["cu"], s["masks"], s["positions"], s["slopes"],
            s["scale"])
    if case["e4m3"]:
        G.paged_attention_tree_fp8(*args, KV_SCALE, KV_SCALE, s["max_len"], s["max_nodes"], s["ws"])
    else:
        G.paged_attention_tree(*args, s["max_len"], s["max_nodes"], s["ws"])
    return {"out": s["out"]}


def _run_keep(s):
    if own:
        import paper_2505_02351_amd as G
        if "set" not in s:
            s["set"] = G.CacheSet(list(s["caches"]))
        G.keep_tokens(s["set"], s["table"], s["start"], s["paths"], s["path_lens"])
    else:
        c, table, start, paths = s["caches"], s["table"].long(), s["start"].long(), s["paths"].long()
        bs = s["case"]["block"]
        i = torch.arange(paths.shape[1], device="cuda")
        there = i < s["path_lens"][:, None]
        row = torch.arange(table.shape[0], device="cuda")[:, None].expand_as(there)[there]
        src, dst = (start[:, None] + paths)[there], (start[:, None] + i)[there]
        c[:, table[row, dst // bs], :, dst % bs] = c[:, table[row, src // bs], :, src % bs]      # (all read, then all written)
    return {"caches": _bits(s["caches"])}


def _run_fork(s):
    if own:
        import paper_2505_02351_amd as G
        G.fork_sequences(s["tables_out"], s["lens_out"], s["tables"], s["lens"], s["refs"], s["parents"], s["case"]["block"])
    else:
        bs, tables, lens, parents = s["case"]["block"], s["tables"], s["lens"], s["parents"].long()
        there = (parents >= 0) & (parents < tables.shape[0])
        p = torch.where(there, parents, 0)
        new = torch.where(there, lens[p], 0)
        j = torch.arange(tables.shape[1], device="cuda")
        before, after = j < (lens[:, None] + bs - 1) // bs, j < (new[:, None] + bs - 1) // bs
        rows = tables[p]
        s["tables_out"].copy_(torch.where(after, rows, s["tables_out"]))
        s["lens_out"].copy_(new)
        s["refs"].index_add_(0, rows.reshape(-1).long(), after.reshape(-1).int())
        s["refs"].index_add_(0, tables.reshape(-1).long(), before.reshape(-1).int(), alpha=-1)
    return {"tables": s["tables_out"], "lens": s["lens_out"], "refs": s["refs"]}


def _run_resize(s):
    if own:
        import paper_2505_02351_amd as G
        B, M, bs = s["case"]["batch"], s["case"]["blocks"], s["case"]["block"]
        if "ws" not in s:
            s["ws"] = torch.empty(G.resize_workspace_bytes(B, M, s["refs"].shape[0]), dtype=torch.uint8, device="cuda")
        G.resize_sequences(s["tables"], s["lens"], s["refs"], s["new"], s["slots"], s["cu"], s["copies"], s["counts"], bs, s["most"], s["ws"])
    else:
        _plain_resize(s)
    return {k: s[k] for k in ("tables", "lens", "refs", "slots", "copies", "counts")}


def _plain_resize(s):
    bs, tables, lens, refs, new, cu = s["case"]["block"], s["tables"], s["lens"], s["refs"], s["new"], s["cu"].long()
    B, M = tables.shape
    j, b = torch.arange(M, device="cuda"), torch.arange(B, device="cuda")
    have, need = (lens + bs - 1) // bs, (new + bs - 1) // bs
    gone = (j >= need[:, None]) & (j < have[:, None])
    refs.index_add_(0, tables.reshape(-1).long(), gone.reshape(-1).int(), alpha=-1)
    # last blocks that are about to be written: replaced where others hold them, but for the last row of those where all of them write
    grows = new > lens
    writes = grows & (lens % bs != 0)
    last = torch.where(writes, tables[b, (lens // bs).clamp(max=M - 1).long()], 0).long()
    writers = torch.zeros_like(refs).index_add_(0, last, writes.int())
    highest = torch.full_like(refs, -1).scatter_reduce_(0, last, torch.where(writes, b, -1).int(), "amax")
    replaced = writes & (refs[last] > 1) & ~((refs[last] == writers[last]) & (highest[last] == b))
    wants = torch.where(grows, need - have, 0) + replaced.int()
    at = wants.cumsum(0) - wants
    free = torch.argsort((refs != 0).int(), stable=True)     # free blocks first, lowest first
    lacking = (wants.sum() - (refs == 0).sum()).clamp(min=0)
    ok = lacking == 0
    refs.index_add_(0, last, (replaced & ok).int(), alpha=-1)
    taken = (at[:, None] + replaced[:, None].int() + (j - have[:, None])).clamp(0, refs.shape[0] - 1)
    added = grows[:, None] & (j >= have[:, None]) & (j < need[:, None]) & ok
    first = free[at.clamp(max=refs.shape[0] - 1)]
    swapped = (replaced & ok)[:, None] & (j == (lens // bs)[:, None])
    pairs = torch.stack([last, first], dim=1).int()
    order = torch.argsort((~(replaced & ok)).int(), stable=True)
    count = (replaced & ok).sum()
    s["copies"].copy_(torch.where((b < count)[:, None], pairs[order], s["copies"]))
    tables.copy_(torch.where(added, free[taken].int(), torch.where(swapped, first[:, None].int(), tables)))
    refs.index_add_(0, tables.reshape(-1).long(), (added | swapped).reshape(-1).int())
    s["counts"].copy_(torch.stack([count, lacking]))
    # where the new tokens go
    t = torch.arange(s["slots"].shape[0], device="cuda")
    row = torch.searchsorted(cu[1:].contiguous(), t, right=True).clamp(max=B - 1)
    pos = lens[row] + (t - cu[row])
    slot = tables[row, (pos // bs).clamp(max=M - 1)].long() * bs + pos % bs
    s["slots"].copy_(torch.where(t < cu[-1], torch.where(ok & (pos < new[row]), slot, -1), s["slots"]))
    lens.copy_(torch.where(grows & ~ok, lens, new))


def _run_compact(s):
    if own:
        import paper_2505_02351_amd as G
        if "ws" not in s:
            s["ws"] = torch.empty(G.compact_workspace_bytes(s["refs"].shape[0]), dtype=torch.uint8, device="cuda")
            s["set"] = G.CacheSet(list(s["caches"]))
        G.compact_blocks(s["tables"], s["lens"], s["refs"], s["copies"], s["counts"], s["case"]["block"], s["ws"])
        G.copy_blocks(s["set"], s["copies"], s["counts"])
    else:
        bs, tables, lens, refs, c = s["case"]["block"], s["tables"], s["lens"], s["refs"], s["caches"]
        used = (refs != 0).sum()
        n = torch.arange(refs.shape[0], device="cuda")
        src, dst = n[(refs != 0) & (n >= used)].flip(0), n[(refs == 0) & (n < used)]
        to = n.clone()
        to[src] = dst
        j = torch.arange(tables.shape[1], device="cuda")
        tables.copy_(torch.where(j < (lens[:, None] + bs - 1) // bs, to[tables.long()].int(), tables))
        refs[dst] = refs[src]
        refs[src] = 0
        s["copies"][:src.shape[0]] = torch.stack([src, dst], dim=1).int()
        s["counts"].copy_(torch.stack([torch.full_like(used, src.shape[0]), used]))
        c[:, dst] = c[:, src]
    return {"caches": _bits(s["caches"]), **{k: s[k] for k in ("tables", "refs", "copies", "counts")}}


def _plain_tree(s):
    """All sequences' keys gathered through their tables and padded to the longest, one masked softmax."""
    case, q, lens, cu = s["case"], s["q"], s["lens"].long(), s["cu"].long()
    B, Hq, Hkv, D, bs = case["batch"], case["heads"], case["kv_heads"], case["dim"], case["block"]
    G, N = Hq // Hkv, s["max_nodes"]
    j = torch.arange(s["max_len"], device="cuda")
    blocks, rows = s["table"][:, j // bs].long(), (j % bs).expand(B, -1)

    def gathered(cache):                                     # [B, Hkv, keys, D]
        x = cache.view(torch.float8_e4m3fn) if case["e4m3"] else cache
        x = x[blocks, :, rows].transpose(1, 2).float()
        return x * torch.tensor(KV_SCALE, dtype=torch.float32) if case["e4m3"] else x

    i, base = torch.arange(N, device="cuda"), lens - (cu[1:] - cu[:-1])
    there = i < (cu[1:] - cu[:-1])[:, None]                  # [B, N]
    token = (cu[:-1, None] + i).clamp(max=q.shape[0] - 1)
    qp = q[token].float().view(B, N, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, N * G, D)
    score = (qp @ gathered(s["k_cache"]).transpose(2, 3)).view(B, Hkv, N, G, -1) * s["scale"]
    c = j - base[:, None]                                    # [B, keys]: which new token a key is
    new = (c >= 0) & (j < lens[:, None])
    bit = c.clamp(0, 32 * s["masks"].shape[1] - 1)
    seen = s["masks"].long()[token].gather(2, (bit // 32)[:, None].expand(-1, N, -1)) >> (bit % 32)[:, None] & 1
    visible = torch.where(new[:, None], seen == 1, (c < 0)[:, None])                                     # [B, N, keys]
    if s["slopes"] is not None:
        pos = torch.where(new, s["positions"][(cu[:-1, None] + c).clamp(0, q.shape[0] - 1)], j)
        dist = (pos[:, None] - s["positions"][token][:, :, None]).float()
        score += s["slopes"].view(Hkv, 1, G, 1) * dist[:, None, :, None]
    score.masked_fill_(~visible[:, None, :, None], -math.inf)
    v = gathered(s["v_cache"]).masked_fill_((j >= lens[:, None])[:, None, :, None], 0.0)
    o = (torch.softmax(score, dim=-1).view(B, Hkv, N * G, -1) @ v).view(B, Hkv, N, G, D)
    return o.permute(0, 2, 1, 3, 4).reshape(B, N, Hq, D)[there].to(q.dtype)


def work(case):
    """Each input once and each output once: of a cache the rows that are attended (common ones once), moved or copied; of
    tables, lengths and reference counts the entries in question."""
    kind = case["kind"]
    if kind == "tree":
        Hq, Hkv, D = case["heads"], case["kv_heads"], case["dim"]
        mine, nodes = _lengths(case)
        P = case["prefix"] * case["block"]
        rows, pairs = P + sum(mine) + sum(nodes), sum(n * (P + m + 1) for m, n in zip(mine, nodes))
        return {"bytes": 2 * rows * Hkv * D * (1 if case["e4m3"] else 2) + 2 * sum(nodes) * Hq * D * 2, "flops": 4 * D * Hq * pairs}
    if kind == "keep":                                       # half of a longest branch moved by each sequence
        row = case["kv_heads"] * case["dim"] * DTYPES[case["dtype"]].itemsize
        return {"bytes": case["batch"] * (case["caches"] * (case["path"] // 2) * 2 * row + 8 + 4 * case["path"]), "flops": 0}
    if kind == "compact":
        block = case["kv_heads"] * case["dim"] * case["block"] * DTYPES[case["dtype"]].itemsize
        used = max(1, int(case["pool"] * case["used"]))
        return {"bytes": int(case["caches"] * used * (1 - used / case["pool"]) * 2 * block + 4 * case["pool"] + 8 * used), "flops": 0}
    if kind == "fork":                                       # rows are half full on average
        entries = case["batch"] * case["blocks"] // 2
        return {"bytes": 8 * entries + 16 * case["batch"], "flops": 0}
    tokens = case["batch"] * (case["change"] + 1) // 2       # each its slot, each block of them an entry and its count
    return {"bytes": 24 * case["batch"] + 8 * tokens + 8 * tokens // case["block"], "flops": 0}


def exact(case, seed):
    """Attention in 64 bits, one head of one sequence at a time; page tables and caches by the definitions, one row and one
    block after another."""
    s = prepare(case, seed)
    if case["kind"] == "tree":
        return {"out": _exact_tree(s)}
    if case["kind"] == "keep":
        return _exact_keep(s)
    s["work"].copy_(s["fresh"])
    h = {k: s[k].cpu().numpy().astype(np.int64) for k in ("tables", "lens", "refs")}
    got = {"fork": _exact_fork, "resize": _exact_resize, "compact": _exact_compact}[case["kind"]](s, **h)
    return {k: torch.from_numpy(v) if isinstance(v, np.ndarray) else v for k, v in got.items()}


def _exact_tree(s):
    case, (mine, nodes) = s["case"], _lengths(s["case"])
    Hkv, D, bs, P = case["kv_heads"], case["dim"], case["block"], case["prefix"] * case["block"]
    group = case["heads"] // Hkv
    one = float(torch.tensor(KV_SCALE, dtype=torch.float32)) if case["e4m3"] else 1.0
    out, t = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda"), 0
    scale = float(torch.tensor(s["scale"], dtype=torch.float32))
    masks = s["masks"].cpu().numpy().view(np.uint32)
    for b in range(case["batch"]):
        n, m = nodes[b], P + mine[b]
        at = torch.arange(m + n, device="cuda")
        phys = s["table"][b].long().repeat_interleave(bs)[:m + n] * bs + at % bs

        def head(cache, g):                                  # [keys, D]
            x = cache[:, g].reshape(-1, D)[phys]
            return (x.view(torch.float8_e4m3fn).float() if case["e4m3"] else x).double() * one

        seen = np.ones((n, m + n), bool)
        for i in range(n):
            seen[i, m:] = [masks[t + i, c // 32] >> np.uint32(c % 32) & 1 == 1 for c in range(n)]
        hidden = torch.from_numpy(~seen).cuda()[:, None]
        pos = s["positions"][t:t + n].double()
        away = (torch.cat([at[:m].double(), pos]) - pos[:, None])[:, None]
        for g in range(Hkv):
            k, v = head(s["k_cache"], g).t().contiguous(), head(s["v_cache"], g)
            x = s["q"][t:t + n, g * group:(g + 1) * group].double()
            sc = (x.reshape(-1, D) @ k).view(n, group, m + n) * scale
            if s["slopes"] is not None:
                sc = sc + s["slopes"][g * group:(g + 1) * group].double()[None, :, None] * away
            w = torch.exp(sc - sc.masked_fill(hidden, -math.inf).amax(dim=2, keepdim=True)).masked_fill(hidden, 0.0)
            o = (w / w.sum(dim=2, keepdim=True)).reshape(-1, m + n) @ v
            out[t:t + n, g * group:(g + 1) * group] = o.view(n, group, D)
        t += n
    return out


def _exact_keep(s):
    c, bs = _bits(s["caches"]), s["case"]["block"]
    table, start, paths, count = (s[k].cpu().numpy() for k in ("table", "start", "paths", "path_lens"))
    for b in range(table.shape[0]):
        for i in range(count[b]):
            src, dst = int(start[b] + paths[b, i]), int(start[b] + i)
            c[:, int(table[b, dst // bs]), :, dst % bs] = c[:, int(table[b, src // bs]), :, src % bs].clone()
    return {"caches": c}


def _exact_fork(s, tables, lens, refs):
    bs, out, new = s["case"]["block"], np.zeros_like(tables), np.zeros_like(lens)
    for i, p in enumerate(s["parents"].tolist()):
        if 0 <= p < len(lens):
            n = -(-lens[p] // bs)
            out[i, :n], new[i] = tables[p, :n], lens[p]
            refs[tables[p, :n]] += 1                         # (a row's blocks are all different)
    for p in range(len(lens)):
        refs[tables[p, :-(-lens[p] // bs)]] -= 1
    return {"tables": out, "lens": new, "refs": refs}


def _exact_resize(s, tables, lens, refs):
    bs, new, cu = s["case"]["block"], s["new"].tolist(), s["cu"].tolist()
    slots, copies, grow = s["slots"].cpu().numpy(), [], []
    for b in range(len(lens)):
        if new[b] > lens[b]:
            grow.append(b)
        else:
            refs[tables[b, -(-new[b] // bs):-(-lens[b] // bs)]] -= 1
            lens[b] = new[b]
    # in order: the last of the writing rows that hold a block by themselves finds it held once
    free, held, plan = np.flatnonzero(refs == 0), refs.copy(), []
    for b in grow:
        j = lens[b] // bs
        if lens[b] % bs and held[tables[b, j]] > 1:
            held[tables[b, j]] -= 1
            plan.append((b, j))
        plan += [(b, j) for j in range(-(-lens[b] // bs), -(-new[b] // bs))]
    lacking = max(len(plan) - len(free), 0)
    if not lacking:
        for (b, j), block in zip(plan, free):
            if j * bs < lens[b]:
                copies.append((tables[b, j], block))
                refs[tables[b, j]] -= 1
            tables[b, j], refs[block] = block, 1
    for b in grow:
        p = np.arange(lens[b], new[b])
        slots[cu[b]:cu[b + 1]] = -1 if lacking else tables[b, p // bs] * bs + p % bs
        lens[b] = lens[b] if lacking else new[b]
    pairs = np.full((len(lens), 2), -1)
    pairs[:len(copies)] = np.array(copies).reshape(-1, 2)
    return {"tables": tables, "lens": lens, "refs": refs, "slots": slots, "copies": pairs, "counts": np.array([len(copies), lacking])}


def _exact_compact(s, tables, lens, refs):
    bs, c, used = s["case"]["block"], _bits(s["caches"]), int((refs > 0).sum())
    src, dst = [n for n in range(len(refs) - 1, used - 1, -1) if refs[n]], [n for n in range(used) if not refs[n]]
    moved = dict(zip(src, dst))
    for a, b in moved.items():
        c[:, b] = c[:, a]
        refs[b], refs[a] = refs[a], 0
    for b in range(len(lens)):
        for j in range(-(-lens[b] // bs)):
            tables[b, j] = moved.get(tables[b, j], tables[b, j])
    pairs = np.full((max(len(refs) // 2, 1), 2), -1)
    pairs[:len(src)] = np.array(list(moved.items())).reshape(-1, 2)
    return {"caches": c, "tables": tables, "refs": refs, "copies": pairs, "counts": np.array([len(src), used])}
