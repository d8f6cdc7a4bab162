"""Plain versions of the page-table calls, one row and one block after another, for the tests."""
import numpy as np


def clamped(lens, M, bs):
    return np.clip(np.asarray(lens, np.int64), 0, M * bs)


def have(length, bs):
    return -(-int(length) // bs)


def resize(tables, lens, refs, new_lens, cu, num_slots, bs):
    """Changed copies of tables, lens, refs; (slots, or -2 where nothing is written), pairs, blocks lacking."""
    tables, refs = tables.copy(), refs.copy()
    M, NB = tables.shape[1], len(refs)
    old, new, lens = clamped(lens, M, bs), clamped(new_lens, M, bs), lens.copy()

    def hold(block, n):
        if 0 <= block < NB:
            refs[block] += n

    grow = []
    for b in range(len(lens)):
        if new[b] > old[b]:
            grow.append(b)
            continue
        for j in range(have(new[b], bs), have(old[b], bs)):
            hold(tables[b, j], -1)
        lens[b] = new[b]
    held, plan = refs.copy(), []
    for b in grow:
        last = tables[b, old[b] // bs] if old[b] % bs else -1
        if 0 <= last < NB and held[last] > 1:
            held[last] -= 1
            plan.append((b, old[b] // bs, True))
        plan += [(b, j, False) for j in range(have(old[b], bs), have(new[b], bs))]
    free = np.flatnonzero(refs == 0)
    lacking = max(len(plan) - len(free), 0)
    pairs = []
    if not lacking:
        for (b, j, copy), block in zip(plan, free):
            if copy:
                pairs.append((tables[b, j], block))
                refs[tables[b, j]] -= 1
            tables[b, j], refs[block] = block, 1
        for b in grow:
            lens[b] = new[b]
    slots = np.full(num_slots, -2, np.int64)
    for b in range(len(lens)):
        for i in range(cu[b + 1] - cu[b]):
            if 0 <= cu[b] + i < num_slots:
                pos = old[b] + i
                slots[cu[b] + i] = tables[b, pos // bs] * bs + pos % bs if b in grow and pos < lens[b] else -1
    return tables, lens, refs, slots, pairs, lacking


def fork(tables, lens, refs, parents, bs):
    """(new rows as lists of blocks, new lens, refs)."""
    refs, M = refs.copy(), tables.shape[1]
    old = clamped(lens, M, bs)
    rows, new = [], []
    for p in parents:
        there = 0 <= p < len(lens)
        new.append(old[p] if there else 0)
        rows.append(tables[p, :have(new[-1], bs)].copy() if there else tables[:0, 0])
        for block in rows[-1]:
            if 0 <= block < len(refs):
                refs[block] += 1
    for p in range(len(lens)):
        for block in tables[p, :have(old[p], bs)]:
            if 0 <= block < len(refs):
                refs[block] -= 1
    return rows, np.array(new, np.int64), refs


def compact(tables, lens, refs, most, bs):
    tables, refs = tables.copy(), refs.copy()
    used = int((refs > 0).sum())
    src, dst = [n for n in range(len(refs) - 1, used - 1, -1) if refs[n] > 0], [n for n in range(used) if refs[n] <= 0]
    pairs = list(zip(src, dst))[:most]
    moved = dict(pairs)
    for a, b in pairs:
        refs[b], refs[a] = refs[a], 0
    for r, n in enumerate(clamped(lens, tables.shape[1], bs)):
        for j in range(have(n, bs)):
            tables[r, j] = moved.get(int(tables[r, j]), tables[r, j])
    return tables, refs, pairs, used


def pool(rng, B, M, bs, spare, shared, just_forked=0.3, full=False):
    """Random tables of B rows of up to M blocks, some of which share blocks with the row before; entries not in use name no block.
    -> (tables, lens, refs)"""
    NB = B * M + spare
    order, at = rng.permutation(NB).astype(np.int32), 0
    tables, lens, refs = np.full((B, M), -7, np.int32), np.zeros(B, np.int32), np.zeros(NB, np.int32)
    for b in range(B):
        lens[b], keep = (M * bs if full else rng.randint(0, M * bs + 1)), 0
        if b and rng.rand() < just_forked:
            lens[b] = lens[b - 1]
            keep = have(lens[b], bs)
        elif b and rng.rand() < shared:
            keep = rng.randint(0, min(lens[b], lens[b - 1]) // bs + 1)
        n = have(lens[b], bs)
        tables[b, :keep] = tables[b - 1, :keep]
        tables[b, keep:n] = order[at:at + n - keep]
        at += n - keep
        refs[tables[b, :n]] += 1
    return tables, lens, refs
