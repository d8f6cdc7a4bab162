"""Attention of trees of new tokens, against plain attention in 64 bits over the keys that each token's mask lets it see."""
import numpy as np
import pytest

import step_reference as R
from test_gpu_common_prefix import Batch, G  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def attend(q, keys, values, visible, distance, slopes, scale):
    """Rows q [n, Hq, D] over keys, values [L, Hkv, D] where visible [n, L], distance [n, L] away -> (out, what the weights average)."""
    n, Hq, D = q.shape
    out, size, group = np.zeros((n, Hq, D)), np.zeros((n, Hq, D)), Hq // keys.shape[1]
    for i in range(n):
        see = np.flatnonzero(visible[i])
        if len(see) == 0:
            continue
        for h in range(Hq):
            s = scale * (keys[see, h // group] @ q[i, h]) + (0.0 if slopes is None else slopes[h] * distance[i, see])
            w = np.exp(s - s.max())
            w /= w.sum()
            out[i, h], size[i, h] = w @ values[see, h // group], w @ np.abs(values[see, h // group])
    return out, size


class Trees(Batch):
    """Batch whose new tokens are trees ("tree"), see any of each other ("any") or themselves and all before them ("line"); bits behind a
    sequence's tokens are set at random."""

    def __init__(self, seed, dtype, Hq, Hkv, D, bs, NP, lens, new, kind="tree", words=None, **kw):
        super().__init__(seed, dtype, Hq, Hkv, D, bs, NP, lens, new, **kw)
        rng = np.random.RandomState(seed)
        words = words or max(-(-max(new) // 32), 1)
        self.seen, self.depth = [], []
        self.masks, self.positions = rng.randint(0, 1 << 32, (self.T, words), dtype=np.uint64).astype(np.uint32), rng.randint(0, 99, self.T).astype(np.int32)
        for b, n in enumerate(new):
            seen, depth = np.zeros((n, n), bool), np.zeros(n, np.int64)
            for i in range(n):
                if kind == "any":
                    seen[i] = rng.rand(n) < rng.choice([0.0, 0.1, 0.5])
                    depth[i] = rng.randint(0, 50)
                elif kind == "line":
                    seen[i, :i + 1], depth[i] = True, i
                else:
                    parent = rng.randint(max(i - 6, -1), i) if i else -1
                    if parent >= 0:
                        seen[i], depth[i] = seen[parent], depth[parent] + 1
                    seen[i, i] = True
            for i in range(n):
                t = self.cu[b] + i
                for c in range(n):
                    bit = np.uint32(1 << c % 32)
                    self.masks[t, c // 32] = self.masks[t, c // 32] | bit if seen[i, c] else self.masks[t, c // 32] & ~bit
                self.positions[t] = lens[b] - n + depth[i]
            self.seen.append(seen)
            self.depth.append(depth)

    def run(self, G, scales="heads", no_cu=False, bounds=(0, 0), positions=True):  # noqa: F811
        import torch
        Hq, Hkv, D = self.shape
        B, most, n = len(self.lens), max(self.lens) + bounds[0], max(max(self.new), 1) + bounds[1]
        need = G.tree_workspace_bytes(self.T, B, Hq, Hkv, D, self.bs, self.NP, most, n)
        raw = torch.full((need + 8192,), 0x7F, dtype=torch.uint8, device="cuda")
        around = torch.full((self.T * Hq * D + 2048,), float("nan"), dtype=self.t, device="cuda")
        out = around[1024:-1024].view(self.T, Hq, D)
        table = torch.full((B, max(self.table.shape[1], -(-most // self.bs))), 1 << 28, dtype=torch.int32)
        table[:, :self.table.shape[1]] = self.table
        args = (out, self.q.cuda(), self.kc, self.vc, self.prefix.cuda(), table.cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda(),
                None if no_cu else torch.from_numpy(self.cu).cuda(), torch.from_numpy(self.masks.view(np.int32)).cuda(),
                torch.from_numpy(self.positions).cuda() if positions else None, None if self.slopes is None else self.slopes.cuda(), self.scale)
        tail = (most, n, raw[4096:-4096])
        if not self.kv8:
            G.paged_attention_tree(*args, *tail)
        elif scales == "heads":
            G.paged_attention_tree_fp8_heads(*args, self.k_scales.cuda(), self.v_scales.cuda(), *tail)
        else:
            G.paged_attention_tree_fp8(*args, 0.0125, 0.02, *tail)
        torch.cuda.synchronize()
        assert (raw[:4096] == 0x7F).all() and (raw[-4096:] == 0x7F).all(), "a kernel wrote outside the workspace"
        assert torch.isnan(around[:1024]).all() and torch.isnan(around[-1024:]).all(), "a kernel wrote outside out"
        return out

    def reference(self, scales="heads"):
        """(out, size) of all tokens."""
        Hq, Hkv, D = self.shape
        P = self.NP * self.bs
        ks, vs = np.ones((1, Hkv, 1)), np.ones((1, Hkv, 1))
        if self.kv8:
            ks, vs = (self.k_scales.double().numpy()[None, :, None], self.v_scales.double().numpy()[None, :, None]) if scales == "heads" else (
                np.float64(np.float32(0.0125)), np.float64(np.float32(0.02)))
        slopes = None if self.slopes is None else self.slopes.double().numpy()
        out, size = np.zeros((self.T, Hq, D)), np.zeros((self.T, Hq, D))
        for b, (L, n) in enumerate(zip(self.lens, self.new)):
            if n == 0:
                continue
            keys = np.concatenate([self.k[-1].double().numpy()[:min(L, P)], self.k[b].double().numpy()]) * ks
            values = np.concatenate([self.v[-1].double().numpy()[:min(L, P)], self.v[b].double().numpy()]) * vs
            base, t = L - n, slice(self.cu[b], self.cu[b] + n)
            visible, at = np.zeros((n, L), bool), np.arange(L)
            visible[:, :max(base, 0)] = True
            there = np.arange(max(base, 0), L)
            visible[:, there] = self.seen[b][:, there - base] & (there >= P)
            where = at.copy()
            where[there] = self.positions[t][there - base]
            out[t], size[t] = attend(self.q[t].double().numpy(), keys, values, visible, where[None] - self.positions[t][:, None], slopes, self.scale)
        return out, size

    def check(self, out, scales="heads"):
        got = out.double().cpu().numpy()
        ref, size = self.reference(scales)
        assert not got[self.cu[-1]:].any()                        # tokens of no sequence
        bar = R.attention_bar(ref, size, self.dtype)
        off = np.abs(got - ref)
        assert (off <= bar).all(), (float(np.nanmax(off / bar)), np.argwhere(~(off <= bar))[:4].tolist())
        assert not got[(size == 0).all(axis=(1, 2))].any()


SHAPES = [
    # Hq, Hkv, D, bs, prefix blocks, lengths, new tokens
    (8, 2, 64, 16, 0, [100], [8]),
    (8, 2, 64, 16, 0, [1, 2, 40], [1, 2, 40]),
    (4, 4, 128, 32, 0, [33, 64, 65, 31], [1, 32, 33, 31]),
    (16, 2, 128, 16, 0, [300, 17, 700], [24, 16, 64]),
    (12, 4, 64, 64, 0, [200, 130, 64], [65, 100, 64]),
    (8, 1, 128, 16, 3, [60, 48 + 5, 200, 99], [12, 5, 31, 0]),
    (32, 8, 128, 32, 8, [256 + 7, 400], [7, 60]),
    (10, 2, 64, 16, 5, [81, 90, 500], [1, 3, 9]),
]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("kind,slopes", [("tree", False), ("tree", True), ("any", True), ("line", True)])
def test_trees(G, shape, dtype, kind, slopes):  # noqa: F811
    t = Trees(len(kind) + len(shape[5]), dtype, *shape, kind=kind, slopes=slopes, pad_tokens=3).upload()
    t.check(t.run(G))


@pytest.mark.parametrize("shape", [SHAPES[1], SHAPES[3], SHAPES[4], SHAPES[5], SHAPES[6]])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("scales", ["heads", "tensor"])
def test_trees_over_8_bit_caches(G, shape, dtype, scales):  # noqa: F811
    t = Trees(5, dtype, *shape, kind="tree", slopes=scales == "heads", kv8=True).upload()
    t.check(t.run(G, scales), scales)


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("B,lens,new,NP", [(1, 5000, 50, 0), (2, 9000, 16, 0), (70, 90, 5, 0), (130, 200, 3, 4), (3, 4100, 40, 200)])
def test_long_contexts_and_many_sequences(G, kv8, B, lens, new, NP):  # noqa: F811
    """Walks of several pieces and of more than 64 blocks, more than 64 sequences, bounds above what there is."""
    rng = np.random.RandomState(B)
    many = [int(rng.randint(max(lens // 2, new + NP * 16), lens + 1)) for _ in range(B)]
    t = Trees(B, "bf16", 8, 2, 64, 16, NP, many, [int(rng.randint(0, new + 1)) for _ in range(B - 1)] + [new], slopes=True, kv8=kv8).upload()
    t.check(t.run(G))
    t.check(t.run(G, bounds=(999, 14)))


@pytest.mark.parametrize("kv8", [False, True])
def test_many_row_tiles_over_a_prefix(G, kv8):  # noqa: F811
    """More row tiles than fill the CUs once in one range of keys, sequences of one, two and four row blocks to a workgroup."""
    rng = np.random.RandomState(2)
    new = [int(n) for n in rng.randint(1, 40, 40)]
    t = Trees(2, "f16", 32, 16, 64, 16, 20, [320 + n + int(rng.randint(0, 90)) for n in new], new, slopes=True, kv8=kv8).upload()
    t.check(t.run(G))


def test_rows_that_see_nothing(G):  # noqa: F811
    """No context and an empty mask: +0, whatever the neighbours see."""
    t = Trees(3, "f16", 8, 2, 64, 16, 0, [40, 3, 70], [40, 3, 33], kind="any")
    t.seen[0][5] = t.seen[0][39] = t.seen[1][:] = False
    for i in (5, 39, 40, 41, 42):
        t.masks[i, :] = 0
        t.masks[i, 1:] = 0xffffff00                                # (bits behind the last token)
    t.upload()
    out = t.run(G)
    t.check(out)
    got = out.cpu().view(-1, 8, 64)
    for i in (5, 39, 40, 41, 42):
        assert (got[i].view(dtype=__import__("torch").int16) == 0).all()


@pytest.mark.parametrize("bound", [0, 9000])
@pytest.mark.parametrize("kv8", [False, True])
def test_contexts_that_hold_only_the_last_of_the_new_tokens(G, bound, kv8):  # noqa: F811
    """Lengths below the number of new tokens: those that lie in front of the first row are not there; none at all: +0.  Under a tight bound
    (one launch) and a wide one (two)."""
    t = Trees(13, "bf16", 16, 4, 64, 16, 0, [3, 0, 40, 1, 31], [5, 4, 40, 33, 0], slopes=True, kv8=kv8, pad_tokens=2).upload()
    t.check(t.run(G, bounds=(bound, 0)))


@pytest.mark.parametrize("NP", [0, 2])
def test_a_batch_of_long_and_short_ones(G, NP):  # noqa: F811
    """Sequences of one piece, which write their output, beside some of several, in one row block of the join."""
    lens, new = [700 if b % 5 == 3 else 40 + b for b in range(20)], [1 + b % 4 for b in range(20)]
    lens[7], new[11] = 6000, 0
    t = Trees(14, "f16", 8, 2, 64, 16, NP, lens, new, slopes=True, pad_tokens=1).upload()
    t.check(t.run(G))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_one_new_token_each(G, dtype):  # noqa: F811
    """A decode step: no prefix sums; tokens that see themselves and one that does not."""
    t = Trees(4, dtype, 16, 4, 128, 16, 2, [33, 64, 100, 47], [1, 1, 1, 1], slopes=True)
    t.seen[2][:] = False
    t.masks[2] = 0xfffffffe
    t.upload()
    t.check(t.run(G, no_cu=True))


def test_new_tokens_in_the_prefix_are_not_seen(G):  # noqa: F811
    """A context that ends in the prefix, or began there with its new tokens."""
    t = Trees(6, "bf16", 8, 2, 64, 16, 4, [50, 70, 64, 5], [20, 10, 3, 9], slopes=True).upload()
    t.check(t.run(G))


def test_positions_without_slopes_are_not_needed(G):  # noqa: F811
    t = Trees(7, "bf16", 8, 2, 64, 16, 0, [50, 70], [20, 10]).upload()
    a, b = t.run(G), t.run(G, positions=False)
    assert a.view(dtype=__import__("torch").int16).equal(b.view(dtype=__import__("torch").int16))
    t.check(a)


@pytest.mark.parametrize("far", [0, 1 << 29])
def test_distances_are_whole_numbers_differences(G, far):  # noqa: F811
    """Slopes go by the positions that tokens are said to have, however far those are from the rows that they lie in."""
    t = Trees(8, "f16", 8, 2, 64, 16, 0, [33, 20], [33, 20], slopes=True)
    t.positions = (t.positions + far).astype(np.int32)
    t.upload()
    t.check(t.run(G))


@pytest.mark.parametrize("kv8,bad", [(False, float("nan")), (False, float("inf")), (False, -float("inf")), (True, float("nan"))])
def test_what_a_row_does_not_see_does_not_reach_it(G, kv8, bad):  # noqa: F811
    """Keys and values that are no finite numbers, of drafts that some rows see and others do not (E4M3: NaN): rows that do not
    see them are as they were, rows that do are no finite numbers in the value's element."""
    import torch
    t = Trees(9, "bf16", 8, 2, 64, 16, 1, [100, 50], [40, 20], slopes=True, kv8=kv8).upload()
    clean = t.run(G)
    t.check(clean)
    node = 3                                                       # of both sequences
    for b in range(2):
        own = t.lens[b] - t.new[b] + node - 16
        t.v[b] = t.v[b].clone().float()
        t.v[b][own, :, 5] = bad
        t.v[b] = t.v[b].to(torch.float8_e4m3fn if kv8 else torch.bfloat16)
    t.upload()
    out = t.run(G).float().cpu()
    for b in range(2):
        for i in range(t.new[b]):
            row, was = out[t.cu[b] + i], clean[t.cu[b] + i].float().cpu()
            if t.seen[b][i, node]:
                assert not torch.isfinite(row[:, 5]).any() and torch.equal(row[:, :5], was[:, :5])
            else:
                assert torch.equal(row, was)
    # a key that some rows see: the others are as they were
    t = Trees(9, "bf16", 8, 2, 64, 16, 1, [100, 50], [40, 20], slopes=True, kv8=kv8)
    for b in range(2):
        k = t.k[b].clone().float()
        k[t.lens[b] - t.new[b] + node - 16] = bad
        t.k[b] = k.to(torch.float8_e4m3fn if kv8 else torch.bfloat16)
    out = t.upload().run(G).float().cpu()
    for b in range(2):
        for i in range(t.new[b]):
            if not t.seen[b][i, node]:
                assert torch.equal(out[t.cu[b] + i], clean[t.cu[b] + i].float().cpu())


def test_a_line_is_the_common_call_s(G):  # noqa: F811
    """A tree without branches: what paged_attention_common gives, to rounding."""
    import torch
    t = Trees(10, "bf16", 16, 4, 128, 16, 4, [200, 90, 65], [9, 26, 1], kind="line", slopes=True).upload()
    a, b = t.run(G), Batch.run(t, G)
    ref, size = t.reference()
    bar = R.attention_bar(ref, size, "bf16")
    assert (np.abs(a.double().cpu().numpy() - b.double().cpu().numpy()) <= 2 * bar).all() and not torch.isnan(a).any()


def test_captured_and_on_another_stream(G):  # noqa: F811
    """One graph, replayed with other lengths, tables, masks and positions in its tensors, between eager calls that share its
    workspace; and on a stream of its own."""
    import torch
    sizes = [([120, 60, 200], [9, 20, 30]), ([55, 300, 31], [16, 1, 31]), ([1, 90, 64], [1, 40, 18]), ([300, 300, 300], [20, 20, 19])]
    all_t = [Trees(20 + i, "f16", 8, 2, 64, 16, 0, lens, new, slopes=True, words=2, pad_tokens=59 - sum(new)).upload() for i, (lens, new) in enumerate(sizes)]
    T, NB = 59, max(t.kc.shape[0] for t in all_t)
    need = G.tree_workspace_bytes(T, 3, 8, 2, 64, 16, 0, 300, 40)
    ws = torch.full((need,), 0xa5, dtype=torch.uint8, device="cuda")
    kc, vc = (torch.zeros(NB, 2, 16, 64, dtype=torch.float16, device="cuda") for _ in range(2))
    q, out = (torch.zeros(T, 8, 64, dtype=torch.float16, device="cuda") for _ in range(2))
    table, lens, cu = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in ((3, 19), (3,), (4,)))
    masks, positions = torch.zeros(T, 2, dtype=torch.int32, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda")
    none, slopes = torch.zeros(0, dtype=torch.int32, device="cuda"), all_t[0].slopes.cuda()

    def call():
        G.paged_attention_tree(out, q, kc, vc, none, table, lens, cu, masks, positions, slopes, all_t[0].scale, 300, 40, ws)

    def load(t):
        kc[:t.kc.shape[0]] = t.kc
        vc[:t.vc.shape[0]] = t.vc
        q.copy_(t.q), lens.copy_(torch.tensor(t.lens)), cu.copy_(torch.from_numpy(t.cu))
        table[:, :t.table.shape[1]] = t.table.cuda()
        masks.copy_(torch.from_numpy(t.masks.view(np.int32))), positions.copy_(torch.from_numpy(t.positions))
        torch.cuda.synchronize()

    load(all_t[0])
    call()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        call()
    for step in range(8):
        t = all_t[step % 4]
        load(t)
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        t.check(out)
        first = out.clone()
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            call()
        torch.cuda.synchronize()
        assert torch.equal(first, out)
