"""Trees of new tokens where a workgroup walks far: over more blocks than a wave holds numbers of at a time, through steps that ask for tiles ahead
without clamps, over row blocks of one, two and four to a workgroup, in a prefix and in own parts; and joins of many pieces.  Each shape says what it is
for, and the library's rules are asked whether it still is.  Against attention in 64 bits."""
import math

import numpy as np
import pytest

import step_reference as R
import tree_walks as W
from test_gpu_common_prefix import G  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu

HELD = 64                   # block numbers of a wave
AHEAD = 8                   # more tiles than are asked for ahead of an unclamped step, with those that end it


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    return W.build(tmp_path_factory.mktemp("walks"))


class Trees:
    """Sequences behind NP common blocks; keys, values and queries of a normal distribution on the GPU.  Blocks of nobody and rows behind a context in its
    last block are no numbers; table entries that no row may follow lead to such a block."""

    def __init__(self, seed, dtype, Hq, Hkv, D, bs, NP, lens, new, kv8, slopes):
        import torch
        self.t = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
        self.dtype, self.shape, self.bs, self.NP, self.lens, self.new, self.kv8 = dtype, (Hq, Hkv, D), bs, NP, lens, new, kv8
        gen, rng, B = torch.Generator("cuda").manual_seed(seed), np.random.RandomState(seed), len(lens)
        own = [max(0, -(-n // bs) - NP) for n in lens]
        pool = NP + sum(own) + 3
        order = rng.permutation(pool).astype(np.int32)
        table, at = np.full((B, NP + max(own)), order[-1], np.int32), NP
        for b in range(B):
            table[b, NP:NP + own[b]] = order[at:at + own[b]]
            at += own[b]
        self.prefix, self.table = torch.from_numpy(order[:NP]).cuda(), torch.from_numpy(table).cuda()
        self.scale, self.ks, self.vs = 1.0 / math.sqrt(D), 0.0125, 0.02

        def cache():
            x = torch.randn(pool, Hkv, bs, D, generator=gen, device="cuda")
            x = (x * 80).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) if kv8 else x.to(self.t)
            bad = 0x7f if kv8 else float("nan")
            x[torch.from_numpy(order[at:]).long().cuda()] = bad
            for b in range(B):
                if own[b] and lens[b] % bs:
                    x[int(table[b, NP + own[b] - 1]), :, lens[b] % bs:] = bad
            return x

        self.kc, self.vc = cache(), cache()
        self.T = sum(new)
        self.q = torch.randn(self.T, Hq, D, generator=gen, device="cuda").to(self.t)
        self.cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        words = -(-max(new) // 32)
        masks, self.positions = np.zeros((self.T, 32 * words), bool), np.zeros(self.T, np.int32)
        for b, n in enumerate(new):
            for i in range(n):
                t, up = self.cu[b] + i, self.cu[b] + i - rng.randint(1, 7)
                if up >= self.cu[b]:
                    masks[t], self.positions[t] = masks[up], self.positions[up] + 1
                else:
                    self.positions[t] = lens[b] - n
                masks[t, i] = True
        self.masks = masks
        self.slopes = torch.exp2(-8.0 * torch.arange(1, Hq + 1) / Hq).cuda() if slopes else None

    def run(self, G):  # noqa: F811
        import torch
        Hq, Hkv, D = self.shape
        most, n = max(self.lens), max(self.new)
        out = torch.full_like(self.q, float("nan"))
        need = G.tree_workspace_bytes(self.T, len(self.lens), Hq, Hkv, D, self.bs, self.NP, most, n)
        ws = torch.full((need,), 0x7f, dtype=torch.uint8, device="cuda")
        masks = torch.from_numpy(np.packbits(self.masks, axis=1, bitorder="little").view(np.int32)).cuda()
        args = (out, self.q, self.kc, self.vc, self.prefix, self.table, torch.tensor(self.lens, dtype=torch.int32).cuda(), torch.from_numpy(self.cu).cuda(),
                masks, torch.from_numpy(self.positions).cuda(), self.slopes, self.scale)
        if self.kv8:
            G.paged_attention_tree_fp8(*args, self.ks, self.vs, most, n, ws)
        else:
            G.paged_attention_tree(*args, most, n, ws)
        torch.cuda.synchronize()
        return out

    def check(self, out):
        import torch
        Hq, Hkv, D = self.shape
        group, P = Hq // Hkv, self.NP * self.bs
        one_k, one_v = (float(np.float32(x)) if self.kv8 else 1.0 for x in (self.ks, self.vs))
        for b, (L, n) in enumerate(zip(self.lens, self.new)):
            if n == 0:
                continue
            base, at, rows = L - n, torch.arange(L, device="cuda"), slice(self.cu[b], self.cu[b] + n)
            blocks = torch.where(at < P, self.prefix[(at // self.bs).clamp(max=max(self.NP - 1, 0))] if self.NP else 0, self.table[b, at // self.bs]).long()
            positions = torch.from_numpy(self.positions[rows]).cuda().double()
            hidden = torch.zeros(n, L, dtype=torch.bool, device="cuda")
            hidden[:, base:] = torch.from_numpy(~self.masks[rows, :n]).cuda()
            hidden[:, base:P] = True                             # (new tokens in the prefix)
            away = torch.cat([at[:base].double(), positions]) - positions[:, None]

            def head(cache, g):
                x = cache[blocks, g, at % self.bs]
                return x.view(torch.float8_e4m3fn).double() if self.kv8 else x.double()

            for g in range(Hkv):
                k, v = head(self.kc, g) * one_k, head(self.vc, g) * one_v
                q = self.q[rows, g * group:(g + 1) * group].double().reshape(n * group, D)
                s = (q @ k.t().contiguous()).view(n, group, L) * self.scale
                if self.slopes is not None:
                    s += self.slopes[g * group:(g + 1) * group].double()[None, :, None] * away[:, None]
                s.masked_fill_(hidden[:, None], -math.inf)
                w = torch.softmax(s, dim=2).view(n * group, L)
                ref, size = (w @ v).cpu().numpy(), (w @ v.abs()).cpu().numpy()
                got = out[rows, g * group:(g + 1) * group].double().reshape(n * group, D).cpu().numpy()
                off, bar = np.abs(got - ref), R.attention_bar(ref, size, self.dtype)
                assert (off <= bar).all(), (b, g, float(np.nanmax(off / bar)), np.argwhere(~(off <= bar))[:4].tolist())


def cus():
    import torch
    return torch.cuda.get_device_properties(0).multi_processor_count


KINDS = [("f16", False), ("bf16", False), ("f16", True), ("bf16", True)]


# Hq, Hkv, D, bs, lengths, new tokens, row blocks to a workgroup
OWN = [
    (32, 8, 128, 16, [11000 + 37 * b for b in range(8)], [8] * 8, 1),
    (32, 8, 128, 16, [10000 + 41 * b for b in range(8)], [16] * 8, 2),
    (16, 2, 128, 16, [36000, 40003], [128, 121], 4),
    (64, 8, 128, 32, [33000, 36001], [64, 50], 4),
    (16, 16, 64, 16, [7000 + 11 * b for b in range(8)], [50] * 8, 2),
    (16, 2, 64, 16, [40000, 36003], [120, 128], 4),
]


@pytest.mark.parametrize("dtype,kv8", KINDS)
@pytest.mark.parametrize("shape", OWN, ids=lambda s: "%d-%d-%d-%d" % (s[0], s[1], s[2], s[6]))
def test_long_walks_of_own_parts(G, rules, shape, dtype, kv8):  # noqa: F811
    Hq, Hkv, D, bs, lens, new, row_waves = shape
    p, own = W.walks(rules, Hq, Hkv, 0, lens, new, cus())
    for o in own:
        assert o.row_waves == row_waves and o.tiles * 32 * (4 // row_waves) > HELD * bs and o.tiles > AHEAD, (p, o)
    t = Trees(1, dtype, Hq, Hkv, D, bs, 0, lens, new, kv8, slopes=D == 64)
    t.check(t.run(G))


# Hq, Hkv, D, bs, prefix blocks, own tokens of each sequence, new tokens, row blocks to a workgroup
PREFIX = [
    (8, 8, 128, 16, 2300, [20, 31], [14, 17], 1),
    (32, 8, 128, 16, 2300, [20, 31], [7, 9], 2),
    (32, 4, 128, 16, 1000, [100 + b for b in range(16)], [20 + b for b in range(16)], 4),
    (32, 8, 64, 16, 1000, [90 + b for b in range(16)], [40 + b for b in range(16)], 4),
]


@pytest.mark.parametrize("dtype,kv8", KINDS)
@pytest.mark.parametrize("shape", PREFIX, ids=lambda s: "%d-%d-%d-%d" % (s[0], s[1], s[2], s[7]))
def test_long_walks_of_a_prefix(G, rules, shape, dtype, kv8):  # noqa: F811
    Hq, Hkv, D, bs, NP, mine, new, row_waves = shape
    lens = [NP * bs + m + n for m, n in zip(mine, new)]
    p, _ = W.walks(rules, Hq, Hkv, NP * bs, lens, new, cus())
    assert p.row_waves == row_waves and p.keys > HELD * bs and p.keys // (32 * (4 // row_waves)) > AHEAD, p
    t = Trees(2, dtype, Hq, Hkv, D, bs, NP, lens, new, kv8, slopes=D == 64)
    t.check(t.run(G))


@pytest.mark.parametrize("dtype,kv8", KINDS)
@pytest.mark.parametrize("D", [64, 128])
def test_a_join_of_written_and_unwritten_rows(G, rules, D, dtype, kv8):  # noqa: F811
    """No prefix, enough rows for the join that gives a workgroup all dims: segments of one piece, which have written their output, share row blocks of 32
    with segments of more than four."""
    new = [3 + b % 5 for b in range(48)]
    lens = [9000 + 100 * b if b % 6 == 2 else 30 + 7 * b for b in range(48)]
    p, own = W.walks(rules, 32, 8, 0, lens, new, cus())
    assert p.slots * 8 * 4 >= 3 * cus() and not p.one_launch
    assert max(o.pieces for o in own) > 4 and sum(o.pieces == 1 for o in own) > 30
    t = Trees(3, dtype, 32, 8, D, 16, 0, lens, new, kv8, slopes=True)
    t.check(t.run(G))


@pytest.mark.parametrize("dtype,kv8", KINDS)
@pytest.mark.parametrize("D", [64, 128])
def test_a_join_of_many_pieces(G, rules, D, dtype, kv8):  # noqa: F811
    """The same join behind a prefix of more than four ranges, with own parts of more than four pieces beside some of none."""
    NP, new = 1600, [9 + b % 4 for b in range(20)]
    lens = [NP * 16 + n + (7000 if b % 5 == 1 else 0 if b % 5 == 3 else 40 * b) for b, n in enumerate(new)]
    lens[3], lens[8] = NP * 16 - 100, NP * 16                # contexts that end in the prefix
    p, own = W.walks(rules, 32, 8, NP * 16, lens, new, cus())
    assert p.slots * 8 * 4 >= 3 * cus() and p.ranges > 4 and max(o.pieces for o in own) > 4 and min(o.pieces for o in own) == 0, (p, own)
    t = Trees(4, dtype, 32, 8, D, 16, NP, lens, new, kv8, slopes=True)
    t.check(t.run(G))
