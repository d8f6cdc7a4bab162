"""Attention with one common prefix for the batch, against plain attention in 64 bits over each sequence's own tokens."""
import math

import numpy as np
import pytest

import step_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    import paper_2505_02351_amd as G
    G.load_library()
    return G


class Batch:
    """Sequences behind a prefix of NP blocks, lens[b] tokens in all of which the last new[b] are query tokens.  What no row may
    read is poisoned: blocks of nobody, rows behind a context in its last block, and own table entries below the prefix."""

    def __init__(self, seed, dtype, Hq, Hkv, D, bs, NP, lens, new, slopes=False, kv8=False, pad_tokens=0, first_block=0):
        import torch
        self.t = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
        self.dtype, self.lens, self.new, self.NP, self.bs, self.kv8 = dtype, list(lens), list(new), NP, bs, kv8
        self.shape = (Hq, Hkv, D)
        B, gen = len(lens), torch.Generator().manual_seed(seed)
        P = NP * bs
        own = [max(0, -(-n // bs) - NP) for n in lens]
        pool = NP + sum(own) + 3
        order = torch.randperm(pool, generator=gen) + first_block
        self.prefix = order[:NP].int()
        width = max([NP + n for n in own] + [1])
        self.table = torch.full((B, width), 1 << 28, dtype=torch.int32)
        at = NP
        for b in range(B):
            self.table[b, NP:NP + own[b]] = order[at:at + own[b]].int()
            at += own[b]

        def values(n):
            x = torch.randn(n, Hkv, D, generator=gen)
            return (x * 80).clamp(-448, 448).to(torch.float8_e4m3fn) if kv8 else x.to(self.t)

        def cache(tokens):
            c = torch.full((pool, Hkv, bs, D), float("nan")).to(torch.float8_e4m3fn if kv8 else self.t)
            for b in range(-1, B):
                n = P if b < 0 else lens[b] - P
                if n <= 0:
                    continue
                j = torch.arange(n)
                blocks = (self.prefix if b < 0 else self.table[b, NP:])[j // bs].long() - first_block
                c[blocks, :, j % bs] = tokens[b]
            return c

        self.k = {b: values(P if b < 0 else max(lens[b] - P, 0)) for b in range(-1, B)}
        self.v = {b: values(P if b < 0 else max(lens[b] - P, 0)) for b in range(-1, B)}
        self.make_cache, self.first_block, self.pool = cache, first_block, pool
        self.T = sum(new) + pad_tokens
        self.q = torch.randn(self.T, Hq, D, generator=gen).to(self.t)
        self.cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.slopes = torch.exp2(-8.0 * torch.arange(1, Hq + 1) / Hq) if slopes else None
        self.scale = 1.0 / math.sqrt(D)
        self.k_scales = torch.linspace(0.011, 0.02, Hkv)
        self.v_scales = torch.linspace(0.02, 0.01, Hkv)

    def upload(self):
        import torch
        self.kc, self.vc = (c.view(torch.uint8).cuda() if self.kv8 else c.cuda() for c in (self.make_cache(self.k), self.make_cache(self.v)))
        return self

    def run(self, G, scales="heads", no_cu=False, bounds=(0, 0)):
        import torch
        Hq, Hkv, D = self.shape
        B = len(self.lens)
        most, n = max(self.lens) + bounds[0], max(max(self.new), 1) + bounds[1]
        need = G.common_prefix_workspace_bytes(self.T, B, Hq, Hkv, D, self.bs, self.NP, most, n)
        raw = torch.full((need + 8192,), 0x7F, dtype=torch.uint8, device="cuda")
        around = torch.full((self.T * Hq * D + 2048,), float("nan"), dtype=self.t, device="cuda")
        out = around[1024:-1024].view(self.T, Hq, D)
        width = max(self.table.shape[1], -(-most // self.bs))
        table = torch.full((B, width), 1 << 28, dtype=torch.int32)
        table[:, :self.table.shape[1]] = self.table
        args = (out, self.q.cuda(), self.kc, self.vc, self.prefix.cuda(), table.cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda(),
                None if no_cu else torch.from_numpy(self.cu).cuda(), None if self.slopes is None else self.slopes.cuda(), self.scale)
        tail = (most, n, raw[4096:-4096])
        if not self.kv8:
            G.paged_attention_common(*args, *tail)
        elif scales == "heads":
            G.paged_attention_common_fp8_heads(*args, self.k_scales.cuda(), self.v_scales.cuda(), *tail)
        else:
            G.paged_attention_common_fp8(*args, 0.0125, 0.02, *tail)
        torch.cuda.synchronize()
        assert (raw[:4096] == 0x7F).all() and (raw[-4096:] == 0x7F).all(), "a kernel wrote outside the workspace"
        assert torch.isnan(around[:1024]).all() and torch.isnan(around[-1024:]).all(), "a kernel wrote outside out"
        return out

    def check(self, out, scales="heads"):
        Hq, Hkv, D = self.shape
        got, P = out.double().cpu().numpy(), self.NP * self.bs
        ks, vs = np.ones((1, Hkv, 1)), np.ones((1, Hkv, 1))
        if self.kv8:
            ks, vs = (self.k_scales.double().numpy()[None, :, None], self.v_scales.double().numpy()[None, :, None]) if scales == "heads" else (
                np.float64(np.float32(0.0125)), np.float64(np.float32(0.02)))
        slopes = None if self.slopes is None else self.slopes.double().numpy()
        keys, values = self.k[-1].double().numpy() * ks, self.v[-1].double().numpy() * vs
        assert not got[self.cu[-1]:].any()                        # tokens of no sequence
        for b, (L, n) in enumerate(zip(self.lens, self.new)):
            rows = slice(self.cu[b], self.cu[b + 1])
            k = np.concatenate([keys, self.k[b].double().numpy() * ks])[:max(L, 0)]
            v = np.concatenate([values, self.v[b].double().numpy() * vs])[:max(L, 0)]
            ref, size = R.attend(self.q[rows].double().numpy(), k, v, np.arange(L - n, L), slopes, self.scale)
            bar = R.attention_bar(ref, size, self.dtype)
            bad = ~(np.abs(got[rows] - ref) <= bar)
            assert not bad.any(), (f"sequence {b} of length {L}, {n} new: {bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(got[rows] - ref))}, "
                                   f"rows {np.unique(np.nonzero(bad)[0])[:5]}, heads {np.unique(np.nonzero(bad)[1])[:5]}")


def ragged(seed, B, lo, hi, P, new_hi):
    rng = np.random.default_rng(seed)
    own = rng.integers(lo, hi + 1, B)
    new = rng.integers(1, new_hi + 1, B)
    return [int(P + o + n) for o, n in zip(own, new)], [int(n) for n in new]


# (Hq, Hkv, D, bs, prefix blocks, sequences, own lo, own hi, new): row blocks of 1, 2 and 4 for the prefix and for own parts
SHAPES = [
    (8, 2, 64, 16, 16, 4, 0, 60, 1),            # 16 rows
    (8, 2, 128, 16, 9, 11, 1, 130, 1),          # 44 rows
    (32, 4, 128, 32, 20, 17, 0, 300, 1),        # 136 rows, several workgroups
    (5, 1, 128, 64, 3, 3, 0, 70, 4),            # a group of 5
    (40, 8, 64, 32, 40, 7, 10, 200, 3),
    (16, 16, 128, 16, 30, 40, 0, 40, 1),        # multi-head
    (64, 8, 128, 16, 33, 5, 63, 300, 9),        # drafts: up to 72 own rows
    (48, 2, 64, 16, 12, 3, 0, 500, 5),          # a group of 24
    (8, 2, 128, 16, 7, 3, 0, 30, 70),           # chunks: up to 280 own rows, causal among themselves
    (4, 4, 64, 64, 1, 70, 0, 20, 3),            # more sequences than lanes
    (8, 1, 128, 16, 150, 2, 1500, 2600, 1),     # own parts in several ranges
]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("slopes", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(G, shape, slopes, dtype):
    Hq, Hkv, D, bs, NP, B, lo, hi, new = shape
    lens, n = ragged(sum(shape), B, lo, hi, NP * bs, new)
    batch = Batch(1, dtype, Hq, Hkv, D, bs, NP, lens, n, slopes).upload()
    batch.check(batch.run(G))


@pytest.mark.parametrize("scales", ["heads", "tensor"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_8_bit_caches(G, shape, dtype, scales):
    Hq, Hkv, D, bs, NP, B, lo, hi, new = shape
    lens, n = ragged(sum(shape), B, lo, hi, NP * bs, new)
    batch = Batch(2, dtype, Hq, Hkv, D, bs, NP, lens, n, D == 64, kv8=True).upload()
    batch.check(batch.run(G, scales), scales)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bounds", [(0, 0), (1, 0), (500, 3), (5000, 0)])
def test_lengths_at_their_ends(G, bounds, D):
    """No prefix, nothing behind it, contexts that end inside it, empty sequences, sequences without new tokens, tokens of nobody;
    bounds that are met or far away."""
    for NP, lens, new in ((0, [1, 17, 33, 2], [1, 1, 2, 2]), (4, [64, 64, 64], [1, 1, 1]), (4, [65, 80, 64, 63], [1, 2, 1, 3]),
                          (5, [0, 3, 40, 100, 0, 81], [1, 1, 1, 1, 0, 2]), (6, [96, 50, 0, 200], [9, 50, 0, 120]), (3, [0, 0], [2, 1])):
        batch = Batch(3, "bf16", 8, 2, D, 16, NP, lens, new, True, pad_tokens=5).upload()
        batch.check(batch.run(G, bounds=bounds))


@pytest.mark.parametrize("new", [[4, 1], [3, 0, 1], [1, 1, 2, 1], [0, 1], [1, 0], [1, 1, 0, 1, 1]])
def test_last_sequence_with_one_new_token(G, new):
    """Prefix sums that look like one new token each in places."""
    batch = Batch(12, "f16", 8, 2, 64, 16, 3, [48 + 20 + 7 * i for i in range(len(new))], new).upload()
    batch.check(batch.run(G))


def test_a_context_shorter_than_its_new_tokens(G):
    """Positions below 0 see nothing."""
    batch = Batch(4, "f16", 8, 2, 64, 16, 2, [3, 40], [5, 2]).upload()
    out = batch.run(G)
    assert not out[:2].any()
    batch.check(out)


@pytest.mark.parametrize("rows", [1, 3, 20])     # one, two and four row blocks of 8-head groups
@pytest.mark.parametrize("dtype,D", [("f16", 64), ("bf16", 128)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_a_row_does_not_see_does_not_reach_it(G, bad, dtype, D, rows):
    """NaN and infinities in the keys and values of later tokens of the same tile."""
    import torch
    n = 4 * rows
    batch = Batch(5, dtype, 8, 1, D, 16, 3, [48 + 10 + n, 48 + 33], [n, 1], True).upload()
    clean = batch.run(G)
    batch.check(clean)
    last = n - 2                                                 # this new token's key and value, and those behind it
    for store, value in ((batch.k, bad), (batch.v, bad)):
        store[0][10 + last, :, ::5] = value
        store[0][10 + last + 1] = value
    batch.upload()
    out = batch.run(G)
    assert torch.isfinite(out[:last]).all() and torch.equal(out[:last], clean[:last]) and torch.equal(out[n:], clean[n:])
    assert not torch.isfinite(out[last]).all(dim=1).any()


@pytest.mark.parametrize("rows", [1, 3, 20])
@pytest.mark.parametrize("dtype,D", [("f16", 64), ("bf16", 128), ("bf16", 64)])
def test_codes_a_row_does_not_see_do_not_reach_it(G, dtype, D, rows):
    """The same for E4M3 caches, whose only such code is NaN."""
    import torch
    n = 4 * rows
    batch = Batch(13, dtype, 8, 1, D, 16, 3, [48 + 10 + n, 48 + 33], [n, 1], True, kv8=True).upload()
    clean = batch.run(G)
    batch.check(clean)
    last = n - 2
    for store in (batch.k, batch.v):
        codes = store[0].view(torch.uint8)
        codes[10 + last, :, ::5] = 0x7F
        codes[10 + last + 1] = 0xFF
    out = batch.upload().run(G)
    assert torch.isfinite(out[:last]).all() and torch.equal(out[:last], clean[:last]) and torch.equal(out[n:], clean[n:])
    assert not torch.isfinite(out[last]).all(dim=1).any()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_value_that_is_seen_is_not_lost(G, dtype):
    """An infinite value in a tile that some row's end cuts reaches the rows that see it, and no others."""
    import torch
    n = 6
    batch = Batch(6, dtype, 8, 1, 128, 16, 2, [32 + 5 + n], [n]).upload()
    clean = batch.run(G)
    batch.v[0][5 + 2, 0, 7], batch.v[0][5 + 4, 0, 9] = float("inf"), -float("inf")
    out = batch.upload().run(G)
    # (bf16 weights are two parts, of which the second may be 0: there the element is NaN instead)
    want = torch.zeros(clean.shape, dtype=torch.bool, device="cuda")
    want[2:, :, 7] = want[4:, :, 9] = True
    assert (torch.isfinite(out) == ~want).all() and (out[~want] == clean[~want]).all()
    assert dtype == "bf16" or (torch.isposinf(out[2:, :, 7]).all() and torch.isneginf(out[4:, :, 9]).all())


@pytest.mark.parametrize("n", [1, 6, 20])        # one, two and four row blocks of 8-head groups
@pytest.mark.parametrize("dtype,kv8,NP", [("f16", False, 3), ("bf16", False, 3), ("bf16", False, 0), ("bf16", True, 3)])
def test_a_query_or_key_that_is_no_number_is_not_lost(G, dtype, kv8, NP, n):
    """A NaN query's row, and the rows that see a NaN key, are NaN, also where no other key of a piece is seen; no others."""
    import torch
    P = 16 * NP
    batch = Batch(14, dtype, 16, 2, 64, 16, NP, [P + n, P + 40], [n, 1], kv8=kv8).upload()
    clean = batch.run(G)
    batch.check(clean)
    batch.q[n - 1, 3] = float("nan")
    want = torch.zeros(clean.shape, dtype=torch.bool, device="cuda")
    want[n - 1, 3] = True
    out = batch.run(G)
    assert torch.equal(torch.isnan(out), want) and torch.equal(out[~want], clean[~want])
    # the first own key of sequence 0, second KV head: its only one behind the prefix where n is 1
    if kv8:
        batch.k[0].view(torch.uint8)[0, 1, 5] = 0x7F
    else:
        batch.k[0][0, 1, 5] = float("nan")
    want[:n, 8:] = True
    out = batch.upload().run(G)
    assert torch.equal(torch.isnan(out), want) and torch.equal(out[~want], clean[~want])


def test_loud_scores_and_zero_scale(G):
    for scale in (0.0, -0.05, 3.0):
        batch = Batch(7, "f16", 8, 2, 64, 16, 9, [200, 170, 144], [1, 2, 1]).upload()
        batch.scale = scale
        out = batch.run(G)
        if abs(scale) < 1:                                       # (at 3 scores reach hundreds: their rounding is beyond the bar's)
            batch.check(out)
        assert np.isfinite(out.double().cpu().numpy()).all()


def test_one_new_token_each_needs_no_prefix_sums(G):
    import torch
    batch = Batch(8, "bf16", 32, 8, 128, 16, 12, [200, 193, 0, 260, 192], [1] * 5, True).upload()
    assert torch.equal(batch.run(G), batch.run(G, no_cu=True))


@pytest.mark.parametrize("kv8", [False, True])
def test_blocks_beyond_4_gib(G, kv8):
    import torch
    batch = Batch(9, "bf16", 8, 8, 128, 64, 5, [400, 350, 330], [1, 2, 1], kv8=kv8)
    kc, vc = batch.make_cache(batch.k), batch.make_cache(batch.v)
    first = 40_000 if not kv8 else 80_000                        # 128 KiB (64 KiB) a block and cache
    batch.kc, batch.vc = (torch.zeros((first + batch.pool, *kc.shape[1:]), dtype=torch.uint8 if kv8 else batch.t, device="cuda") for _ in range(2))
    for big, small in ((batch.kc, kc), (batch.vc, vc)):
        big[first:] = small.view(big.dtype).cuda() if kv8 else small.cuda()
    batch.prefix += first
    batch.table += first
    batch.check(batch.run(G))


def test_the_other_calls_on_full_tables(G):
    """What optgqa_paged_attention and optgqa_paged_prefill give, to twice their roundings."""
    import torch
    Hq, Hkv, D, bs, NP = 32, 4, 128, 32, 30
    for new_hi in (1, 6):
        lens, new = ragged(5, 9, 3, 400, NP * bs, new_hi)
        batch = Batch(10, "bf16", Hq, Hkv, D, bs, NP, lens, new, True).upload()
        out = batch.run(G)
        full = batch.table.clone()
        full[:, :NP] = batch.prefix
        want = torch.empty_like(out)
        q, tab, ln, sl = batch.q.cuda(), full.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), batch.slopes.cuda()
        if new_hi == 1:
            G.paged_attention(want, q, batch.kc, batch.vc, tab, ln, sl, batch.scale, max(lens), -1)
        else:
            G.paged_prefill(want, q, batch.kc, batch.vc, tab, ln, torch.from_numpy(batch.cu).cuda(), sl, batch.scale, max(new))
        assert (out.float() - want.float()).abs().max() < 2e-2


def test_a_captured_call_replays(G):
    import torch
    batch = Batch(11, "bf16", 32, 8, 128, 16, 40, [700, 650, 641, 800], [1, 3, 1, 2]).upload()
    Hq, Hkv, D = batch.shape
    q, out = batch.q.cuda(), torch.empty(batch.T, Hq, D, dtype=batch.t, device="cuda")
    lens = torch.tensor(batch.lens, dtype=torch.int32).cuda()
    ws = torch.empty(G.common_prefix_workspace_bytes(batch.T, 4, Hq, Hkv, D, 16, 40, 800, 3), dtype=torch.uint8, device="cuda")
    args = (out, q, batch.kc, batch.vc, batch.prefix.cuda(), batch.table.cuda(), lens, torch.from_numpy(batch.cu).cuda(), None, batch.scale, 800, 3, ws)
    G.paged_attention_common(*args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.paged_attention_common(*args)
    for i in range(4):
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(i)).to(batch.t))
        lens[1] -= 3
        graph.replay()
        got = out.clone()
        out.zero_()
        ws.fill_(0xFF)
        G.paged_attention_common(*args)
        assert torch.equal(got, out)
