"""CPU: the workspace of attention with one common prefix.  A server sizes it once, for its largest batch, prompt and context; every
call that is smaller in any of these has to fit."""
import os
import random

import pytest

import common_prefix_plan as P


@pytest.fixture(scope="module")
def G():
    import paper_2505_02351_amd as G
    if not os.path.exists(G.LIB_PATH):
        from paper_2505_02351_amd import build
        build.build()
    G.load_library()
    return G


HEADS = [(32, 8, 128), (32, 4, 128), (64, 8, 128), (8, 2, 64), (40, 8, 64), (16, 16, 128), (8, 1, 128), (5, 1, 64), (512, 512, 64)]


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("blocks,own", [(2048, 2048), (128, 1023), (0, 700), (33, 512), (1, 0)])
def test_a_smaller_batch_fits(G, Hq, Hkv, D, blocks, own):
    """Decode steps and drafts of 1 to 128 sequences in the workspace of one more."""
    for new in (1, 5):
        before = 0
        for B in range(1, 129):
            need = G.common_prefix_workspace_bytes(B * new, B, Hq, Hkv, D, 16, blocks, 16 * blocks + own + new, new)
            assert need >= before > 0 or B == 1, (B, new)
            before = need


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("B,own", [(64, 512), (3, 60), (17, 2048)])
def test_a_shorter_prefix_fits(G, Hq, Hkv, D, B, own):
    """Prefixes of 0 to 2 048 blocks in the workspace of one block more, with the same tokens behind it and with the same whole length."""
    before = 0
    for blocks in list(range(0, 140)) + list(range(140, 2049, 53)):
        need = G.common_prefix_workspace_bytes(B, B, Hq, Hkv, D, 16, blocks, 16 * blocks + own, 1)
        assert need >= before > 0 or blocks == 0, blocks
        assert need >= G.common_prefix_workspace_bytes(B, B, Hq, Hkv, D, 16, max(blocks - 1, 0), 16 * blocks + own, 1)
        before = need


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
def test_no_argument_makes_it_smaller(G, Hq, Hkv, D):
    """Random sizes; tokens, sequences, prefix, longest context and new tokens of a sequence each made smaller by itself, by a little
    and by much, and all of them together."""
    rng = random.Random(Hq * 1000 + Hkv)

    def size(a):
        return G.common_prefix_workspace_bytes(a[0], a[1], Hq, Hkv, D, 16, a[2], a[3], a[4])

    def some(hi):
        return int(round(hi ** rng.random()))

    for _ in range(3000):
        new, B = some(300), some(200)
        blocks = rng.choice([0, some(4096)])
        a = [min(B * new, some(20000)), B, blocks, rng.choice([16 * blocks, 16 * blocks + some(50000), some(16 * blocks + 1)]), new]
        need = size(a)
        assert need > 0, a
        less = [x if i in (2, 3) and x == 0 else rng.choice([max(x - 1, min(x, 1)), max(min(some(max(x, 1)), x), min(x, 1))]) for i, x in enumerate(a)]
        assert size(less) <= need, (a, less)
        for i in range(5):
            one = a[:i] + [less[i]] + a[i + 1:]
            assert size(one) <= need, (a, one)


@pytest.mark.parametrize("cus", [256, 304, 32, 1])
def test_the_pieces_of_a_call_fit(cus, tmp_path_factory):
    lib, rng = P.build(tmp_path_factory.mktemp("rules")), random.Random(cus)

    def some(hi):
        return int(round(hi ** rng.random()))

    for _ in range(20000):
        Hq, Hkv, _ = rng.choice(HEADS)
        new, B = some(300), some(200)
        blocks = rng.choice([0, some(4096)])
        p = P.plan(lib, B * new, B, Hq, Hkv, 16 * blocks, 16 * blocks + some(50000), new, cus)
        assert 0 < p.pieces <= p.held, (Hq, Hkv, B, new, blocks)
