"""Verification of drafted tokens against a plain sequential implementation in 64 bits: whole numbers, equal."""
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


def strided(x, pad):
    """x on the GPU with rows `pad` elements longer, NaN between them."""
    import torch
    wide = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=x.dtype, device="cuda")
    wide[:, :x.shape[1]] = x.cuda()
    return wide[:, :x.shape[1]]


def check(G, target, draft, ids, counts, accept_u, sample_u, width, pad=0):
    import torch
    B, V = len(counts), target.shape[1]
    cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    tokens, accepted = torch.full((B, width), -7, dtype=torch.int64, device="cuda"), torch.full((B,), -7, dtype=torch.int32, device="cuda")
    raw = torch.full((G.verify_drafts_workspace_bytes(B, V) + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    G.verify_drafts(tokens, accepted, strided(target, pad), None if draft is None else strided(draft, pad), torch.from_numpy(ids).cuda(),
                    torch.from_numpy(cu).cuda(), torch.from_numpy(accept_u).cuda(), torch.from_numpy(sample_u).cuda(), raw[256:-256])
    assert (raw[:256] == 0x5A).all() and (raw[-256:] == 0x5A).all()
    want = R.verify(target.double().numpy(), None if draft is None else draft.double().numpy(), ids, cu, accept_u.astype(np.float64),
                    sample_u.astype(np.float64), width)
    assert np.array_equal(accepted.cpu().numpy(), want[1])
    assert np.array_equal(tokens.cpu().numpy(), want[0])
    return want


def inputs(seed, counts, V, dtype, sampled):
    import torch
    gen, rng, T, B = torch.Generator().manual_seed(seed), np.random.default_rng(seed), int(sum(counts)), len(counts)
    logits = 2 * torch.randn(T + B, V, generator=gen)
    target = torch.softmax(logits, 1).to(dtype)
    rows = np.array([i + b for b in range(B) for i in range(sum(counts[:b]), sum(counts[:b + 1]))], np.int64)
    noisy = logits[torch.from_numpy(rows)] + 0.5 * torch.randn(T, V, generator=gen)
    draft = torch.softmax(noisy, 1)
    ids = torch.multinomial(draft, 1, generator=gen)[:, 0].numpy() if T else np.zeros(0, np.int64)
    return target, draft.to(dtype) if sampled else None, ids, rng.random(T, np.float32), rng.random(B, np.float32)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("sampled", [True, False])
@pytest.mark.parametrize("V", [1, 2, 5, 4095, 4096, 4097, 32000, 50021])
@pytest.mark.parametrize("pad", [0, 1, 8])
def test_random_drafts(G, V, pad, sampled, dtype):
    import torch
    rng = np.random.default_rng(V + pad)
    for B, most in ((1, 4), (7, 5)):
        counts = [int(c) for c in rng.integers(0, most + 1, B)]
        target, draft, ids, a, s = inputs(V + B, counts, V, getattr(torch, dtype), sampled)
        want = check(G, target, draft, ids, counts, a, s, most + 1, pad)
        assert (want[0][np.arange(B), want[1]] >= 0).all()


@pytest.mark.parametrize("sampled", [True, False])
@pytest.mark.parametrize("V", [1023, 1024, 1025, 16384, 16385, 32767, 32768, 32769, 33793])
def test_draws_from_every_chunk(G, V, sampled):
    """Vocabularies around a chunk of 1 024, a wave's of 16 and the 32 that one launch takes; draws spread over the whole row."""
    import torch
    counts = [i % 3 for i in range(67)]
    target, draft, ids, a, s = inputs(V, counts, V, torch.float32, sampled)
    s[:] = np.linspace(0.0, 0.9999, len(s), dtype=np.float32)
    want = check(G, target, draft, ids, counts, a, s, 3)
    drawn = want[0][np.arange(67), want[1]]
    # (what the oracle drew: most chunks)
    assert (drawn >= 0).all() and 2 * np.unique(drawn // 1024).size >= min(-(-V // 1024), 32)


def test_many_drafts_and_many_sequences(G):
    """More drafts than a wave has lanes, and more than max_drafts; hundreds of sequences; a vocabulary of many chunks."""
    import torch
    counts = [70, 0, 129, 64, 65, 1]
    target, draft, ids, a, s = inputs(1, counts, 300, torch.float32, True)
    a[:] = 0.0                                                   # kept wherever p(x) > 0
    a[[69, 70 + 66]] = 0.9999
    ids[70 + 66] = int(np.argmax(np.where(draft[70 + 66] > target[70 + 66 + 2], draft[70 + 66] / target[70 + 66 + 2], 0)))
    want = check(G, target, draft, ids, counts, a, s, 130)
    assert want[1].max() > 64
    check(G, target, draft, ids, counts, a, s, 67)               # no more than 66 are looked at
    counts = [int(c) for c in np.random.default_rng(2).integers(0, 4, 300)]
    check(G, *inputs(3, counts, 700, torch.float32, True)[:3], counts, *inputs(3, counts, 700, torch.float32, True)[3:], 4)
    counts = [2, 3]
    t = inputs(4, counts, 1_300_003, torch.float32, True)        # 318 chunks
    check(G, *t[:3], counts, *t[3:], 4)


def test_no_drafts_at_all(G):
    import torch
    for width in (1, 3):
        target, _, ids, a, s = inputs(5, [0, 0, 0], 1000, torch.float32, False)
        check(G, target, None, ids, [0, 0, 0], a, s, width)


def test_numbers_at_their_ends(G):
    """Random numbers of 0 and next to 1; equal, dyadic probabilities, where every draw lies on a border."""
    import torch
    V, counts = 8192, [1] * 6
    u = np.array([0.0, 1 - 2.0 ** -24, 0.5, 0.25, 0.125, 1.0 / 8192], np.float32)
    flat = torch.full((12, V), 1.0 / V)
    draft = torch.zeros(6, V)
    draft[:, :V // 2] = 2.0 / V
    ids = np.full(6, 17, np.int64)
    want = check(G, flat, draft, ids, counts, np.full(6, 0.75, np.float32), u, 2)
    assert (want[1] == 0).all() and want[0][0, 0] == V // 2      # left: the upper half, equal parts
    check(G, flat, draft, ids, counts, np.zeros(6, np.float32), u, 2)
    check(G, flat, draft, ids, counts, np.full(6, 0.5, np.float32), u, 2)       # u q == p: not kept


def test_probabilities_that_are_none(G):
    """Rows of zeros, NaN, infinities and negative numbers; q above p everywhere; ids that no vocabulary has."""
    import torch
    V, counts = 5000, [1, 2, 1, 1, 1, 3]
    target, draft, ids, a, s = inputs(6, counts, V, torch.float32, True)
    target[0] = 0.0                                              # sequence 0: nothing kept, nothing to draw from
    target[1] = 0.0                                              # (its second row)
    target[2, ::3], target[2, 1::3] = float("nan"), float("inf")
    draft[1, 2::3] = float("nan")                                # sequence 1: p alone where p - q is no number
    target[2, ids[1]] = 0.0
    a[1] = 0.5
    draft[3] = target[5] * 2                                     # sequence 2: q above p, nothing left
    a[3] = 0.9
    ids[4], ids[5] = -1, V                                       # sequences 3 and 4: no drafts
    target[11, ::2] = -1.0
    want = check(G, target, draft, ids, counts, a, s, 4)
    assert want[0][0, 0] == -1 and want[1][3] == 0 and want[1][4] == 0
    check(G, target, None, ids, counts, a, s, 4)
    only = torch.zeros(2, V)
    only[:, 4321] = 0.3                                          # a certain draft where p has nothing else: drawn again
    want = check(G, only, None, np.array([4321]), [1], np.array([0.5], np.float32), np.array([0.7], np.float32), 2)
    assert want[1][0] == 0 and want[0][0, 0] == 4321


def test_a_captured_verification_replays(G):
    import torch
    counts = [3, 1, 4]
    target, draft, ids, a, s = inputs(8, counts, 9000, torch.float32, True)
    dev = [strided(target, 0), strided(draft, 0), torch.from_numpy(ids).cuda(), torch.tensor([0, 3, 4, 8], dtype=torch.int32).cuda(),
           torch.from_numpy(a).cuda(), torch.from_numpy(s).cuda()]
    tokens, accepted = torch.empty(3, 5, dtype=torch.int64, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")
    ws = torch.empty(G.verify_drafts_workspace_bytes(3, 9000), dtype=torch.uint8, device="cuda")
    G.verify_drafts(tokens, accepted, *dev, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.verify_drafts(tokens, accepted, *dev, ws)
    for i in range(4):
        dev[4].copy_(torch.rand(8, generator=torch.Generator().manual_seed(i)))
        dev[5].copy_(torch.rand(3, generator=torch.Generator().manual_seed(50 + i)))
        graph.replay()
        got = tokens.clone(), accepted.clone()
        tokens.zero_()
        ws.fill_(0x77)
        G.verify_drafts(tokens, accepted, *dev, ws)
        assert torch.equal(got[0], tokens) and torch.equal(got[1], accepted)
