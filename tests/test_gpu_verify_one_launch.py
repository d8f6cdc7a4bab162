"""Verification of rows of up to 32 chunks, which are one launch: its time on the GPU, and entries that are no probabilities."""
import numpy as np
import pytest

from test_gpu_verify import G, check, inputs, strided  # noqa: F401  (G: a fixture)

pytestmark = pytest.mark.gpu


def replayed(G, V, B=1, drafts=4, calls=40):
    """GPU time of a call among others in a replayed graph, us."""
    import torch
    counts = [drafts] * B
    target, draft, ids, a, s = inputs(V, counts, V, torch.float32, True)
    dev = [strided(target, 0), strided(draft, 0), torch.from_numpy(ids).cuda(), (torch.arange(B + 1, device="cuda") * drafts).int(), torch.from_numpy(a).cuda(),
           torch.from_numpy(s).cuda()]
    tokens, accepted = torch.empty(B, drafts + 1, dtype=torch.int64, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    ws = torch.empty(G.verify_drafts_workspace_bytes(B, V), dtype=torch.uint8, device="cuda")
    G.verify_drafts(tokens, accepted, *dev, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(calls):
            G.verify_drafts(tokens, accepted, *dev, ws)
    e = [torch.cuda.Event(enable_timing=True) for _ in "ab"]

    held = tokens, accepted, dev, ws                             # (what the graph reads and writes lives as long as it may be replayed)

    def once():
        assert held
        e[0].record()
        graph.replay()
        e[1].record()
        torch.cuda.synchronize()
        return e[0].elapsed_time(e[1]) / calls * 1e3

    return once


@pytest.mark.parametrize("B", [1, 4])
def test_a_row_of_32_chunks_takes_no_longer_than_one_of_33(G, B):
    """In a graph, where launches cost the host nothing: 8.7 us against 6.9 when the first was one workgroup's on one CU and the
    second, in two launches, nine workgroups'."""
    one, two = replayed(G, 32 * 1024, B), replayed(G, 33 * 1024, B)
    for _ in range(3):
        one(), two()
    a, b = (sorted(x)[7] for x in zip(*((one(), two()) for _ in range(15))))
    print(f"32 chunks {a:.2f} us, 33 {b:.2f}")
    assert a <= 1.1 * b


@pytest.mark.parametrize("B,V", [(1, 32000), (3, 21 * 1024), (63, 22000), (64, 22000), (2, 20 * 1024)])
def test_a_captured_call_gives_the_bits_of_a_direct_one(G, B, V):
    """On both sides of where a captured call has two launches and a direct one has one; every replay after new random numbers."""
    import torch
    counts = [i % 5 for i in range(B)]
    target, draft, ids, a, s = inputs(V + B, counts, V, torch.float32, True)
    cu = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda()
    dev = [strided(target, 0), strided(draft, 0), torch.from_numpy(ids).cuda(), cu, torch.from_numpy(a).cuda(), torch.from_numpy(s).cuda()]
    tokens, accepted = torch.empty(B, 5, dtype=torch.int64, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    ws = torch.empty(G.verify_drafts_workspace_bytes(B, V), dtype=torch.uint8, device="cuda")
    G.verify_drafts(tokens, accepted, *dev, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.verify_drafts(tokens, accepted, *dev, ws)
    for i in range(4):
        dev[4].copy_(torch.rand(len(a), generator=torch.Generator().manual_seed(i)))
        dev[5].copy_(torch.rand(B, generator=torch.Generator().manual_seed(50 + i)))
        graph.replay()
        got = tokens.clone(), accepted.clone()
        tokens.zero_()
        ws.fill_(0x77)
        G.verify_drafts(tokens, accepted, *dev, ws)
        assert torch.equal(got[0], tokens) and torch.equal(got[1], accepted)


@pytest.mark.parametrize("sampled", [True, False])
@pytest.mark.parametrize("V", [700, 5000, 40000])
def test_entries_that_are_no_probabilities(G, V, sampled):
    """Infinities of both signs, NaN, negative and subnormal numbers in p and q, against one another."""
    import torch
    odd = torch.tensor([float("inf"), -float("inf"), float("nan"), -1.0, -0.0, 0.0, 1e-40, 3e-40, 2.0 ** -149, 3.4e38, -3.4e38, 0.5])
    counts = [1] * 30
    rng = np.random.default_rng(V)
    target, draft, ids, a, s = inputs(V, counts, V, torch.float32, True)
    for x in (target, draft):
        where = torch.from_numpy(rng.random(x.shape) < 0.5)
        x[where] = odd[torch.from_numpy(rng.integers(0, len(odd), int(where.sum())))]
    for b in range(0, 30, 3):                                    # nothing but subnormal numbers to draw from
        target[2 * b:2 * b + 2] = torch.where(torch.from_numpy(rng.random((2, V)) < 0.3), torch.tensor(3e-40), torch.tensor(-1.0))
        draft[b] = torch.where(torch.from_numpy(rng.random(V) < 0.5), torch.tensor(1e-40), torch.tensor(0.0))
    check(G, target, draft if sampled else None, ids, counts, a, s, 2)
