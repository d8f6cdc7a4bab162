"""The example of drafted trees: trees change a token only where two are as good, and whatever sequences do - fork, take branches, shrink,
move - the caches hold their tokens' rows."""
import os
import sys

import pytest

import page_reference as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import drafted_trees
    return drafted_trees


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_it_runs(E, dtype, capsys):
    tokens, plain = E.main(["--sequences", "4", "--prompt", "50", "--tokens", "12", "--dtype", dtype, "--check"])
    print(capsys.readouterr().out)
    assert tokens.shape == plain.shape == (4, 12)


@pytest.mark.parametrize("width,depth,prompt,tokens", [(3, 3, 300, 24), (1, 5, 16, 40), (8, 4, 77, 30)])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_trees_change_a_token_only_where_two_are_as_good(E, dtype, width, depth, prompt, tokens):
    """The two runs add attention's pieces in other orders, so activations x differ by some roundings: in each of 2 layers and the
    output by up to half a step eps / 2 of themselves, at random.  A logit is a sum of x times weights of variance 1 / width, so it
    moves by sqrt(3) eps / 2 rms(x), six times that at the very most, below 5.2 eps rms(x), and by its own rounding, half a step in
    both runs.  Where the first other token of a sequence stands, its logit may lie twice that below the first one's, no more."""
    import torch
    torch.manual_seed(width + depth)
    model, B = E.Model(getattr(torch, dtype)), 8
    text, starts = torch.randint(0, model.vocab, (prompt,)).cuda(), torch.randint(0, model.vocab, (B,)).cuda()
    drafted, _ = E.Server(model, text, B, tokens, E.Tree(width, depth)).decode(starts, tokens)
    server, said, logits = E.Server(model, text, B, tokens, E.Tree(0, 0)), [], model.logits

    def recorded(x):
        said.append((x.float(), logits(x)))
        return said[-1][1]

    model.logits = recorded                                      # (once a step of one token each)
    plain, steps = server.decode(starts, tokens)
    assert steps == len(said) == tokens
    eps, same = torch.finfo(getattr(torch, dtype)).eps, 0
    for b in range(B):
        differ = (plain[b] != drafted[b]).nonzero()
        same += int(differ[0]) if len(differ) else tokens
        if not len(differ):
            continue
        i = int(differ[0])
        x, row = said[i][0][b], said[i][1][b]
        top, other = float(row[plain[b, i]]), float(row[drafted[b, i]])
        assert top == float(row.max())
        bar = 2 * eps * (abs(top) + 5.2 * float(x.square().mean().sqrt()))
        assert 0 <= top - other <= bar, f"sequence {b}, token {i}: logits {top} and {other}, {bar} apart at most"
    print(f"{same} of {B * tokens} tokens checked")
    assert same >= B * tokens // 4


@pytest.mark.parametrize("prompt", [37, 64])
def test_caches_hold_the_sequences_tokens(E, prompt):
    """A row of the first layer's caches is made of its token and its position alone: after trees, forks and compactions each
    sequence's rows are those of the prompt and of what it and those it came from have said (to the rounding of a product that is
    computed for other numbers of rows: 512 terms, half a step of bf16 and of the turned value each)."""
    import torch
    torch.manual_seed(3)
    model, B = E.Model(torch.bfloat16), 7
    text, last = torch.randint(0, model.vocab, (prompt,)).cuda(), torch.randint(0, model.vocab, (B,)).cuda()
    server = E.Server(model, text, B, 120, E.Tree(4, 3))
    mine = [text.tolist() for _ in range(B)]
    for step in range(12):
        got, kept, following = server.step(last)
        for b, (row, n, token) in enumerate(zip(got.tolist(), kept.tolist(), last.tolist())):
            mine[b] += [token] + row[:n - 1]
        last = following
        if step % 3 == 1:
            parents = torch.randint(0, B, (B,)).cuda()
            server.fork(parents)
            mine, last = [list(mine[p]) for p in parents.tolist()], last[parents]
            if step > 6:
                last = torch.randint(0, model.vocab, (B,)).cuda()
        if step % 4 == 3:
            used = server.tidy()
            assert used == int((server.refs > 0).sum()) and bool((server.refs[:used] > 0).all())
        assert server.lens.tolist() == [len(x) for x in mine]
    table, held = server.tables.long().cpu(), torch.zeros(server.pool, dtype=torch.int64)
    for b in range(B):
        n = len(mine[b])
        used = P.have(n, server.block)
        held += torch.bincount(table[b, :used], minlength=server.pool)
        at = torch.arange(n)
        x = model.embed[torch.tensor(mine[b]).cuda()]
        _, k, v = model.rows(0, x)
        turned = torch.empty(k.shape, dtype=k.dtype, device="cuda")
        E.G.rotary_embedding(turned, k, None, None, at.int().cuda(), model.freqs, magnitude=model.magnitude)
        for cache, want in zip(server.layers[0], (turned, v)):
            rows = cache[table[b, at // server.block].cuda(), :, (at % server.block).cuda()].float()
            size = want.float().abs().amax(dim=-1, keepdim=True)     # (a pair's larger half decides what turning rounds)
            assert bool(((rows - want.float()).abs() <= 4 * 2.0 ** -8 * size).all()), b
    assert torch.equal(held, server.refs.long().cpu())
