"""Drafted steps of the example against steps of one token: the tokens are the same up to a place where two of them have the same logit
to within rounding."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("drafts,prompt,tokens", [(3, 272, 20), (1, 512, 48), (6, 16, 40)])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_drafts_change_a_token_only_where_two_are_as_good(dtype, drafts, prompt, tokens):
    """The two runs add attention's pieces in other orders, so activations x differ by some roundings: in each of 2 layers and the
    output by up to half a step eps / 2 of themselves, at random.  A logit is a sum of x times weights of variance 1 / width, so it
    moves by sqrt(3) eps / 2 rms(x), six times that at the very most, below 5.2 eps rms(x), and by its own rounding, half a step in
    both runs.  Where the first other token of a sequence stands, its logit may lie twice that below the first one's, no more."""
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import drafted_steps as E
    torch.manual_seed(2 + drafts)
    model, B = E.Model(getattr(torch, dtype)), 8
    text, starts = torch.randint(0, model.vocab, (prompt,)).cuda(), torch.randint(0, model.vocab, (B,)).cuda()
    drafted, _ = E.Server(model, text, B, tokens, drafts).decode(starts, tokens, drafts)
    said, logits = [], model.logits

    def recorded(x):
        said.append((x.float(), logits(x)))
        return said[-1][1]

    server = E.Server(model, text, B, tokens, 0)
    model.logits = recorded                                      # (once a step of one token each)
    plain, steps = server.decode(starts, tokens, 0)
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
