"""The example of drafted steps behind a common prompt: it runs, and its drafts change no token."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_drafted_steps_give_the_tokens_of_single_steps(dtype, capsys):
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import drafted_steps
    tokens, plain = drafted_steps.main(["--sequences", "6", "--prompt", "272", "--tokens", "20", "--drafts", "3", "--dtype", dtype, "--check"])
    print(capsys.readouterr().out)
    # Logits are sums of 512 products of numbers near 1, rounded to 2 bytes; a step of several tokens and one of one add attention's
    # pieces in other orders, so two logits that lie within a rounding of each other may change places, and what follows in that
    # sequence with them: up to the first such place the tokens are the same.
    agree = (tokens == plain).int().cumprod(dim=1).sum(dim=1)
    assert int((agree == tokens.shape[1]).sum()) >= 4 and int(agree.min()) >= 1
