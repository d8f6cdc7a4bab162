"""Rotary positions of more tokens than one launch has workgroups for."""
import numpy as np
import pytest

import step_reference as R
from test_gpu_verify import G  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("append", [False, True])
def test_more_than_2_to_the_24_tokens(G, append):
    """A workgroup for each token of 9 narrow heads (4 and 5 where they are appended, 14 in all): 2^24 workgroups of 256 threads are 2^32 threads.  In place; the
    first tokens, those around the border and the last ones are checked, and that nothing behind the last is written."""
    import torch
    D, rot, Hq, Hkv = 64, 24, 4 if append else 9, 5 if append else 0
    T = (1 << 24) + 37
    width = (Hq + 2 * Hkv) * D if append else Hq * D
    freqs, _ = G.rotary_frequencies(rot, 10000.0)
    rows = torch.empty(T + 1, width, dtype=torch.bfloat16, device="cuda")
    some = torch.randn(4099, width, generator=torch.Generator("cuda").manual_seed(3), device="cuda").bfloat16()
    at = torch.arange(T + 1, device="cuda")
    for i in range(0, T + 1, 4099):
        rows[i:i + 4099] = some[:min(4099, T + 1 - i)]
    positions = (at[:T] % 100003).int()
    q = rows[:T, :Hq * D].view(T, Hq, D)
    checked = torch.cat([torch.arange(0, 70), torch.arange((1 << 24) - 70, T)])
    before = rows[checked.cuda()].cpu()
    if append:
        k, v = (rows[:T, (Hq + i * Hkv) * D:(Hq + (i + 1) * Hkv) * D].view(T, Hkv, D) for i in range(2))
        # (the checked tokens' rows are kept, all others are padding)
        slots = torch.full((T,), -1, dtype=torch.int64, device="cuda")
        slots[checked.cuda()] = torch.arange(len(checked), device="cuda")
        caches = [torch.zeros(-(-len(checked) // 16), Hkv, 16, D, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
        G.rotary_and_cache(q, q, k, v, *caches, slots, positions, freqs.cuda())
    else:
        G.rotary_embedding(q, q, None, None, positions, freqs.cuda())
    torch.cuda.synchronize()
    x, pos = before.double().numpy().reshape(len(checked), -1, D), checked.numpy() % 100003
    pairs = [(rows[checked.cuda()].cpu().double().numpy().reshape(len(checked), -1, D)[:, :Hq], x[:, :Hq])]
    if append:
        kept = [c.cpu().double().permute(0, 2, 1, 3).reshape(-1, Hkv, D)[:len(checked)].numpy() for c in caches]
        assert np.array_equal(kept[1], x[:, Hq + Hkv:])
        pairs.append((kept[0], x[:, Hq:Hq + Hkv]))
    for got, base in pairs:
        ref = R.rotate(base, pos, freqs.numpy(), False)
        slack = R.rotate_slack(base, freqs.numpy(), False)
        bar = R.half_step(np.abs(ref) + slack, R.EPS["bf16"], R.SMALLEST["bf16"]) + slack
        assert (np.abs(got - ref) <= bar).all(), np.unique(np.nonzero(np.abs(got - ref) > bar)[0])[:10]
    assert torch.equal(rows[T].cpu(), some[T % 4099].cpu())
