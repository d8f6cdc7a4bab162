"""Attention with one common prefix at positions that 24 bits do not hold, with slopes: a key's distance has to be exact where it is near."""
import numpy as np
import pytest

import step_reference as R
from test_gpu_common_prefix import G  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("prefix,own", [((1 << 24) + 64, 100), (64, (1 << 24) + 1000), (1 << 27, 37)])
def test_near_keys_of_far_positions(G, prefix, own, dtype):
    """Tables that name the same few blocks again and again, so that contexts of 2^24 to 2^27 tokens need no memory.  With a slope of
    1 / 4 and more a key 1 024 behind weighs below exp(-200): the last 2 048 keys are the reference."""
    import torch
    t, Hq, D, bs, new = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype], 4, 64, 64, 3
    gen = torch.Generator().manual_seed(80)
    kc, vc = (torch.randn(23, 1, bs, D, generator=gen).to(t) for _ in range(2))
    q = torch.randn(new, Hq, D, generator=gen).to(t)
    L, NP, slopes = prefix + own + new, prefix // bs, torch.tensor([0.25, 0.5, 0.75, 1.0])
    table = (torch.arange(-(-L // bs)) * 7 % 23).int()
    common, mine = table[:NP].clone(), table[None].clone()
    mine[0, :NP] = 1 << 28                                       # (not read)
    out = torch.empty(new, Hq, D, dtype=t, device="cuda")
    ws = torch.empty(G.common_prefix_workspace_bytes(new, 1, Hq, 1, D, bs, NP, L, new), dtype=torch.uint8, device="cuda")
    G.paged_attention_common(out, q.cuda(), kc.cuda(), vc.cuda(), common.cuda(), mine.cuda(), torch.tensor([L], dtype=torch.int32).cuda(),
                             torch.tensor([0, new], dtype=torch.int32).cuda(), slopes.cuda(), 0.125, L, new, ws)
    near = np.arange(L - 2048, L)
    block, row = table.numpy()[near // bs], near % bs
    keys, values = (c.double().numpy()[block, 0, row][:, None] for c in (kc, vc))
    ref, size = R.attend(q.double().numpy(), keys, values, np.arange(2048 - new, 2048), slopes.double().numpy(), 0.125)
    bad = ~(np.abs(out.double().cpu().numpy() - ref) <= R.attention_bar(ref, size, dtype))
    assert not bad.any(), f"{bad.sum()} of {bad.size} off by up to {np.abs(out.double().cpu().numpy() - ref).max()}"
