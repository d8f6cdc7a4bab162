"""Attention with one common prefix where scores are so large that 32 bits hold them to whole numbers only."""
import numpy as np
import pytest

import step_reference as R
from test_gpu_common_prefix import G, Batch  # noqa: F401  (G: a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("NP,own,new", [(40, 3, 1), (3, 300, 1), (3, 60, 12)])
def test_scores_of_any_size(G, NP, own, new, D, dtype):
    """Keys that are all the same: every score of a row is one number, from 2^2 to 2^31 binary orders and of either sign.  A score, and a
    row's reference, are known to a unit in the last place of 32 bits, so a weight is off by that many binary orders, twice, beside what
    the other tests allow; however many that are, the output is a mean of the values: finite, and between the least and the largest."""
    import torch
    B = 38 if new == 1 else 4
    batch = Batch(90, dtype, 8, 2, D, 16, NP, [16 * NP + own + i for i in range(B)], [new] * B)
    batch.scale = 1.0
    for part in batch.k:
        batch.k[part][:] = 1408.0
    rows = torch.arange(batch.T * 8).reshape(batch.T, 8)
    batch.q[:] = (torch.exp2(2 + (rows * 5 % 117) / 4.0) / (1408.0 * D) * (1 - 2 * (rows % 2)))[:, :, None].to(batch.t)
    got = batch.upload().run(G).double().cpu().numpy()
    score = np.abs(batch.q[:, :, 0].double().numpy()) * 1408.0 * D / np.log(2.0)
    unit = np.exp2(np.floor(np.log2(np.maximum(score, 1.0))) - 23)
    off = np.exp2(np.minimum(2 * unit, 40.0)) - 1.0
    for b in range(B):
        for i in range(new):
            t = batch.cu[b] + i
            sees = batch.lens[b] - new + i + 1
            v = np.concatenate([batch.v[-1].double().numpy(), batch.v[b].double().numpy()])[:sees]
            for h in range(8):
                mine = v[:, h // 4]
                ref, size = mine.mean(axis=0), np.abs(mine).mean(axis=0)
                slack = 2 * off[t, h] * (size + np.abs(ref))
                bar = R.attention_bar(ref, size, dtype) + slack * (1 + R.EPS[dtype])
                edge = R.attention_bar(np.abs(mine).max(axis=0), np.abs(mine).max(axis=0), dtype)
                x = got[t, h]
                assert np.isfinite(x).all(), (b, i, h, score[t, h])
                assert (np.abs(x - ref) <= bar).all() and (x <= mine.max(axis=0) + edge).all() and (x >= mine.min(axis=0) - edge).all(), (b, i, h, score[t, h])
