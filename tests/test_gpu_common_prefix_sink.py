"""Attention with one common prefix where one key has most of the weight and tens of thousands of others share what is left: what
every one of them weighs lies many binary orders below the largest weight, what they weigh together does not."""
import numpy as np
import pytest

import step_reference as R
from test_gpu_common_prefix import G, Batch  # noqa: F401  (G: a fixture)

pytestmark = pytest.mark.gpu

# (Hq, Hkv, prefix blocks of 16, sequences, own cached tokens, new tokens): all of a long prefix in one range, for four row blocks; in several
# ranges, for one and for two row blocks; an own part alone, for one, two and four row blocks
WALKS = [(64, 8, 2048, 64, 20, 8), (8, 2, 2048, 3, 20, 1), (32, 2, 512, 3, 20, 1), (8, 8, 0, 1, 4000, 7), (16, 2, 0, 2, 4000, 7), (16, 2, 0, 2, 4000, 16)]


@pytest.mark.parametrize("dtype,kv8", [("f16", False), ("f16", True), ("bf16", False)])
@pytest.mark.parametrize("walk", WALKS)
@pytest.mark.parametrize("at", ["first", "middle", "last"])
@pytest.mark.parametrize("below", [12.0, 21.25, 23.5])
def test_what_many_small_weights_add_up_to(G, below, at, walk, dtype, kv8):
    """One key with a value of 0, all others `below` binary orders under it with values of 1.  The others' weights are normal
    numbers of the type they are rounded to down to 24 orders below the largest, so the bar of the other tests holds."""
    import torch
    Hq, Hkv, NP, B, own, new = walk
    batch = Batch(20, dtype, Hq, Hkv, 64, 16, NP, [16 * NP + own + new] * B, [new] * B, kv8=kv8)
    sink = {"first": 0, "middle": 1000, "last": 16 * NP + own - 1}[at]
    k_scale, v_scale = (float(np.float32(0.0125)), float(np.float32(0.02))) if kv8 else (1.0, 1.0)
    # scores: 0 for the one key, -below for the others
    batch.q[:] = 0.0
    batch.q[:, :, 3] = 8.0
    away = torch.tensor([-below * np.log(2.0) / (batch.scale * 8.0 * k_scale)]).clamp(min=-448.0).to(torch.float8_e4m3fn if kv8 else batch.t)
    if kv8:                                                      # (the codes are coarse: the query takes what they leave)
        batch.q[:, :, 3] *= float(-below * np.log(2.0) / (batch.scale * 8.0 * k_scale) / away.double())
    for b in range(-1, B):
        for tokens in (batch.k, batch.v):
            tokens[b] = torch.zeros(tokens[b].shape).to(tokens[b].dtype)
        batch.k[b][:, :, 3] = away
        batch.v[b][:] = torch.ones(1).to(batch.v[b].dtype)
    for b in range(B):
        part, i = (-1, sink) if sink < 16 * NP else (b, sink - 16 * NP)
        batch.k[part][i], batch.v[part][i] = (torch.zeros(Hkv, 64).to(batch.k[b].dtype) for _ in range(2))
    got = batch.upload().run(G, "tensor").double().cpu().numpy()
    score = float(np.float32(batch.scale)) * float(batch.q[0, 0, 3].double()) * float(away.double()) * k_scale
    others = (16 * NP + own + np.tile(np.arange(new), B)) * np.exp(score)            # (each row sees itself, and the one key)
    ref = np.broadcast_to((v_scale * others / (1.0 + others))[:, None, None], got.shape)
    bad = ~(np.abs(got - ref) <= R.attention_bar(ref, ref, dtype))
    assert not bad.any(), f"{bad.sum()} of {bad.size} off: {got[bad][:3]} for {ref[bad][:3]}"
