"""Attention with one common prefix where a workgroup walks through more blocks than the 64 numbers that its lanes hold, and where a row
has more pieces than the join takes at once: what long prefixes and contexts always come to.  That the calls are cut that way is
asked of the library's own rules."""
import numpy as np
import pytest

import common_prefix_plan as P
import step_reference as R
from test_gpu_common_prefix import G, Batch  # noqa: F401  (G: a fixture)

pytestmark = pytest.mark.gpu

# (query type, scales of 8-bit caches or "", head_dim)
FORMS = [("f16", "", 128), ("f16", "", 64), ("bf16", "", 128), ("bf16", "", 64), ("f16", "heads", 64), ("bf16", "tensor", 128)]


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    return P.build(tmp_path_factory.mktemp("rules"))


def plan(rules, batch):
    import torch
    Hq, Hkv, _ = batch.shape
    return P.plan(rules, batch.T, len(batch.lens), Hq, Hkv, batch.NP * batch.bs, max(batch.lens), max(max(batch.new), 1),
                  torch.cuda.get_device_properties(0).multi_processor_count)


def reference(batch, scales):
    """What step_reference.attend gives for every sequence (out, and what its weights average), a KV head at a time: the prefix's scores of
    all rows are one product."""
    (Hq, Hkv, D), P, T = batch.shape, batch.NP * batch.bs, batch.T
    ks = vs = np.ones(Hkv)
    if batch.kv8:
        ks, vs = (batch.k_scales.double().numpy(), batch.v_scales.double().numpy()) if scales == "heads" else (
            np.full(Hkv, np.float64(np.float32(x))) for x in (0.0125, 0.02))
    group = Hq // Hkv
    pos = np.concatenate([np.arange(n - m, n) for n, m in zip(batch.lens, batch.new)])
    q = batch.q.double().numpy().reshape(T, Hkv, group, D)
    slopes = np.zeros(Hq) if batch.slopes is None else batch.slopes.double().numpy()
    out, size = np.zeros((T, Hkv, group, D)), np.zeros((T, Hkv, group, D))

    def piece(rows, g, keys, values, first):
        """(maximum, weights' sum, weighted values, weighted magnitudes) of rows over keys first, first + 1, .."""
        at = first + np.arange(len(keys))
        s = batch.scale * q[rows, g] @ keys.T + slopes[g * group:(g + 1) * group, None] * (at - pos[rows, None, None])
        s = np.where(at <= pos[rows, None, None], s, -np.inf)
        m = np.maximum(s.max(axis=2, keepdims=True, initial=-np.inf), -1e300)
        w = np.exp(s - m)
        return m, w.sum(axis=2, keepdims=True), w @ values, w @ np.abs(values)

    every = np.arange(T)
    for g in range(Hkv):
        def of(store, part, scale):
            return store[part][:, g].double().numpy() * scale
        common = piece(every, g, of(batch.k, -1, ks[g]), of(batch.v, -1, vs[g]), 0)
        for b in range(len(batch.lens)):
            rows = every[batch.cu[b]:batch.cu[b + 1]]
            m1, l1, o1, a1 = (x[rows] for x in common)
            m2, l2, o2, a2 = piece(rows, g, of(batch.k, b, ks[g]), of(batch.v, b, vs[g]), P)
            m = np.maximum(m1, m2)
            f1, f2 = np.exp(m1 - m), np.exp(m2 - m)
            out[rows, g], size[rows, g] = (f1 * o1 + f2 * o2) / (f1 * l1 + f2 * l2), (f1 * a1 + f2 * a2) / (f1 * l1 + f2 * l2)
    return out.reshape(T, Hq, D), size.reshape(T, Hq, D)


def test_the_reference(G):
    """Against step_reference.attend."""
    batch = Batch(70, "f16", 6, 2, 64, 16, 2, [40, 33, 32], [2, 1, 3], True)
    got = reference(batch, "")
    for b, (n, m) in enumerate(zip(batch.lens, batch.new)):
        keys, values = (np.concatenate([s[-1].double().numpy(), s[b].double().numpy()])[:n] for s in (batch.k, batch.v))
        rows = slice(batch.cu[b], batch.cu[b + 1])
        want = R.attend(batch.q[rows].double().numpy(), keys, values, np.arange(n - m, n), batch.slopes.double().numpy(), batch.scale)
        assert all(np.allclose(x[rows], y, rtol=1e-12, atol=1e-13) for x, y in zip(got, want))


def check(G, batch, scales):
    """Against 64 bits; the same call twice has the same bits."""
    import torch
    out = batch.upload().run(G, scales)
    ref, size = reference(batch, scales)
    bad = ~(np.abs(out.double().cpu().numpy() - ref) <= R.attention_bar(ref, size, batch.dtype))
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, rows {np.unique(np.nonzero(bad)[0])[:5]}, heads {np.unique(np.nonzero(bad)[1])[:5]}"
    assert torch.equal(out, batch.run(G, scales))


@pytest.mark.parametrize("dtype,scales,D", FORMS)
@pytest.mark.parametrize("T,row_waves", [(20, 1), (40, 2), (70, 4)])
@pytest.mark.parametrize("bs,NP", [(16, 150), (32, 81)])
def test_a_range_of_more_than_64_blocks(G, rules, bs, NP, T, row_waves, dtype, scales, D):
    """As many KV heads as leave one range: 2 400 and 2 592 keys of the prefix in a walk."""
    batch = Batch(30 + T, dtype, 144, 144, D, bs, NP, [bs * NP + 5 + 3 * (i % 4) for i in range(T)], [1] * T, D == 64, bool(scales))
    p = plan(rules, batch)
    assert p.row_waves == row_waves and p.row_tiles == 1 and p.ranges == 1 and p.keys > 64 * bs
    check(G, batch, scales)


@pytest.mark.parametrize("dtype,scales,D", FORMS)
@pytest.mark.parametrize("new,row_waves", [(1, 1), (40, 2), (70, 4)])
@pytest.mark.parametrize("own", [2250])
def test_an_own_piece_of_more_than_64_blocks(G, rules, own, new, row_waves, dtype, scales, D):
    """As many segments as there are shares, each one piece of up to 145 blocks; a prefix in front of them and none."""
    for NP in (2, 0):
        lens = [16 * NP + own + new - i for i in range(8)]
        batch = Batch(40 + new, dtype, 16, 16, D, 16, NP, lens, [new] * 8, D == 64, bool(scales))
        p = plan(rules, batch)
        step = 32 * (4 // row_waves)
        steps = [-(-(n - 16 * NP) // step) for n in lens]        # (rows of one tile: segments are sequences times KV heads)
        share = max(-(-sum(steps) * 16 // p.shares), 1)
        assert p.own_row_waves == row_waves and max(-(-s // -(-s // share)) for s in steps) * step > 64 * 16
        check(G, batch, scales)


@pytest.mark.parametrize("dtype,scales,D", FORMS)
@pytest.mark.parametrize("B,row_waves,NP", [(6, 1, 336), (6, 1, 420), (15, 2, 336), (20, 4, 168)])
def test_more_ranges_than_the_join_takes_at_once(G, rules, B, row_waves, NP, dtype, scales, D):
    """16 pieces of the prefix are a round of the join's four waves: 18 to 42 of them, with own parts and without."""
    lens = [16 * NP + 7 * (i % 5) + 1 for i in range(B)]
    batch = Batch(50 + B, dtype, 8, 2, D, 16, NP, lens, [1] * B, D == 64, bool(scales))
    p = plan(rules, batch)
    assert p.row_waves == row_waves and p.ranges > 16 and (row_waves == 1 or p.ranges > 32)
    check(G, batch, scales)


@pytest.mark.parametrize("dtype,scales,D", FORMS)
def test_more_own_pieces_than_the_join_takes_at_once(G, rules, dtype, scales, D):
    """8 own pieces of a row are a round: one sequence's long own part, dealt to all shares."""
    lens = [48 + 5000, 48 + 11, 48]
    batch = Batch(60, dtype, 8, 2, D, 16, 3, lens, [2, 1, 1], True, bool(scales))
    p = plan(rules, batch)
    steps = [-(-(n - 48) // 128) for n in lens]
    share = max(-(-sum(steps) * 2 // p.shares), 1)
    assert p.own_row_waves == 1 and -(-steps[0] // share) > 16
    check(G, batch, scales)
