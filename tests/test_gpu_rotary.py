"""Rotary positions and the rotated cache appends against plain 64-bit arithmetic."""
import math

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


def torch_type(dtype):
    import torch
    return {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]


def rows(seed, T, H, D, dtype, pad=0, offset=0):
    """[T, H, D] of N(0, 1), a slice of longer rows that starts `offset` elements in."""
    import torch
    gen = torch.Generator().manual_seed(seed)
    wide = torch.randn(T, offset + H * D + pad, generator=gen).to(torch_type(dtype)).cuda()
    return wide[:, offset:offset + H * D].unflatten(1, (H, D))


def host(t):
    return t.double().cpu().numpy()


def close(got, ref, slack, dtype, what):
    bar = R.half_step(np.abs(ref) + slack, R.EPS[dtype], R.SMALLEST[dtype]) + slack
    bad = ~(np.abs(host(got) - ref) <= bar)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, worst {np.abs(host(got) - ref).max()}"


def positions_of(seed, T, far=131072):
    rng = np.random.default_rng(seed)
    p = rng.integers(0, far, T).astype(np.int32)
    p[:min(T, 4)] = [far * 8 + 7, 0, 1, -5][:min(T, 4)]
    return p


# (T, Hq, Hkv, D, rot): one token; few; more than a workgroup's tokens; many workgroups of several tokens; odd groups; rot that is no multiple of 16
SHAPES = [(1, 8, 2, 64, 64), (3, 5, 1, 128, 128), (67, 32, 4, 128, 64), (4500, 4, 2, 64, 16), (2100, 40, 8, 128, 96), (33, 6, 3, 64, 34),
          (9, 3, 3, 128, 2), (1025, 2, 1, 128, 126)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv,D,rot", SHAPES)
def test_rotary_embedding(G, T, Hq, Hkv, D, rot, backward, interleaved, dtype):
    import torch
    q, k = rows(1, T, Hq, D, dtype, pad=16), rows(2, T, Hkv, D, dtype)
    freqs, m = G.rotary_frequencies(rot, 10000.0, G.ROTARY_YARN, 8.0, 4096.0)
    pos = positions_of(T, T)
    out = [torch.full((T, H, D), float("nan"), dtype=q.dtype, device="cuda") for H in (Hq, Hkv)]
    G.rotary_embedding(out[0], q, out[1], k, torch.from_numpy(pos).cuda(), freqs.cuda(), interleaved=interleaved, magnitude=m, backward=backward)
    for got, x, name in zip(out, (q, k), "qk"):
        ref = R.rotate(host(x), pos, freqs.numpy(), interleaved, m, backward)
        close(got, ref, R.rotate_slack(host(x), freqs, interleaved, m), dtype, name)
        assert torch.equal(got[..., rot:], x[..., rot:])        # what passes through does so bit for bit


@pytest.mark.parametrize("pad,offset", [(1, 0), (0, 1), (3, 5), (8, 8), (4, 2)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rows_of_any_alignment_in_place(G, interleaved, pad, offset):
    import torch
    T, Hq, Hkv, D = 19, 3, 2, 64
    q, k = rows(3, T, Hq, D, "bf16", pad, offset), rows(4, T, Hkv, D, "bf16", pad, offset)
    freqs, _ = G.rotary_frequencies(D)
    pos = positions_of(5, T)
    args = torch.from_numpy(pos).cuda(), freqs.cuda()
    want = [torch.empty(x.shape, dtype=x.dtype, device="cuda") for x in (q, k)]
    G.rotary_embedding(want[0], q, want[1], k, *args, interleaved=interleaved)
    for w, x in zip(want, (q, k)):
        close(w, R.rotate(host(x), pos, freqs.numpy(), interleaved), R.rotate_slack(host(x), freqs, interleaved), "bf16", "out of place")
    around = q._base.clone()
    around[:, offset:offset + Hq * D] = want[0].flatten(1)
    G.rotary_embedding(q, q, k, k, *args, interleaved=interleaved)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    assert torch.equal(q._base, around)                          # nothing beside the rows
    only = torch.empty_like(want[0])
    G.rotary_embedding(only, want[0], None, None, *args, interleaved=interleaved, backward=True)
    G.rotary_embedding(only, only, None, None, *args, interleaved=interleaved)
    assert (only.float() - want[0].float()).abs().max() < 0.1    # there and back, two roundings


def test_the_gradient_is_that_of_the_rotation(G):
    """Against the formula's transpose: <R x, y> = <x, R^T y> for random y; and against differences of the operator itself."""
    import torch
    T, H, D, rot = 6, 2, 64, 48
    freqs, m = G.rotary_frequencies(rot, 10000.0, G.ROTARY_YARN, 4.0, 512.0)
    pos = torch.arange(100, 100 + T, dtype=torch.int32).cuda()
    for interleaved in (False, True):
        call = dict(interleaved=interleaved, magnitude=m)
        x, y = rows(7, T, H, D, "f16"), rows(8, T, H, D, "f16")
        fx, gy = torch.empty_like(x), torch.empty_like(y)
        G.rotary_embedding(fx, x, None, None, pos, freqs.cuda(), **call)
        G.rotary_embedding(gy, y, None, None, pos, freqs.cuda(), backward=True, **call)
        a, b = (fx.double() * y.double()).sum().item(), (x.double() * gy.double()).sum().item()
        # each term is off by half a step of one factor, N(0, m) by N(0, 1): random signs, 6 sigma
        assert abs(a - b) < 6 * math.sqrt(2 * x.numel()) * 2.0 ** -11 * m
        for d in (0, 1, rot // 2, rot - 1, rot, D - 1):          # the column of the transpose: differences along e_d
            step = torch.zeros_like(x)
            step[:, :, d] = 1.0
            up, down = torch.empty_like(x), torch.empty_like(x)
            G.rotary_embedding(up, step, None, None, pos, freqs.cuda(), **call)
            G.rotary_embedding(down, -step, None, None, pos, freqs.cuda(), **call)
            column = (up.double() - down.double()) / 2
            want = (column * y.double()).sum(dim=2)
            # two terms, each off by half a step of the column's entry and of the gradient's sum
            bar = 2.0 ** -11 * (2 * m * y.double().abs().amax(dim=2) * 2) + 1e-6
            assert ((gy[:, :, d].double() - want).abs() <= bar).all(), d


@pytest.mark.parametrize("scaling", range(5))
def test_far_positions(G, scaling):
    """Positions up to 2^31 - 1, whose angles 32 bits do not hold."""
    import torch
    q = rows(9, 5, 2, 128, "f16")
    freqs, m = G.rotary_frequencies(128, 500000.0, scaling, 8.0, 8192.0)
    pos = np.array([2**31 - 1, 2**30 + 1, -2**31, 999_983, 16_777_217], np.int32)
    out = torch.empty_like(q)
    G.rotary_embedding(out, q, None, None, torch.from_numpy(pos).cuda(), freqs.cuda(), magnitude=m)
    # two products in 64 bits here and one in the reference, of up to 2^31 radians: 3 * 2^31 * 2^-53 = 0.7e-6 of a radian beside the slack's 1e-6
    close(out, R.rotate(host(q), pos, freqs.numpy(), False, m), 2 * R.rotate_slack(host(q), freqs, False, m), "f16", "far")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv,D,rot", SHAPES)
def test_append_is_the_two_calls(G, T, Hq, Hkv, D, rot, interleaved, dtype):
    """Bits of rotary_embedding followed by reshape_and_cache; padding tokens' rows are not stored, and nothing else changes."""
    import torch
    bs = 32 if D == 128 else 16
    qkv = rows(11, T, Hq + 2 * Hkv, D, dtype, pad=8 * (T % 2))
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    freqs = G.rotary_frequencies(rot)[0].cuda()
    pos = torch.from_numpy(positions_of(T + 1, T)).cuda()
    blocks = -(-T // bs) + 2
    slots = torch.randperm(blocks * bs, generator=torch.Generator().manual_seed(T))[:T]
    slots[T // 2] = -1
    slots = slots.cuda()
    shape = (blocks, Hkv, bs, D)
    caches = [torch.full(shape, float("nan"), dtype=q.dtype, device="cuda") for _ in range(4)]
    want_q, want_k = torch.empty(T, Hq, D, dtype=q.dtype, device="cuda"), torch.empty(T, Hkv, D, dtype=q.dtype, device="cuda")
    G.rotary_embedding(want_q, q, want_k, k, pos, freqs, interleaved=interleaved, magnitude=1.25)
    G.reshape_and_cache(want_k, v, caches[0], caches[1], slots)
    got_q = torch.full_like(want_q, float("nan"))
    G.rotary_and_cache(got_q, q, k, v, caches[2], caches[3], slots, pos, freqs, interleaved=interleaved, magnitude=1.25)
    assert torch.equal(got_q, want_q)
    for a, b in ((caches[0], caches[2]), (caches[1], caches[3])):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv,D,rot", [s for s in SHAPES if s[0] < 2000])
def test_append_to_8_bit_caches(G, T, Hq, Hkv, D, rot, interleaved, dtype, per_head):
    import torch
    bs = 64
    q, k, v = rows(12, T, Hq, D, dtype), rows(13, T, Hkv, D, dtype), rows(14, T, Hkv, D, dtype)
    k[0, 0, 0] = 500.0                                           # saturates
    freqs = G.rotary_frequencies(rot)[0]
    pos = positions_of(T + 2, T)
    blocks = -(-T // bs) + 1
    slots = np.random.default_rng(T).permutation(blocks * bs)[:T]
    slots[T // 2] = -1 if T > 1 else slots[T // 2]
    kc, vc = (torch.full((blocks, Hkv, bs, D), 0x55, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks = torch.linspace(0.01, 0.03, Hkv, device="cuda") if per_head else torch.full((Hkv,), 0.0125, device="cuda")
    vs = torch.linspace(0.05, 0.01, Hkv, device="cuda") if per_head else torch.full((Hkv,), 0.02, device="cuda")
    q_out = torch.empty_like(q)
    args = (q_out, q, k, v, kc, vc, torch.from_numpy(slots).cuda(), torch.from_numpy(pos).cuda(), freqs.cuda())
    if per_head:
        G.rotary_and_cache_fp8_heads(*args, ks, vs, interleaved=interleaved)
    else:
        G.rotary_and_cache_fp8(*args, 0.0125, 0.02, interleaved=interleaved)
    close(q_out, R.rotate(host(q), pos, freqs.numpy(), interleaved), R.rotate_slack(host(q), freqs, interleaved), dtype, "q")
    live = slots >= 0
    stored = np.zeros((blocks, bs), bool)
    stored[slots[live] // bs, slots[live] % bs] = True
    for cache, x, scales, slack in ((kc, R.rotate(host(k), pos, freqs.numpy(), interleaved), ks, R.rotate_slack(host(k), freqs, interleaved)),
                                    (vc, host(v), vs, np.zeros(v.shape))):
        assert (cache.cpu().numpy().transpose(0, 2, 1, 3)[~stored] == 0x55).all()
        got = cache.view(torch.float8_e4m3fn).float().cpu().numpy()[slots[live] // bs, :, slots[live] % bs].astype(np.float64)
        inv = 1.0 / scales.cpu().numpy().astype(np.float64)[:, None]
        t, s = (x * inv)[live], (slack * inv + np.abs(x * inv) * 2.0 ** -22)[live]      # (32 bits: the inverse, the product)
        ref = np.clip(t, -448, 448)
        assert (np.abs(got - ref) <= R.half_step(np.abs(ref) + s, R.EPS["e4m3"], R.SMALLEST["e4m3"]) + s).all()


def test_non_finite_rows_stay_in_their_pairs(G):
    import torch
    q = rows(15, 4, 2, 64, "bf16")
    q[1, 0, 3], q[2, 1, 40] = float("nan"), float("inf")
    freqs, _ = G.rotary_frequencies(32)
    out = torch.empty_like(q)
    G.rotary_embedding(out, q, None, None, torch.arange(7, 11, dtype=torch.int32).cuda(), freqs.cuda())
    bad = ~torch.isfinite(out).cpu()
    want = torch.zeros_like(bad)
    want[1, 0, 3] = want[1, 0, 19] = want[2, 1, 40] = True       # dim 40 passes through
    assert torch.equal(bad, want)


def test_a_captured_append_replays(G):
    """A graph of the append on a side stream, replayed over other inputs, with eager calls between."""
    import torch
    T, Hq, Hkv, D, bs = 37, 8, 2, 128, 16
    q, k, v = (rows(20 + i, T, H, D, "bf16") for i, H in enumerate((Hq, Hkv, Hkv)))
    freqs = G.rotary_frequencies(D)[0].cuda()
    pos, slots = torch.arange(T, dtype=torch.int32).cuda(), torch.arange(T).cuda()
    q_out, kc, vc = torch.empty_like(q), torch.zeros(4, Hkv, bs, D, dtype=q.dtype, device="cuda"), torch.zeros(4, Hkv, bs, D, dtype=q.dtype, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        G.rotary_and_cache(q_out, q, k, v, kc, vc, slots, pos, freqs)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.rotary_and_cache(q_out, q, k, v, kc, vc, slots, pos, freqs)
    for i in range(3):
        q.copy_(rows(30 + i, T, Hq, D, "bf16"))
        k.copy_(rows(40 + i, T, Hkv, D, "bf16"))
        pos.add_(1000)
        graph.replay()
        got = q_out.clone(), kc.clone()
        q_out.zero_(), kc.zero_()
        G.rotary_and_cache(q_out, q, k, v, kc, vc, slots, pos, freqs)
        torch.cuda.synchronize()
        assert torch.equal(got[0], q_out) and torch.equal(got[1], kc)
