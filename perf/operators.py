"""The operators of a step of drafted tokens for a batch behind one common prompt, as cases that can be
timed: rotary positions (and their gradient), the cache append with the rotation on the way, attention
whose common prefix is computed once for the batch, and the verification of drafted tokens.

``run`` computes them in plain torch operations in 32 bits (64 for angles and for the sums that a draw
is looked up in), or, with ``own``, through the package's entry points.  Head counts, head sizes, block sizes,
batches and lengths are those of the configured workloads (workloads.py) and odd ones of the same ranges;
vocabularies are generic sizes.
"""
import math
import random

import torch

own = False

KV_SCALE = 0.0125           # E4M3 caches of N(0, 1) data: +-448 codes cover +-5.6 sigma
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _rotary(name, kind, dtype, tokens, heads, kv_heads, dim, rot, interleaved, pos, scaling="none", block=16):
    return {"name": name, "kind": kind, "dtype": dtype, "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "rot": rot, "interleaved": interleaved, "pos_hi": pos, "scaling": scaling, "block": block}


def _common(name, dtype, batch, heads, kv_heads, dim, block, prefix, mine, new=(1, 1), alibi=False, e4m3=False):
    """prefix: common blocks; mine: range of a sequence's own cached tokens behind them; new: range of new tokens."""
    return {"name": name, "kind": "common", "dtype": dtype, "batch": batch, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "block": block, "prefix": prefix, "own_lo": mine[0], "own_hi": mine[1], "new_lo": new[0], "new_hi": new[1],
            "alibi": alibi, "e4m3": e4m3}


def _verify(name, dtype, batch, vocab, drafts, sampled=True):
    return {"name": name, "kind": "verify", "dtype": dtype, "batch": batch, "vocab": vocab, "drafts_lo": drafts[0],
            "drafts_hi": drafts[1], "sampled": sampled}


def listed():
    return [
        # rotary positions of one new token of a small model: the launch is all there is
        _rotary("rotary_one", "rotary", "f16", 1, 8, 2, 64, 64, False, 127),
        # eight whole prompts of 2560 tokens, long-context frequencies
        _rotary("rotary_prompts", "rotary", "bf16", 20480, 32, 8, 128, 128, False, 131071, "yarn"),
        # the gradient, interleaved pairs in half of the head, an odd number of tokens
        _rotary("rotary_gradient", "gradient", "f16", 4099, 40, 8, 128, 64, True, 8191, "linear"),
        # a decode step's append: one token each of a full batch
        _rotary("append_batch64", "append", "bf16", 64, 32, 4, 128, 128, False, 8191, block=32),
        # ragged chunks into 8-bit caches
        _rotary("append_e4m3_chunks", "append_e4m3", "bf16", 2943, 32, 8, 128, 96, True, 4095, "linear", block=32),
        # a few requests behind a short common prompt
        _common("common_few_short", "f16", 4, 8, 2, 64, 16, 16, (0, 60)),
        # a full batch behind a system prompt of 4096 tokens, slopes
        _common("common_batch64", "bf16", 64, 32, 4, 128, 32, 128, (127, 1023), alibi=True),
        # a full batch behind a document of 32768 tokens
        _common("common_long", "bf16", 64, 32, 8, 128, 16, 2048, (1023, 2047)),
        # drafted tokens: 2 to 9 queries a sequence
        _common("common_drafts", "f16", 16, 64, 8, 128, 16, 512, (63, 511), new=(2, 9)),
        # 8-bit caches
        _common("common_e4m3", "bf16", 32, 32, 8, 128, 16, 512, (255, 1023), e4m3=True),
        # one sequence, four drafts from a small vocabulary
        _verify("verify_one", "f32", 1, 32000, (4, 4)),
        # a full batch, four to eight drafts, a large odd vocabulary
        _verify("verify_batch64", "f32", 64, 128255, (4, 8)),
    ]


def _log(rng, lo, hi):
    """A whole number, spread over the logarithm of lo .. hi."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    case = _draw(rng)
    del case["name"]
    return case


def _draw(rng):
    kind = rng.choice(["rotary", "gradient", "append", "append_e4m3", "common", "common", "common", "common_e4m3", "verify", "verify"])
    if kind == "verify":
        batch, vocab, most = _log(rng, 1, 64), _log(rng, 1000, 128255), rng.randint(1, 8)
        return _verify("", rng.choice(["f32", "f32", "f16", "bf16"]), batch, vocab, (rng.randint(0, most), most), rng.random() < 0.8)
    heads, kv_heads = rng.choice([(8, 2), (16, 4), (32, 8), (32, 4), (64, 8), (40, 8), (16, 16)])
    dim, block, dtype = rng.choice([64, 128, 128]), rng.choice([16, 32, 64]), rng.choice(["f16", "bf16"])
    if kind in ("common", "common_e4m3"):
        batch = _log(rng, 2, 64)
        prefix, hi, new = _log(rng, 128, 32768), _log(rng, 8, 2047), rng.choice([1, 1, 1, rng.randint(2, 9)])
        while batch * new * heads * prefix * dim > 1.7e10 or batch * (prefix + hi) * kv_heads * dim > 2.2e9:
            prefix = prefix * 2 // 3
        return _common("", dtype, batch, heads, kv_heads, dim, block, -(-prefix // block), (hi // 4, hi), (max(1, new // 2), new),
                       rng.random() < 0.4, kind == "common_e4m3")
    tokens = _log(rng, 1, 20480)
    while tokens * (heads + kv_heads) * dim > 20480 * 40 * 128:
        tokens = tokens * 2 // 3
    rot = rng.choice([dim, dim, dim // 2, dim // 4 * 3, dim // 4])
    return _rotary("", kind, dtype, tokens, heads, kv_heads, dim, rot, rng.random() < 0.5, _log(rng, 100, 131071),
                   rng.choice(["none", "linear", "yarn"]), block)


def _frequencies(rot, scaling):
    """Radians a token of each pair in 64 bits, and the factor of the rotated values: base 10000; linear: positions
    divided by 4; yarn: by 16 from 8192 tokens on, pairs of 32 turns and more in them untouched, those of one turn and
    less divided, a ramp between."""
    i = torch.arange(0, rot, 2, dtype=torch.float64)
    f = 10000.0 ** (-i / rot)
    if scaling == "linear":
        return f / 4.0, 1.0
    if scaling == "yarn":
        def pair(turns):
            return rot * math.log(8192 / (turns * 2 * math.pi)) / (2 * math.log(10000.0))
        lo, hi = max(math.floor(pair(32.0)), 0), min(math.ceil(pair(1.0)), rot - 1)
        ramp = ((i / 2 - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f * (1 - ramp) + f / 16.0 * ramp, 0.1 * math.log(16.0) + 1.0
    return f, 1.0


def _lengths(case):
    """(own cached tokens, new tokens) of each sequence: the case's own, whatever the seed."""
    rng = random.Random("%(batch)d %(own_lo)d %(own_hi)d %(new_lo)d %(new_hi)d" % case)
    mine = [rng.randint(case["own_lo"], case["own_hi"]) for _ in range(case["batch"])]
    return mine, [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["batch"])]


def _drafts(case):
    rng = random.Random("%(batch)d %(vocab)d %(drafts_lo)d %(drafts_hi)d" % case)
    return [rng.randint(case["drafts_lo"], case["drafts_hi"]) for _ in range(case["batch"])]


def _starts(counts):
    return torch.tensor([sum(counts[:b]) for b in range(len(counts) + 1)], dtype=torch.int32)


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    kind = case["kind"]

    def normal(*shape, dtype):
        return torch.randn(*shape, generator=gen, device="cuda").to(dtype)

    if kind == "common":
        return _prepare_common(case, gen, normal)
    if kind == "verify":
        return _prepare_verify(case, gen)
    dt, T, Hq, Hkv, D, bs = DTYPES[case["dtype"]], case["tokens"], case["heads"], case["kv_heads"], case["dim"], case["block"]
    freqs, magnitude = _frequencies(case["rot"], case["scaling"])
    # q, k and v as one projection makes them: side by side in a row of each token
    qkv = normal(T, (Hq + 2 * Hkv) * D, dtype=dt)
    q, k, v = (x.view(T, -1, D) for x in qkv.split([Hq * D, Hkv * D, Hkv * D], dim=1))
    s = {"case": case, "q": q, "k": k, "v": v, "freqs": freqs.cuda(), "magnitude": magnitude,
         "positions": torch.randint(0, case["pos_hi"] + 1, (T,), generator=gen, device="cuda", dtype=torch.int32),
         "q_out": torch.empty(T, Hq, D, dtype=dt, device="cuda")}
    if kind in ("rotary", "gradient"):
        s["k_out"] = torch.empty(T, Hkv, D, dtype=dt, device="cuda")
        return s
    blocks = -(-T // bs) + 3
    s["slots"] = torch.randperm(blocks * bs, generator=gen, device="cuda")[:T]
    shape = (blocks, Hkv, bs, D)
    if kind == "append_e4m3":
        s["k_cache"], s["v_cache"] = (torch.zeros(shape, dtype=torch.uint8, device="cuda") for _ in range(2))
        s["k_scales"] = KV_SCALE * (1 + torch.rand(Hkv, generator=gen, device="cuda"))
        s["v_scales"] = KV_SCALE * (1 + torch.rand(Hkv, generator=gen, device="cuda"))
    else:
        s["k_cache"], s["v_cache"] = (torch.zeros(shape, dtype=dt, device="cuda") for _ in range(2))
    return s


def _prepare_common(case, gen, normal):
    dt, (mine, new) = DTYPES[case["dtype"]], _lengths(case)
    B, Hq, Hkv, D, bs, NP = case["batch"], case["heads"], case["kv_heads"], case["dim"], case["block"], case["prefix"]
    lens = [NP * bs + m + n for m, n in zip(mine, new)]
    need = [-(-n // bs) for n in lens]
    # the pool: the common blocks, every sequence's own and some of other requests, dealt in random order
    pool = NP + sum(n - NP for n in need) + 16
    order = torch.randperm(pool, generator=gen, device="cuda").int().cpu()
    table = torch.zeros(B, max(need), dtype=torch.int32)
    at = NP
    for b in range(B):
        table[b, :NP] = order[:NP]
        table[b, NP:need[b]] = order[at:at + need[b] - NP]
        at += need[b] - NP
    shape = (pool, Hkv, bs, D)
    if case["e4m3"]:
        def cache():
            x = torch.randn(shape, generator=gen, device="cuda") * (1.0 / KV_SCALE)
            return x.clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        def cache():
            return normal(*shape, dtype=dt)
    h = torch.arange(1, Hq + 1, dtype=torch.float64)
    q = normal(sum(new), Hq, D, dtype=dt)
    return {"case": case, "q": q, "out": torch.empty_like(q), "k_cache": cache(), "v_cache": cache(), "table": table.cuda(),
            "prefix": order[:NP].cuda(), "lens": torch.tensor(lens, dtype=torch.int32).cuda(), "cu": _starts(new).cuda(),
            "slopes": torch.exp2(-8.0 * h / Hq).float().cuda() if case["alibi"] else None, "scale": 1.0 / math.sqrt(D),
            "max_len": max(lens), "max_new": max(new)}


def _prepare_verify(case, gen):
    B, V, dt, drafts = case["batch"], case["vocab"], DTYPES[case["dtype"]], _drafts(case)
    T = sum(drafts)
    # the draft model's logits are the target's and some noise: most of its tokens are good ones
    logits = 2.5 * torch.randn(T + B, V, generator=gen, device="cuda")
    target = torch.softmax(logits, dim=1)
    rows = torch.tensor([i + b for b in range(B) for i in range(sum(drafts[:b]), sum(drafts[:b + 1]))], dtype=torch.int64).cuda()
    noisy = logits[rows] + 0.7 * torch.randn(T, V, generator=gen, device="cuda")
    gumbel = -torch.log(-torch.log(torch.rand(T, V, generator=gen, device="cuda").clamp_(1e-20, 1 - 1e-7)))
    tokens = (noisy + gumbel).argmax(dim=1) if T else torch.zeros(0, dtype=torch.int64, device="cuda")
    return {"case": case, "target": target.to(dt), "draft": torch.softmax(noisy, dim=1).to(dt) if case["sampled"] else None,
            "draft_tokens": tokens, "cu": _starts(drafts).cuda(),
            "accept_u": torch.rand(T, generator=gen, device="cuda"), "sample_u": torch.rand(B, generator=gen, device="cuda"),
            "tokens": torch.empty(B, case["drafts_hi"] + 1, dtype=torch.int64, device="cuda"),
            "accepted": torch.empty(B, dtype=torch.int32, device="cuda")}


def run(s):
    kind = s["case"]["kind"]
    if own:
        return _own(s, kind)
    if kind == "verify":
        return _plain_verify(s)
    if kind == "common":
        return {"out": _plain_common(s)}
    q = _rotate(s, s["q"], kind == "gradient")
    k = _rotate(s, s["k"], kind == "gradient")
    if kind in ("rotary", "gradient"):
        return {"q": q.to(s["q"].dtype), "k": k.to(s["k"].dtype)}
    bs, slots, kc, vc, v = s["case"]["block"], s["slots"], s["k_cache"], s["v_cache"], s["v"]
    if kind == "append_e4m3":
        def codes(x, scales):
            return (x * (1.0 / scales)[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        k, v = codes(k, s["k_scales"]), codes(v.float(), s["v_scales"])
    kc[slots // bs, :, slots % bs] = k.to(kc.dtype)
    vc[slots // bs, :, slots % bs] = v
    return {"q": q.to(s["q"].dtype), "k_cache": _values(kc), "v_cache": _values(vc)}


def _values(cache):
    """8-bit codes as the type whose values they are."""
    return cache.view(torch.float8_e4m3fn) if cache.dtype == torch.uint8 else cache


def _own(s, kind):
    import paper_2505_02351_amd as G
    case = s["case"]
    if kind == "verify":
        if "ws" not in s:
            s["ws"] = torch.empty(G.verify_drafts_workspace_bytes(case["batch"], case["vocab"]), dtype=torch.uint8, device="cuda")
        G.verify_drafts(s["tokens"], s["accepted"], s["target"], s["draft"], s["draft_tokens"], s["cu"], s["accept_u"], s["sample_u"], s["ws"])
        return {"tokens": s["tokens"], "accepted": s["accepted"]}
    if kind == "common":
        B, Hq, Hkv, D, bs = case["batch"], case["heads"], case["kv_heads"], case["dim"], case["block"]
        if "ws" not in s:
            n = G.common_prefix_workspace_bytes(s["q"].shape[0], B, Hq, Hkv, D, bs, case["prefix"], s["max_len"], s["max_new"])
            s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        args = (s["out"], s["q"], s["k_cache"], s["v_cache"], s["prefix"], s["table"], s["lens"], s["cu"], s["slopes"], s["scale"])
        if case["e4m3"]:
            G.paged_attention_common_fp8(*args, KV_SCALE, KV_SCALE, s["max_len"], s["max_new"], s["ws"])
        else:
            G.paged_attention_common(*args, s["max_len"], s["max_new"], s["ws"])
        return {"out": s["out"]}
    q_out, q, k, v, positions, freqs = s["q_out"], s["q"], s["k"], s["v"], s["positions"], s["freqs"]
    how = {"interleaved": case["interleaved"], "magnitude": s["magnitude"]}
    if kind in ("rotary", "gradient"):
        G.rotary_embedding(q_out, q, s["k_out"], k, positions, freqs, backward=kind == "gradient", **how)
        return {"q": q_out, "k": s["k_out"]}
    if kind == "append_e4m3":
        G.rotary_and_cache_fp8_heads(q_out, q, k, v, s["k_cache"], s["v_cache"], s["slots"], positions, freqs, s["k_scales"], s["v_scales"], **how)
    else:
        G.rotary_and_cache(q_out, q, k, v, s["k_cache"], s["v_cache"], s["slots"], positions, freqs, **how)
    return {"q": q_out, "k_cache": _values(s["k_cache"]), "v_cache": _values(s["v_cache"])}


def _rotate(s, x, backward):
    """x [T, heads, D] rotated by its positions, in 32 bits (angles in 64)."""
    rot, x = s["case"]["rot"], x.float()
    angle = s["positions"].double()[:, None] * s["freqs"]
    cos = (angle.cos() * s["magnitude"]).float()[:, None]
    sin = (angle.sin() * s["magnitude"]).float()[:, None] * (-1.0 if backward else 1.0)
    if s["case"]["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _plain_common(s):
    """All sequences' keys gathered through their tables and padded to the longest, one masked softmax."""
    case, q, lens, cu = s["case"], s["q"], s["lens"].long(), s["cu"].long()
    B, Hq, Hkv, D, bs = case["batch"], case["heads"], case["kv_heads"], case["dim"], case["block"]
    G, N = Hq // Hkv, s["max_new"]
    j = torch.arange(s["max_len"], device="cuda")
    blocks, rows = s["table"][:, j // bs].long(), (j % bs).expand(B, -1)

    def gathered(cache):                                     # [B, Hkv, keys, D]
        x = _values(cache)[blocks, :, rows].transpose(1, 2).float()
        return x * torch.tensor(KV_SCALE, dtype=torch.float32) if case["e4m3"] else x

    i = torch.arange(N, device="cuda")
    there = i < (cu[1:] - cu[:-1])[:, None]                  # [B, N]
    pos = lens[:, None] - (cu[1:] - cu[:-1])[:, None] + i
    token = (cu[:-1, None] + i).clamp(max=q.shape[0] - 1)
    qp = q[token].float().view(B, N, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, N * G, D)
    score = (qp @ gathered(s["k_cache"]).transpose(2, 3)).view(B, Hkv, N, G, -1) * s["scale"]
    dist = (j - pos[:, :, None]).float()                     # [B, N, keys]
    if s["slopes"] is not None:
        score += s["slopes"].view(Hkv, 1, G, 1) * dist[:, None, :, None]
    score.masked_fill_((dist > 0)[:, None, :, None], -math.inf)
    v = gathered(s["v_cache"]).masked_fill_((j >= lens[:, None])[:, None, :, None], 0.0)
    o = (torch.softmax(score, dim=-1).view(B, Hkv, N * G, -1) @ v).view(B, Hkv, N, G, D)
    return o.permute(0, 2, 1, 3, 4).reshape(B, N, Hq, D)[there].to(q.dtype)


def _plain_verify(s):
    case, cu, p, q = s["case"], s["cu"].long(), s["target"], s["draft"]
    B, V, K = case["batch"], case["vocab"], case["drafts_hi"]
    count, first, i = cu[1:] - cu[:-1], cu[:-1] + torch.arange(B, device="cuda"), torch.arange(K + 1, device="cuda")
    most = max(s["draft_tokens"].shape[0] - 1, 0)
    at = (cu[:-1, None] + i[:K]).clamp(max=most)             # [B, K]
    there = i[:K] < count[:, None]
    if s["draft_tokens"].shape[0]:
        x, u = s["draft_tokens"][at], s["accept_u"][at].double()
        px = p[(first[:, None] + i[:K]).clamp(max=p.shape[0] - 1), x].double()
        qx = q[at, x].double() if q is not None else torch.ones_like(u)
        good = there & (u * qx < px)
    else:
        x, good = torch.zeros_like(at), there
    n = good.long().cumprod(dim=1).sum(dim=1)                # accepted drafts
    left = p[first + n].double()
    rejected = n < count
    if s["draft_tokens"].shape[0]:
        r = (cu[:-1] + n).clamp(max=most)
        minus = q[r].double() if q is not None else torch.nn.functional.one_hot(s["draft_tokens"][r], V).double() * left
        rest = (left - minus).clamp(min=0)
        left = torch.where((rejected & (rest.sum(dim=1) > 0))[:, None], rest, left)
    sums = left.cumsum(dim=1)
    token = (sums > s["sample_u"].double()[:, None] * sums[:, -1:]).int().argmax(dim=1)
    tokens = torch.where(i < n[:, None], torch.cat([x, x[:, :1] if K else x.new_zeros(B, 1)], dim=1), -1)
    return {"tokens": torch.where(i == n[:, None], token[:, None], tokens), "accepted": n.int()}


def work(case):
    """Each input once and each output once: of a cache the rows that are attended (common ones once) or written; of the
    probabilities one row for each sequence and the drafts' own entries."""
    kind = case["kind"]
    if kind == "verify":
        e, drafts = DTYPES[case["dtype"]].itemsize, _drafts(case)
        rows = 2 if case["sampled"] else 1
        return {"bytes": case["batch"] * (rows * case["vocab"] * e + 8 * (case["drafts_hi"] + 1) + 12) + sum(drafts) * (rows * e + 12),
                "flops": 3 * case["batch"] * case["vocab"]}
    Hq, Hkv, D = case["heads"], case["kv_heads"], case["dim"]
    if kind == "common":
        mine, new = _lengths(case)
        P = case["prefix"] * case["block"]
        rows = P + sum(m + n for m, n in zip(mine, new))
        pairs = sum(n * (P + m) + n * (n + 1) // 2 for m, n in zip(mine, new))
        return {"bytes": 2 * rows * Hkv * D * (1 if case["e4m3"] else 2) + 2 * sum(new) * Hq * D * 2, "flops": 4 * D * Hq * pairs}
    T = case["tokens"]
    if kind in ("rotary", "gradient"):
        return {"bytes": 4 * T * (Hq + Hkv) * D + 4 * T, "flops": 3 * T * (Hq + Hkv) * case["rot"]}
    out = 1 if kind == "append_e4m3" else 2
    return {"bytes": T * D * (4 * Hq + 2 * Hkv * (2 + out)) + 12 * T, "flops": 3 * T * (Hq + Hkv) * case["rot"]}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "verify":
        return _exact_verify(s)
    if case["kind"] == "common":
        return {"out": _exact_common(s)}
    T, D, rot = case["tokens"], case["dim"], case["rot"]
    sign = -1.0 if case["kind"] == "gradient" else 1.0
    # as complex numbers: pairs (dim a, dim b) times m exp(i angle)
    if case["interleaved"]:
        a, b = torch.arange(0, rot, 2), torch.arange(1, rot, 2)
    else:
        a, b = torch.arange(rot // 2), torch.arange(rot // 2, rot)
    angle = s["positions"].double()[:, None] * s["freqs"]
    factor = torch.polar(torch.full_like(angle, s["magnitude"]), sign * angle)[:, None, :]

    def turned(x):
        y = x.double()
        z = torch.complex(y[..., a.cuda()], y[..., b.cuda()]) * factor
        y[..., a.cuda()], y[..., b.cuda()] = z.real, z.imag
        return y

    if case["kind"] in ("rotary", "gradient"):
        return {"q": turned(s["q"]), "k": turned(s["k"])}
    blocks, rows = s["slots"] // case["block"], s["slots"] % case["block"]
    caches = {}
    for name, x in (("k", turned(s["k"])), ("v", s["v"].double())):
        c = torch.zeros(s[name + "_cache"].shape, dtype=torch.float64, device="cuda")
        if case["kind"] == "append_e4m3":
            x = x / s[name + "_scales"].double()[:, None]
        c[blocks, :, rows] = x
        caches[name + "_cache"] = c
    return {"q": turned(s["q"]), **caches}


def _exact_common(s):
    case, (mine, new) = s["case"], _lengths(s["case"])
    Hq, Hkv, D, bs = case["heads"], case["kv_heads"], case["dim"], case["block"]
    group, P = Hq // Hkv, case["prefix"] * case["block"]
    one = float(torch.tensor(KV_SCALE, dtype=torch.float32)) if case["e4m3"] else 1.0
    out, t = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda"), 0
    scale = float(torch.tensor(s["scale"], dtype=torch.float32))
    for b in range(case["batch"]):
        n = P + mine[b] + new[b]
        at = torch.arange(n, device="cuda")
        phys = s["table"][b].long().repeat_interleave(bs)[:n] * bs + at % bs

        def head(cache, g):                                  # [n, D]
            x = cache[:, g].reshape(-1, D)[phys]
            return (x.view(torch.float8_e4m3fn).float() if case["e4m3"] else x).double() * one

        pos = torch.arange(n - new[b], n, device="cuda")
        for g in range(Hkv):
            k, v = head(s["k_cache"], g).t().contiguous(), head(s["v_cache"], g)
            x = s["q"][t:t + new[b], g * group:(g + 1) * group].double()            # [new, group, D]
            sc = (x.reshape(-1, D) @ k).view(new[b], group, n) * scale
            away = (at - pos[:, None]).double()[:, None]
            if s["slopes"] is not None:
                sc = sc + s["slopes"][g * group:(g + 1) * group].double()[None, :, None] * away
            w = torch.exp(sc - sc.masked_fill(away > 0, -math.inf).amax(dim=2, keepdim=True)).masked_fill(away > 0, 0.0)
            o = (w / w.sum(dim=2, keepdim=True)).reshape(-1, n) @ v
            out[t:t + new[b], g * group:(g + 1) * group] = o.view(new[b], group, D)
        t += new[b]
    return out


def _exact_verify(s):
    import numpy as np
    case = s["case"]
    p, cu, x = s["target"].double().cpu().numpy(), s["cu"].tolist(), s["draft_tokens"].tolist()
    q = None if s["draft"] is None else s["draft"].double().cpu().numpy()
    au, su = s["accept_u"].double().tolist(), s["sample_u"].double().tolist()
    tokens, accepted = np.full((case["batch"], case["drafts_hi"] + 1), -1, np.int64), []
    for b in range(case["batch"]):
        n, row = 0, cu[b] + b
        while n < cu[b + 1] - cu[b]:
            i = cu[b] + n
            if not au[i] * (1.0 if q is None else q[i, x[i]]) < p[row + n, x[i]]:
                break
            tokens[b, n], n = x[i], n + 1
        dist = p[row + n].copy()
        if n < cu[b + 1] - cu[b]:
            if q is None:
                dist[x[cu[b] + n]] = 0.0
            else:
                dist = np.maximum(dist - q[cu[b] + n], 0.0)
            if dist.sum() <= 0:
                dist = p[row + n]
        sums = np.cumsum(dist)
        tokens[b, n] = np.searchsorted(sums, su[b] * sums[-1], side="right")
        accepted.append(n)
    return {"tokens": torch.from_numpy(tokens).cuda(), "accepted": torch.tensor(accepted, dtype=torch.int32).cuda()}
