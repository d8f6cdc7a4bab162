"""Plain 64-bit versions (numpy) of the operators around a step's attention, for the tests."""
import numpy as np


def rotate(x, positions, freqs, interleaved, magnitude=1.0, backward=False):
    """x [T, H, D] turned by its positions."""
    y = np.array(x, dtype=np.float64)
    rot = 2 * len(freqs)
    a = np.asarray(positions, np.float64)[:, None] * np.asarray(freqs, np.float64)
    c, s = magnitude * np.cos(a)[:, None], magnitude * np.sin(a)[:, None] * (-1 if backward else 1)
    i, j = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if interleaved else (np.arange(rot // 2), np.arange(rot // 2, rot))
    u, v = y[..., i].copy(), y[..., j].copy()
    y[..., i], y[..., j] = u * c - v * s, v * c + u * s
    return y


def rotate_slack(x, freqs, interleaved, magnitude=1.0):
    """What 32-bit arithmetic may cost an element of rotate(): sine and cosine to 2 units of 2^-24 and the angle's remainder
    to 2^-24 of a half turn, on each of the two terms, and three roundings: below 1e-6 of the pair's sum of magnitudes."""
    m = np.abs(np.array(x, np.float64))
    rot = 2 * len(freqs)
    i, j = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if interleaved else (np.arange(rot // 2), np.arange(rot // 2, rot))
    both = m[..., i] + m[..., j]
    slack = np.zeros_like(m)
    slack[..., i] = slack[..., j] = 1e-6 * abs(magnitude) * both
    return slack


def half_step(ref, eps, smallest):
    """Half a step of the output type at ref: eps / 2 of the value, at least half of its smallest step."""
    return np.maximum(np.abs(ref) * (eps / 2), smallest / 2)


EPS = {"f16": 2.0 ** -10, "bf16": 2.0 ** -7, "e4m3": 2.0 ** -3}
SMALLEST = {"f16": 2.0 ** -24, "bf16": 2.0 ** -133, "e4m3": 2.0 ** -9}


def verify(target, draft, draft_tokens, cu, accept_u, sample_u, width):
    """(tokens [B, width], accepted [B]); target, draft float64 rows (draft may be None)."""
    V, B = target.shape[1], len(cu) - 1
    tokens, accepted = np.full((B, width), -1, np.int64), np.zeros(B, np.int32)

    def counted(x):
        return np.where(np.isfinite(x) & (x > 0), x, 0.0)

    for b in range(B):
        n, count, row = 0, min(cu[b + 1] - cu[b], width - 1), cu[b] + b
        while n < count:
            i, x = cu[b] + n, draft_tokens[cu[b] + n]
            if not (0 <= x < V and accept_u[i] * (1.0 if draft is None else draft[i, x]) < target[row + n, x]):
                break
            tokens[b, n] = x
            n += 1
        rest = counted(target[row + n])
        if n < count and 0 <= draft_tokens[cu[b] + n] < V:
            i, x = cu[b] + n, draft_tokens[cu[b] + n]
            if draft is None:
                less = rest.copy()
                less[x] = 0.0
            else:
                with np.errstate(invalid="ignore"):
                    less = counted(target[row + n] - draft[i])
            rest = less if less.sum() > 0 else rest
        sums = np.cumsum(rest)
        over = (rest > 0) & (sums > sample_u[b] * sums[-1])
        tokens[b, n] = np.argmax(over) if over.any() else -1
        accepted[b] = n
    return tokens, accepted


def attend(q, keys, values, positions, slopes, scale):
    """Rows q [n, Hq, D] at `positions` over keys, values [L, Hkv, D] up to each row's position -> (out, what the weights
    average: sum of weight * |value|).  A row that sees no key is 0."""
    n, Hq, D = q.shape
    L, Hkv, _ = keys.shape
    out, size = np.zeros((n, Hq, D)), np.zeros((n, Hq, D))
    for i in range(n):
        see = int(min(max(positions[i] + 1, 0), L))
        if see == 0:
            continue
        for h in range(Hq):
            g = h // (Hq // Hkv)
            s = scale * (keys[:see, g] @ q[i, h])
            if slopes is not None:
                s = s + slopes[h] * (np.arange(see) - positions[i])
            w = np.exp(s - s.max())
            w /= w.sum()
            out[i, h] = w @ values[:see, g]
            size[i, h] = w @ np.abs(values[:see, g])
    return out, size


# Relative error of a softmax weight in the kernels: rounded to fp16 once, or kept to 16 bits as two bf16; and 1.2e-4 for the
# score (128 products summed in 32 bits, of magnitudes that add up to some 10: 128 * 10 * 2^-24, with the exponential's
# argument and value).
WEIGHT = {"f16": 2.0 ** -11 + 1.2e-4, "bf16": 2.0 ** -16 + 1.2e-4}


def attention_bar(ref, size, dtype):
    """What a kernel's output may differ from attend()'s: weights off by WEIGHT on both sides of the quotient, one rounding."""
    slack = WEIGHT[dtype] * (size + np.abs(ref))
    return half_step(np.abs(ref) + slack, EPS[dtype], SMALLEST[dtype]) + slack
