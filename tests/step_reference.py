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
