"""The AdamW step in plain numpy: in 64 bits, and with states in 8 bits."""
import numpy as np

from .mx4 import philox_blocks

FORMATS = {"m": (7, 448.0), "v": (15, 61440.0)}  # exponent bias and largest number; three mantissa bits


def step(p, g, m, v, t, lr, beta1, beta2, eps, decay, scale=1.0):
    """The new (p, m, v) in 64 bits."""
    g = np.asarray(g, np.float64) * scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    mh, vh = m / (1 - beta1 ** t), v / (1 - beta2 ** t)
    return p * (1 - lr * decay) - lr * mh / (np.sqrt(vh) + eps), m, v


def moments32(g, m, v, beta1, beta2, scale=1.0):
    """The new moments as the 8-bit states see them: every operation rounded to 32 bits."""
    f = np.float32
    g = np.asarray(g, f) * f(scale)
    return m * f(beta1) + g * f(1 - beta1), v * f(beta2) + (g * g) * f(1 - beta2)


def numbers(kind):
    """The numbers of a format by code: 128 of m's (and their negatives), 256 of v's."""
    bias, _ = FORMATS[kind]
    c = np.arange(128 if kind == "m" else 256)
    e, f = c >> 3, c & 7
    return np.where(e > 0, (8 + f) * 2.0 ** (e - 3.0 - bias), f * 2.0 ** (-2.0 - bias))


def read(codes, scales, kind):
    n = numbers(kind)
    c = codes.astype(int)
    x = np.where(c & 128, -n[c & 127], n[c & 127]) if kind == "m" else n[c]
    s = np.repeat(scales.astype(np.float64), 32)[: len(codes)]
    return np.where(s == 255, np.nan, x * np.exp2(s - 127))


def write(x, words16, kind):
    """x (32-bit values of one tensor) with 16 random bits each -> codes and scales."""
    bias, most = FORMATS[kind]
    n = numbers(kind)
    x = np.asarray(x, np.float32)
    codes, scales = np.zeros(len(x), np.uint8), np.zeros(-(-len(x) // 32), np.uint8)
    least = 2.0 ** (1 - bias)
    for j in range(len(scales)):
        b = np.abs(x[32 * j:32 * j + 32].astype(np.float64))
        if not np.all(np.isfinite(b)):
            scales[j] = 255
            continue
        s = 0
        while b.max() > most * 2.0 ** (s - 127):
            s += 1
        scales[j] = s
        t = b / 2.0 ** (s - 127)
        # below the least normal number: the step of the least binade, the place in it rounded to 32 bits
        t = np.where(t < least, (t + least).astype(np.float32).astype(np.float64) - least, t)
        lo = np.searchsorted(n, t, side="right") - 1
        step = np.where(lo < 8, least / 8, np.exp2(np.floor(np.log2(np.maximum(n[lo], least)))) / 8)
        f = np.floor((t - n[lo]) / step * 2 ** 20)
        up = f + 16 * words16[32 * j:32 * j + 32].astype(np.int64) + 8 >= 2 ** 20
        codes[32 * j:32 * j + 32] = lo + up + (128 * np.signbit(x[32 * j:32 * j + 32]) if kind == "m" else 0)
    return codes, scales


def random_words(n, t, seed, first=0):
    """The words of elements first .. first + n - 1 (first a multiple of 4) of a tensor with its own seed at step t."""
    return philox_blocks(first // 4 + np.arange(-(-n // 4), dtype=np.uint64), t, 8, seed).reshape(-1)[:n]
