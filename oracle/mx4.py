"""4-bit microscaled matrices in plain 64-bit numpy, from the definition of the format."""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
WORD = 0xFFFFFFFF


def philox_blocks(blocks, epoch, purpose, seed):
    """Philox4x32-10 words [n, 4] of the blocks (a uint64 array) of one random stream."""
    b = np.asarray(blocks, np.uint64)
    c = [b & WORD, b >> np.uint64(32), np.full_like(b, epoch), np.full_like(b, purpose)]
    k0, k1 = seed & WORD, seed >> 32 & WORD
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), q & np.uint64(WORD),
             (p >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p & np.uint64(WORD)]
        k0, k1 = (k0 + 0x9E3779B9) & WORD, (k1 + 0xBB67AE85) & WORD
    return np.stack(c, 1).astype(np.uint32)


def random_bytes(rows, cols, epoch, purpose, seed):
    per = -(-cols // 16)
    w = philox_blocks(np.arange(rows * per, dtype=np.uint64), epoch, purpose, seed)
    return w.astype("<u4").view(np.uint8).reshape(rows, per * 16)


def scale_of(block):
    """The scale byte of a block: the smallest s with max <= 6 * 2^(s - 127)."""
    if not np.all(np.isfinite(block)):
        return 255
    most = np.max(np.abs(block))
    s = 0
    while most > 6 * 2.0 ** (s - 127):
        s += 1
    return s


def quantize(x, stochastic=False, epoch=0, purpose=6, seed=0):
    """x [rows, cols] -> codes, one a value, [rows, 128 groups], and scales [rows, 4 groups]."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    groups = -(-cols // 128)
    codes = np.zeros((rows, 128 * groups), np.uint8)
    scales = np.zeros((rows, 4 * groups), np.uint8)
    r = random_bytes(rows, cols, epoch, purpose, seed) if stochastic and x.size else None
    for i in range(rows):
        for j in range(0, cols, 32):
            block = x[i, j:j + 32]
            s = scale_of(block)
            scales[i, j // 32] = s
            if s == 255:
                continue
            t = np.abs(block) / 2.0 ** (s - 127)
            if stochastic:
                lo = np.searchsorted(GRID, t, side="right") - 1
                hi = np.minimum(lo + 1, 7)
                f = (t - GRID[lo]) / np.where(hi > lo, GRID[hi] - GRID[lo], 1)
                c = np.where(f * 512 >= 511 - 2 * r[i, j:j + len(block)].astype(int), hi, lo)
            else:
                d = np.abs(t[:, None] - GRID)
                c = np.argmin(d + 1e-9 * (np.arange(8) % 2) * (d <= d.min(1)[:, None]), 1)  # half way: the even code
            codes[i, j:j + len(block)] = c + 8 * np.signbit(block)
    return codes, scales


def pack(codes):
    return codes[:, 0::2] | codes[:, 1::2] << 4


def unpack(packed):
    return np.stack((packed & 15, packed >> 4), 2).reshape(packed.shape[0], -1)


def values(codes, scales):
    """What codes (one a value) and scales stand for."""
    v = np.where(codes & 8, -1.0, 1.0) * GRID[codes & 7]
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return v * np.repeat(s, 32, 1)
