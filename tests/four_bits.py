"""What 4-bit quantisation, dropout and layer norm are, written from their definitions in binary64 and whole numbers on
the host; no code of the library's."""
import numpy as np

LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
VALUES = np.concatenate([LEVELS, -LEVELS])
BLOCK = 32
FOR_DROPOUT, FOR_ROWS, FOR_COLUMNS = 1, 2, 3


def philox(counter, key):
    """Philox4x32-10 of arrays: counter [n, 4], key (2 numbers) -> [n, 4]."""
    c = [counter[:, i].astype(np.uint64) for i in range(4)]
    k0, k1 = int(key[0]), int(key[1])
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), p1 & low, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p0 & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, 1)


def draws(groups, what, seed, step):
    """[len(groups), 8] 16-bit numbers."""
    groups = np.asarray(groups, np.uint64)
    low = np.uint64(0xFFFFFFFF)
    counter = np.zeros((len(groups), 4), np.uint64)
    counter[:, 0] = groups & low
    counter[:, 1] = groups >> np.uint64(32) | np.uint64(what << 24)
    counter[:, 2], counter[:, 3] = step & 0xFFFFFFFF, step >> 32
    words = philox(counter, (seed & 0xFFFFFFFF, seed >> 32))
    out = np.empty((len(groups), 8), np.int64)
    out[:, 0::2], out[:, 1::2] = words & np.uint64(0xFFFF), words >> np.uint64(16)
    return out


def blocks_of(k):
    return -(-k // BLOCK)


def quantized(x, along="rows", seed=None, step=0):
    """(numbers 0 .. 15 [rows, k], scale bytes [blocks, rows]) of x, turned over along columns."""
    x = np.asarray(x, np.float64)
    x = x if along == "rows" else x.T
    rows, k = x.shape
    blocks = blocks_of(k)
    wide = np.zeros((rows, blocks * BLOCK))
    wide[:, :k] = x
    wide = wide.reshape(rows, blocks, BLOCK)
    with np.errstate(all="ignore"):
        largest = np.abs(wide).max(2)
        broken = ~np.isfinite(wide).all(2)
        largest = np.where(broken, 0, largest)
        power = np.full(largest.shape, -127)
        for e in range(-127, 127):
            over = largest >= 7 * 2.0 ** e if seed is None else largest > 6 * 2.0 ** e
            power = np.where(over, e + 1, power)
        t = np.abs(np.where(broken[:, :, None], 0, wide)) / (2.0 ** power)[:, :, None]
        at = np.clip(np.searchsorted(LEVELS, t, side="right") - 1, 0, 6)
        fraction = (t - LEVELS[at]) / (LEVELS[at + 1] - LEVELS[at])
        if seed is None:
            up = (fraction > 0.5) | ((fraction == 0.5) & (at % 2 == 1))
        else:
            u = draws(np.arange(rows * blocks * 4), FOR_ROWS if along == "rows" else FOR_COLUMNS, seed, step)
            up = u.reshape(rows, blocks, BLOCK) + 0.5 < 65536 * fraction
    q = (at + up) | (np.signbit(wide) * 8)
    q = np.where(broken[:, :, None], 0, q).reshape(rows, -1)[:, :k]
    return q.astype(np.uint8), np.where(broken, 255, power + 127).astype(np.uint8).T


def packed(q):
    """Two numbers a byte, the even one in the lower half."""
    rows, k = q.shape
    wide = np.zeros((rows, (k + 1) // 2 * 2), np.uint8)
    wide[:, :k] = q
    return wide[:, 0::2] | wide[:, 1::2] << 4


def unpacked(b, k):
    out = np.empty((b.shape[0], 2 * b.shape[1]), np.uint8)
    out[:, 0::2], out[:, 1::2] = b & 15, b >> 4
    return out[:, :k]


def values(q, scale):
    """Binary64 values of numbers [rows, k] with scales [blocks, rows]."""
    factor = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return VALUES[q] * np.repeat(factor.T, BLOCK, 1)[:, :q.shape[1]]


def kept(rows, cols, p, seed, step):
    """Dropout's mask, and the factor of what is kept."""
    below = int(np.rint(p * 65536))
    u = draws(np.arange(-(-rows * cols // 8)), FOR_DROPOUT, seed, step).reshape(-1)[:rows * cols].reshape(rows, cols)
    return u >= below, 65536 / (65536 - below) if below < 65536 else 0.0
