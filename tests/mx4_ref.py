"""Plain definition of microscaled 4-bit numbers in 64 bits (not collected by pytest)."""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
ORDER = [0, 2, 4, 6, 1, 3, 5, 7]


def words(rows, cols, seed, stream):
    """The Philox4x32-10 word of each element: word i % 4 of block i / 4."""
    n, u = rows * cols, np.uint64
    low, half = u(0xFFFFFFFF), u(32)
    at = np.arange((n + 3) // 4, dtype=u)
    c = [at & low, at >> half, np.full_like(at, stream & 0xFFFFFFFF), np.full_like(at, stream >> 32)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p, q = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(q >> half) ^ c[1] ^ u(k[0]), q & low, (p >> half) ^ c[3] ^ u(k[1]), p & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, 1).reshape(-1)[:n].reshape(rows, cols)


def encode(x, word=None):
    """(codes [rows, cols], scales [rows, blocks]) of x, blocks of 32 along its rows; word: random words, for stochastic rounding."""
    rows, cols = x.shape
    blocks = -(-cols // 32)
    codes, scales = np.zeros((rows, blocks * 32), int), np.zeros((rows, blocks), int)
    y = np.zeros((rows, blocks * 32))
    y[:, :cols] = x
    r = np.zeros((rows, blocks * 32), np.uint64)
    if word is not None:
        r[:, :cols] = word
    for b in range(blocks):
        part = y[:, 32 * b:32 * b + 32]
        top = np.abs(part).max(1)
        finite = np.isfinite(top)
        s = np.zeros(rows, int)
        for _ in range(256):                                    # the smallest scale that covers the block
            s += finite & (top > 6 * 2.0 ** (s - 127.0))
        scales[:, b] = np.where(finite, s, 255)
        m = np.where(finite[:, None], np.abs(part), 0) / 2.0 ** (s - 127.0)[:, None]
        below = np.searchsorted(GRID, m, side="right") - 1      # GRID[below] <= m
        above = np.minimum(below + 1, 7)
        gap = np.where(above > below, GRID[above] - GRID[below], 1)
        share = (m - GRID[below]) / gap
        if word is None:
            up = (share > 0.5) | ((share == 0.5) & (below % 2 == 1))
        else:
            up = (r[:, 32 * b:32 * b + 32] >> np.uint64(10)) < np.floor(share * 2.0 ** 22).astype(np.uint64)
        codes[:, 32 * b:32 * b + 32] = np.where(up, above, below) + 8 * np.signbit(part)
    return codes[:, :cols], scales


def values(codes, scales):
    unit = np.where(scales == 255, np.nan, 2.0 ** (scales - 127.0))
    return np.where(codes >= 8, -1, 1) * GRID[codes % 8] * np.repeat(unit, 32, 1)[:, :codes.shape[1]]


def unpack(data, scales, cols):
    """(codes, scales) of the layout, with all of the last panel's columns."""
    panels, rows, _ = data.shape
    codes = np.stack([data & 15, data >> 4], -1).reshape(panels, rows, 256)
    s = np.empty_like(scales)
    s[:, :, ORDER] = scales
    return codes.transpose(1, 0, 2).reshape(rows, -1).astype(int), s.transpose(1, 0, 2).reshape(rows, -1).astype(int)
