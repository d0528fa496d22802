"""Plain implementation of the microscaled 4-bit form in float64 (numpy), for the tests: grid search instead of bit tricks, and no code or
table of the library."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def blocks(cols):
    return -(-cols // 32)


def pitch(cols):
    return -(-blocks(cols) // 4) * 4


def fmix32(h):
    h = np.asarray(h, np.uint32).copy()
    h ^= h >> np.uint32(16)
    h *= np.uint32(0x85EBCA6B)
    h ^= h >> np.uint32(13)
    h *= np.uint32(0xC2B2AE35)
    return h ^ (h >> np.uint32(16))


def draws(first, count, seed):
    """The 16-bit draws of elements first .. first + count (first even)."""
    pair = np.arange(first // 2, (first + count + 1) // 2, dtype=np.uint64)
    low = np.uint64(0xFFFFFFFF)
    key = fmix32((np.uint64(seed) + np.uint64(0x9E3779B9) * (pair >> np.uint64(32))) & low)
    h = fmix32((pair & low).astype(np.uint32) ^ key)
    return np.stack([h & np.uint32(0xFFFF), h >> np.uint32(16)], 1).reshape(-1)[:count]


def quantize(x, stochastic=False, seed=0, first=0):
    """x [rows, cols], any float type -> codes uint8 [rows, 16 * blocks], scales uint8 [rows, blocks].  first: number of the first element."""
    x = np.asarray(x).astype(np.float64)
    rows, cols = x.shape
    nb = blocks(cols)
    full = np.zeros((rows, nb * 32))
    full[:, :cols] = x
    full = full.reshape(rows, nb, 32)
    with np.errstate(all="ignore"):
        peak = np.abs(full).max(2)
        bad = ~np.isfinite(full).all(2)
        peak = np.where(bad | (peak == 0), 1.0, peak)
        e = np.where(np.abs(full).max(2) == 0, -300, np.frexp(peak)[1] - 1 - 2)
        if stochastic:
            e = np.where(peak > 6 * np.ldexp(1.0, e), e + 1, e)
        e = np.clip(e, -127, 125)
        a = np.where(bad[..., None], 0.0, np.abs(full)) / np.ldexp(1.0, e)[..., None]
    if stochastic:
        lower = (np.searchsorted(GRID, a, side="right") - 1).astype(np.int64)
        upper = np.minimum(lower + 1, 7)
        gap = np.where(upper > lower, GRID[upper] - GRID[lower], 1.0)
        u = draws(first, rows * nb * 32, seed).reshape(a.shape).astype(np.float64)
        code = np.where((u + 0.5) / 65536 < (a - GRID[lower]) / gap, upper, lower)
    else:
        code = np.zeros(a.shape, np.int64)
        best = np.abs(a - GRID[0])
        for c in range(1, 8):
            d = np.abs(a - GRID[c])
            take = (d < best) | ((d == best) & (c % 2 == 0))
            code, best = np.where(take, c, code), np.where(take, d, best)
    code = np.where(bad[..., None], 0, code + 8 * np.signbit(full)).astype(np.uint8)
    codes = (code[..., 0::2] | (code[..., 1::2] << 4)).reshape(rows, nb * 16)
    return codes, np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes, scales, cols):
    """float64 [rows, cols]."""
    rows, nb = scales.shape[0], blocks(cols)
    b = codes[:, :nb * 16]
    code = np.stack([b & 15, b >> 4], 2).reshape(rows, nb, 32)
    s = scales[:, :nb].astype(np.int64)
    with np.errstate(invalid="ignore"):
        v = np.where(code >= 8, -1.0, 1.0) * GRID[code & 7] * np.where(s == 255, np.nan, np.ldexp(1.0, s - 127))[..., None]
    return v.reshape(rows, nb * 32)[:, :cols]


def place(codes, scales, cols, extra=0, fill=0xFF):
    """The same with the least pitch (and `extra` blocks, a multiple of 4), everything past a row's blocks filled with `fill`."""
    rows, nb = scales.shape[0], blocks(cols)
    p = pitch(cols) + extra
    c = np.full((rows, 16 * p), fill, np.uint8)
    s = np.full((rows, p), fill, np.uint8)
    c[:, :16 * nb] = codes[:, :16 * nb]
    s[:, :nb] = scales[:, :nb]
    return c, s


def random_matrix(rng, rows, cols, low=125, high=130):
    """Codes and scale bytes (from low to below high) of a random matrix, codes past a row's end 0."""
    nb = blocks(cols)
    code = rng.integers(0, 16, (rows, nb * 32), dtype=np.uint8)
    code[:, cols:] = 0
    return code[:, 0::2] | (code[:, 1::2] << 4), rng.integers(low, high, (rows, nb), dtype=np.uint8)
