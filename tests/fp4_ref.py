"""MXFP4 in float64, written from the format: the quantiser, the values of codes, and the library's layouts by
their definitions (one element at a time, no reshaping shared with the kernels)."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
TILE_BYTES, QUAD_BYTES = 4352, 1088


def quantise(x):
    """x [R][C] -> (codes [R][C] 0..15, scale bytes [R][C / 32])."""
    x = np.asarray(x, np.float64)
    R, C = x.shape
    b = x.reshape(R, C // 32, 32)
    bad = ~np.isfinite(b).all(axis=2)
    b = np.where(bad[:, :, None], 0.0, b)
    m = np.abs(b).max(axis=2)
    _, ex = np.frexp(m)  # m = mant 2^ex, mant in [0.5, 1): floor(log2 m) = ex - 1
    e = np.where(m > 0, np.maximum(ex - 3, -127), 0)
    a = np.abs(b) * np.exp2(-e.astype(np.float64))[:, :, None]
    # Nearest level; of two at one distance the even code; past the last level, the last.
    hi = np.clip(np.searchsorted(LEVELS, a, side="left"), 1, 7)
    lo = hi - 1
    d_hi, d_lo = LEVELS[hi] - a, a - LEVELS[lo]
    code = np.where((d_hi < d_lo) | ((d_hi == d_lo) & (hi % 2 == 0)), hi, lo)
    code = code | np.where(np.signbit(b), 8, 0)
    code = np.where(bad[:, :, None], 0, code)
    return code.reshape(R, C).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def values(code, scale):
    """float64 values of codes [R][C] under scale bytes [R][C / 32]."""
    v = LEVELS[code & 7] * np.where(code & 8, -1.0, 1.0)
    s = np.where(scale == 255, np.nan, np.exp2(scale.astype(np.float64) - 127))
    return v * np.repeat(s, 32, axis=1)


def rowmajor(code, scale):
    return (code[:, 0::2] | (code[:, 1::2] << 4)).astype(np.uint8), scale


def frag16(code, scale):
    """Quad fragments of 16 rows x 128 columns: byte positions from the layout's definition."""
    R, C = code.shape
    by, _ = rowmajor(code, scale)
    out = np.zeros((R // 16, C // 128, QUAD_BYTES), np.uint8)
    for rb in range(R // 16):
        for kq in range(C // 128):
            for lane in range(64):
                row, g = 16 * rb + lane % 16, lane // 16
                for b in range(4):
                    c = (128 * kq + 32 * b + 8 * g) // 2
                    out[rb, kq, 16 * lane + 4 * b: 16 * lane + 4 * b + 4] = by[row, c: c + 4]
            for i in range(16):
                out[rb, kq, 1024 + 4 * i: 1024 + 4 * i + 4] = scale[16 * rb + i, 4 * kq: 4 * kq + 4]
    return out.reshape(-1)


def tile32(code, scale):
    """Tiles of 32 rows x 256 columns; code 0 and scale 127 past the matrix."""
    R, C = code.shape
    by, _ = rowmajor(code, scale)
    rbs, cbs = -(-R // 32), -(-C // 256)
    out = np.zeros((rbs, cbs, TILE_BYTES), np.uint8)
    out[:, :, 4096:] = 127
    for row in range(R):
        rb, r = divmod(row, 32)
        for blk in range(C // 32):
            cb, in_tile = divmod(blk, 8)
            j, h = divmod(in_tile, 2)
            lane = 32 * h + r
            out[rb, cb, 1024 * j + 16 * lane: 1024 * j + 16 * lane + 16] = by[row, 16 * blk: 16 * blk + 16]
            out[rb, cb, 4096 + 4 * lane + j] = scale[row, blk]
    return out.reshape(-1)


def awkward(rng, R, C):
    """Rows of every kind of block: normal ones over many magnitudes, zeros (both signs), values on and next to
    the midpoints, saturating ones, subnormals, the largest finite values, infinities and NaN."""
    x = rng.standard_normal((R, C)) * np.exp2(rng.integers(-20, 20, (R, C // 32))).repeat(32, axis=1)
    b = x.reshape(R, C // 32, 32)
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 6.0, 4.0, 0.5, 1.0, 2.0, 3.0, 1.5, 0.0])
    kinds = rng.integers(0, 10, (R, C // 32))
    for r in range(R):
        for k in range(C // 32):
            kind, v = kinds[r, k], b[r, k]
            if kind == 0:
                v[:] = np.where(rng.random(32) < 0.5, 0.0, -0.0)
            elif kind in (1, 2):
                v[:] = np.concatenate([ties, -ties]) * 2.0 ** int(rng.integers(-30, 30))
                if kind == 2:
                    v *= 1 + rng.choice([-1, 0, 1], 32) * 2.0 ** -7
            elif kind == 3:
                v[:] = rng.standard_normal(32) * 2.0 ** -130
            elif kind == 4:
                v[:] = rng.standard_normal(32) * 2.0 ** 124
            elif kind == 5 and rng.random() < 0.5:
                v[int(rng.integers(32))] = rng.choice([np.inf, -np.inf, np.nan])
    return x
