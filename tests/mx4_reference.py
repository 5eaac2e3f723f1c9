"""MX4 by its definition, in 64 bits, for the tests (numpy; no code of the library)."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize(x):
    """x [rows][cols] -> (codes uint8 [rows][nb*16], scales uint8 [rows][nb])."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    nb = -(-cols // 32)
    v = np.zeros((rows, nb * 32))
    v[:, :cols] = x
    v = v.reshape(rows, nb, 32)
    a = np.abs(v)
    with np.errstate(all="ignore"):
        amax = a.max(2)
        bad = ~np.isfinite(amax)
        _, e = np.frexp(np.where(bad, 1.0, amax))          # amax = f * 2^e, f in [.5, 1)
        byte = np.clip(e - 1 - 2 + 127, 0, 254)
        byte = np.where(amax == 0, 0, byte)
        q = a / np.ldexp(1.0, byte - 127)[:, :, None]
        below = (LEVELS[None, None, None, :] <= q[..., None]).sum(-1) - 1   # largest level not above q
        below = np.clip(below, 0, 7)
        up = np.minimum(below + 1, 7)
        d_lo, d_up = q - LEVELS[below], LEVELS[up] - q
        take_up = (d_up < d_lo) | ((d_up == d_lo) & (up % 2 == 0))
    code = np.where(take_up & (below < 7), up, below) + 8 * np.signbit(v)
    code = np.where(bad[:, :, None], 0, code).astype(np.uint8)
    byte = np.where(bad, 255, byte).astype(np.uint8)
    code = code.reshape(rows, nb * 32)
    return (code[:, 0::2] | (code[:, 1::2] << 4)).astype(np.uint8), byte


def values(codes, scales):
    """fp64 [..., nb*32] of codes [..., nb*16] and scales [..., nb]."""
    codes, scales = np.asarray(codes), np.asarray(scales)
    half = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    v = np.where(half & 8, -1.0, 1.0) * LEVELS[half & 7]
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(int) - 127))
    return v * np.repeat(s, 32, -1)
