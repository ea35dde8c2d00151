"""Microscaled 4-bit floating point in plain numpy, 64 bits: the definition, element by element (test infrastructure)."""
import numpy as np

VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def padded(cols):
    return -(-cols // 128) * 128


def quantize(x):
    """(codes rows x padded, scales rows x padded / 32) of the rows of x (float64 holding the input type's values)."""
    rows, cols = x.shape
    b = np.zeros((rows, padded(cols)))
    b[:, :cols] = x
    b = b.reshape(rows, -1, 32)
    most = np.abs(b).max(-1)
    with np.errstate(invalid="ignore"):
        bad = ~np.isfinite(b).all(-1)
    _, e = np.frexp(np.where(bad, 1.0, most))
    shared = np.where(most == 0, -127, np.maximum(e - 3, -127))
    with np.errstate(invalid="ignore"):
        v = np.abs(b) / np.exp2(shared.astype(float))[..., None]
    # the nearest value; of two at the same distance the one with the even mantissa (the even code)
    v = np.where(bad[..., None], 0.0, v)
    lo = np.clip(np.searchsorted(VALUES, v, side="right") - 1, 0, 7)
    hi = np.minimum(lo + 1, 7)
    down, up = v - VALUES[lo], VALUES[hi] - v
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = code + 8 * np.signbit(b)
    code = np.where(bad[..., None], 0, code)
    return code.reshape(rows, -1).astype(np.uint8), np.where(bad, 255, shared + 127).astype(np.uint8)


def pack(codes):
    return codes[:, 0::2] | codes[:, 1::2] << 4


def values(codes, scales):
    """What codes (rows x padded) and scales (rows x padded / 32) stand for, float64."""
    v = np.where(codes & 8, -1.0, 1.0) * VALUES[codes & 7]
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(float) - 127))
    return (v.reshape(codes.shape[0], -1, 32) * s[..., None]).reshape(codes.shape)


def random_codes(rng, rows, cols, low=126, high=128):
    """Random elements and scales of a rows x cols matrix, its padding zero."""
    codes = rng.integers(0, 16, (rows, padded(cols))).astype(np.uint8)
    codes[:, cols:] = 0
    scales = rng.integers(low, high, (rows, padded(cols) // 32)).astype(np.uint8)
    scales[:, -(-cols // 32):] = 0
    return codes, scales
