"""The microscaled formats in 64 bits, from the tables of their magnitudes (shared by tests)."""
import numpy as np

TABLE = {"fp4": np.array([0, .5, 1, 1.5, 2, 3, 4, 6]),
         "fp8": np.array([c % 8 * 2.0 ** -9 if c < 8 else (1 + c % 8 / 8) * 2.0 ** (c // 8 - 7) for c in range(127)])}
TOP = {"fp4": 2, "fp8": 8}


def quantize(x, fmt):
    """(codes with sign bit, scale bytes) of the rows of x, padded to 128 columns."""
    t = TABLE[fmt]
    rows, cols = x.shape
    b = np.zeros((rows, -(-cols // 128) * 4, 32))
    b.reshape(rows, b.shape[1] * 32)[:, :cols] = x
    fine = np.isfinite(b).all(2)
    b = np.where(fine[:, :, None], b, 0)
    amax = np.abs(b).max(2)
    e = np.where(amax > 0, np.frexp(amax)[1] - 1 - TOP[fmt], -127).clip(-127, 127).astype(int)
    a = np.ldexp(np.abs(b), -e[:, :, None])
    hi = np.searchsorted(t, a).clip(0, len(t) - 1)           # t[hi] >= a, or the largest
    lo = np.maximum(hi - 1, 0)
    up, down = t[hi] - a, a - t[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)) | (a >= t[-1]), hi, lo)
    code = np.where(a == 0, 0, code)
    sign = np.signbit(b) & fine[:, :, None]
    code = code + sign * (8 if fmt == "fp4" else 128)
    return code.reshape(rows, code.shape[1] * 32).astype(np.uint8), np.where(fine, e + 127, 255).astype(np.uint8)


def unpack(values, fmt):
    v = values.astype(np.uint8)
    if fmt == "fp8":
        return v
    out = np.empty((v.shape[0], v.shape[1] * 2), dtype=np.uint8)
    out[:, 0::2], out[:, 1::2] = v & 15, v >> 4
    return out


def values_of(codes, scales, fmt, cols):
    bit = 8 if fmt == "fp4" else 128
    c = codes.astype(int)
    v = TABLE[fmt][np.minimum(c % bit, len(TABLE[fmt]) - 1)] * np.where(c >= bit, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(int) - 127))
    return (v.reshape(*s.shape, 32) * s[:, :, None]).reshape(v.shape)[:, :cols]


def rounded(x, fmt):
    return values_of(*quantize(x, fmt), fmt, x.shape[1])
