"""Block-scaled values in 64 bits, for tests: the definition, written apart from
the library's kernels."""
import numpy as np

TOP = {"fp4": 6.0, "fp8": 448.0}
DIGITS = {"fp4": 2, "fp8": 4}         # significant binary digits
LEAST = {"fp4": 1.0, "fp8": 2.0 ** -6}  # smallest normal value


def blocks(x):
    rows, cols = x.shape
    return np.pad(x, ((0, 0), (0, -cols % 32))).reshape(rows, -1, 32)


def scale_exp(x, fmt):
    """e of every block's scale 2^e: the least e >= -127 with max |x| <= F 2^e."""
    big = np.abs(blocks(np.asarray(x, np.float64))).max(2)
    m, p = np.frexp(big)               # big = m 2^p, m in [1/2, 1)
    fm, fp = np.frexp(TOP[fmt])
    e = p - fp + (m > fm)
    return np.where(big > 0, np.maximum(e, -127), -127)


def step(u, fmt):
    """Distance of neighbouring values of the format around u."""
    a = np.maximum(np.abs(u), LEAST[fmt])
    return np.exp2(np.floor(np.log2(a)) - (DIGITS[fmt] - 1))


def held(x, fmt):
    """The values that x [rows, cols] goes to; NaN in blocks that are not finite."""
    x = np.asarray(x, np.float64)
    b = blocks(x)
    bad = ~np.isfinite(b).all(2)
    b = np.where(bad[:, :, None], 0.0, b)
    e = scale_exp(b.reshape(len(x), -1), fmt)
    u = b * np.exp2(-e.astype(np.float64))[:, :, None]
    s = step(u, fmt)
    v = np.round(u / s) * s * np.exp2(e.astype(np.float64))[:, :, None]  # halves to even
    v = np.where(bad[:, :, None], np.nan, v)
    return v.reshape(len(x), -1)[:, : x.shape[1]]
