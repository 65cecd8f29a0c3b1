"""Plain 64-bit forms (numpy, from the formulas) of microscaled 4-bit floating point and of clipping by the global norm.  Codes are kept one to a byte."""
import numpy as np

VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])
MIDDLES = (VALUES[:7] + VALUES[1:8]) / 2                       # between codes k and k + 1


def scale_exponent(a, fit):
    """Exponent of the scale of a block whose largest magnitude is a, a finite number."""
    a = max(float(a), 2.0 ** -100)
    e = int(np.frexp(a)[1]) - 1 - 2                            # floor(log2 a) - 2
    if fit and a > 6 * 2.0 ** e:
        e += 1
    return min(e, 125)


def nearest(x):
    """Codes of the values nearest to x, ties to even, saturating; the sign of a zero stays."""
    a = np.abs(x)
    code = np.zeros(a.shape, dtype=np.int64)
    for k, m in enumerate(MIDDLES):
        code += (a > m) | ((a == m) & (k % 2 == 1))
    return (code | (np.signbit(x).astype(np.int64) << 3)).astype(np.uint8)


def quantize(x, block_rows=1, fit=False):
    """x [rows][cols] -> (codes [rows][cols], scale bytes [rows][blocks])."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    blocks = -(-cols // 32)
    codes, scales = np.zeros((rows, cols), dtype=np.uint8), np.zeros((rows, blocks), dtype=np.uint8)
    for r in range(0, rows, block_rows):
        for b in range(blocks):
            at = np.s_[r:r + block_rows, 32 * b:32 * b + 32]
            t = x[at]
            if not np.isfinite(t).all():
                scales[r:r + block_rows, b] = 255
                continue
            e = scale_exponent(np.abs(t).max(), fit)
            scales[r:r + block_rows, b] = e + 127
            codes[at] = nearest(t * 2.0 ** -e)
    return codes, scales


def pack(codes):
    codes = np.concatenate([codes, np.zeros((codes.shape[0], codes.shape[1] % 2), dtype=np.uint8)], axis=1)
    return codes[:, ::2] | codes[:, 1::2] << 4


def unpack(packed, cols):
    return np.stack([packed & 15, packed >> 4], axis=2).reshape(packed.shape[0], -1)[:, :cols]


def values(codes, scales):
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return VALUES[codes] * np.repeat(s, 32, axis=1)[:, :codes.shape[1]]


def norm(grads, scale=1.0):
    return float(np.float64(np.float32(scale)) * np.sqrt(sum(float((np.asarray(g, dtype=np.float64) ** 2).sum()) for g in grads)))


def factor(norm, max_norm, scale=1.0):
    """From the norm as it is held, in 32 bits."""
    norm, max_norm, scale = np.float32(norm), np.float32(max_norm), np.float32(scale)
    with np.errstate(all="ignore"):
        return np.float64(scale) if norm <= max_norm else np.float64(scale) * (np.float64(max_norm) / np.float64(norm))
