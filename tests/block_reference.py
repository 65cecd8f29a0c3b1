"""Plain 64-bit forms of the training-side operators (numpy, from the formulas): block quantisation to 8-bit floating point, the
product of two such matrices, distillation from lists.  They take and give numpy arrays; 8-bit codes are uint8."""
import numpy as np

PAD_ID = 0xFFFFFFFF
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}


def _decode(fmt):
    """The 256 codes' values."""
    exp_bits, man_bits, bias = (4, 3, 7) if fmt == "e4m3" else (5, 2, 15)
    out = np.empty(256)
    for c in range(256):
        s, e, m = -1.0 if c & 0x80 else 1.0, (c >> man_bits) & ((1 << exp_bits) - 1), c & ((1 << man_bits) - 1)
        if fmt == "e4m3" and (c & 0x7F) == 0x7F:
            v = np.nan
        elif fmt == "e5m2" and e == 31:
            v = np.inf if m == 0 else np.nan
        elif e == 0:
            v = m * 2.0 ** (1 - bias - man_bits)
        else:
            v = (1 + m / (1 << man_bits)) * 2.0 ** (e - bias)
        out[c] = s * v
    return out


DECODE = {f: _decode(f) for f in LARGEST}


def round_to_format(x, fmt):
    """Values -> the format's nearest values, ties to the even code.  Finite inputs are within the format's range here."""
    grid = DECODE[fmt][:0x7F if fmt == "e4m3" else 0x7C]          # ascending, non-negative, finite
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    hi = np.clip(np.searchsorted(grid, a), 0, len(grid) - 1)
    lo = np.maximum(hi - 1, 0)
    below, above = a - grid[lo], grid[hi] - a
    at = np.where(above < below, hi, np.where(below < above, lo, np.where(hi % 2 == 0, hi, lo)))
    v = np.copysign(grid[at], x)
    v = np.where(np.isnan(x), np.nan, v)
    return np.where(np.isinf(x), np.nan if fmt == "e4m3" else x, v)


def quantize(x, fmt, block_rows=1, pow2=False):
    """x [rows][cols] (any float type) -> (values the codes stand for without their scales, scales f32)."""
    x = np.asarray(x, dtype=np.float32)
    rows, cols = x.shape
    R, C = -(-rows // block_rows), -(-cols // 128)
    scales = np.empty((R, C), dtype=np.float32)
    out = np.empty((rows, cols))
    one = np.float32(1.0)
    for r in range(R):
        for c in range(C):
            t = x[r * block_rows:(r + 1) * block_rows, c * 128:(c + 1) * 128]
            a = np.abs(t[np.isfinite(t)]).max(initial=np.float32(0.0))
            a = max(np.float32(a), np.float32(2.0 ** -100))
            if pow2:
                f, e = np.frexp(np.float64(a) / LARGEST[fmt])      # exact quotient's exponent: the divisor is 7 * 2^k
                s = np.float32(2.0 ** (e - 1 if float(a) == LARGEST[fmt] * 2.0 ** int(e - 1) else e))
            else:
                s = np.float32(a) / np.float32(LARGEST[fmt])
            scales[r, c] = s
            with np.errstate(invalid="ignore"):
                out[r * block_rows:(r + 1) * block_rows, c * 128:(c + 1) * 128] = round_to_format((t * (one / s)).astype(np.float64), fmt)
    return out, scales


def spread(scales, rows, cols, block_rows):
    s = np.repeat(scales.astype(np.float64), 128, axis=1)[:, :cols]
    return np.repeat(s, block_rows, axis=0)[:rows]


def product(a, a_scales, b, b_scales, b_block_rows):
    """(out, sum of the products' magnitudes) of two matrices of code values."""
    x = a * spread(a_scales, a.shape[0], a.shape[1], 1)
    y = b * spread(b_scales, b.shape[0], b.shape[1], b_block_rows)
    return x @ y.T, np.abs(x) @ np.abs(y).T


def distill(logits, ids, values, scale, teacher_scale, teacher_lse=None, grad_loss=None):
    """(loss [R], gradient [R][V], what the gradient's terms add up to in magnitude [R][V], largest argument of an exponential [R])."""
    R, V = logits.shape
    loss, grad, size, reach = np.zeros(R), np.zeros((R, V)), np.zeros((R, V)), np.zeros(R)
    scale, teacher_scale = float(np.float32(scale)), float(np.float32(teacher_scale))
    for r in range(R):
        g = 1.0 if grad_loss is None else float(grad_loss[r])
        p = np.zeros(V)
        with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
            z = teacher_scale * values[r].astype(np.float64)
            entry = (ids[r].astype(np.int64) < V) & ~(z == -np.inf)
            s = scale * logits[r].astype(np.float64)
            if not entry.any() or (s == -np.inf).all():
                continue
            top = np.max(s)
            e = np.exp(s - top)
            log_q = s - top - np.log(e.sum())
            zt = np.max(z[entry])
            lse = zt + np.log(np.exp(z[entry] - zt).sum()) if teacher_lse is None else float(teacher_lse[r])
            np.add.at(p, ids[r][entry].astype(np.int64), np.exp(z[entry] - lse))
            on = np.zeros(V, dtype=bool)
            on[ids[r][entry].astype(np.int64)] = True
            q = np.exp(log_q)
            at = on & ~(p == 0)
            loss[r] = (p[at] * (np.log(p[at]) - log_q[at])).sum()
            c, ratio = 1.0, 0.0
            if teacher_lse is not None and not on.all():
                p_r, q_r = max(0.0, 1.0 - p.sum()), q[~on].sum()
                if p_r > 0:
                    loss[r] += p_r * (np.log(p_r) - np.log(q_r))
                ratio = p_r / q_r if q_r > 0 else 0.0
                c = 1.0 - ratio
            grad[r] = g * scale * np.where(on, q - p, c * q)
            size[r] = np.abs(g) * scale * np.where(on, q + p, (1.0 + ratio) * q)
            near = s[on & (s > -np.inf)]
            reach[r] = max(np.abs(near - top).max(initial=0.0), np.abs(z[entry] - lse).max(), abs(np.log(e.sum())), 1.0)
    return loss, grad, size, reach
