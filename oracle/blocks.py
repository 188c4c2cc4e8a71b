"""Operators of gated recurrent blocks in fp64 numpy, from their formulas: root-mean-square norm with the residual's addition,
8-bit numbers in blocks, products of them, the gated linear recurrence, and AdamW.  Whole tensors; what is split over workers
is cut by the caller."""
import numpy as np

BLOCK = 128


# ---- root-mean-square norm ------------------------------------------------

def norm_forward(x, r, g, eps):
    """(s, y, rstd) of rows: s = x + r, y = s / sqrt(mean(s^2) + eps) * g."""
    s = x if r is None else x + r
    rstd = 1.0 / np.sqrt((s * s).mean(1) + eps)
    return s, s * rstd[:, None] * g, rstd


def norm_adjoint(s, g, rstd, dy, dsum):
    """(gradient of x and r, gradient of g)."""
    n = s * rstd[:, None]
    e = dy * g
    dx = rstd[:, None] * (e - n * (e * n).mean(1, keepdims=True))
    return (dx if dsum is None else dx + dsum), (dy * n).sum(0)


# ---- 8-bit numbers --------------------------------------------------------

def e4m3_values():
    """The value of every code; 0x7f and 0xff are NaN."""
    code = np.arange(256)
    exponent, mantissa = (code >> 3) & 15, code & 7
    size = np.where(exponent > 0, (8 + mantissa) * 2.0 ** (exponent - 10.0), mantissa * 2.0 ** -9)
    size[[0x7F, 0xFF]] = np.nan
    return np.where(code & 0x80, -size, size)


def scale_byte(block):
    """Biased exponent of the smallest power of two, at least 2^-126, that 448 times of is no less than any magnitude."""
    sizes = np.abs(block[~np.isnan(block)])
    top = sizes.max() if sizes.size else 0.0
    if np.isinf(top):
        return 255
    byte = 1
    while top > 448.0 * 2.0 ** (byte - 127):
        byte += 1
    return byte


def round_e4m3(y):
    """Codes of magnitudes up to 448, ties to the even code; NaN stays NaN."""
    values = e4m3_values()[:0x7F]
    size = np.abs(y)
    below = np.clip(np.searchsorted(values, size, side="right") - 1, 0, 0x7E)
    above = np.minimum(below + 1, 0x7E)
    lo, hi = size - values[below], values[above] - size
    up = (above > below) & ((hi < lo) | ((hi == lo) & (below % 2 == 1)))
    code = np.where(up, above, below).astype(np.uint8)
    code = np.where(np.isnan(y), 0x7F, code).astype(np.uint8)
    return code | np.where(np.signbit(y), 0x80, 0).astype(np.uint8)


def quantise(x, rows, cols):
    """Codes of a matrix, one scale byte for each rows x cols of it (the last ones cut): (codes, bytes)."""
    R, K = x.shape
    codes = np.zeros((R, K), np.uint8)
    scales = np.zeros((-(-R // rows), -(-K // cols)), np.uint8)
    for i in range(scales.shape[0]):
        for k in range(scales.shape[1]):
            at = (slice(i * rows, (i + 1) * rows), slice(k * cols, (k + 1) * cols))
            byte = scale_byte(x[at])
            scales[i, k] = byte
            if byte == 255:
                with np.errstate(invalid="ignore"):
                    codes[at] = round_e4m3(x[at] * 0.0)  # (it stands for NaN throughout)
            else:
                codes[at] = round_e4m3(x[at] * 2.0 ** (127 - byte))
    return codes, scales


def values_of(codes, scales, rows, cols):
    """What codes and scale bytes stand for."""
    scale = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    scale = scale.repeat(rows, 0)[:codes.shape[0]].repeat(cols, 1)[:, :codes.shape[1]]
    return e4m3_values()[codes] * scale


# ---- gated linear recurrence ----------------------------------------------

def gates(a, x, sigmoid):
    """(factor, input) of every step."""
    if not sigmoid:
        return a, x
    with np.errstate(over="ignore"):
        f = 1.0 / (1.0 + np.exp(-a))
    return f, (1.0 - f) * x


def scan_forward(a, x, h0, lengths, sigmoid):
    """(h of all steps, last states); a, x: [n, steps, channels]."""
    f, u = gates(a, x, sigmoid)
    h, state = np.zeros_like(u), h0.copy()
    for t in range(a.shape[1]):
        live = lengths > t
        state[live] = f[live, t] * state[live] + u[live, t]
        h[live, t] = state[live]
    return h, state


def scan_adjoint(a, x, h, h0, lengths, dh, dhT, sigmoid):
    """(gradients of a, of x, of h0) for gradients dh of all states and dhT of the last."""
    f, _ = gates(a, x, sigmoid)
    da, dx, back = np.zeros_like(f), np.zeros_like(f), dhT.copy()
    for t in range(a.shape[1] - 1, -1, -1):
        live = lengths > t
        d = back[live] + dh[live, t]
        before = h[live, t - 1] if t else h0[live]
        if sigmoid:
            da[live, t] = d * (before - x[live, t]) * f[live, t] * (1 - f[live, t])
            dx[live, t] = d * (1 - f[live, t])
        else:
            da[live, t], dx[live, t] = d * before, d
        back[live] = f[live, t] * d
    return da, dx, back


# ---- AdamW ----------------------------------------------------------------

def adamw(p, g, m, v, lr, beta1, beta2, eps, weight_decay, step):
    """(p, m, v) after one step."""
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    return p * (1 - lr * weight_decay) - lr * (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps), m, v
