"""CPU oracle of the calls that learn the head from tokens and serve it in integers (TEST
INFRASTRUCTURE ONLY): cross entropy, gradient norm and clipping, the integer layout and
product, in numpy at 64 bits from their definitions."""
import numpy as np


def cross_entropy(x, w, targets, weight):
    """(loss, lse, dx, dw, dz) of hidden states x [rows x dim] under w [vocab x dim]."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    z = x @ w.T
    top = z.max(1)
    lse = top + np.log(np.exp(z - top[:, None]).sum(1))
    some = (targets >= 0) & (targets < w.shape[0])
    at = np.where(some, targets, 0)
    rows = np.arange(len(x))
    loss = np.where(some, lse - z[rows, at], 0.0)
    g = np.where(some, weight, 0.0)
    dz = np.exp(z - lse[:, None])
    dz[rows, at] -= 1.0
    dz = np.where(g[:, None] == 0, 0.0, dz * g[:, None])
    xs = np.where(g[:, None] == 0, 0.0, x)
    return loss, lse, dz @ w, dz.T @ xs, dz


def grad_norm(tensors):
    return np.sqrt(sum((np.asarray(t, np.float64) ** 2).sum() for t in tensors))


def clip_factor(norm, max_norm):
    """What gradients are multiplied by, as the library rounds it: a float32 quotient."""
    norm = np.float32(norm)
    return np.float32(max_norm) / norm if np.isfinite(norm) and norm > np.float32(max_norm) else np.float32(1)


def integer_layout(x):
    """(codes [rows x P], scales [rows]) of x [rows x dim]; the roundings to float32 are the
    definition's."""
    x = np.asarray(x, np.float32)
    rows, dim = x.shape
    codes = np.zeros((rows, -(-dim // 128) * 128), np.int8)
    scales = np.zeros(rows, np.float32)
    for r in range(rows):
        finite = np.abs(x[r][np.isfinite(x[r])])
        m = finite.max() if finite.size else np.float32(0)
        if m > np.float32(2.0) ** -100:
            with np.errstate(over="ignore", invalid="ignore"):
                y = x[r] * (np.float32(127) * (np.float32(1) / m))
            codes[r, :dim] = np.where(np.isnan(y), 0, np.clip(np.rint(y), -127, 127)).astype(np.int8)
            scales[r] = m / np.float32(127)
        if np.isnan(x[r]).any():
            scales[r] = np.nan
    return codes, scales


def integer_product(a, a_scales, w, w_scales):
    """(sums, results before the last rounding) of two layouts."""
    sums = a.astype(np.int64) @ w.astype(np.int64).T
    return sums, sums * a_scales.astype(np.float64)[:, None] * w_scales.astype(np.float64)
