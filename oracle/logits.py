"""CPU oracle of the calls on the head's logits (TEST INFRASTRUCTURE ONLY): the
8-bit layout and product, sampling and distillation, in numpy at 64 bits from
their definitions."""
import numpy as np

BLOCK = 128


# ---- 8-bit layout (OCP e4m3: sign, 4 exponent bits biased by 7, 3 fraction bits) ----

def e4m3_values():
    """The 256 codes' values; 0x7f and 0xff are NaN."""
    c = np.arange(256)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e > 0, (1 + f / 8.0) * 2.0 ** (e - 7.0), f / 8.0 * 2.0 ** -6)
    v[(c & 127) == 127] = np.nan
    return np.where(c >= 128, -v, v)


def e4m3_nearest(x):
    """Codes of the values nearest to x, ties to the even code; beyond 448 saturates."""
    v = e4m3_values()[:127]
    mid = (v[1:] + v[:-1]) / 2
    a = np.minimum(np.abs(x), 448.0)
    lo = np.searchsorted(mid, a, side="left")   # values at a midpoint stay low
    hi = np.searchsorted(mid, a, side="right")
    code = np.where(lo == hi, lo, np.where(lo % 2 == 0, lo, hi))
    code = np.where(np.isnan(x), 127, code) + np.where(np.signbit(x), 128, 0)
    return code.astype(np.uint8)


def fp8_layout(x, block_rows):
    """(codes [rows x P], scales [blocks x Q]) of x [rows x dim] (float)."""
    x = np.asarray(x, np.float64)
    rows, dim = x.shape
    kb, nb = -(-dim // BLOCK), -(-rows // block_rows)
    full = np.zeros((nb * block_rows, kb * BLOCK))
    full[:rows, :dim] = x
    t = full.reshape(nb, block_rows, kb, BLOCK)
    amax = np.where(np.isfinite(t), np.abs(t), 0).max((1, 3))
    e = np.full(amax.shape, -127)
    at = amax > 0
    e[at] = np.ceil(np.log2(amax[at] / 448.0)).astype(int)
    e += amax > 448.0 * 2.0 ** e
    e -= at & (amax <= 448.0 * 2.0 ** (e - 1))
    e = np.maximum(e, -127)
    scales = np.full((nb, -(-kb // 4) * 4), 127, np.uint8)
    scales[:, :kb] = e + 127
    codes = e4m3_nearest(t / 2.0 ** e[:, None, :, None]).reshape(full.shape)
    return codes[:rows], scales


def fp8_values(codes, scales, block_rows):
    """The numbers that a layout stands for."""
    rows, pitch = codes.shape
    f = 2.0 ** (scales[:, :pitch // BLOCK].astype(np.float64) - 127)
    f = np.repeat(np.repeat(f, block_rows, 0)[:rows], BLOCK, 1)
    return e4m3_values()[codes] * f


# ---- sampling ----

def sample(l, T, top_k, top_p, min_p, u):
    """One row.  (token, prob, margin): margin is how near, relative to the sums they
    compare, the nearest of the decisions that the answer rests on was to going
    the other way."""
    l = np.where(np.isnan(l), -np.inf, np.asarray(l, np.float64))
    top = l.max()
    if top == -np.inf:
        return -1, 0.0, 1.0
    if not T > 0:
        return int(np.argmax(l)), 1.0, 1.0
    with np.errstate(invalid="ignore", over="ignore"):
        d = np.where(l == top, 0.0, (l - top) / T)
    w = np.where(l == -np.inf, 0.0, np.rint(2.0 ** 31 * np.exp(d)))
    order = np.lexsort((np.arange(l.size), -w))
    w, same, margin = w[order], l[order], 1.0
    if 0 < top_k < w.size:
        if same[top_k - 1] != same[top_k] and w[top_k - 1] > 0:
            margin = (w[top_k - 1] - w[top_k]) / w[top_k - 1]
        w = np.where(np.arange(w.size) < top_k, w, 0.0)
    if top_p < 1:
        cum = w.cumsum()
        part = max(1.0, np.floor(max(top_p, 0.0) * cum[-1]))
        n = int(np.searchsorted(cum, part))
        margin = min(margin, np.abs(cum - part)[max(0, n - 1):n + 1].min() / cum[-1] if part > 1 else 1.0)
        w = np.where(np.arange(w.size) <= n, w, 0.0)
    if min_p > 0:
        least = np.rint(min(min_p, 1.0) * 2.0 ** 31)
        if least < 2.0 ** 31:
            margin = min(margin, np.abs(w - least).min() / least)
        w = np.where(w >= least, w, 0.0)
    cum = w.cumsum()
    z = cum[-1]
    at = np.floor(min(max(u, 0.0), 1.0) * z) if u == u else 0.0
    at = min(at, z - 1)
    n = int(np.searchsorted(cum, at, side="right"))
    edges = np.concatenate([[0.0], cum])[[n, n + 1]]
    near = [abs(at - edges[0])] if n > 0 else []
    near += [abs(at - edges[1])] if edges[1] < z else []
    margin = min([margin] + [x / z for x in near])
    # Its place among its neighbours: both weights of a comparison are off, so a gap
    # counts as 1 / 1.7 of itself; equal logits stand in the order of their tokens.
    for i in (n - 1, n + 1):
        if 0 <= i < w.size and w[i] > 0 and same[i] != same[n]:
            margin = min(margin, abs(w[i] - w[n]) / w[n] / 1.7)
    return int(order[n]), w[n] / z, margin


# ---- distillation ----

def distill(s, ids, t, tau, weight):
    """(loss, lse, grad, p, q) of rows s [rows x vocab], ids and t [rows x K]; p and q are the
    two distributions over the vocabulary."""
    s, t = np.asarray(s, np.float64) / tau, np.asarray(t, np.float64) / tau
    rows, vocab = s.shape
    # log p from differences to the row's largest: 64 bits do not show a sum beside -1e38.
    top = s.max(1)
    none = top == -np.inf  # the student leaves nothing: p is 0
    with np.errstate(invalid="ignore", divide="ignore"):
        logp = s - np.where(none, 0.0, top)[:, None]
        total = np.log(np.exp(logp).sum(1))
        lse = top + total
        logp = np.where(none[:, None], -np.inf, logp - total[:, None])
    loss, grad = np.zeros(rows), np.zeros(s.shape)
    p, q = np.zeros(s.shape), np.zeros(s.shape)
    for r in range(rows):
        there = (ids[r] >= 0) & (ids[r] < vocab)
        at, z = ids[r][there], t[r][there]
        if not at.size or z.max() == -np.inf:
            continue
        logq = z - z.max()
        logq -= np.log(np.exp(logq).sum())
        qk = np.exp(logq)
        use = qk > 0
        np.add.at(q[r], at, qk)
        loss[r] = tau ** 2 * (qk[use] * (logq[use] - logp[r][at[use]])).sum()
        p[r] = np.exp(logp[r])
        if weight[r] != 0:
            grad[r] = weight[r] * tau * (p[r] - q[r])
    return loss, lse, grad, p, q
