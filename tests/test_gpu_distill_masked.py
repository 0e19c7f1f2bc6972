"""Distillation of rows whose student logits are masked as a whole, or lie so far from zero that
a float32 log-sum-exp does not show the sum of their exponentials.

Where a row's log-sum-exp is above 4096 in magnitude, probabilities come from differences to the
largest logit m: an exponent (x - m) / tau of at most 104 in magnitude (beyond that it is 0) is
rounded to 2^-22 of itself, the exponential is within 2^-22 and a sum adds at most 400 terms:
p within 2e-5 + 2^-22 104 of itself, twice with the sum's.  Elsewhere 104 is |x|max, as for any
other row.  The loss adds q-weighted terms of that error and of 2^-22 of (s - m) / tau."""
import numpy as np
import pytest
import torch

from oracle import logits as O

from .test_gpu_distill import BF16, F32, TORCH, Call, inputs

pytestmark = pytest.mark.gpu

KINDS = ["nothing", "lowest", "lowest, some nothing", "lowest but one", "-1e9", "-1e9 but one", "-1e4", "far below",
         "far above", "largest", "nothing but one", "plain"]


def masked(seed, vocab, dtype):
    """A row of each kind."""
    s, ids, t, weight = inputs(seed, len(KINDS), vocab, 9, short=False)
    low, n = torch.finfo(TORCH[dtype]).min, np.arange(vocab)
    for r, kind in enumerate(KINDS):
        if kind == "nothing":
            s[r] = -np.inf
        elif kind.startswith("lowest"):
            s[r] = low
        elif kind.startswith("-1e9"):
            s[r] = -1e9
        elif kind == "-1e4":
            s[r] = -1e4
        elif kind == "far below":
            s[r] = -1e6 + np.round(s[r]) * 8192  # bfloat16 keeps steps of 8192 there
        elif kind == "far above":
            s[r] = 3e5 + np.round(s[r]) * 2048
        elif kind == "largest":
            s[r] = np.where(n % 3 == 0, -low, low)
        elif kind == "nothing but one":
            s[r] = -np.inf
            s[r, vocab - 1] = 1.5
        if kind == "lowest, some nothing":
            s[r, n % 7 != 0] = -np.inf
        elif kind in ("lowest but one", "-1e9 but one"):
            s[r, vocab // 2] = -3.0
    return s, ids, t, weight


def check(c, ids, weight, loss, lse, grad):
    s, t = c.seen()
    with np.errstate(over="ignore"):
        wl, wlse, wg, p, q = O.distill(s, ids, t, c.tau, weight)
    got = lse.double().cpu().numpy()
    over = np.abs(wlse) > torch.finfo(torch.float32).max
    np.testing.assert_array_equal(got[over], np.sign(wlse[over]) * np.inf)
    assert (np.abs(got[~over] - wlse[~over]) <= 2e-5 + 2.0 ** -22 * np.abs(wlse[~over])).all()
    x = s.astype(np.float64) / c.tau
    most = np.abs(np.where(np.isfinite(x), x, 0)).max(1)
    eps = 2e-5 + 2.0 ** -22 * np.where(np.abs(wlse) > 4095, 104, most)
    top = x.max(1)
    ref = np.where(top == -np.inf, 0, top)
    far = np.abs(np.take_along_axis(x, ids, 1) - ref[:, None])
    far = np.where(np.isfinite(far), far, 0).max(1)
    if loss is not None:
        got = loss.double().cpu().numpy()
        over = c.tau ** 2 * far > 1e38
        inf = np.isinf(wl)
        np.testing.assert_array_equal(np.isposinf(got[inf]), True)
        ok = ~inf & ~over
        bound = c.tau ** 2 * (2 * eps + 1e-5 * (far + 20)) + 1e-6 * np.abs(wl)
        assert (np.abs(got[ok] - wl[ok]) <= bound[ok]).all(), (got[ok], wl[ok])
        assert (got[~inf & over] > 1e37).all()
    if grad is not None:
        got = grad[:, :c.vocab].double().cpu().numpy()
        f = np.abs(weight[:, None]) * c.tau
        bound = f * (p * 2 * eps[:, None] + q * 2e-5) + np.abs(wg) * (2.0 ** -8 if c.dtype == BF16 else 1e-6) + 1e-37
        bad = ~(np.abs(got - wg) <= bound)
        assert not bad.any(), (sorted({KINDS[r % len(KINDS)] for r in np.argwhere(bad)[:, 0]}), got[bad][:4], wg[bad][:4])


@pytest.mark.parametrize("tau", [2.0, 0.5, 1.0])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [37, 700, 40003, 151936])
def test_masked_rows(vocab, dtype, tau):
    s, ids, t, weight = masked(vocab, vocab, dtype)
    c = Call(s, ids, t, tau, dtype, pad=vocab % 2, gpad=vocab % 2)
    w = torch.from_numpy(weight).cuda()
    loss, lse = c.loss()
    check(c, ids, weight, loss, lse, None)
    grad = c.grad(lse, w)
    check(c, ids, weight, loss, lse, grad)
    both = c.both(w)
    check(c, ids, weight, *both)
    # One call or two, in a place of its own or the logits': the same bits.
    for x, y in zip(both, (loss, lse, grad)):
        assert torch.equal(x, y)
    keep = c.s.clone()
    c.grad(lse, w, grad=c.s)
    assert torch.equal(c.s[:, :vocab], grad[:, :vocab])
    c.s.copy_(keep)
    c.both(w, grad=c.s)
    assert torch.equal(c.s[:, :vocab], grad[:, :vocab])


def test_a_student_that_leaves_nothing():
    """No probability anywhere: the loss is infinite, the gradient -tau q; 0 without a teacher."""
    vocab, tau = 50000, 2.0
    ids = np.array([[5, 40000, 7], [5, 40000, 7], [-1, -1, -1]])
    t = np.array([[1.0, 2.0, 3.0], [1.0, -np.inf, 3.0], [0.0, 0.0, 0.0]])
    c = Call(np.full((3, vocab), -np.inf), ids, t, tau)
    loss, lse, grad = c.both(None)
    q = np.exp(t[:2] / tau)
    q /= q.sum(1, keepdims=True)
    assert torch.isinf(loss[:2]).all() and loss[2] == 0 and (lse == -np.inf).all()
    want = np.zeros((3, vocab))
    want[np.arange(2)[:, None], ids[:2]] = -tau * q
    np.testing.assert_allclose(grad.cpu().numpy(), want, rtol=1e-5, atol=0)


@pytest.mark.parametrize("tau", [3.0, 0.3, 1.0])
@pytest.mark.parametrize("tdtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [900, 40003])
def test_teachers_far_from_zero(vocab, tdtype, tau):
    """Lists whose logits lie far from 0, or at masks' values: q depends on differences alone
    ((t - m) / tau is rounded to 2^-22 of itself, at most 104 where q is not 0)."""
    rows = 8
    s, ids, t, weight = inputs(vocab, rows, vocab, 40, short=False)
    low = torch.finfo(TORCH[tdtype]).min
    step = 8192.0 if tdtype == BF16 else 0.5  # what the type keeps there
    for r, at in enumerate((1e6, -1e6, 3e5, -2e6)):
        t[r] = np.round((at + np.round(t[r] * 2) * step) / step) * step
    t[4], t[5], t[6] = low, -1e9, -low
    t[7, ::2] = low
    c = Call(s, ids, t, tau, F32, tdtype)
    w = torch.from_numpy(weight).cuda()
    loss, lse = c.loss()
    check(c, ids, weight, loss, lse, c.grad(lse, w))
    check(c, ids, weight, *c.both(w))


def test_infinite_teachers_are_not_hidden():
    """NaN or +infinity in a list: the loss is NaN, and so is the gradient at the listed tokens;
    elsewhere it is the student's.  Lists of -infinity and padding alone have no weight."""
    vocab, tau = 33000, 2.0
    s, _, _, _ = inputs(9, 5, vocab, 3, short=False)
    ids = np.tile([[7, 32999, 12000]], (5, 1))
    t = np.zeros((5, 3))
    t[0], t[1, 1], t[2] = np.nan, np.inf, np.inf
    t[3], ids[3, 1] = -np.inf, -1
    c = Call(s, ids, t, tau)
    loss, lse = c.loss()
    for loss, lse, grad in ((loss, lse, c.grad(lse, None)), c.both(None)):
        assert loss[:3].isnan().all() and loss[3] == 0 and torch.isfinite(loss[4]) and torch.isfinite(lse).all()
        at = torch.from_numpy(ids[0].astype(np.int64)).cuda()
        assert grad[:3, at].isnan().all() and grad[:3].isnan().sum() == 9
        assert not grad[3].any() and torch.isfinite(grad[4]).all()
