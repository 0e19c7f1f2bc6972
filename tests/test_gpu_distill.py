"""The distillation loss and its gradient against the 64-bit oracle, and the gradient
against differences of the oracle's loss.

Bounds, with x = s / tau.  An exponential's argument x - m is rounded to 2^-23 of
itself and of x (at most 2^-23 (|x - m| + |x|)), the hardware exponential is within
2^-22, and the sum adds at most 400 partial sums one after another (2^-24 each):
log-sum-exp within 2e-5 + 2^-22 |x|max.  The loss adds q-weighted terms of that
error (q within 1e-5).  A probability p: relative error as of the log-sum-exp's
absolute one, twice."""
import numpy as np
import pytest
import torch

from oracle import logits as O
from paper_2607_07388_amd import tfe

from . import harness as H

pytestmark = pytest.mark.gpu

F32, BF16 = tfe.TFE_F32, tfe.TFE_BF16
TORCH = {F32: torch.float32, BF16: torch.bfloat16}


def tensor(x, dtype, pad=0):
    rows, cols = x.shape
    t = torch.full((rows, cols + pad), float("nan"), dtype=TORCH[dtype], device="cuda")
    t[:, :cols] = torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().to(TORCH[dtype])
    return t


def inputs(seed, rows, vocab, K, short=True):
    rng = np.random.default_rng(seed)
    s = rng.standard_normal((rows, vocab)) * 2 - 0.5 * np.log(1 + np.arange(vocab))
    ids = np.stack([rng.permutation(vocab)[:K] if K <= vocab else
                    np.concatenate([rng.permutation(vocab), np.full(K - vocab, -1)]) for _ in range(rows)])
    t = rng.standard_normal((rows, K)) * 3
    if short and K > 1:
        ids[::3, K - K // 3:] = -1
        t[::3, K - K // 3:] = np.nan  # padding may hold anything
    return s, ids.astype(np.int32), t, rng.uniform(0.2, 2.0, rows).astype(np.float32)


class Call:
    def __init__(self, s, ids, t, tau, dtype=F32, tdtype=F32, pad=0, gpad=0):
        self.rows, self.vocab = s.shape
        self.tau, self.dtype, self.tdtype, self.K = tau, dtype, tdtype, ids.shape[1]
        self.s, self.t = tensor(s, dtype, pad), tensor(t, tdtype)
        self.ids = torch.from_numpy(np.ascontiguousarray(ids, np.int32)).cuda()
        self.ldg = self.vocab + gpad
        self.size = tfe.tfe_distill_workspace(self.rows, self.vocab)
        self.space = torch.full((self.size + 64,), 0xA5, dtype=torch.uint8, device="cuda")
        self.front = (self.s, dtype, self.vocab + pad, self.rows, self.vocab, self.ids, self.t, tdtype, self.K, tau)

    def seen(self):
        return self.s[:, :self.vocab].float().cpu().numpy(), self.t.float().cpu().numpy()

    def new(self):
        return (torch.full((self.rows,), -9.0, device="cuda"), torch.full((self.rows,), -9.0, device="cuda"),
                torch.full((self.rows, self.ldg), -9.0, dtype=TORCH[self.dtype], device="cuda"))

    def loss(self, stream=None):
        loss, lse, _ = self.new()
        tfe.tfe_distill_loss(*self.front, loss, lse, self.space, self.size, stream or H.cur_stream())
        return loss, lse

    def grad(self, lse, weight, stream=None, grad=None):
        grad = self.new()[2] if grad is None else grad
        tfe.tfe_distill_grad(*self.front, lse, weight, grad, self.ldg, stream or H.cur_stream())
        return grad

    def both(self, weight, stream=None, grad=None):
        loss, lse, g = self.new()
        grad = g if grad is None else grad
        tfe.tfe_distill_loss_grad(*self.front, weight, loss, lse, grad, self.ldg, self.space, self.size,
                                  stream or H.cur_stream())
        return loss, lse, grad


def check_values(c, ids, weight, loss, lse, grad):
    s, t = c.seen()
    wl, wlse, wg, p, q = O.distill(s, ids, t, c.tau, weight)
    x = np.abs(np.where(np.isfinite(s), s, 0) / c.tau).max(1)
    eps = 2e-5 + 2.0 ** -22 * x
    if lse is not None:
        assert (np.abs(lse.cpu().numpy() - wlse) <= eps).all()
    if loss is not None:
        got = loss.cpu().numpy()
        bound = c.tau ** 2 * (2 * eps + 1e-5 * (x + 20)) + 1e-6 * np.abs(wl)
        assert (np.abs(got - wl) <= bound).all(), (got - wl, bound)
    if grad is not None:
        got = grad[:, :c.vocab].float().cpu().numpy()
        f = np.abs(weight[:, None]) * c.tau
        bound = f * (p * 2 * eps[:, None] + q * 2e-5) + np.abs(wg) * (2.0 ** -8 if c.dtype == BF16 else 1e-6) + 1e-37
        bad = np.abs(got - wg) > bound
        assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], wg[bad][:4])
        assert (grad[:, c.vocab:] == -9).all()


SIZES = [(1, 1, 1), (2, 2, 1), (3, 5, 5), (4, 64, 7), (5, 65, 256), (7, 1000, 17), (3, 4099, 64), (300, 333, 33),
         (2, 33333, 128), (1, 151936, 256), (5, 151936, 64), (1, 1 << 18, 3), (600, 2000, 9), (300, 40001, 33),
         (1001, 17000, 5)]


@pytest.mark.parametrize("dtype,tdtype", [(F32, F32), (BF16, F32), (F32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("rows,vocab,K", SIZES)
def test_loss_and_gradient(rows, vocab, K, dtype, tdtype):
    s, ids, t, weight = inputs(rows + vocab + K, rows, vocab, K)
    c = Call(s, ids, t, 1.0 + (vocab % 3), dtype, tdtype, pad=vocab % 2, gpad=vocab % 4)
    w = torch.from_numpy(weight).cuda()
    loss, lse = c.loss()
    grad = c.grad(lse, w)
    check_values(c, ids, weight, loss, lse, grad)
    loss, lse, grad = c.both(w)
    check_values(c, ids, weight, loss, lse, grad)
    assert (c.space[c.size:] == 0xA5).all()


@pytest.mark.parametrize("tau", [0.05, 0.7, 20.0])
def test_temperatures(tau):
    s, ids, t, weight = inputs(1, 6, 3000, 40)
    c = Call(s, ids, t, tau)
    check_values(c, ids, weight, *c.both(torch.from_numpy(weight).cuda()))


@pytest.mark.parametrize("rows,vocab", [(4, 500), (2, 40000), (300, 500)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place_and_without_weights(rows, vocab, dtype):
    s, ids, t, _ = inputs(2, rows, vocab, 20)
    ones = np.ones(rows, np.float32)
    c = Call(s, ids, t, 2.0, dtype)
    want = c.both(None)
    check_values(c, ids, ones, *want)
    loss, lse = c.loss()
    keep = c.s.clone()
    c.grad(lse, None, grad=c.s)
    again = c.s.clone()
    c.s.copy_(keep)
    loss, lse, g = c.both(None, grad=c.s)
    for x, y in zip((loss, lse, g, again), want + (want[2],)):
        assert torch.equal(x, y)


def test_gradient_against_differences():
    """The formula's gradient is the loss' slope: central differences of the oracle in 64 bits at
    every coordinate of small rows, with ids listed twice among them."""
    rng = np.random.default_rng(3)
    rows, vocab, K, tau, h = 3, 23, 6, 1.7, 1e-5
    s = rng.standard_normal((rows, vocab)).astype(np.float32).astype(float)
    ids = rng.integers(0, vocab, (rows, K))
    ids[0, 1] = ids[0, 0]
    ids[1, 2:5] = 4
    ids[2, 5] = -1
    t = rng.standard_normal((rows, K)).astype(np.float32).astype(float)
    weight = np.array([1.0, 0.5, 2.0], np.float32)
    slope = np.zeros((rows, vocab))
    for v in range(vocab):
        up, down = s.copy(), s.copy()
        up[:, v] += h
        down[:, v] -= h
        slope[:, v] = weight * (O.distill(up, ids, t, tau, weight)[0] - O.distill(down, ids, t, tau, weight)[0]) / (2 * h)
    c = Call(s, ids, t, tau)
    w = torch.from_numpy(weight).cuda()
    loss, lse, grad = c.both(w)
    # Differences: h^2 / 6 of a third derivative below 10, and 1e-16 / h of rounding.
    np.testing.assert_allclose(grad.cpu().numpy(), slope, rtol=0, atol=2e-5)
    check_values(c, ids, weight, loss, lse, grad)
    np.testing.assert_allclose(grad.double().sum(1).cpu().numpy(), 0, atol=1e-5)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab", [(10, 700), (10, 50000), (400, 700)])
def test_empty_rows_masks_and_padding(rows, vocab, dtype):
    K = 12
    s, ids, t, weight = inputs(4, rows, vocab, K, short=False)
    ids[0] = -1                                # no teacher
    t[1] = -np.inf                             # no weight anywhere
    ids[2, 3:], t[2, 3:] = vocab, np.inf       # beyond the vocabulary
    ids[3, 0], t[3, 0] = -(2 ** 31), np.nan
    s[4, vocab // 2:] = torch.finfo(TORCH[dtype]).min  # masked by the type's lowest value
    ids[4] = np.arange(K)
    s[5, vocab // 2:] = -np.inf
    ids[5] = np.arange(K)
    t[6, 1:] = -np.inf                         # one entry has all
    weight[7], s[7] = 0.0, np.nan              # left out, whatever it holds
    s[8, ids[8, 2]], t[8, 2] = -np.inf, -np.inf  # no weight, no probability: no term
    c = Call(s, ids, t, 2.0, dtype)
    w = torch.from_numpy(weight).cuda()
    loss, lse = c.loss()
    parts = (loss, lse, c.grad(lse, w))
    for loss, lse, grad in (parts, c.both(w)):
        assert loss[0] == 0 and loss[1] == 0 and not grad[:2].float().abs().any()
        assert not grad[7].float().abs().any()
        keep = np.array([r for r in range(rows) if r != 7])
        k = torch.from_numpy(keep).cuda()
        sub = Call(c.seen()[0][keep], ids[keep], t[keep], 2.0, dtype)
        check_values(sub, ids[keep], weight[keep], loss[k], lse[k], grad[k])


def test_where_the_student_gives_nothing():
    """A token the teacher lists and the student excludes: infinite loss, finite gradient."""
    s, ids, t, weight = inputs(5, 2, 100, 4, short=False)
    s[0, ids[0, 1]] = -np.inf
    c = Call(s, ids, t, 1.0)
    loss, lse, grad = c.both(None)
    assert loss[0] == float("inf") and torch.isfinite(loss[1]) and torch.isfinite(grad).all()
    q = O.distill(np.zeros((2, 100)), ids, t, 1.0, np.ones(2))[4]
    np.testing.assert_allclose(float(grad[0, ids[0, 1]]), -q[0, ids[0, 1]], rtol=1e-5)


def test_nan_is_not_hidden():
    s, ids, t, _ = inputs(6, 3, 5000, 4, short=False)
    s[0, 4321] = np.nan
    t[1, 2] = np.nan
    c = Call(s, ids, t, 1.0)
    loss, lse, grad = c.both(None)
    assert loss[0].isnan() and lse[0].isnan() and grad[0].isnan().all()
    assert loss[1].isnan() and grad[1, torch.from_numpy(ids[1].astype(np.int64)).cuda()].isnan().all()
    assert torch.isfinite(loss[2]) and torch.isfinite(grad[2]).all()


@pytest.mark.parametrize("rows,vocab", [(3, 50000), (300, 900)])
def test_twice_the_same_and_captured(rows, vocab):
    """The same inputs give the same bits, eagerly, on another stream and in a graph's replays."""
    s, ids, t, weight = inputs(7, rows, vocab, 30)
    c = Call(s, ids, t, 2.0, BF16)
    w = torch.from_numpy(weight).cuda()
    want = c.both(w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = c.both(w, side.cuda_stream)
    side.synchronize()
    for x, y in zip(other, want):
        assert torch.equal(x, y)
    out = c.new()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tfe.tfe_distill_loss_grad(*c.front, w, out[0], out[1], out[2], c.ldg, c.space, c.size,
                                  torch.cuda.current_stream().cuda_stream)
    keep = c.s.clone()
    for k in range(3):
        c.s.copy_(keep * (0.5 + 0.5 * (k % 2)))
        eager = c.both(w)
        g.replay()
        for x, y in zip(out, eager):
            assert torch.equal(x, y)


def test_no_rows():
    assert tfe.tfe_distill_loss(None, F32, 10, 0, 10, None, None, F32, 4, 1.0, None, None, None, 0) == 0
    assert tfe.tfe_distill_grad(None, F32, 10, 0, 10, None, None, F32, 4, 1.0, None, None, None, 10) == 0
    assert tfe.tfe_distill_loss_grad(None, F32, 10, 0, 10, None, None, F32, 4, 1.0, None, None, None, None, 10,
                                     None, 0) == 0
