"""The norm of many gradients and their clipping, through the C ABI, against 64 bits.

The norm is a float64 sum of exact squares, rounded to float32: off by 2^-24 of itself (the float64
sum by far less).  A clipped number is a float32 product: the oracle's product in float32 to the bit,
rounded to bfloat16 where the gradient is."""
import numpy as np
import pytest
import torch

from oracle import learn as O
from paper_2607_07388_amd import tfe

from . import harness as H

pytestmark = pytest.mark.gpu

F32, BF16 = tfe.TFE_F32, tfe.TFE_BF16
TORCH = {F32: torch.float32, BF16: torch.bfloat16}


class Grads:
    """Tensors of (rows, cols, pad, shift, dtype); `place`: clipped in place, or elsewhere."""

    def __init__(self, shapes, seed=1, scale=1.0, place=False, out_pad=0):
        rng = np.random.default_rng(seed)
        self.grads, self.outs, entries = [], [], []
        for rows, cols, pad, shift, dtype in shapes:
            opad = pad if place else out_pad
            g = torch.full((rows * (cols + pad) + shift,), float("nan"), dtype=TORCH[dtype], device="cuda")[shift:]
            g = g.view(rows, cols + pad)
            g[:, :cols] = torch.from_numpy((rng.standard_normal((rows, cols)) * scale).astype(np.float32)).cuda()
            o = g if place else torch.full((rows * (cols + opad) + shift,), -7.0, dtype=TORCH[dtype],
                                           device="cuda")[shift:].view(rows, cols + opad)
            self.grads.append(g[:, :cols])
            self.outs.append(o[:, :cols])
            entries.append((g, o, rows, cols, cols + pad, cols + opad, dtype))
        self.entries, self.n = entries, len(entries)
        self.list = tfe.make_grad_tensors(entries)
        self.size = tfe.tfe_grad_workspace(self.list, self.n)
        self.norm = torch.full((1,), -7.0, device="cuda")

    def space(self):
        return torch.full((max(16, self.size),), 0x7F, dtype=torch.uint8, device="cuda"), self.size

    def seen(self):
        return [g.float().cpu().numpy() for g in self.grads]

    def measure(self):
        tfe.tfe_grad_norm(self.list, self.n, self.norm, *self.space(), H.cur_stream())
        return self.norm

    def clip(self, most):
        tfe.tfe_grad_norm_clip(self.list, self.n, most, self.norm, *self.space(), H.cur_stream())
        return self.norm

    def check(self, seen, most):
        norm = O.grad_norm(seen)
        got = float(self.norm)
        assert abs(got - norm) <= 2.0 ** -23 * norm
        by = O.clip_factor(got, most)
        for s, o in zip(seen, self.outs):
            want = torch.from_numpy(s * by).to(o.dtype)
            assert torch.equal(o.cpu(), want)
        for (g, o, rows, cols, ldg, ldo, _) in self.entries:
            pad = o[:, cols:].float()
            assert pad.isnan().all() if o is g else (pad == -7).all()


ONE = (1, 1, 0, 0, F32)
SETS = {
    "one": [ONE], "one_bf16": [(1, 1, 0, 0, BF16)], "vector": [(1, 8193, 0, 1, F32)],
    "odd": [(1, 7, 0, 1, BF16), (3, 5, 0, 0, F32), (1, 100001, 0, 3, BF16), (1, 16383, 0, 1, F32)],
    "pitched": [(300, 77, 3, 1, F32), (1000, 8, 8, 0, BF16), (129, 1000, 24, 0, BF16), (2, 1, 5, 0, F32),
                (70, 512, 4, 0, F32)],
    "many": [(1 + k % 3, 1 + 37 * k % 501, k % 2, k % 5, k % 2) for k in range(81)],
    "more": [(1, 1 + 97 * k % 1303, 0, k % 3, F32 if k % 7 else BF16) for k in range(333)],
    "empty": [(0, 5, 0, 0, F32), (1, 40, 0, 0, F32), (3, 0, 2, 0, BF16)],
    "large": [(1, 5000003, 0, 1, F32), (2000, 1024, 0, 0, BF16), ONE]}


@pytest.mark.parametrize("place", [False, True])
@pytest.mark.parametrize("name", SETS)
def test_norm_and_clip(name, place):
    g = Grads(SETS[name], place=place, out_pad=0 if place else 3)
    seen = g.seen()
    assert abs(float(g.measure()) - O.grad_norm(seen)) <= 2.0 ** -23 * O.grad_norm(seen)
    measured = g.norm.clone()
    g.clip(0.37)
    assert torch.equal(measured, g.norm)
    g.check(seen, 0.37)


@pytest.mark.parametrize("place", [False, True])
def test_two_calls_are_one(place):
    a, b = (Grads(SETS["odd"] + SETS["pitched"], place=place) for _ in range(2))
    a.clip(1.5)
    b.measure()
    tfe.tfe_grad_clip(b.list, b.n, 1.5, b.norm, H.cur_stream())
    assert torch.equal(a.norm, b.norm) and all(torch.equal(x, y) for x, y in zip(a.outs, b.outs))


@pytest.mark.parametrize("place", [False, True])
def test_below_the_limit(place):
    """A norm at or below the limit changes nothing: copies elsewhere, nothing in place."""
    g = Grads(SETS["odd"], place=place)
    seen = g.seen()
    limit = float(g.measure())
    g.clip(limit)
    g.check(seen, limit)
    assert all(np.array_equal(o.float().cpu().numpy(), s) for o, s in zip(g.outs, seen))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("place", [False, True])
def test_not_finite(bad, place):
    """The norm shows it, and the gradients stay as they are."""
    g = Grads(SETS["odd"], place=place)
    g.grads[2][0, 5000] = bad
    before = [x.clone() for x in g.grads]
    g.clip(0.1)
    assert float(g.norm) == float("inf") if bad == bad else g.norm.isnan().all()
    for x, y in zip(g.outs, before):
        assert torch.equal(x.nan_to_num(5.0, 6.0, 7.0), y.nan_to_num(5.0, 6.0, 7.0))


@pytest.mark.parametrize("scale", [1e-30, 1e-22, 1e18, 1e30])
def test_squares_outside_float32(scale):
    g = Grads([(1, 5000, 0, 0, F32), (1, 3001, 0, 1, BF16)], scale=scale)
    seen = g.seen()
    g.clip(scale)
    g.check(seen, scale)


def test_zeros_and_limit_zero():
    g = Grads(SETS["odd"], scale=0.0)
    g.clip(0.0)
    assert float(g.norm) == 0 and all((o == 0).all() for o in g.outs)
    g = Grads(SETS["odd"])
    g.clip(0.0)
    assert all((o == 0).all() for o in g.outs)


def test_nothing():
    norm = torch.full((1,), -7.0, device="cuda")
    t = tfe.make_grad_tensors([])
    tfe.tfe_grad_norm(t, 0, norm, None, 0, H.cur_stream())
    assert float(norm) == 0
    norm.fill_(-7)
    tfe.tfe_grad_norm_clip(t, 0, 1.0, norm, None, 0, H.cur_stream())
    assert float(norm) == 0
    e = Grads([(0, 5, 0, 0, F32), (4, 0, 0, 0, BF16)])
    assert float(e.clip(1.0)) == 0
    tfe.tfe_grad_clip(e.list, e.n, 1.0, e.norm, H.cur_stream())


def test_a_norm_from_elsewhere():
    """Clipped by a norm joined from several ranks', larger than these gradients' own."""
    g = Grads(SETS["odd"])
    seen = g.seen()
    g.norm.fill_(1e4)
    tfe.tfe_grad_clip(g.list, g.n, 50.0, g.norm, H.cur_stream())
    for s, o in zip(seen, g.outs):
        assert torch.equal(o.cpu(), torch.from_numpy(s * O.clip_factor(1e4, 50.0)).to(o.dtype))


@pytest.mark.parametrize("name", ["odd", "more"])
def test_captured_and_on_another_stream(name):
    a, b = Grads(SETS[name], seed=1), Grads(SETS[name], seed=2)
    a.clip(0.5)
    want = [o.clone() for o in a.outs], a.norm.clone()
    b.clip(0.5)
    other = [o.clone() for o in b.outs], b.norm.clone()
    side = torch.cuda.Stream()
    for o in a.outs:
        o.fill_(-7)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.clip(0.5)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a.outs, want[0])) and torch.equal(a.norm, want[1])
    c, space = Grads(SETS[name], seed=3), a.space()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tfe.tfe_grad_norm_clip(c.list, c.n, 0.5, c.norm, *space, H.cur_stream())
    for src, (outs, norm) in ((a, want), (b, other), (a, want), (b, other)):
        for x, y in zip(c.grads, src.grads):
            x.copy_(y)
        g.replay()
        c2 = Grads(SETS["one"])
        c2.clip(1.0)
        torch.cuda.synchronize()
        assert torch.equal(c.norm, norm) and all(torch.equal(x, y) for x, y in zip(c.outs, outs))


def test_norm_does_not_look_at_out():
    g = torch.randn((700, 96), device="cuda")
    t = tfe.make_grad_tensors([(g, None, 700, 96, 96, 0, F32), (g, None, 1, 700 * 96, 0, 0, F32)])
    size, norm = tfe.tfe_grad_workspace(t, 2), torch.zeros(1, device="cuda")
    tfe.tfe_grad_norm(t, 2, norm, torch.empty(size, dtype=torch.uint8, device="cuda"), size, H.cur_stream())
    want = O.grad_norm([g.cpu().numpy()] * 2)
    assert abs(float(norm) - want) <= 2.0 ** -23 * want


def test_more_than_2_to_the_32_elements():
    n = (1 << 32) + 4099
    g = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    g[-1] = 3.0
    t = tfe.make_grad_tensors([(g, g, 1, n, n, n, BF16)])
    size, norm = tfe.tfe_grad_workspace(t, 1), torch.zeros(1, device="cuda")
    tfe.tfe_grad_norm_clip(t, 1, 32768.0, norm, torch.empty(size, dtype=torch.uint8, device="cuda"), size, H.cur_stream())
    want = np.sqrt(n + 8.0)
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    by = O.clip_factor(float(norm), 32768.0)
    assert (g[:-1] == torch.tensor(by).bfloat16().cuda()).all() and g[-1] == torch.tensor(by * np.float32(3)).bfloat16()


@pytest.mark.parametrize("place", [False, True])
def test_more_tensors_with_rows_apart_than_a_launch_has(place):
    shapes = [(2 + k % 3, 3 + k % 7, 1 + k % 4, k % 3, k % 2) for k in range(50)] + [(1, 1024 * k, 0, 0, F32) for k in (1, 2)]
    g = Grads(shapes, place=place)
    seen = g.seen()
    g.clip(0.9)
    g.check(seen, 0.9)
