"""A head from its learning to its answers: cross entropy of the tokens that came next, gradients
clipped by their norm, an update; then the projection in integers, logits and drawn tokens.

One step's numbers against 64 bits: gradients are off by at most 2^-7 of their norm in bfloat16 and
2^-15 in float32 (the roundings of dz and of the result), a clipped gradient by one rounding more."""
import numpy as np
import pytest
import torch

from oracle import learn as O
from paper_2607_07388_amd import tfe

from . import harness as H

pytestmark = pytest.mark.gpu

F32, BF16 = tfe.TFE_F32, tfe.TFE_BF16


class Head:
    def __init__(self, rows=96, vocab=1500, dim=136, dtype=F32, seed=1):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.rows, self.vocab, self.dim, self.dtype = rows, vocab, dim, dtype
        self.hidden = torch.randn((rows, dim), generator=g, device="cuda").bfloat16()
        self.master = torch.randn((vocab, dim), generator=g, device="cuda") * 0.1
        self.w = self.master.bfloat16()
        self.targets = torch.randint(-1, vocab, (rows,), generator=g, device="cuda").int()
        kind = dict(dtype=torch.float32 if dtype == F32 else torch.bfloat16, device="cuda")
        self.loss, self.lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        self.gh, self.gw = torch.empty((rows, dim), **kind), torch.empty((vocab, dim), **kind)
        self.norm = torch.empty(1, device="cuda")
        self.list = tfe.make_grad_tensors([(t, t, t.shape[0], dim, dim, dim, dtype) for t in (self.gh, self.gw)])
        size = max(tfe.tfe_cross_entropy_workspace(rows, vocab, dim), tfe.tfe_grad_workspace(self.list, 2))
        self.space = torch.empty(size, dtype=torch.uint8, device="cuda")

    def grads(self):
        tfe.tfe_cross_entropy_loss_grad(self.hidden, self.dim, self.w, self.dim, self.targets, self.rows, self.vocab,
                                        self.dim, None, self.loss, self.lse, self.gh, self.dim, self.gw, self.dim,
                                        self.dtype, 0, self.space, self.space.numel(), H.cur_stream())

    def step(self, rate=0.05, most=1.0):
        self.grads()
        tfe.tfe_grad_norm_clip(self.list, 2, most, self.norm, self.space, self.space.numel(), H.cur_stream())
        self.master.add_(self.gw.float(), alpha=-rate)
        self.w.copy_(self.master)

    def exact(self):
        return O.cross_entropy(self.hidden.float().cpu().numpy(), self.w.float().cpu().numpy(),
                               self.targets.cpu().numpy(), np.ones(self.rows))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_step(dtype):
    h = Head(dtype=dtype)
    loss, lse, dx, dw, _ = h.exact()
    h.grads()
    most = 2.0 ** -15 if dtype == F32 else 2.0 ** -7
    for got, want in ((h.gh, dx), (h.gw, dw)):
        assert np.linalg.norm(got.double().cpu().numpy() - want) <= most * np.linalg.norm(want)
    seen = [t.float().cpu().numpy() for t in (h.gh, h.gw)]
    h.step(most=0.5)
    norm = O.grad_norm(seen)
    assert abs(float(h.norm) - norm) <= 2.0 ** -23 * norm and norm > 0.5
    by = O.clip_factor(float(h.norm), 0.5)
    for s, t in zip(seen, (h.gh, h.gw)):
        assert torch.equal(t.cpu(), torch.from_numpy(s * by).to(t.dtype))
    after = O.grad_norm([t.float().cpu().numpy() for t in (h.gh, h.gw)])
    assert abs(after - 0.5) <= 2.0 ** -8 * 0.5


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_steps_captured_are_steps(dtype):
    """A captured step replayed between eager work of another head that shares nothing with it."""
    a, b, other = Head(dtype=dtype), Head(dtype=dtype), Head(dtype=dtype, seed=5)
    for _ in range(4):
        a.step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.step()
    b.master.copy_(Head(dtype=dtype).master)
    b.w.copy_(b.master)
    for _ in range(4):
        g.replay()
        other.step()
        torch.cuda.synchronize()
    assert torch.equal(a.master, b.master) and torch.equal(a.norm, b.norm) and torch.equal(a.loss, b.loss)


def test_accumulated_over_batches():
    """Gradients of two batches added in float32 are those of both batches as one."""
    h = Head(rows=128)
    _, _, _, dw, _ = h.exact()
    total = torch.zeros_like(h.gw)
    half = h.rows // 2
    for k in range(2):
        rows = slice(k * half, (k + 1) * half)
        tfe.tfe_cross_entropy_loss_grad(h.hidden[rows], h.dim, h.w, h.dim, h.targets[rows], half, h.vocab, h.dim, None,
                                        h.loss[rows], h.lse[rows], h.gh[rows], h.dim, total, h.dim, F32, 1, h.space,
                                        h.space.numel(), H.cur_stream())
    assert np.linalg.norm(total.double().cpu().numpy() - dw) <= 2.0 ** -15 * np.linalg.norm(dw)


@pytest.mark.parametrize("rows", [1, 16, 96])
def test_learned_then_served_in_integers(rows):
    """The tokens that are drawn from integer logits are the oracle's layout's."""
    h = Head()
    for _ in range(8):
        h.step()
    pitch = -(-h.dim // 128) * 128
    codes = torch.empty((h.vocab, pitch), dtype=torch.int8, device="cuda")
    scales = torch.empty(h.vocab, device="cuda")
    tfe.tfe_integer_quantize(h.w, BF16, h.dim, h.vocab, h.dim, codes, scales, H.cur_stream())
    logits = torch.empty((rows, h.vocab), device="cuda")
    size = tfe.tfe_integer_workspace(rows, h.dim)
    tfe.tfe_integer_linear(h.hidden, BF16, h.dim, codes, scales, rows, h.vocab, h.dim, logits, F32, h.vocab,
                           torch.empty(size, dtype=torch.uint8, device="cuda"), size, H.cur_stream())
    a, b = (O.integer_layout(t.float().cpu().numpy()) for t in (h.hidden[:rows], h.w))
    _, exact = O.integer_product(*a, *b)
    got = logits.double().cpu().numpy()
    assert (np.abs(got - exact) <= 4 * 2.0 ** -24 * np.abs(exact)).all()
    token = torch.empty(rows, dtype=torch.int32, device="cuda")
    size = tfe.tfe_sample_workspace(rows, h.vocab)
    tfe.tfe_sample(logits, F32, h.vocab, rows, h.vocab, torch.zeros(rows, device="cuda"), None, None, None,
                   torch.zeros(rows, device="cuda"), token, None,
                   torch.empty(max(16, size), dtype=torch.uint8, device="cuda"), size, H.cur_stream())
    assert torch.equal(token.long(), logits.argmax(1))
