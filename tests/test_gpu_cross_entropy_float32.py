"""Float32 gradients of cross entropy are those of a dz in float32.

W's first rows are unit vectors and the others 0, so that logits are numbers of the hidden states,
without an error, and the hidden states' gradient is dz itself.  lse is given.  u = 2^-24: the
exponential at d = z - lse is off by 3 |d| u (d, log2(e) and their product are each rounded) and 4 u
(its own rounding, the weight's), the one subtracted at the target by 2 u, and a sum of what dz is
kept as, with the product's other factor, by 8 u of itself.  A dz of 16 bits is off by up to 2^-18 = 64 u."""
import numpy as np
import pytest
import torch

from paper_2607_07388_amd import tfe

from . import harness as H

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32 = tfe.TFE_F32


# Rows of each tile of logits, both tiles of dW.
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("rows,vocab,dim", [(1, 200, 64), (5, 3000, 200), (100, 131073, 72), (300, 50000, 64), (700, 90000, 300)])
def test_dz_is_float32(rows, vocab, dim, weighted):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = (torch.rand((rows, dim), generator=g, device="cuda") * 3 + 12).bfloat16()
    w = torch.zeros((vocab, dim), dtype=torch.bfloat16, device="cuda")
    w[:dim].fill_diagonal_(1)
    t = torch.randint(0, dim, (rows,), generator=g, device="cuda").int()
    weight = torch.rand(rows, generator=g, device="cuda") + 0.5 if weighted else None
    z = x.double()
    lse = (z.exp().sum(1) + (vocab - dim)).log().float()
    size = tfe.tfe_cross_entropy_workspace(rows, vocab, dim)
    space = torch.empty(size, dtype=torch.uint8, device="cuda")

    def grads(weight):
        gx, gw = torch.empty((rows, dim), device="cuda"), torch.empty((vocab, dim), device="cuda")
        tfe.tfe_cross_entropy_grad(x, dim, w, dim, t, rows, vocab, dim, lse, weight, gx, dim, gw, dim, F32, 0, space,
                                   size, H.cur_stream())
        return gx.double(), gw.double()

    by = (weight.double() if weighted else torch.ones(rows, device="cuda").double())[:, None]
    d = z - lse.double()[:, None]
    hit = torch.zeros_like(z).scatter_(1, t.long()[:, None], 1.0)
    dz = (d.exp() - hit) * by
    off = by * (d.exp() * (3 * d.abs() + 4) + 2 * hit) * U + 8 * U * dz.abs()
    gx, _ = grads(weight)
    worst = float(((gx - dz).abs() / off).max())
    assert worst <= 1, "dH: %g of the bound" % worst
    # dW of one row that takes part: a product for each number.
    r = rows // 2
    alone = torch.zeros(rows, device="cuda")
    alone[r] = by[r, 0].float()
    _, gw = grads(alone)
    want, off = dz[r][:, None] * z[r], (off[r][:, None] + 8 * U * dz[r].abs()[:, None]) * z[r]
    worst = float(((gw[:dim] - want).abs() / off).max())
    assert worst <= 1, "dW: %g of the bound" % worst
    # The tokens of logit 0.
    p = np.exp(-float(lse[r])) * float(by[r])
    rest = (gw[dim:] - p * z[r]).abs().max() / (p * float(z[r].max()))
    assert float(rest) <= (3 * abs(float(lse[r])) + 16) * U
