"""Gradients that lie between each other's rows, or are listed twice, through the C ABI against 64 bits.

The norm is a float64 sum rounded to float32, off by 2^-24 of itself; clipped numbers are the
oracle's float32 products, to the bit."""
import numpy as np
import pytest
import torch

from oracle import learn as O
from paper_2607_07388_amd import tfe

from . import harness as H

pytestmark = pytest.mark.gpu

F32, BF16 = tfe.TFE_F32, tfe.TFE_BF16


def clip(entries, most):
    t, n = tfe.make_grad_tensors(entries), len(entries)
    size, norm = tfe.tfe_grad_workspace(t, n), torch.zeros(1, device="cuda")
    tfe.tfe_grad_norm_clip(t, n, most, norm, torch.empty(size, dtype=torch.uint8, device="cuda"), size, H.cur_stream())
    return float(norm)


@pytest.mark.parametrize("dtype,kind", [(F32, torch.float32), (BF16, torch.bfloat16)])
@pytest.mark.parametrize("rows,cols", [(70, 64), (33, 37), (1000, 3)])
def test_columns_of_one_matrix(rows, cols, dtype, kind):
    """Three parts of each row as tensors of their own, in place."""
    g = torch.randn((rows, 3 * cols), generator=torch.Generator("cuda").manual_seed(rows), device="cuda").to(kind)
    seen = g.float().cpu().numpy()
    norm = clip([(g[:, k * cols:], g[:, k * cols:], rows, cols, 3 * cols, 3 * cols, dtype) for k in (2, 0, 1)], 0.7)
    assert abs(norm - O.grad_norm([seen])) <= 2.0 ** -23 * norm
    assert torch.equal(g.cpu(), torch.from_numpy(seen * O.clip_factor(norm, 0.7)).to(kind))


def test_listed_twice():
    """It counts twice in the norm, and goes to two places."""
    g = torch.randn(5000, generator=torch.Generator("cuda").manual_seed(3), device="cuda")
    a, b = torch.empty_like(g), torch.empty_like(g)
    norm = clip([(g, a, 1, 5000, 5000, 5000, F32), (g, b, 1, 5000, 5000, 5000, F32)], 2.0)
    seen = g.cpu().numpy()
    assert abs(norm - O.grad_norm([seen] * 2)) <= 2.0 ** -23 * norm
    want = torch.from_numpy(seen * O.clip_factor(norm, 2.0))
    assert torch.equal(a.cpu(), want) and torch.equal(b.cpu(), want)


@pytest.mark.parametrize("n", [100, 700])
def test_many_in_any_order(n):
    flat = torch.randn(n * 33, generator=torch.Generator("cuda").manual_seed(n), device="cuda")
    seen = flat.cpu().numpy()
    parts = [flat[k * 33:(k + 1) * 33] for k in np.random.default_rng(n).permutation(n)]
    norm = clip([(p, p, 1, 33, 33, 33, F32) for p in parts], 1.0)
    assert abs(norm - O.grad_norm([seen])) <= 2.0 ** -23 * norm
    assert torch.equal(flat.cpu(), torch.from_numpy(seen * O.clip_factor(norm, 1.0)))
