"""The 8-bit product's sums: float32 whatever the type of the results and however many rows.

The products of two codes are exact, so a sum in float32 is within P 2^-24 sum |a w| of the
exact one (P terms), and exact where every partial sum has at most 24 significant bits.  A
bfloat16 result is that sum rounded once, by at most 2^-8 of itself."""
import numpy as np
import pytest
import torch

from oracle import logits as O
from paper_2607_07388_amd import tfe

from . import harness as H
from .test_gpu_quantized import BF16, F32, TORCH, quantize

pytestmark = pytest.mark.gpu


def matmul(ac, asc, wc, wsc, n, dim, out_dtype):
    rows = ac.shape[0]
    out = torch.full((rows, n), -7.0, dtype=TORCH[out_dtype], device="cuda")
    tfe.tfe_quantized_matmul(ac, asc, wc, wsc, rows, n, dim, out, out_dtype, n, H.cur_stream())
    return out


# Rows that stay in shared memory, both kinds of tiles, ragged ends; one row too wide for shared memory.
SHAPES = [(100, 515, 1024), (300, 2000, 1300), (65, 255, 640), (513, 66000, 256),
          (1, 300, 1024), (16, 300, 512), (64, 1000, 1000), (1, 40, 65536)]


@pytest.mark.parametrize("rows,n,dim", SHAPES)
def test_small_results_of_large_terms(rows, n, dim):
    """Two terms of 2^16 that cancel and small ones: every partial sum is a multiple of 1/16 below
    2^17 in magnitude, 21 bits."""
    rng = np.random.default_rng(rows + n + dim)
    some = min(dim, 512)
    x, w = np.zeros((rows, dim)), np.zeros((n, dim))
    at = np.sort(rng.permutation(dim)[:some])
    x[:, at] = rng.integers(-3, 4, (rows, some)) / 4
    w[:, at] = rng.integers(-3, 4, (n, some)) / 4
    first, last = at[0], at[-1]
    x[:, [first, last]] = 256
    w[:, first], w[:, last] = 256, -256
    ac, asc, _ = quantize(x, F32, 1)
    wc, wsc, _ = quantize(w, F32, 128)
    a, v = O.fp8_values(ac.cpu().numpy(), asc.cpu().numpy(), 1), O.fp8_values(wc.cpu().numpy(), wsc.cpu().numpy(), 128)
    exact = torch.from_numpy(a @ v.T)
    for out_dtype in (F32, BF16):
        got = matmul(ac, asc, wc, wsc, n, dim, out_dtype).cpu()
        assert torch.equal(got, exact.to(TORCH[out_dtype])), (got.double() - exact).abs().max()


@pytest.mark.parametrize("rows,n,dim", SHAPES)
def test_bfloat16_results_are_the_float32_ones_rounded(rows, n, dim):
    rng = np.random.default_rng(rows * 3 + n + dim)
    ac, asc, _ = quantize(rng.standard_normal((rows, dim)) * 2.0 ** rng.integers(-6, 6, (rows, 1)), F32, 1)
    wc, wsc, _ = quantize(rng.standard_normal((n, dim)) * 0.1, F32, 128)
    want = matmul(ac, asc, wc, wsc, n, dim, F32)
    assert torch.equal(matmul(ac, asc, wc, wsc, n, dim, BF16), want.to(torch.bfloat16))
    few = slice(0, min(n, 300))
    a = O.fp8_values(ac.cpu().numpy(), asc.cpu().numpy(), 1)
    v = O.fp8_values(wc.cpu().numpy(), wsc.cpu().numpy(), 128)[few, :a.shape[1]]
    bound = a.shape[1] * 2.0 ** -24 * (np.abs(a) @ np.abs(v).T)
    assert (np.abs(want[:, few].double().cpu().numpy() - a @ v.T) <= bound).all()


@pytest.mark.parametrize("out_dtype", [F32, BF16])
def test_a_row_has_the_same_results_in_any_batch(out_dtype):
    rows, n, dim = 600, 66000, 640
    rng = np.random.default_rng(1)
    ac, asc, _ = quantize(rng.standard_normal((rows, dim)), F32, 1)
    wc, wsc, _ = quantize(rng.standard_normal((n, dim)) * 0.1, F32, 128)
    want = matmul(ac, asc, wc, wsc, n, dim, out_dtype)
    for few in (1, 16, 48, 64, 65, 200, 300):
        assert torch.equal(matmul(ac[:few], asc[:few], wc, wsc, n, dim, out_dtype), want[:few]), few
