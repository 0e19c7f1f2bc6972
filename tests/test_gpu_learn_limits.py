"""The calls that learn the head near the ends of what they take: lists that pass the caches by, rows apart over
more than 2^32 elements, the longest pitches that are read in place and longer ones.

A norm is a float64 sum rounded to float32: off by 2^-24 of itself, and 2^-23 is asked for.  A matrix at another pitch
has the same numbers: results are equal."""
import numpy as np
import pytest
import torch

from oracle import learn as O
from paper_2607_07388_amd import tfe

from . import harness as H

pytestmark = pytest.mark.gpu

F32, BF16 = tfe.TFE_F32, tfe.TFE_BF16
TORCH = {F32: torch.float32, BF16: torch.bfloat16}


def norm_of(entries):
    t, n = tfe.make_grad_tensors(entries), len(entries)
    size, norm = tfe.tfe_grad_workspace(t, n), torch.full((1,), -7.0, device="cuda")
    tfe.tfe_grad_norm(t, n, norm, torch.full((size,), 0x7F, dtype=torch.uint8, device="cuda"), size, H.cur_stream())
    return float(norm)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tensors", [3, 40])
def test_norm_of_more_than_the_cache_holds(tensors, dtype):
    """Tensors of odd sizes, one off its alignment, one with rows apart."""
    g = torch.Generator(device="cuda").manual_seed(tensors)
    total = (300 << 20) // (4 if dtype == F32 else 2)
    entries, want = [], 0.0
    for k in range(tensors):
        n = total // tensors + 2 * k + 1
        x = torch.randn(n + 1, generator=g, device="cuda").to(TORCH[dtype])[k % 2:][:n]
        entries.append((x, None, 1, n, n, 0, dtype))
        want += float(x.double().square().sum())
    x = torch.randn((1000, 200), generator=g, device="cuda").to(TORCH[dtype])
    entries.append((x, None, 1000, 177, 200, 0, dtype))
    want = np.sqrt(want + float(x[:, :177].double().square().sum()))
    assert abs(norm_of(entries) - want) <= 2.0 ** -23 * want


@pytest.mark.parametrize("cols,ld", [(65536, 65544), (65537, 65540)])
def test_rows_apart_over_more_than_2_to_the_32_elements(cols, ld):
    rows = 65900
    g = torch.ones((rows, ld), dtype=torch.bfloat16, device="cuda")
    g[:, cols:] = float("nan")
    g[-1, cols - 1], g[rows // 2, 5] = 3.0, 3.0
    t, norm = tfe.make_grad_tensors([(g, g, rows, cols, ld, ld, BF16)]), torch.zeros(1, device="cuda")
    size = tfe.tfe_grad_workspace(t, 1)
    tfe.tfe_grad_norm_clip(t, 1, 32768.0, norm, torch.empty(size, dtype=torch.uint8, device="cuda"), size, H.cur_stream())
    want = np.sqrt(rows * cols + 16.0)
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    by = O.clip_factor(float(norm), 32768.0)
    threes = torch.tensor(by * np.float32(3)).bfloat16()
    assert g[-1, cols - 1] == threes and g[rows // 2, 5] == threes
    g[-1, cols - 1] = g[rows // 2, 5] = float(torch.tensor(by).bfloat16())
    assert (g[:, :cols] == float(torch.tensor(by).bfloat16())).all() and g[:, cols:].isnan().all()


LONGEST = 1 << 21


@pytest.mark.parametrize("rows,vocab,dim,which,ld", [
    (40, 1000, 64, "w", LONGEST), (40, 1000, 64, "w", LONGEST + 8), (600, 45000, 72, "hidden", LONGEST),
    (600, 45000, 72, "hidden", LONGEST + 8), (100, 1500, 136, "both", LONGEST)])
def test_long_pitches(rows, vocab, dim, which, ld):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn((rows, dim), generator=g, device="cuda").bfloat16()
    w = (torch.randn((vocab, dim), generator=g, device="cuda") * 0.2).bfloat16()
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda").int()
    size = tfe.tfe_cross_entropy_workspace(rows, vocab, dim)
    space = torch.empty(size, dtype=torch.uint8, device="cuda")

    def call(x, ldx, w, ldw):
        loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        gx, gw = torch.empty((rows, dim), device="cuda"), torch.empty((vocab, dim), device="cuda")
        tfe.tfe_cross_entropy_loss_grad(x, ldx, w, ldw, t, rows, vocab, dim, None, loss, lse, gx, dim, gw, dim, F32, 0,
                                        space, size, H.cur_stream())
        return loss, lse, gx, gw

    def far(m):
        out = torch.full((m.shape[0], ld), float("nan"), dtype=torch.bfloat16, device="cuda")
        out[:, :dim] = m
        return out

    want = call(x, dim, w, dim)
    assert all(o.isfinite().all() for o in want)
    got = call(*((far(x), ld) if which != "w" else (x, dim)), *((far(w), ld) if which != "hidden" else (w, dim)))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
