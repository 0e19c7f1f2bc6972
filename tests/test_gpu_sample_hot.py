"""tfe_sample at temperatures where neighbouring logits' weights differ by less than the
exponential's error, so that weights need not fall with the logits.  A bfloat16 row and the
same numbers as a float32 row have the same weights, so their tokens and probabilities have to
be equal to the bit; the two are counted in different ways, the float32 row's order by the
weights themselves."""
import numpy as np
import pytest
import torch

from paper_2607_07388_amd import tfe

from .test_gpu_sample import BF16, F32, draw

pytestmark = pytest.mark.gpu


def rows_of(kind, rows, vocab, seed):
    g = torch.Generator()
    g.manual_seed(seed)
    if kind == "every value":  # both signs, 2^-9 to 2^8, each more or less often
        bits = torch.arange(118 << 7, 135 << 7, dtype=torch.int32)
        v = (torch.cat([bits, bits + 0x8000]) << 16).view(torch.float32)
        return v[torch.randint(0, v.numel(), (rows, vocab), generator=g)]
    if kind == "large":        # 16 to 256, steps of 1/8 to 1
        return (torch.rand((rows, vocab), generator=g) * 240 + 16).bfloat16().float()
    if kind == "negative":
        return -(torch.rand((rows, vocab), generator=g) * 200).bfloat16().float()
    return (torch.randn((rows, vocab), generator=g) * 2 - 0.8 * torch.log1p(torch.arange(vocab).float())).bfloat16().float()


@pytest.mark.parametrize("T", [8.0, 60.0, 300.0, 2500.0, 1e5, 1e7])
@pytest.mark.parametrize("kind", ["every value", "large", "negative", "language"])
@pytest.mark.parametrize("vocab", [6007, 70001])
def test_hot_rows_like_float32_ones(vocab, kind, T):
    rows = 160
    l = rows_of(kind, rows, vocab, vocab + int(T)).cuda()
    rng = np.random.default_rng(int(T) + vocab)
    n = np.arange(rows)
    k = np.where(n & 1, rng.integers(1, vocab, rows), 0)
    p = np.where(n & 2, rng.uniform(0.05, 0.999, rows), 1.0)
    m = np.where(n & 4, rng.uniform(0.1, 0.9999, rows), 0.0)
    u = rng.random(rows)
    temp = T * rng.uniform(0.7, 1.4, rows)
    token, prob = draw(l.bfloat16(), BF16, vocab, rows, vocab, temp, k, p, m, u)
    want, wp = draw(l, F32, vocab, rows, vocab, temp, k, p, m, u)
    assert (token >= 0).all(), np.flatnonzero(token < 0)
    np.testing.assert_array_equal(token, want)
    np.testing.assert_array_equal(prob, wp)


def test_a_hot_row_does_not_depend_on_its_batch():
    """Few rows are split over blocks, many have a block each."""
    rows, vocab = 140, 20011
    l = rows_of("every value", rows, vocab, 3).bfloat16().cuda()
    rng = np.random.default_rng(1)
    u, p, T = rng.random(rows), rng.uniform(0.2, 0.99, rows), rng.uniform(50, 5000, rows)
    token, prob = draw(l, BF16, vocab, rows, vocab, T, None, p, None, u)
    for r0 in range(0, rows, 35):
        at = slice(r0, r0 + 35)
        tk, pr = draw(l[at].contiguous(), BF16, vocab, 35, vocab, T[at], None, p[at], None, u[at])
        np.testing.assert_array_equal(tk, token[at])
        np.testing.assert_array_equal(pr, prob[at])
