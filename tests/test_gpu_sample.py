"""tfe_sample against the 64-bit oracle.

The weights' relative error against exact ones: (l - M), 1 / T and their product
are rounded (3 2^-24 of an exponent of at most 22.2, beyond which a weight is 0),
the exponential is within 2^-23 and the weight rounded by half a unit of 2^31:
below 4.2e-6 for weights that matter.  Where every comparison that an answer
rests on is decided by more than 5e-6 of what it compares, the token has to be
the oracle's and its probability within 1e-5.  Elsewhere (the far tail's steps are
smaller than that) it has to lie, in the order of weights known to their error,
between the oracle's answers for settings and u moved by 1e-5 to either side."""
import numpy as np
import pytest
import torch

from oracle import logits as O
from paper_2607_07388_amd import tfe

from . import harness as H

pytestmark = pytest.mark.gpu

F32, BF16 = tfe.TFE_F32, tfe.TFE_BF16
TORCH = {F32: torch.float32, BF16: torch.bfloat16}
CLEAR = 5e-6
WEIGHT = 4.2e-6  # a weight's relative error


class Out:
    def __init__(self, rows):
        self.token = torch.full((rows,), -9, dtype=torch.int32, device="cuda")
        self.prob = torch.full((rows,), -9.0, dtype=torch.float32, device="cuda")

    def numpy(self):
        return self.token.cpu().numpy(), self.prob.cpu().numpy()


def dev(x, dtype):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x, dtype)).cuda()


def draw(logits, dtype, ld, rows, vocab, T=None, k=None, p=None, m=None, u=None, stream=None):
    out = Out(rows)
    size = tfe.tfe_sample_workspace(rows, vocab)
    space = torch.full((size + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    args = [dev(T, np.float32), dev(k, np.int32), dev(p, np.float32), dev(m, np.float32), dev(u, np.float32)]
    tfe.tfe_sample(logits, dtype, ld, rows, vocab, *args, out.token, out.prob, space, size,
                   stream or H.cur_stream())
    torch.cuda.synchronize()
    assert (space[size:] == 0xA5).all()
    return out.numpy()


def tensor(l, dtype, pad=0):
    rows, vocab = l.shape
    t = torch.full((rows, vocab + pad), float("inf"), dtype=TORCH[dtype], device="cuda")
    t[:, :vocab] = torch.from_numpy(np.ascontiguousarray(l, np.float32)).cuda().to(TORCH[dtype])
    return t, vocab + pad


def check(l, dtype, T=None, k=None, p=None, m=None, u=None, pad=0):
    rows, vocab = l.shape
    t, ld = tensor(l, dtype, pad)
    seen = t[:, :vocab].float().cpu().numpy()
    u = np.random.default_rng(vocab + rows).random(rows).astype(np.float32) if u is None else u
    token, prob = draw(t, dtype, ld, rows, vocab, T, k, p, m, u)
    for r in range(rows):
        pick = lambda x, d: d if x is None else float(np.float32(x[r]))  # noqa: E731
        at = [pick(T, 1.0), 0 if k is None else int(k[r]), pick(p, 1.0), pick(m, 0.0), float(np.float32(u[r]))]
        want, wp, margin = O.sample(seen[r], *at)
        if margin >= CLEAR:
            assert token[r] == want, (r, token[r], want, margin)
            assert abs(prob[r] - wp) <= 1e-5 * wp, (r, prob[r], wp)
            continue
        near = [O.sample(seen[r], at[0], at[1], at[2] * (1 + i * 1e-5) if at[2] < 1 else 1.0,
                         at[3] * (1 + j * 1e-5), at[4] + n * 1e-5)[0]
                for i in (-1, 1) for j in (-1, 1) for n in (-1, 1)]
        l64 = seen[r].astype(float)
        w = np.exp((l64[near] - l64[token[r]]) / at[0])
        assert w.min() <= 1 + 2 * WEIGHT and w.max() >= 1 - 2 * WEIGHT, (r, token[r], want, margin)


def language(seed, rows, vocab, sigma=1.5):
    rng = np.random.default_rng(seed)
    l = rng.standard_normal((rows, vocab)) * sigma - 0.8 * np.log(1 + np.arange(vocab))
    l[np.arange(rows)[:, None], rng.integers(0, vocab, (rows, 8))] = rng.standard_normal((rows, 8)) * 2 + 3
    return l


def settings(seed, rows, vocab):
    """Every combination of filters, in turn."""
    rng = np.random.default_rng(seed)
    n = np.arange(rows)
    T = rng.uniform(0.3, 1.5, rows)
    T[n % 11 == 10] = 0.0
    k = np.where(n & 1, rng.integers(1, max(2, min(vocab, 100)), rows), 0)
    p = np.where(n & 2, rng.uniform(0.3, 0.999, rows), 1.0)
    m = np.where(n & 4, rng.uniform(0.001, 0.2, rows), 0.0)
    return T, k, p, m


@pytest.mark.parametrize("rows,vocab,dtype,pad", [
    (24, 1, F32, 0), (24, 2, BF16, 1), (24, 7, F32, 0), (48, 63, BF16, 2), (48, 64, F32, 1), (48, 1000, BF16, 0),
    (24, 4097, F32, 3), (16, 33333, BF16, 5), (9, 151936, F32, 0), (16, 151936, BF16, 1), (3, 1 << 18, F32, 0),
    (300, 3001, BF16, 0), (1, 151936, BF16, 0), (2, 50000, F32, 7)])
def test_filters(rows, vocab, dtype, pad):
    check(language(rows + vocab, rows, vocab), dtype, *settings(vocab, rows, vocab), pad=pad)


@pytest.mark.parametrize("rows,vocab", [(5, 3001), (2, 151936)])
def test_no_settings(rows, vocab):
    """Every optional array left out: temperature 1, nothing filtered."""
    check(language(3, rows, vocab), F32)


@pytest.mark.parametrize("which", ["k", "p", "m", "T"])
@pytest.mark.parametrize("rows,vocab", [(40, 5000), (6, 151936)])
def test_one_setting(rows, vocab, which):
    T, k, p, m = settings(1, rows, vocab)
    every = {"T": np.maximum(T, 0.3), "k": np.maximum(k, 1), "p": np.minimum(p, 0.97), "m": np.maximum(m, 0.01)}
    check(language(4, rows, vocab), BF16, **{which: every[which]})


@pytest.mark.parametrize("vocab", [300, 5000, 151936])
def test_flat_rows(vocab):
    """Equal logits: every token has the same weight, the order is the tokens'."""
    rows = 6
    l = np.zeros((rows, vocab))
    l[1] = -3.5
    l[2] = np.finfo(np.float32).min  # a mask's value in every place
    l[3, : vocab // 2] = 1.0
    u = np.array([0.0, 0.25, 0.5, 0.99, 0.7, 1.0 - 2.0 ** -24], np.float32)
    check(l, F32, u=u)
    token, prob = draw(*tensor(l[:1].repeat(4, 0), F32)[:1], F32, vocab, 4, vocab, u=[0.0, 0.25, 0.5, 0.75])
    np.testing.assert_array_equal(token, np.floor(vocab * np.array([0, 0.25, 0.5, 0.75])).astype(int))
    np.testing.assert_allclose(prob, 1 / vocab, rtol=1e-6)
    # Of equal ones, top-k and top-p keep the lowest tokens.
    token, prob = draw(tensor(l[:1].repeat(3, 0), F32)[0], F32, vocab, 3, vocab, k=[7, 0, 7], p=[1.0, 0.5, 0.5],
                       u=[0.999, 0.999, 0.999])
    half = vocab // 2 if vocab % 2 == 0 else vocab // 2 + 1
    np.testing.assert_array_equal(token, [6, int(np.float32(0.999).astype(float) * half), 3])


@pytest.mark.parametrize("vocab", [700, 40000])
def test_narrow_rows(vocab):
    """Logits so near each other that thousands share every coarse step of the weights."""
    rng = np.random.default_rng(8)
    l = rng.standard_normal((12, vocab)) * 0.01
    T, k, p, m = settings(2, 12, vocab)
    k = np.where(k > 0, vocab // 3, 0)
    m[:] = 0
    check(l, F32, np.maximum(T, 0.5), k, p, m)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masks_infinities_and_nan(dtype):
    vocab = 2000
    base = language(9, 8, vocab)
    base[0, :] = -np.inf                      # nothing left: -1
    base[1, 5:] = -np.inf                     # five tokens left
    base[2, ::2] = np.nan                     # NaN is never drawn
    base[3, :] = np.nan
    base[4, 100], base[4, 50] = np.inf, np.inf  # they share all
    base[5, 1:] = torch.finfo(TORCH[dtype]).min
    base[6, :] = -np.inf
    base[6, 77] = -1e30
    u = np.full(8, 0.6, np.float32)
    for p in (None, np.full(8, 0.9)):
        t, ld = tensor(base, dtype)
        token, prob = draw(t, dtype, ld, 8, vocab, p=p, u=u)
        assert token[0] == -1 and prob[0] == 0 and token[3] == -1 and prob[3] == 0
        assert 0 <= token[1] < 5 and token[2] % 2 == 1
        assert token[4] == 100 and prob[4] == 0.5
        assert token[5] == 0 and prob[5] == 1 and token[6] == 77 and prob[6] == 1
        check(base[[1, 2, 5, 6, 7]], dtype, p=None if p is None else p[:5], u=u[:5])
    # Greedy: the first of the largest.
    token, prob = draw(t, dtype, ld, 8, vocab, T=np.zeros(8), u=u)
    assert token[4] == 50 and prob[4] == 1 and token[0] == -1


def test_settings_out_of_range():
    l = language(10, 12, 500)
    nan = np.float32(np.nan)
    T = [nan, -1.0, 0.0, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0]
    k = [0, 0, 0, -5, 10 ** 9, 0, 0, 0, 0, 0, 0, 0]
    p = [1.0, 1.0, 1.0, 1.0, 1.0, nan, 1.5, -2.0, 0.0, 1.0, 1.0, 1.0]
    m = [0.0] * 8 + [0.0, nan, -1.0, 7.0]
    u = [0.5, 0.5, 0.5, 0.3, 0.3, 0.3, 0.3, 0.9, 0.9, 0.3, 0.3, 0.9]
    t, ld = tensor(l, F32)
    token, prob = draw(t, F32, ld, 12, 500, T, k, p, m, u)
    best = l.astype(np.float32).argmax(1)
    for r in (0, 1, 2, 7, 8, 11):
        assert token[r] == best[r] and prob[r] == 1
    rest = np.array([3, 4, 5, 6, 9, 10])
    plain, pp = draw(tensor(l[rest], F32)[0], F32, ld, 6, 500, u=np.array(u)[rest])
    np.testing.assert_array_equal(token[rest], plain)
    np.testing.assert_array_equal(prob[rest], pp)
    lo, _ = draw(t, F32, ld, 12, 500, u=[-1.0, nan, 0.0] * 4)
    zero, _ = draw(t, F32, ld, 12, 500, u=[0.0] * 12)
    np.testing.assert_array_equal(lo, zero)
    hi, _ = draw(t, F32, ld, 12, 500, u=[1.0, 5.0, float("inf")] * 4)
    w = np.rint(2.0 ** 31 * np.exp(l.astype(np.float32).astype(float) - l.max(1, keepdims=True)))
    for r in range(12):
        assert w[r, hi[r]] == min(w[r][w[r] > 0]) or w[r, hi[r]] < 2


def test_extreme_temperatures():
    l = language(11, 4, 3000)
    t, ld = tensor(l, F32)
    seen = l.astype(np.float32)
    token, _ = draw(t, F32, ld, 4, 3000, T=[1e-30, 1e-40, 1e30, float("inf")], u=[0.9, 0.9, 0.5, 0.5])
    assert token[0] == seen[0].argmax() and token[1] == seen[1].argmax()
    # Infinitely hot: all alike, in the order of the tokens.
    assert token[3] == 1500 and token[2] == 1500


def test_order_and_distribution():
    """u runs over [0, 1): each token comes as often as its probability says, larger ones first."""
    l = np.log(np.array([[0.1, 0.4, 0.2, 0.3]]))
    n = 1000
    u = (np.arange(n) + 0.5) / n
    token, prob = draw(tensor(l.repeat(n, 0), F32)[0], F32, 4, n, 4, u=u)
    np.testing.assert_array_equal(token, np.repeat([1, 3, 2, 0], [400, 300, 200, 100]))
    np.testing.assert_allclose(prob, np.exp(l[0])[token], rtol=1e-5)


@pytest.mark.parametrize("rows", [1, 5, 64, 300])
def test_same_rows_same_tokens_however_many(rows):
    """A row's token does not depend on the batch it comes in (nor, so, on how it is split)."""
    l = language(12, 5, 40001)
    T, k, p, m = settings(6, 5, 40001)
    u = np.array([0.1, 0.35, 0.6, 0.85, 0.99])
    want = [draw(tensor(l[r:r + 1], BF16)[0], BF16, 40001, 1, 40001, T[r:r + 1], k[r:r + 1], p[r:r + 1], m[r:r + 1],
                 u[r:r + 1]) for r in range(5)]
    n = np.arange(rows) % 5
    token, prob = draw(tensor(l[n], BF16)[0], BF16, 40001, rows, 40001, T[n], k[n], p[n], m[n], u[n])
    np.testing.assert_array_equal(token, np.array([w[0][0] for w in want])[n])
    np.testing.assert_array_equal(prob, np.array([w[1][0] for w in want])[n])


@pytest.mark.parametrize("rows", [2, 300])
def test_captured_and_on_another_stream(rows):
    vocab = 5000
    ls = [tensor(language(20 + i, rows, vocab), F32)[0] for i in range(3)]
    T, k, p, m = (dev(x, d) for x, d in zip(settings(3, rows, vocab), (np.float32, np.int32, np.float32, np.float32)))
    u = dev(np.random.default_rng(1).random(rows), np.float32)
    size = tfe.tfe_sample_workspace(rows, vocab)

    def call(l, out, space, stream):
        tfe.tfe_sample(l, F32, vocab, rows, vocab, T, k, p, m, u, out.token, out.prob, space, size, stream)

    scratch = lambda: torch.empty(max(16, size), dtype=torch.uint8, device="cuda")  # noqa: E731
    want = []
    for l in ls:
        o = Out(rows)
        call(l, o, scratch(), H.cur_stream())
        want.append(o)
    side, o, space = torch.cuda.Stream(), Out(rows), scratch()
    side.wait_stream(torch.cuda.current_stream())
    call(ls[1], o, space, side.cuda_stream)
    side.synchronize()
    assert torch.equal(o.token, want[1].token) and torch.equal(o.prob, want[1].prob)
    l, o = ls[0].clone(), Out(rows)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(l, o, space, torch.cuda.current_stream().cuda_stream)
    for i in (1, 2, 0, 1):
        l.copy_(ls[i])
        g.replay()
        assert torch.equal(o.token, want[i].token) and torch.equal(o.prob, want[i].prob)


def test_no_rows_and_no_probabilities():
    assert tfe.tfe_sample(None, F32, 10, 0, 10, None, None, None, None, None, None, None, None, 0) == 0
    l = language(13, 3, 100)
    t, ld = tensor(l, F32)
    want, _ = draw(t, F32, ld, 3, 100, u=[0.2, 0.5, 0.8])
    token = torch.empty(3, dtype=torch.int32, device="cuda")
    size = tfe.tfe_sample_workspace(3, 100)
    tfe.tfe_sample(t, F32, ld, 3, 100, None, None, None, None, dev([0.2, 0.5, 0.8], np.float32), token, None,
                   torch.empty(max(16, size), dtype=torch.uint8, device="cuda"), size, H.cur_stream())
    np.testing.assert_array_equal(token.cpu().numpy(), want)


@pytest.mark.parametrize("vocab", [2999, 70001])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_many_rows_of_every_kind(vocab, dtype):
    """Batches whose rows each have a block of their own: masks, infinities, NaN, flat and
    narrow rows, logits near zero, beyond 256 and of the type's lowest value, with every
    combination of filters."""
    kinds, rows = 12, 132
    rng = np.random.default_rng(vocab)
    l = language(30, rows, vocab)
    kind = np.arange(rows) // 11 % kinds
    for r in range(rows):
        k = kind[r]
        if k == 1:
            l[r] = 1.25
        elif k == 2:
            l[r, rng.random(vocab) < 0.7] = -np.inf
        elif k == 3:
            l[r, ::3] = np.nan
        elif k == 4:
            l[r, vocab // 3:] = torch.finfo(TORCH[dtype]).min
        elif k == 5:
            l[r] = rng.standard_normal(vocab) * 2e-3       # small ones alone
        elif k == 6:
            l[r] = rng.standard_normal(vocab) * 0.02       # around zero
        elif k == 7:
            l[r] += 300.0                                  # beyond the binned range
        elif k == 8:
            l[r] -= 300.0
        elif k == 9:
            l[r] = np.round(l[r])                          # heavy ties
        elif k == 10:
            l[r] = -np.abs(l[r]) - 1.0                     # no positive one
    T, k, p, m = settings(31, rows, vocab)
    T = np.where(kind == 11, 8.0, T)  # hot: the tail's weights matter
    check(l, dtype, T, k, p, m, pad=vocab % 3)
    t, ld = tensor(l, dtype)
    u = rng.random(rows)
    token, prob = draw(t, dtype, ld, rows, vocab, T, k, p, m, u)
    for r0 in range(0, rows, 44):  # fewer rows: split over blocks instead
        at = slice(r0, r0 + 44)
        tk, pr = draw(t[at].contiguous(), dtype, ld, 44, vocab, T[at], k[at], p[at], m[at], u[at])
        np.testing.assert_array_equal(tk, token[at])
        np.testing.assert_array_equal(pr, prob[at])


def test_many_rows_without_a_token():
    rows = 140
    l = np.full((rows, 300), -np.inf)
    l[1::2] = np.nan
    l[7, 3] = 2.0
    for dtype in (F32, BF16):
        t, ld = tensor(l, dtype)
        token, prob = draw(t, dtype, ld, rows, 300, u=np.full(rows, 0.5))
        assert token[7] == 3 and prob[7] == 1
        rest = np.arange(rows) != 7
        assert (token[rest] == -1).all() and (prob[rest] == 0).all()
