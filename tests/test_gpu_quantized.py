"""The 8-bit layout and product through the C ABI against the 64-bit oracle.

Codes and scales have to be the oracle's.  A product's exact terms are summed in
float32, so a float32 result is within P 2^-24 sum |a w| of the exact one (P
terms, each addition rounds a partial sum of at most sum |a w| by 2^-24).  A
bfloat16 result may come from the 8-bit matrix instruction, whose sums are
allowed 2^-11 sum |a w|, and is rounded by 2^-8 of itself at most."""
import numpy as np
import pytest
import torch

from oracle import logits as O
from paper_2607_07388_amd import tfe

from . import harness as H

pytestmark = pytest.mark.gpu

F32, BF16 = tfe.TFE_F32, tfe.TFE_BF16
TORCH = {F32: torch.float32, BF16: torch.bfloat16}


def device(x, dtype, pad=0):
    """x on the GPU, its rows `pad` elements further apart; (tensor, pitch)."""
    rows, cols = x.shape
    t = torch.full((rows, cols + pad), float("nan"), dtype=TORCH[dtype], device="cuda")
    t[:, :cols] = torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().to(TORCH[dtype])
    return t, cols + pad


def pitches(dim):
    kb = -(-dim // 128)
    return kb * 128, -(-kb // 4) * 4


def quantize(x, dtype, block_rows, pad=0):
    rows, dim = x.shape
    t, ld = device(x, dtype, pad)
    p, q = pitches(dim)
    codes = torch.full((rows, p), 0x55, dtype=torch.uint8, device="cuda")
    scales = torch.full((-(-rows // block_rows), q), 0x55, dtype=torch.uint8, device="cuda")
    tfe.tfe_quantize(t, dtype, ld, rows, dim, block_rows, codes, scales, H.cur_stream())
    seen = t[:, :dim].float().cpu().numpy()
    return codes, scales, seen


def same_codes(got, want):
    got = got.cpu().numpy()
    nan = (want & 127) == 127
    np.testing.assert_array_equal((got & 127) == 127, nan)
    # A zero's sign has no meaning in a product.
    np.testing.assert_array_equal(np.where(nan | (want == 128), 0, want),
                                  np.where(nan | (got == 128), 0, got))


@pytest.mark.parametrize("rows,dim,block_rows,dtype,pad", [
    (1, 1, 1, F32, 0), (3, 127, 1, BF16, 1), (5, 128, 1, F32, 3), (7, 129, 1, BF16, 0),
    (64, 1024, 1, BF16, 0), (33, 1000, 1, F32, 5), (2, 4097, 1, BF16, 7),
    (1, 1, 128, F32, 0), (127, 130, 128, BF16, 1), (128, 512, 128, F32, 0),
    (129, 513, 128, BF16, 0), (300, 1000, 128, F32, 3)])
def test_layout(rows, dim, block_rows, dtype, pad):
    rng = np.random.default_rng(rows + dim)
    x = rng.standard_normal((rows, dim)) * 2.0 ** rng.integers(-20, 20, (rows, 1))
    codes, scales, seen = quantize(x, dtype, block_rows, pad)
    want_codes, want_scales = O.fp8_layout(seen, block_rows)
    same_codes(codes, want_codes)
    np.testing.assert_array_equal(scales.cpu().numpy(), want_scales)


def test_layout_of_every_rounding_case():
    """Every code, every midpoint of neighbours and the values beside it, as they stand."""
    v = O.e4m3_values()[:127]
    mid = (v[1:] + v[:-1]) / 2
    x = np.concatenate([v, mid, np.nextafter(mid.astype(np.float32), np.float32(0)),
                        np.nextafter(mid.astype(np.float32), np.float32(1e9))])
    x = np.concatenate([x, -x])
    x = np.concatenate([x, np.zeros(-x.size % 127)]).reshape(-1, 127)
    x = np.concatenate([x, np.full((x.shape[0], 1), 448.0)], 1)  # scale 1 in every row
    codes, scales, seen = quantize(x, F32, 1)
    want_codes, want_scales = O.fp8_layout(seen, 1)
    assert (want_scales[:, 0] == 127).all()
    same_codes(codes, want_codes)
    np.testing.assert_array_equal(scales.cpu().numpy(), want_scales)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_layout_of_extremes(block_rows):
    """Zeros, infinities, NaN, the largest and the least numbers."""
    x = np.ones((130, 256), np.float32)
    x[0] = 0
    x[1, 3], x[1, 4], x[1, 200] = np.inf, -np.inf, np.nan
    x[2] = np.finfo(np.float32).max
    x[3] = np.finfo(np.float32).tiny
    x[4] = 1e-42
    x[5, 128:] = -np.inf
    if block_rows == 128:
        x[2] = 1
    codes, scales, seen = quantize(x, F32, block_rows)
    want_codes, want_scales = O.fp8_layout(seen, block_rows)
    same_codes(codes, want_codes)
    np.testing.assert_array_equal(scales.cpu().numpy(), want_scales)


def check_product(got, a, w, out_dtype):
    exact = a @ w.T
    size = np.abs(a) @ np.abs(w).T
    got = got.float().cpu().numpy().astype(np.float64)
    if out_dtype == F32:
        bound = a.shape[1] * 2.0 ** -24 * size
    else:
        bound = 2.0 ** -8 * np.abs(exact) + 2.0 ** -11 * size
    bad = np.abs(got - exact) > bound + 1e-37
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], exact[bad][:5], bound[bad][:5])


SHAPES = [(1, 1, 1), (1, 17, 128), (2, 300, 129), (16, 64, 256), (17, 1000, 1024), (33, 129, 1000),
          (64, 4096, 512), (65, 255, 640), (100, 3001, 256), (128, 513, 1024), (130, 1025, 384),
          (257, 777, 1000), (300, 2000, 1300), (513, 1300, 512), (1030, 515, 256), (3, 130, 5000)]


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("rows,n,dim", SHAPES)
def test_product(rows, n, dim, out_dtype):
    rng = np.random.default_rng(rows * 7 + n + dim)
    x = rng.standard_normal((rows, dim)) * 2.0 ** rng.integers(-6, 6, (rows, 1))
    w = rng.standard_normal((n, dim)) * 0.1 * 2.0 ** rng.integers(-4, 4, (1, dim))
    ac, asc, _ = quantize(x, F32, 1)
    wc, wsc, _ = quantize(w, F32, 128)
    pad = n % 3
    out = torch.full((rows, n + pad), -7.0, dtype=TORCH[out_dtype], device="cuda")
    tfe.tfe_quantized_matmul(ac, asc, wc, wsc, rows, n, dim, out, out_dtype, n + pad, H.cur_stream())
    a = O.fp8_values(ac.cpu().numpy(), asc.cpu().numpy(), 1)
    v = O.fp8_values(wc.cpu().numpy(), wsc.cpu().numpy(), 128)
    check_product(out[:, :n], a, v, out_dtype)
    assert (out[:, n:] == -7).all()
    # In one call, from the hidden states; the workspace and what lies behind it.
    size = tfe.tfe_quantized_workspace(rows, dim)
    space = torch.full((size + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    t, ld = device(x, F32, 1)
    again = torch.full_like(out, -7.0)
    tfe.tfe_quantized_linear(t, F32, ld, wc, wsc, rows, n, dim, again, out_dtype, n + pad, space, size,
                       H.cur_stream())
    check_product(again[:, :n], a, v, out_dtype)
    assert (again[:, n:] == -7).all() and (space[size:] == 0xA5).all()


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("rows,n,dim", [(1, 515, 1024), (64, 260, 1000), (200, 700, 512), (600, 515, 128)])
def test_small_integers_are_exact(rows, n, dim, out_dtype):
    """Integers of at most 15 in magnitude are codes; their products' sums here are below 2^8
    (sparse), so each is a float32 and a bfloat16."""
    rng = np.random.default_rng(n)
    x = rng.integers(-2, 3, (rows, dim)).astype(np.float64) * (rng.random((rows, dim)) < 16 / dim)
    w = rng.integers(-2, 3, (n, dim)).astype(np.float64)
    x[:, 0], w[:, 0] = 0, 0
    exact = x @ w.T
    assert np.abs(exact).max() < 256
    ac, asc, _ = quantize(x, BF16, 1)
    wc, wsc, _ = quantize(w, BF16, 128)
    out = torch.empty((rows, n), dtype=TORCH[out_dtype], device="cuda")
    tfe.tfe_quantized_matmul(ac, asc, wc, wsc, rows, n, dim, out, out_dtype, n, H.cur_stream())
    np.testing.assert_array_equal(out.float().cpu().numpy(), exact)


@pytest.mark.parametrize("rows", [1, 20, 200])
@pytest.mark.parametrize("out_dtype", [F32, BF16])
def test_nan_and_infinity_stay_in_their_rows(rows, out_dtype):
    rng = np.random.default_rng(5)
    x = rng.standard_normal((rows, 300))
    w = rng.standard_normal((500, 300))
    x[rows // 2, 7] = np.nan
    wc, wsc, _ = quantize(w, F32, 128)
    t, ld = device(x, F32)
    out = torch.empty((rows, 500), dtype=TORCH[out_dtype], device="cuda")
    size = tfe.tfe_quantized_workspace(rows, 300)
    tfe.tfe_quantized_linear(t, F32, ld, wc, wsc, rows, 500, 300, out, out_dtype, 500,
                       torch.empty(size, dtype=torch.uint8, device="cuda"), size, H.cur_stream())
    nan = out.isnan().cpu().numpy()
    assert nan[rows // 2].all() and nan.sum() == 500


@pytest.mark.parametrize("rows,out_dtype", [(1, F32), (64, BF16), (300, BF16), (300, F32)])
def test_captured_and_on_another_stream(rows, out_dtype):
    """A linear call captured in a graph and replayed on inputs that change in between, and one
    on a stream of its own, give the eager answers."""
    rng = np.random.default_rng(rows)
    n, dim = 1000, 512
    wc, wsc, _ = quantize(rng.standard_normal((n, dim)), F32, 128)
    xs = [device(rng.standard_normal((rows, dim)), BF16)[0] for _ in range(3)]
    size = tfe.tfe_quantized_workspace(rows, dim)

    def call(x, out, space, stream):
        tfe.tfe_quantized_linear(x, BF16, dim, wc, wsc, rows, n, dim, out, out_dtype, n, space, size, stream)

    new = lambda: torch.empty((rows, n), dtype=TORCH[out_dtype], device="cuda")  # noqa: E731
    scratch = lambda: torch.empty(size, dtype=torch.uint8, device="cuda")  # noqa: E731
    want = [new() for _ in xs]
    space = scratch()
    for x, o in zip(xs, want):
        call(x, o, space, H.cur_stream())
    side, o = torch.cuda.Stream(), new()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(xs[1], o, scratch(), side.cuda_stream)
    side.synchronize()
    assert torch.equal(o, want[1])
    x, o, space = xs[0].clone(), new(), scratch()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(x, o, space, torch.cuda.current_stream().cuda_stream)
    for k in (1, 2, 0, 1):
        x.copy_(xs[k])
        g.replay()
        assert torch.equal(o, want[k])


def test_no_rows():
    wc, wsc, _ = quantize(np.ones((4, 4)), F32, 128)
    assert tfe.tfe_quantized_linear(None, F32, 4, wc, wsc, 0, 4, 4, None, F32, 4, None, 0) == 0


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("rows,n,dim", [(400, 70000, 130), (513, 66000, 384), (300, 66001, 520)])
def test_large_tiles(rows, n, dim, out_dtype):
    """Enough columns and rows for the largest tiles, with ragged ends."""
    rng = np.random.default_rng(n)
    ac, asc, _ = quantize(rng.standard_normal((rows, dim)), F32, 1)
    wc, wsc, _ = quantize(rng.standard_normal((n, dim)) * 0.1, F32, 128)
    out = torch.full((rows, n), -7.0, dtype=TORCH[out_dtype], device="cuda")
    tfe.tfe_quantized_matmul(ac, asc, wc, wsc, rows, n, dim, out, out_dtype, n, H.cur_stream())
    a = O.fp8_values(ac.cpu().numpy(), asc.cpu().numpy(), 1)
    w = O.fp8_values(wc.cpu().numpy(), wsc.cpu().numpy(), 128)
    some = np.unique(np.concatenate([np.arange(0, n, 97), np.arange(n - 300, n), np.arange(300)]))
    at = torch.from_numpy(some).cuda()
    check_product(out[:, at], a, w[some], out_dtype)


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [3, 100])
def test_extreme_scales(rows, out_dtype):
    """Blocks at either end of the scales: hidden states of 1e-36 and of 1e30 under weights of
    1e30 and 1e-30."""
    rng = np.random.default_rng(rows)
    x = rng.uniform(0.5, 1, (rows, 256)) * np.where(np.arange(rows)[:, None] % 2 == 0, 1e-36, 1e30)
    w = rng.uniform(-1, 1, (200, 256)) * np.where(np.arange(256) < 128, 1e30, 1e-30)
    ac, asc, seen = quantize(x, F32, 1)
    wc, wsc, _ = quantize(w, F32, 128)
    out = torch.empty((rows, 200), dtype=TORCH[out_dtype], device="cuda")
    x[1::2, :128] = 0
    ac, asc, _ = quantize(x, F32, 1)
    tfe.tfe_quantized_matmul(ac, asc, wc, wsc, rows, 200, 256, out, out_dtype, 200, H.cur_stream())
    check_product(out, O.fp8_values(ac.cpu().numpy(), asc.cpu().numpy(), 1),
                  O.fp8_values(wc.cpu().numpy(), wsc.cpu().numpy(), 128), out_dtype)
