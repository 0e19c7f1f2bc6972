"""The integer layout and product through the C ABI against the 64-bit oracle.

Codes and scales are the oracle's to the bit.  A product's sum is exact; it is converted to float32
and multiplied by two scales, three roundings of 2^-24, and a bfloat16 result by 2^-8 more."""
import numpy as np
import pytest
import torch

from oracle import learn as O
from paper_2607_07388_amd import tfe

from . import harness as H

pytestmark = pytest.mark.gpu

F32, BF16 = tfe.TFE_F32, tfe.TFE_BF16
TORCH = {F32: torch.float32, BF16: torch.bfloat16}


def device(x, dtype, pad=0):
    rows, cols = x.shape
    t = torch.full((rows, cols + pad), float("nan"), dtype=TORCH[dtype], device="cuda")
    t[:, :cols] = torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().to(TORCH[dtype])
    return t, cols + pad


def quantize(x, dtype, pad=0):
    rows, dim = x.shape
    t, ld = device(x, dtype, pad)
    codes = torch.full((rows, -(-dim // 128) * 128), 0x55, dtype=torch.int8, device="cuda")
    scales = torch.full((rows,), -7.0, device="cuda")
    tfe.tfe_integer_quantize(t, dtype, ld, rows, dim, codes, scales, H.cur_stream())
    return codes, scales, t[:, :dim].float().cpu().numpy()


@pytest.mark.parametrize("rows,dim,dtype,pad", [
    (1, 1, F32, 0), (3, 127, BF16, 1), (5, 128, F32, 3), (7, 129, BF16, 0), (64, 1024, BF16, 0), (33, 1000, F32, 5),
    (2, 4097, BF16, 7), (9, 513, F32, 0), (1, 65536, BF16, 0), (300, 1000, BF16, 3), (1, 65535, F32, 1)])
def test_layout(rows, dim, dtype, pad):
    rng = np.random.default_rng(rows + dim)
    x = rng.standard_normal((rows, dim)) * 2.0 ** rng.integers(-90, 90, (rows, 1))
    codes, scales, seen = quantize(x, dtype, pad)
    want_codes, want_scales = O.integer_layout(seen)
    np.testing.assert_array_equal(codes.cpu().numpy(), want_codes)
    np.testing.assert_array_equal(scales.cpu().numpy(), want_scales)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_layout_of_odd_rows(dtype):
    """Zeros, infinities, NaN, rows too small for a scale, ties, the type's largest numbers, subnormals."""
    big = 3e38
    x = np.zeros((12, 300))
    x[1, 299] = 2.0 ** -101
    x[2, 7] = 2.0 ** -100
    x[3, 7] = 2.0 ** -99
    x[4, :3] = np.inf, -np.inf, 1.0
    x[5, 290] = np.nan
    x[6, :] = np.nan
    x[7, :4] = big, -big, big / 2, big / 300
    x[8, :254] = (np.arange(254) - 127) / 2.0
    x[9, 0] = -np.inf
    x[10, :3] = 1e-45, 1e-40, 1e-38
    x[11, :3] = 1e-45, 1e-38, 1.0
    codes, scales, seen = quantize(x, dtype)
    want_codes, want_scales = O.integer_layout(seen)
    np.testing.assert_array_equal(codes.cpu().numpy(), want_codes)
    np.testing.assert_array_equal(scales.cpu().numpy(), want_scales)


def check(out, sums, exact, out_dtype):
    got = out.double().cpu().numpy()
    bound = (4 * 2.0 ** -24 + (2.0 ** -8 if out_dtype == BF16 else 0)) * np.abs(exact) + 1e-37
    assert (np.abs(got - exact) <= bound).all()


SHAPES = [(1, 1, 1), (1, 16, 128), (1, 1000, 300), (2, 257, 129), (7, 300, 128), (16, 515, 1000), (17, 129, 256),
          (33, 1024, 640), (48, 777, 1024), (64, 2000, 1000), (65, 300, 130), (100, 1111, 512), (128, 128, 4096),
          (200, 333, 1000), (257, 700, 130), (300, 5001, 256), (600, 1100, 100), (5, 40, 65536), (70, 90, 30000),
          (64, 40, 2048), (40, 100, 1500)]


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("rows,n,dim", SHAPES)
def test_product(rows, n, dim, out_dtype):
    rng = np.random.default_rng(rows * 7 + n + dim)
    pad = int(rng.integers(0, 4))
    ac, asc, seen = quantize(rng.standard_normal((rows, dim)), BF16)
    wc, wsc, _ = quantize(rng.standard_normal((n, dim)) * rng.uniform(0.01, 1, (n, 1)), F32)
    sums, exact = O.integer_product(ac.cpu().numpy(), asc.cpu().numpy(), wc.cpu().numpy(), wsc.cpu().numpy())
    size = tfe.tfe_integer_workspace(rows, dim)
    space = torch.full((size,), 0x7F, dtype=torch.uint8, device="cuda")
    t, ld = device(seen, BF16, 5)
    a, b = (torch.full((rows, n + pad), -7.0, dtype=TORCH[out_dtype], device="cuda") for _ in range(2))
    tfe.tfe_integer_matmul(ac, asc, wc, wsc, rows, n, dim, a, out_dtype, n + pad, H.cur_stream())
    tfe.tfe_integer_linear(t, BF16, ld, wc, wsc, rows, n, dim, b, out_dtype, n + pad, space, size, H.cur_stream())
    check(a[:, :n], sums, exact, out_dtype)
    assert torch.equal(a, b) and (a[:, n:] == -7).all()


@pytest.mark.parametrize("rows", [1, 3, 16, 40, 64, 65, 130, 300])
def test_sums_are_exact(rows):
    """Codes at their limits, the longest rows: sums near 2^30, scales 1, so that float32 results are
    the sums rounded once."""
    dim, n = 65536, 70
    rng = np.random.default_rng(rows)
    a = rng.integers(-127, 128, (rows, dim)).astype(np.int8)
    w = rng.integers(-127, 128, (n, dim)).astype(np.int8)
    a[0], w[0], w[1] = 127, 127, -127
    at, wt = torch.from_numpy(a).cuda(), torch.from_numpy(w).cuda()
    one = torch.ones(max(rows, n), device="cuda")
    out = torch.empty((rows, n), device="cuda")
    tfe.tfe_integer_matmul(at, one, wt, one, rows, n, dim, out, F32, n, H.cur_stream())
    sums = torch.mm(at.double(), wt.double().t().contiguous())
    assert sums.abs().max() == 127 ** 2 * dim and torch.equal(out, sums.float())


def test_a_row_does_not_depend_on_its_batch():
    rng = np.random.default_rng(4)
    n, dim = 1500, 384
    ac, asc, _ = quantize(rng.standard_normal((600, dim)), F32)
    wc, wsc, _ = quantize(rng.standard_normal((n, dim)), F32)
    for out_dtype in (F32, BF16):
        want = torch.empty((600, n), dtype=TORCH[out_dtype], device="cuda")
        tfe.tfe_integer_matmul(ac, asc, wc, wsc, 600, n, dim, want, out_dtype, n, H.cur_stream())
        for rows in (1, 2, 16, 17, 33, 64, 65, 128, 257, 599):
            out = torch.empty((rows, n), dtype=TORCH[out_dtype], device="cuda")
            tfe.tfe_integer_matmul(ac, asc, wc, wsc, rows, n, dim, out, out_dtype, n, H.cur_stream())
            assert torch.equal(out, want[:rows])


@pytest.mark.parametrize("rows", [1, 20, 200, 300])
@pytest.mark.parametrize("out_dtype", [F32, BF16])
def test_nan_stays_in_its_row(rows, out_dtype):
    rng = np.random.default_rng(5)
    x = rng.standard_normal((rows, 300))
    w = rng.standard_normal((500, 300))
    x[rows // 2, 7], w[11, 3] = np.nan, np.nan
    wc, wsc, _ = quantize(w, F32)
    t, ld = device(x, F32)
    out = torch.empty((rows, 500), dtype=TORCH[out_dtype], device="cuda")
    size = tfe.tfe_integer_workspace(rows, 300)
    tfe.tfe_integer_linear(t, F32, ld, wc, wsc, rows, 500, 300, out, out_dtype, 500,
                           torch.empty(size, dtype=torch.uint8, device="cuda"), size, H.cur_stream())
    nan = out.isnan().cpu().numpy()
    assert nan[rows // 2].all() and nan[:, 11].all() and nan.sum() == 500 + rows - 1


@pytest.mark.parametrize("rows,out_dtype", [(1, F32), (64, BF16), (300, BF16), (300, F32)])
def test_captured_and_on_another_stream(rows, out_dtype):
    rng = np.random.default_rng(rows)
    n, dim = 1000, 512
    wc, wsc, _ = quantize(rng.standard_normal((n, dim)), F32)
    xs = [device(rng.standard_normal((rows, dim)), BF16)[0] for _ in range(3)]
    size = tfe.tfe_integer_workspace(rows, dim)
    new = lambda: torch.empty((rows, n), dtype=TORCH[out_dtype], device="cuda")  # noqa: E731
    scratch = lambda: torch.empty(size, dtype=torch.uint8, device="cuda")  # noqa: E731

    def call(x, out, space, stream):
        tfe.tfe_integer_linear(x, BF16, dim, wc, wsc, rows, n, dim, out, out_dtype, n, space, size, stream)

    want, space = [new() for _ in xs], scratch()
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
        call(x, o, space, H.cur_stream())
    for k in (1, 2, 0, 1):
        x.copy_(xs[k])
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want[k])


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("rows,n,dim", [(1, 151936, 1024), (64, 151935, 1000), (400, 70000, 130), (513, 66001, 384),
                                        (3, 1 << 20, 64), (20, 100001, 256)])
def test_large(rows, n, dim, out_dtype):
    g = torch.Generator(device="cuda").manual_seed(n)
    pitch = -(-dim // 128) * 128
    a, w = (torch.randint(-127, 128, (k, pitch), generator=g, device="cuda").to(torch.int8) for k in (rows, n))
    a[:, dim:], w[:, dim:] = 0, 0
    asc, wsc = (torch.rand(k, generator=g, device="cuda") + 0.5 for k in (rows, n))
    out = torch.full((rows, n), -7.0, dtype=TORCH[out_dtype], device="cuda")
    tfe.tfe_integer_matmul(a, asc, w, wsc, rows, n, dim, out, out_dtype, n, H.cur_stream())
    # Sums below 2^24 are exact in float32 products too.
    want = (torch.mm(a.double(), w.double().t().contiguous()) * asc.double()[:, None]).mul_(wsc.double())
    off = (out.double() - want).abs_()
    assert (off <= (4 * 2.0 ** -24 + (2.0 ** -8 if out_dtype == BF16 else 0)) * want.abs_()).all()


def test_more_than_2_to_the_32_results():
    rows, n, dim = 30000, 151936, 128
    g = torch.Generator(device="cuda").manual_seed(1)
    a, w = (torch.randint(-127, 128, (k, dim), generator=g, device="cuda").to(torch.int8) for k in (rows, n))
    asc, wsc = (torch.rand(k, generator=g, device="cuda") + 0.5 for k in (rows, n))
    out = torch.full((rows, n), -7.0, dtype=torch.bfloat16, device="cuda")
    tfe.tfe_integer_matmul(a, asc, w, wsc, rows, n, dim, out, BF16, n, H.cur_stream())
    for at in (0, 14000, 28250, 29900):
        want = torch.mm(a[at:at + 100].double(), w.double().t().contiguous()) * asc[at:at + 100, None].double() * wsc.double()
        assert ((out[at:at + 100].double() - want).abs() <= (4 * 2.0 ** -24 + 2.0 ** -8) * want.abs()).all()
