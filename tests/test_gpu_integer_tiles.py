"""The integer product in every tile that its rules choose, number by number against 64 bits on the GPU.

The shapes reach, with 256 compute units, tiles of 128 x 128, 256 x 256 and 128 x 64, one to eight and
more steps of the width, edges in either direction.  Sums are below 2^53: exact in float64.  A result
is the sum converted to float32 and multiplied by two scales, three roundings of 2^-24, and one of 2^-8 for
bfloat16."""
import pytest
import torch

from paper_2607_07388_amd import tfe

from . import harness as H

pytestmark = pytest.mark.gpu

F32, BF16 = tfe.TFE_F32, tfe.TFE_BF16
TORCH = {F32: torch.float32, BF16: torch.bfloat16}


class Case:
    def __init__(self, rows, n, dim):
        g = torch.Generator(device="cuda").manual_seed(rows + n + dim)
        self.rows, self.n, self.dim, pitch = rows, n, dim, -(-dim // 128) * 128
        self.a, self.w = (torch.randint(-127, 128, (k, pitch), generator=g, device="cuda").to(torch.int8) for k in (rows, n))
        self.a[:, dim:], self.w[:, dim:] = 0, 0
        self.sa, self.sw = (torch.rand(k, generator=g, device="cuda") + 0.5 for k in (rows, n))

    def run(self, out_dtype, pad=0, rows=None):
        rows = rows or self.rows
        out = torch.full((rows, self.n + pad), -7.0, dtype=TORCH[out_dtype], device="cuda")
        tfe.tfe_integer_matmul(self.a, self.sa, self.w, self.sw, rows, self.n, self.dim, out, out_dtype, self.n + pad,
                               H.cur_stream())
        assert (out[:, self.n:] == -7).all()
        return out[:, :self.n]

    def check(self, out, out_dtype):
        want = torch.mm(self.a.double(), self.w.double().t().contiguous())
        want.mul_(self.sa.double()[:, None]).mul_(self.sw.double())
        off = out.double().sub_(want).abs_()
        assert (off <= (4 * 2.0 ** -24 + (2.0 ** -8 if out_dtype == BF16 else 0)) * want.abs_()).all()


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("rows,n,dim,pad", [
    (257, 40001, 1000, 0), (100, 33001, 1024, 3), (65, 32768, 2100, 1), (128, 151936, 1024, 0), (600, 20003, 300, 5),  # 128 x 128
    (512, 66001, 1000, 1), (1024, 66000, 1024, 0), (2048, 151936, 1024, 0), (700, 70001, 3000, 2),  # 256 x 256
    (70, 20000, 1024, 0), (300, 5001, 1300, 7)])  # 128 x 64
def test_numbers(rows, n, dim, pad, out_dtype):
    c = Case(rows, n, dim)
    c.check(c.run(out_dtype, pad), out_dtype)


@pytest.mark.parametrize("out_dtype", [F32, BF16])
def test_a_row_does_not_depend_on_its_batch(out_dtype):
    """Rows in LDS under W's stream, tiles of 128 x 128 and of 256 x 256."""
    c = Case(600, 66001, 1000)
    want = c.run(out_dtype)
    c.check(want, out_dtype)
    for rows in (1, 16, 17, 64, 65, 128, 200, 257, 511, 512, 513, 599):
        assert torch.equal(c.run(out_dtype, rows=rows), want[:rows])


@pytest.mark.parametrize("rows,n", [(100, 33001), (600, 66001)])
def test_laid_out_in_the_same_call(rows, n):
    """tfe_integer_linear's results are those of its two parts."""
    dim = 1000
    c = Case(rows, n, dim)
    x = torch.randn((rows, dim + 3), generator=torch.Generator("cuda").manual_seed(2), device="cuda")
    tfe.tfe_integer_quantize(x, F32, dim + 3, rows, dim, c.a, c.sa, H.cur_stream())
    out = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda")
    size = tfe.tfe_integer_workspace(rows, dim)
    tfe.tfe_integer_linear(x, F32, dim + 3, c.w, c.sw, rows, n, dim, out, BF16, n,
                           torch.full((size,), 0x7F, dtype=torch.uint8, device="cuda"), size, H.cur_stream())
    c.check(out, BF16)
    assert torch.equal(out, c.run(BF16))
