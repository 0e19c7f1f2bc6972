"""Cross entropy in every tile that its rules choose, number by number against 64 bits on the GPU.

The shapes reach, with 256 compute units: logits in tiles of 64, 128 and 256 rows; dW in tiles of 128 x
128 and 256 x 256, one and several across, in one piece of the vocabulary and in later ones, W in place
and copied; one to sixteen steps of the width, one to forty of the rows; lists of up to 64 rows a
block of 128 tokens and longer ones.

Bounds, u = 2^-24.  A logit is a float32 sum of dim exact products: off by at most E = dim u max_v
sum |x w|.  lse by that and below 400 u + 8 u of itself (300 additions, exponentials off by 2 u d + 2 u at
distance d), the loss, lse minus a logit, by 2 E + 400 u and roundings of the parts.  So p = exp(z - lse)
is off by p (2 E + 400 u + 8 u |lse|), and by 2 u where 1 is subtracted; dz is rounded by 2^-8 of itself
for bfloat16 gradients, by 4 u with its weight for float32 ones.  A gradient's n products add n u of
their magnitudes (twice that with the parts that are joined), its own rounding 2^-8 (u) of it."""
import pytest
import torch

from paper_2607_07388_amd import tfe

from . import harness as H

pytestmark = pytest.mark.gpu

F32, BF16 = tfe.TFE_F32, tfe.TFE_BF16
TORCH = {F32: torch.float32, BF16: torch.bfloat16}
U = 2.0 ** -24


class Case:
    def __init__(self, rows, vocab, dim, pad=0, tokens=None):
        g = torch.Generator(device="cuda").manual_seed(rows + vocab + dim)
        self.rows, self.vocab, self.dim, self.ld = rows, vocab, dim, dim + pad
        self.x, self.w = (torch.full((n, self.ld), float("nan"), dtype=torch.bfloat16, device="cuda") for n in (rows, vocab))
        self.x[:, :dim] = torch.randn((rows, dim), generator=g, device="cuda")
        # Logits of about the same spread whatever the width.
        self.w[:, :dim] = torch.randn((vocab, dim), generator=g, device="cuda") * (1.5 / dim ** 0.5)
        t = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
        if tokens:  # everybody's targets are a few tokens all over the vocabulary
            t = t % tokens * (vocab // tokens) + vocab // tokens // 2
        t[::9] = -1
        t[4::13] = vocab - 1  # the last row of W
        self.t = t.int()
        self.g = torch.rand(rows, generator=g, device="cuda") + 0.5
        self.g[3::17] = 0

    def run(self, dtype, out_pad=0, old=None):
        f32 = dict(dtype=torch.float32, device="cuda")
        loss, lse = torch.full((self.rows,), -7.0, **f32), torch.full((self.rows,), -7.0, **f32)
        gx, gw = (torch.full((n, self.dim + out_pad), -7.0, dtype=TORCH[dtype], device="cuda") for n in (self.rows, self.vocab))
        if old is not None:
            gw[:, :self.dim] = old
        size = tfe.tfe_cross_entropy_workspace(self.rows, self.vocab, self.dim)
        space = torch.full((size,), 0x7F, dtype=torch.uint8, device="cuda")
        tfe.tfe_cross_entropy_loss_grad(self.x, self.ld, self.w, self.ld, self.t, self.rows, self.vocab, self.dim, self.g,
                                        loss, lse, gx, self.dim + out_pad, gw, self.dim + out_pad, dtype,
                                        int(old is not None), space, size, H.cur_stream())
        for o in (gx, gw):
            assert (o[:, self.dim:] == -7).all()
        return loss, lse, gx[:, :self.dim], gw[:, :self.dim]

    def check(self, got, dtype):
        x, w = self.x[:, :self.dim].double(), self.w[:, :self.dim].double()
        wt, xa = w.t().contiguous(), x.abs()
        e = self.dim * U * torch.mm(xa, wt.abs().contiguous()).amax(1)
        z = torch.mm(x, wt)
        lse = z.logsumexp(1)
        there = (self.t >= 0) & (self.t < self.vocab)
        at = torch.where(there, self.t, 0).long()[:, None]
        loss = (lse - z.gather(1, at)[:, 0]) * there
        far = 2 * e + 400 * U + 8 * U * lse.abs()
        near(got[0], loss, far + 4 * U * loss)
        near(got[1], lse, far)
        by = (self.g.double() * there)[:, None]
        p = z.sub_(lse[:, None]).exp_()
        off = p * (far[:, None] * by)
        dz = p.scatter_add_(1, at, -torch.ones_like(by)).mul_(by)
        size = dz.abs()
        off.scatter_add_(1, at, 2 * U * by).add_(size, alpha=2.0 ** -8 + 4 * U if dtype == BF16 else 4 * U)
        last = 2.0 ** -8 if dtype == BF16 else U
        want = torch.mm(dz, w)
        near(got[2], want, (1 + last) * torch.mm(off.add(size, alpha=2 * self.vocab * U), w.abs()) + last * want.abs())
        live = x * (by != 0)
        want = torch.mm(dz.t().contiguous(), live)
        near(got[3], want, (1 + last) * torch.mm(off.add_(size, alpha=2 * self.rows * U).t().contiguous(), live.abs()) + last * want.abs())


def near(got, want, bound):
    assert got.isfinite().all()
    worst = float(((got.double() - want).abs() - bound).max())
    assert worst <= 0, "%g beyond the bound" % worst


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab,dim,pad", [
    (100, 131073, 72, 0), (65, 140000, 1024, 0), (128, 131073, 201, 3),  # 128 rows a tile
    (600, 45000, 520, 0), (257, 40001, 999, 2), (300, 50000, 1024, 8),  # 256 rows
    (2100, 150000, 520, 0), (2560, 110000, 263, 1),  # in pieces
    (513, 3001, 1024, 0), (64, 151936, 1024, 0)])  # 64 rows
def test_numbers(rows, vocab, dim, pad, dtype):
    c = Case(rows, vocab, dim, pad)
    c.check(c.run(dtype, out_pad=pad), dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab,dim", [(30000, 20000, 24), (30000, 9000, 5000), (20000, 16384, 600), (300, 25000, 16384),
                                            (1 << 20, 300, 16), (5, 1 << 18, 16), (1, 1, 16384)])
def test_many_rows_and_wide_ones(rows, vocab, dim, dtype):
    """Every list of targets long, several tokens a block; pieces of a few thousand tokens; the longest rows."""
    c = Case(rows, vocab, dim)
    c.check(c.run(dtype), dtype)


def test_training_batch():
    """4096 rows of 151936 x 1024: five pieces."""
    c = Case(4096, 151936, 1024)
    c.check(c.run(BF16), BF16)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tokens", [1, 3, 40])
@pytest.mark.parametrize("rows,vocab,dim,pad", [(100, 131073, 72, 0), (600, 45000, 520, 0), (2100, 150000, 260, 0), (700, 90000, 333, 2)])
def test_common_targets(rows, vocab, dim, pad, tokens, dtype):
    """Lists of hundreds of rows in large tiles, of this piece and later ones; the same bits again."""
    c = Case(rows, vocab, dim, pad, tokens)
    got = c.run(dtype, out_pad=pad)
    c.check(got, dtype)
    assert all(torch.equal(a, b) for a, b in zip(got, c.run(dtype, out_pad=pad)))


@pytest.mark.parametrize("rows,vocab,dim,out_pad", [(600, 45000, 520, 0), (2100, 150000, 300, 3), (100, 131073, 72, 1)])
def test_accumulated(rows, vocab, dim, out_pad):
    c = Case(rows, vocab, dim)
    gw = c.run(F32)[3]
    old = torch.randn((vocab, dim), generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    assert torch.equal(c.run(F32, out_pad, old)[3], gw + old)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_that_take_no_part(dtype):
    """In large tiles: they may hold anything, and the others do not change."""
    c = Case(600, 45000, 264)
    want = c.run(dtype)
    none = (c.t < 0) | (c.g == 0)
    c.x[none] = float("nan")
    got = c.run(dtype)
    assert torch.equal(got[2], want[2]) and torch.equal(got[3], want[3]) and torch.equal(got[0][~none], want[0][~none])
