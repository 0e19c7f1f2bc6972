"""Loss and gradient in one call over rows of several parts: the parts tell each other their
sums.  What a part has not been told within its wait it computes itself, so that the results
are the same to the bit however long it waits and whatever else the GPU does."""
import numpy as np
import pytest
import torch

from paper_2607_07388_amd import tfe

from . import harness as H
from .test_gpu_distill import BF16, F32, Call, check_values, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,tdtype", [(F32, F32), (BF16, F32), (F32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("rows,vocab,K", [(1, 1 << 18, 3), (5, 151936, 64), (3, 16392, 7), (40, 40001, 33), (9, 33001, 256)])
def test_without_waiting(monkeypatch, rows, vocab, K, dtype, tdtype):
    """No poll, one and a few: parts compute the sums of most others themselves."""
    s, ids, t, weight = inputs(rows + vocab + K, rows, vocab, K)
    c = Call(s, ids, t, 2.0, dtype, tdtype, pad=vocab % 2, gpad=vocab % 4)
    w = torch.from_numpy(weight).cuda()
    want = c.both(w)
    check_values(c, ids, weight, *want)
    for limit in ("0", "1", "8"):
        monkeypatch.setenv("TFE_DISTILL_WAIT_LIMIT", limit)
        for x, y in zip(c.both(w), want):
            assert torch.equal(x, y), limit


def test_nan_and_infinity_without_waiting(monkeypatch):
    s, ids, t, weight = inputs(3, 6, 50000, 5, short=False)
    s[0, 49999], s[1, 7], s[2, 20000] = np.nan, np.inf, -np.inf
    s[3, :40000] = -np.inf
    c = Call(s, ids, t, 2.0)
    want = c.both(None)
    assert want[0][:2].isnan().all() and want[2][:2].isnan().all()
    monkeypatch.setenv("TFE_DISTILL_WAIT_LIMIT", "0")
    for x, y in zip(c.both(None), want):
        assert torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0)) and torch.equal(x.isnan(), y.isnan())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place_of_the_logits(monkeypatch, dtype):
    """The gradient over the logits themselves: the same bits, whatever the waits."""
    s, ids, t, weight = inputs(4, 30, 151936, 20)
    c = Call(s, ids, t, 2.0, dtype)
    w = torch.from_numpy(weight).cuda()
    want, keep = c.both(w), c.s.clone()
    for limit in (None, "0"):
        if limit:
            monkeypatch.setenv("TFE_DISTILL_WAIT_LIMIT", limit)
        c.s.copy_(keep)
        for x, y in zip(c.both(w, grad=c.s), want):
            assert torch.equal(x, y)


def test_many_calls_at_once():
    """Twelve calls in flight on twelve streams beside products that fill compute units."""
    rows, vocab = 200, 1 << 18
    s, ids, t, weight = inputs(5, rows, vocab, 9)
    w = torch.from_numpy(weight).cuda()
    calls = [Call(s * (1 + k / 8), ids, t, 2.0, BF16 if k % 2 else F32) for k in range(4)]
    want = [c.both(w) for c in calls]
    n, dim = 100000, 512
    codes = torch.zeros((n, dim), dtype=torch.uint8, device="cuda")
    scales = torch.full((-(-n // 128), 4), 127, dtype=torch.uint8, device="cuda")
    logits = torch.empty((1024, n), dtype=torch.bfloat16, device="cuda")
    ones = torch.full((1024, 4), 127, dtype=torch.uint8, device="cuda")
    streams = [torch.cuda.Stream() for _ in range(13)]
    spaces = [torch.empty(calls[0].size, dtype=torch.uint8, device="cuda") for _ in range(12)]
    outs = [calls[k % 4].new() for k in range(12)]
    torch.cuda.synchronize()
    for _ in range(4):
        for _ in range(3):
            tfe.tfe_quantized_matmul(codes, ones, codes, scales, 1024, n, dim, logits, BF16, n,
                                     streams[12].cuda_stream)
        for k, (loss, lse, grad) in enumerate(outs):
            c = calls[k % 4]
            tfe.tfe_distill_loss_grad(*c.front, w, loss, lse, grad, c.ldg, spaces[k], c.size, streams[k].cuda_stream)
    torch.cuda.synchronize()
    for k, out in enumerate(outs):
        for x, y in zip(out, want[k % 4]):
            assert torch.equal(x, y), k
