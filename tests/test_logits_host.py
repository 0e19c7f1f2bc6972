"""Refusals of the calls on the head's logits (checked on the host, before anything is
enqueued), their workspaces' sizes, and pins of their oracle."""
import numpy as np
import pytest

from oracle import logits as O
from paper_2607_07388_amd import tfe

F32, BF16 = tfe.TFE_F32, tfe.TFE_BF16
P = 1 << 16  # an address that is never read

CALLS = {
    "tfe_quantize": dict(x=P, dtype=F32, ldx=100, rows=4, dim=100, block_rows=1, codes=P, scales=P),
    "tfe_quantized_matmul": dict(a=P, a_scales=P, w=P, w_scales=P, rows=4, out_dim=50, dim=100, out=P, out_dtype=F32, ldo=50),
    "tfe_quantized_linear": dict(x=P, dtype=F32, ldx=100, w=P, w_scales=P, rows=4, out_dim=50, dim=100, out=P,
                           out_dtype=F32, ldo=50, workspace=P, workspace_bytes=1 << 20),
    "tfe_sample": dict(logits=P, dtype=F32, ld=100, rows=4, vocab=100, temperature=None, top_k=None, top_p=None,
                       min_p=None, u=P, token=P, prob=None, workspace=P, workspace_bytes=1 << 24),
    "tfe_distill_loss": dict(logits=P, dtype=F32, ld=100, rows=4, vocab=100, teacher_ids=P, teacher_logits=P,
                             teacher_dtype=F32, K=8, temperature=1.0, loss=P, lse=P, workspace=P,
                             workspace_bytes=1 << 24),
    "tfe_distill_grad": dict(logits=P, dtype=F32, ld=100, rows=4, vocab=100, teacher_ids=P, teacher_logits=P,
                             teacher_dtype=F32, K=8, temperature=1.0, lse=P, grad_loss=None, grad=P, ldg=100),
    "tfe_distill_loss_grad": dict(logits=P, dtype=F32, ld=100, rows=4, vocab=100, teacher_ids=P, teacher_logits=P,
                                  teacher_dtype=F32, K=8, temperature=1.0, grad_loss=None, loss=P, lse=P, grad=P + 64,
                                  ldg=100, workspace=P, workspace_bytes=1 << 24),
}
BIG = 1 << 20
WRONG = [
    ("tfe_quantize", dict(x=None), "null"), ("tfe_quantize", dict(x=P + 2), "aligned"),
    ("tfe_quantize", dict(dtype=2), "dtype"), ("tfe_quantize", dict(ldx=99), "pitch"),
    ("tfe_quantize", dict(rows=-1), "rows"), ("tfe_quantize", dict(rows=BIG + 1), "rows"),
    ("tfe_quantize", dict(dim=0), "dim"), ("tfe_quantize", dict(dim=65537, ldx=65537), "dim"),
    ("tfe_quantize", dict(block_rows=64), "block_rows"), ("tfe_quantize", dict(codes=None), "codes"),
    ("tfe_quantize", dict(codes=P + 8), "codes"), ("tfe_quantize", dict(scales=P + 2), "scales"),
    ("tfe_quantized_matmul", dict(a=None), "codes"), ("tfe_quantized_matmul", dict(w=P + 4), "codes"),
    ("tfe_quantized_matmul", dict(a_scales=None), "scales"), ("tfe_quantized_matmul", dict(w_scales=P + 1), "scales"),
    ("tfe_quantized_matmul", dict(out=None), "out"), ("tfe_quantized_matmul", dict(out=P + 1, out_dtype=BF16), "out"),
    ("tfe_quantized_matmul", dict(ldo=49), "pitch"), ("tfe_quantized_matmul", dict(out_dim=0), "out_dim"),
    ("tfe_quantized_matmul", dict(out_dim=BIG + 1, ldo=BIG + 1), "out_dim"), ("tfe_quantized_matmul", dict(out_dtype=-1), "dtype"),
    ("tfe_quantized_linear", dict(workspace=None), "workspace"), ("tfe_quantized_linear", dict(workspace=P + 8), "workspace"),
    ("tfe_quantized_linear", dict(workspace_bytes=4 * 132 - 1), "workspace"), ("tfe_quantized_linear", dict(x=None), "x"),
    ("tfe_quantized_linear", dict(w=None), "codes"), ("tfe_quantized_linear", dict(ldx=7), "pitch"),
    ("tfe_sample", dict(logits=None), "logits"), ("tfe_sample", dict(dtype=5), "dtype"),
    ("tfe_sample", dict(ld=99), "pitch"), ("tfe_sample", dict(vocab=0), "vocab"),
    ("tfe_sample", dict(vocab=(1 << 18) + 1, ld=1 << 19), "vocab"), ("tfe_sample", dict(rows=BIG + 1), "rows"),
    ("tfe_sample", dict(u=None), "u"), ("tfe_sample", dict(token=None), "token"),
    ("tfe_sample", dict(logits=P + 1, dtype=BF16), "aligned"),
] + [(c, w, t) for c in ("tfe_distill_loss", "tfe_distill_grad", "tfe_distill_loss_grad") for w, t in [
    (dict(logits=None), "logits"), (dict(teacher_ids=None), "teacher_ids"), (dict(teacher_logits=None), "teacher_logits"),
    (dict(teacher_dtype=3), "dtype"), (dict(K=0), "K"), (dict(K=257), "K"), (dict(temperature=0.0), "temperature"),
    (dict(temperature=float("nan")), "temperature"), (dict(temperature=float("inf")), "temperature"),
    (dict(temperature=1e-45), "temperature"), (dict(temperature=-1.0), "temperature"), (dict(lse=None), "lse"),
    (dict(ld=10), "pitch"), (dict(vocab=0), "vocab"), (dict(rows=-3), "rows")]
] + [("tfe_distill_grad", dict(grad=None), "grad"), ("tfe_distill_grad", dict(ldg=99), "pitch"),
     ("tfe_distill_grad", dict(grad=P, ldg=101), "place"), ("tfe_distill_loss", dict(loss=None), "loss"),
     ("tfe_distill_loss_grad", dict(grad=None), "grad")]


@pytest.mark.parametrize("call,change,word", WRONG)
def test_refusals(call, change, word):
    with pytest.raises(tfe.TfeError) as e:
        getattr(tfe, call)(**{**CALLS[call], **change})
    assert e.value.status == tfe.TFE_ERR_INVALID_ARG and word in str(e.value)


@pytest.mark.parametrize("call", sorted(CALLS))
def test_no_rows_enqueue_nothing(call):
    """No rows need no pointers (and no GPU)."""
    args = {k: None if v == P or v == P + 64 else v for k, v in CALLS[call].items()}
    assert getattr(tfe, call)(**{**args, "rows": 0}) == tfe.TFE_OK


def test_workspace_sizes():
    assert tfe.tfe_quantized_workspace(0, 1) == 0 and tfe.tfe_quantized_workspace(3, 1) == 3 * 132
    assert tfe.tfe_quantized_workspace(64, 1024) == 64 * (1024 + 8)
    for f in (tfe.tfe_sample_workspace, tfe.tfe_distill_workspace):
        assert f(0, 1) == 0
        sizes = [f(r, 151936) for r in (1, 2, 64, 256, 4096, 1 << 20)]
        assert min(sizes) >= 0 and max(sizes) < 1 << 31
        for bad in ((-1, 10), ((1 << 20) + 1, 10), (1, 0), (1, (1 << 18) + 1)):
            with pytest.raises(tfe.TfeError):
                f(*bad)
    for bad in ((-1, 10), ((1 << 20) + 1, 10), (1, 0), (1, 65537)):
        with pytest.raises(tfe.TfeError):
            tfe.tfe_quantized_workspace(*bad)


# ---- pins of the oracle ----

def test_oracle_codes():
    v = O.e4m3_values()
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[7] == 7 * 2.0 ** -9 and v[8] == 2.0 ** -6
    assert v[56] == 1 and v[126] == 448 and np.isnan(v[127]) and v[0x80 | 56] == -1
    for c in range(127):
        assert O.e4m3_nearest(v[c]) == c and O.e4m3_nearest(-v[c]) == (c | 128)
        if c < 126:
            mid = (v[c] + v[c + 1]) / 2
            assert O.e4m3_nearest(mid) == c + c % 2
            assert O.e4m3_nearest(mid * (1 - 1e-9)) == c and O.e4m3_nearest(mid * (1 + 1e-9)) == c + 1
    assert O.e4m3_nearest(np.inf) == 126 and O.e4m3_nearest(-500.0) == 254


def test_oracle_layout():
    x = np.zeros((3, 130))
    x[0, 0], x[0, 129], x[1, 5], x[2, 129] = 448, 449, -1, 2.0 ** -140
    codes, scales = O.fp8_layout(x, 1)
    assert codes.shape == (3, 256) and scales.shape == (3, 4)
    np.testing.assert_array_equal(scales, [[127, 128, 127, 127], [119, 0, 127, 127], [0, 0, 127, 127]])
    np.testing.assert_array_equal(O.fp8_values(codes, scales, 1)[1, :130], x[1])
    codes, scales = O.fp8_layout(np.full((129, 128), 3.0), 128)
    assert scales.shape == (2, 4) and (scales[:, 0] == 127 - 7).all() and (O.fp8_values(codes, scales, 128) == 3).all()


def test_oracle_sampling():
    l = np.log([0.1, 0.4, 0.2, 0.3])
    got = lambda u, T=1.0, k=0, p=1.0, m=0.0: O.sample(l, T, k, p, m, u)[:2]  # noqa: E731
    assert [got(u)[0] for u in (0.0, 0.39, 0.41, 0.69, 0.71, 0.89, 0.91)] == [1, 1, 3, 3, 2, 2, 0]
    assert [got(u, k=2)[0] for u in (0.5, 0.6, 0.99)] == [1, 3, 3] and abs(got(0.5, k=2)[1] - 4 / 7) < 1e-8
    assert got(0.99, p=0.45)[0] == 3 and got(0.99, p=0.39)[0] == 1 and got(0.99, p=0.0)[0] == 1
    assert got(0.99, m=0.6)[0] == 3 and got(0.99, m=0.8)[0] == 1 and got(0.99, T=0.0) == (1, 1.0)
    assert got(0.99, k=3, p=0.5)[0] == 3  # of 0.9 in all, 0.4 does not reach a half
    assert O.sample(np.zeros(4), 1.0, 0, 1.0, 0.0, 0.5)[0] == 2
    assert O.sample(np.full(3, -np.inf), 1.0, 0, 1.0, 0.0, 0.5)[:2] == (-1, 0.0)


def test_oracle_distillation():
    s = np.log([[0.5, 0.25, 0.25]])
    loss, lse, grad, p, q = O.distill(s, np.array([[0, 1]]), np.log([[0.5, 0.5]]), 1.0, np.ones(1))
    assert abs(loss[0] - (0.5 * np.log(1) + 0.5 * np.log(2))) < 1e-12 and abs(lse[0]) < 1e-12
    np.testing.assert_allclose(grad, [[0.0, -0.25, 0.25]], atol=1e-12)
    assert O.distill(s, np.array([[-1, 3]]), np.zeros((1, 2)), 1.0, np.ones(1))[0][0] == 0
    same = O.distill(s, np.array([[0, 1, 2]]), s, 2.0, np.ones(1))
    assert abs(same[0][0]) < 1e-12 and np.abs(same[2]).max() < 1e-12
