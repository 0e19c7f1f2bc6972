"""Refusals of the calls that learn the head from tokens and serve it in integers (checked on the
host, before anything is enqueued), their workspaces' sizes, and pins of their oracle."""
import numpy as np
import pytest

from oracle import learn as O
from paper_2607_07388_amd import tfe

F32, BF16 = tfe.TFE_F32, tfe.TFE_BF16
P = 1 << 16  # an address that is never read
SPACE = 1 << 34

HEAD = dict(hidden=P, ldh=100, w=2 * P, ldw=100, targets=P, rows=4, vocab=50, dim=100)
GRADS = dict(grad_hidden=3 * P, ldgh=100, grad_w=4 * P, ldgw=100, grad_dtype=F32, accumulate=0)
WORK = dict(workspace=P, workspace_bytes=SPACE)
CALLS = {
    "tfe_cross_entropy_loss": dict(HEAD, loss=P, lse=P, **WORK),
    "tfe_cross_entropy_grad": dict(HEAD, lse=P, grad_loss=None, **GRADS, **WORK),
    "tfe_cross_entropy_loss_grad": dict(HEAD, grad_loss=None, loss=P, lse=P, **GRADS, **WORK),
    "tfe_integer_quantize": dict(x=P, dtype=F32, ldx=100, rows=4, dim=100, codes=P, scales=P),
    "tfe_integer_matmul": dict(a=P, a_scales=P, w=P, w_scales=P, rows=4, out_dim=50, dim=100, out=P, out_dtype=F32,
                               ldo=50),
    "tfe_integer_linear": dict(x=P, dtype=F32, ldx=100, w=P, w_scales=P, rows=4, out_dim=50, dim=100, out=P,
                               out_dtype=F32, ldo=50, **WORK),
    "tfe_grad_norm": dict(tensors=P, n=0, norm=P, **WORK),
    "tfe_grad_clip": dict(tensors=P, n=0, max_norm=1.0, norm=P),
    "tfe_grad_norm_clip": dict(tensors=P, n=0, max_norm=1.0, norm=P, **WORK),
}
BIG = 1 << 20
LOSS, GRAD, BOTH = "tfe_cross_entropy_loss", "tfe_cross_entropy_grad", "tfe_cross_entropy_loss_grad"
WRONG = [(c, d, m) for c in (LOSS, GRAD, BOTH) for d, m in [
    (dict(hidden=None), "hidden"), (dict(hidden=P + 1), "aligned"), (dict(ldh=99), "pitch"), (dict(w=None), "w"),
    (dict(ldw=99), "pitch"), (dict(targets=None), "targets"), (dict(targets=P + 2), "targets"),
    (dict(rows=-1), "rows"), (dict(rows=BIG + 1), "rows"), (dict(vocab=0), "vocab"),
    (dict(vocab=(1 << 18) + 1), "vocab"), (dict(dim=0), "dim"), (dict(dim=16385, ldh=16385, ldw=16385), "dim"),
    (dict(workspace=None), "workspace"), (dict(workspace=P + 8), "workspace"), (dict(workspace_bytes=100), "workspace"),
    (dict(lse=None), "lse")]]
WRONG += [(c, d, m) for c in (GRAD, BOTH) for d, m in [
    (dict(grad_hidden=None), "grad_hidden"), (dict(grad_w=None), "grad_w"), (dict(ldgh=99), "pitch"),
    (dict(ldgw=99), "pitch"), (dict(grad_dtype=2), "dtype"), (dict(grad_w=4 * P + 2), "aligned"),
    (dict(grad_w=2 * P), "place"), (dict(grad_hidden=P), "place"), (dict(grad_hidden=4 * P), "place"),
    (dict(grad_dtype=BF16, accumulate=1), "accumulate"), (dict(grad_loss=P + 1), "grad_loss")]]
WRONG += [(LOSS, dict(loss=None), "loss"), (BOTH, dict(loss=P + 1), "loss"), (GRAD, dict(lse=P + 1), "lse")]
Q, M, L = "tfe_integer_quantize", "tfe_integer_matmul", "tfe_integer_linear"
WRONG += [
    (Q, dict(x=None), "null"), (Q, dict(x=P + 2), "aligned"), (Q, dict(dtype=3), "dtype"), (Q, dict(ldx=99), "pitch"),
    (Q, dict(rows=-1), "rows"), (Q, dict(rows=BIG + 1), "rows"), (Q, dict(dim=0), "dim"),
    (Q, dict(dim=65537, ldx=65537), "dim"), (Q, dict(codes=None), "codes"), (Q, dict(codes=P + 8), "codes"),
    (Q, dict(scales=None), "scales"), (Q, dict(scales=P + 2), "scales"),
    (M, dict(a=None), "codes"), (M, dict(w=P + 4), "codes"), (M, dict(a_scales=None), "scales"),
    (M, dict(w_scales=P + 1), "scales"), (M, dict(out=None), "out"), (M, dict(ldo=49), "pitch"),
    (M, dict(out_dim=0), "out_dim"), (M, dict(out_dim=BIG + 1, ldo=BIG + 1), "out_dim"), (M, dict(out_dtype=2), "dtype"),
    (L, dict(x=None), "x"), (L, dict(w=None), "codes"), (L, dict(w_scales=None), "scales"),
    (L, dict(out=P + 1, out_dtype=BF16), "aligned"), (L, dict(workspace=None), "workspace"),
    (L, dict(workspace_bytes=10), "workspace"), (L, dict(workspace=P + 4), "workspace")]
WRONG += [(c, d, m) for c in ("tfe_grad_norm", "tfe_grad_clip", "tfe_grad_norm_clip") for d, m in [
    (dict(n=-1), "tensors"), (dict(n=BIG + 1), "tensors"), (dict(tensors=None, n=1), "tensors"),
    (dict(norm=None), "norm"), (dict(norm=P + 2), "norm")]]
WRONG += [(c, dict(max_norm=m), "max_norm") for c in ("tfe_grad_clip", "tfe_grad_norm_clip")
          for m in (-1.0, float("inf"), float("nan"))]


@pytest.mark.parametrize("call,change,says", WRONG)
def test_refusals(call, change, says):
    args = dict(CALLS[call], **change)
    for f in (getattr(tfe, call), tfe._BY_CTYPES.get(call, getattr(tfe, call))):
        with pytest.raises(tfe.TfeError) as e:
            f(*args.values())
        assert e.value.status == tfe.TFE_ERR_INVALID_ARG and says in str(e.value)


TENSOR = dict(grad=P, out=2 * P, rows=3, cols=5, ldg=5, ldo=5, dtype=F32)
TENSORS = [
    (dict(grad=None), True, "null"), (dict(grad=P + 2), True, "aligned"), (dict(dtype=7), True, "dtype"),
    (dict(rows=-1), True, "rows"), (dict(cols=-1), True, "rows"), (dict(ldg=4), True, "pitch"),
    (dict(rows=1 << 31), True, "rows"), (dict(rows=2, cols=1 << 31, ldg=1 << 31, ldo=1 << 31), True, "rows"),
    (dict(rows=1 << 30, cols=1 << 20, ldg=1 << 20, ldo=1 << 20), True, "elements"),
    (dict(out=None), False, "null"), (dict(ldo=4), False, "pitch"), (dict(out=P, ldo=6), False, "in place")]


@pytest.mark.parametrize("change,norm_too,says", TENSORS)
def test_refused_tensors(change, norm_too, says):
    good = tuple(TENSOR.values())
    bad = tuple(dict(TENSOR, **change).values())
    t = tfe.make_grad_tensors([good, bad])
    calls = [lambda: tfe.tfe_grad_clip(t, 2, 1.0, P), lambda: tfe.tfe_grad_norm_clip(t, 2, 1.0, P, P, SPACE)]
    if norm_too:
        calls += [lambda: tfe.tfe_grad_norm(t, 2, P, P, SPACE), lambda: tfe.tfe_grad_workspace(t, 2)]
    else:
        assert tfe.tfe_grad_workspace(t, 2) > 0
    for f in calls:
        with pytest.raises(tfe.TfeError) as e:
            f()
        assert e.value.status == tfe.TFE_ERR_INVALID_ARG and says in str(e.value)


def test_workspaces():
    size = tfe.tfe_cross_entropy_workspace
    assert size(0, 100, 100) == 0
    assert size(1, 100, 100) > 0
    # The logits are not kept: of 65536 rows the workspace is far below them, and grows with the rows.
    assert size(65536, 151936, 1024) < 65536 * 151936 * 2 // 8
    for bad in ((-1, 10, 10), (1, 0, 10), (1, 1 << 19, 10), (1, 10, 0), (BIG + 1, 10, 10)):
        with pytest.raises(tfe.TfeError):
            size(*bad)
    assert tfe.tfe_integer_workspace(0, 10) == 0 and tfe.tfe_integer_workspace(3, 130) >= 3 * (256 + 4)
    for bad in ((-1, 10), (1, 0), (1, 65537)):
        with pytest.raises(tfe.TfeError):
            tfe.tfe_integer_workspace(*bad)


def test_no_rows():
    assert tfe.tfe_cross_entropy_loss(None, 8, P, 8, None, 0, 4, 8, None, None, None, 0) == 0
    assert tfe.tfe_integer_linear(None, F32, 4, None, None, 0, 4, 4, None, F32, 4, None, 0) == 0
    assert tfe.tfe_integer_matmul(None, None, None, None, 0, 4, 4, None, F32, 4) == 0
    assert tfe.tfe_integer_quantize(None, F32, 4, 0, 4, None, None) == 0


def test_tensors_are_kept():
    class Tensor:
        def data_ptr(self):
            return P
    t = Tensor()
    g = tfe.make_grad_tensors([(t, t, 1, 4, 4, 4, F32)])
    assert g.kept == [(t, t)] and g.array[0].grad == P and g.data_ptr() == g.address


# ---- the oracle ----------------------------------------------------------------------------


def test_oracle_cross_entropy():
    x, w = np.eye(3)[:2], np.log([[0.5, 0.2, 1], [0.25, 0.2, 1], [0.25, 0.6, 1]])
    loss, lse, dx, dw, dz = O.cross_entropy(x, w, np.array([1, 2]), np.array([1.0, 2.0]))
    np.testing.assert_allclose(loss, [np.log(4), -np.log(0.6)], atol=1e-12)
    np.testing.assert_allclose(lse, 0, atol=1e-12)
    np.testing.assert_allclose(dz, [[0.5, -0.75, 0.25], [0.4, 0.4, -0.8]], atol=1e-12)
    np.testing.assert_allclose(dx, dz @ w, atol=1e-12)
    np.testing.assert_allclose(dw, np.c_[dz.T, np.zeros(3)], atol=1e-12)
    loss, _, dx, dw, _ = O.cross_entropy(x, w, np.array([-1, 3]), np.ones(2))
    assert not loss.any() and not dx.any() and not dw.any()


def test_oracle_gradients_are_differences():
    rng = np.random.default_rng(3)
    x, w, t, g = rng.standard_normal((5, 7)), rng.standard_normal((11, 7)), np.array([0, 10, -1, 4, 4]), rng.random(5)
    _, _, dx, dw, _ = O.cross_entropy(x, w, t, g)
    total = lambda x, w: (O.cross_entropy(x, w, t, g)[0] * g).sum()  # noqa: E731
    h = 1e-6
    for a, d in ((x, dx), (w, dw)):
        for i in np.ndindex(a.shape):
            old = a[i]
            a[i] = old + h
            up = total(x, w)
            a[i] = old - h
            down = total(x, w)
            a[i] = old
            assert abs((up - down) / (2 * h) - d[i]) < 1e-7


def test_oracle_integers():
    x = np.array([[1, -2, 127, 63.5, 62.5], [0, 0, 0, 0, 2.0 ** -101], [np.inf, -np.inf, 1, 0, -0.5],
                  [np.nan, 1, 2, 3, 4]])
    codes, scales = O.integer_layout(x)
    assert codes.shape == (4, 128)
    np.testing.assert_array_equal(codes[:3, :5], [[1, -2, 127, 64, 62], [0] * 5, [127, -127, 127, 0, -64]])
    assert scales[0] == 1 and scales[1] == 0 and scales[2] == np.float32(1) / np.float32(127) and np.isnan(scales[3])
    sums, out = O.integer_product(codes[:1], scales[:1], codes[:1], np.float32([2.0]))
    assert sums[0, 0] == 1 + 4 + 127 ** 2 + 64 ** 2 + 62 ** 2 and out[0, 0] == 2.0 * sums[0, 0]


def test_oracle_clipping():
    assert O.grad_norm([np.array([3.0]), np.array([[4.0], [12.0]])]) == 13
    assert O.clip_factor(4, 1.0) == 0.25 and O.clip_factor(0.5, 1.0) == 1 and O.clip_factor(1, 1.0) == 1
    assert O.clip_factor(np.inf, 1.0) == 1 and O.clip_factor(np.nan, 1.0) == 1 and O.clip_factor(2, 0.0) == 0
