"""The calls on logits through the native module: plain arguments reach the library as
they are, in their order; other forms go to the ctypes function."""
import ctypes
import inspect

import pytest
import torch

from paper_2607_07388_amd import _calls, tfe

V, I, L, F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
HEAD = (V, I, L, L, I, V, V, I, I, F)
TYPES = {
    "tfe_quantized_linear": (V, I, L, V, V, L, I, I, V, I, L, V, L),
    "tfe_sample": (V, I, L, L, I, V, V, V, V, V, V, V, V, L),
    "tfe_distill_loss": HEAD + (V, V, V, L),
    "tfe_distill_grad": HEAD + (V, V, V, L),
    "tfe_distill_loss_grad": HEAD + (V, V, V, V, L, V, L),
}


@pytest.fixture(params=sorted(TYPES))
def bound(request):
    name, native, handed = request.param, [], []
    fn = ctypes.CFUNCTYPE(ctypes.c_int, *TYPES[name], V)(lambda *a: native.append(a) or 0)

    def slow(*a, **k):
        handed.append((a, k))
        return "slow"

    every = {n: (slow, 1) for n in tfe._BY_CTYPES}
    every[name] = (slow, ctypes.cast(fn, V).value)
    _calls.bind(lambda st: st, every)
    yield name, native, handed
    tfe._bind_calls()


def arguments(name):
    """Distinct values of each argument's type; int64 ones beyond int32."""
    return [100 + i if t is V else 7 + i if t is I else (1 << 40) + i if t is L else 0.5 + i
            for i, t in enumerate(TYPES[name])]


def test_plain_arguments(bound):
    name, native, handed = bound
    a = arguments(name)
    assert getattr(_calls, name)(*a) == 0 and getattr(_calls, name)(*a, 9) == 0
    assert native == [tuple(a) + (None,), tuple(a) + (9,)] and not handed
    t = torch.zeros(4)
    b = [t[1:] if ty is V else x for x, ty in zip(a, TYPES[name])]
    assert getattr(_calls, name)(*b) == 0
    assert native[-1] == tuple(t.data_ptr() + 4 if ty is V else x for x, ty in zip(a, TYPES[name])) + (None,)
    none = [None if ty is V else x for x, ty in zip(a, TYPES[name])]
    assert getattr(_calls, name)(*none) == 0 and native[-1][0] is None


def test_other_forms(bound):
    name, native, handed = bound
    a = arguments(name)
    forms = [(a[:-1], {}), (a, {"stream": 3}), (a + [1, 2], {})]
    for i, ty in enumerate(TYPES[name]):
        bad = {V: "x", I: 1 << 31, L: 1 << 63, F: 1}[ty]
        forms.append((a[:i] + [bad] + a[i + 1:], {}))
    for x, kw in forms:
        assert getattr(_calls, name)(*x, **kw) == "slow"
    assert not native and len(handed) == len(forms)


def test_signatures_and_errors():
    for name, f in tfe._BY_CTYPES.items():
        assert list(inspect.signature(getattr(tfe, name)).parameters) == list(inspect.signature(f).parameters)
    with pytest.raises(tfe.TfeError) as e:
        tfe.tfe_sample(None, 0, 10, 1, 10, None, None, None, None, None, None, None, None, 0)
    assert e.value.status == tfe.TFE_ERR_INVALID_ARG and "logits" in str(e.value)
