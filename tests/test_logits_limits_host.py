"""Arguments at the ends of their ranges, as the host checks them."""
import pytest

from paper_2607_07388_amd import tfe

from .test_logits_host import CALLS


@pytest.mark.parametrize("call", ["tfe_distill_loss", "tfe_distill_grad", "tfe_distill_loss_grad"])
@pytest.mark.parametrize("tau", [3.0e-39, 4.2e-39])
def test_temperatures_whose_factor_is_infinite(call, tau):
    """1 / tau is finite there, log2(e) / tau, by which the kernels multiply, is not."""
    with pytest.raises(tfe.TfeError) as e:
        getattr(tfe, call)(**{**CALLS[call], "temperature": tau})
    assert e.value.status == tfe.TFE_ERR_INVALID_ARG and "temperature" in str(e.value)


@pytest.mark.parametrize("call", ["tfe_distill_loss", "tfe_distill_grad", "tfe_distill_loss_grad"])
def test_the_least_temperature(call):
    assert getattr(tfe, call)(**{**CALLS[call], "rows": 0, "temperature": 4.3e-39}) == tfe.TFE_OK
