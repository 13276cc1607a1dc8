"""Compensation factors that the operators around the quantised layer refuse: a
factor that does not fit would be dropped in silence or read past its end."""
import pytest
import torch

from paper_2603_04800_amd import ops


# ------------------------------------------------------------------ the experts' layer
def _experts(l_down, r_up):
    return ops.ExpertLinear(torch.ones(2, 64), torch.zeros(3, 32, 64, dtype=torch.int8), torch.ones(3, 32), l_down, r_up)


def test_expert_factors_without_an_axis():
    with pytest.raises(ValueError, match="l_down"):         # one non-text modality, without its axis
        _experts(torch.ones(3, 16, 64), torch.ones(3, 32, 16))
    with pytest.raises(ValueError, match="l_down"):         # one layer's factors
        _experts(torch.ones(1, 16, 64), torch.ones(1, 32, 16))
    with pytest.raises(ValueError, match="r_up"):
        _experts(torch.ones(3, 1, 16, 64), torch.ones(3, 32, 16))


def test_expert_factors_come_together():
    with pytest.raises(ValueError, match="together"):
        _experts(None, torch.ones(3, 1, 32, 16))
    with pytest.raises(ValueError, match="together"):
        _experts(torch.ones(3, 1, 16, 64), None)


def test_expert_factors_that_fit():
    assert _experts(torch.ones(3, 1, 16, 64), torch.ones(3, 1, 32, 16)).rank == 16
    assert _experts(torch.ones(3, 1, 0, 64), torch.ones(3, 1, 32, 0)).rank == 0
    assert _experts(None, None).rank == 0
