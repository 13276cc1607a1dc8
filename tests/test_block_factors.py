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
    assert _experts(torch.ones(3, 1, 0, 64), torch.ones(3, 1, 32, 16)).rank == 0          # not read
    assert _experts(None, None).rank == 0


# ------------------------------------------------------------------ the layer with an epilogue
def _fused(match, error=ValueError, l_down=None, r_up=None, wq=None, w_scale=None, inv=None):
    wq = torch.zeros(32, 64, dtype=torch.int8) if wq is None else wq
    lin = ops.Linear(torch.ones(2, 64) if inv is None else inv, wq, torch.ones(32) if w_scale is None else w_scale,
                     l_down, r_up)
    with pytest.raises(error, match=match):
        lin.fused(torch.ones(4, 64), torch.zeros(4, dtype=torch.int32))


def test_a_layers_factors_fit():
    ld, ru = torch.ones(1, 16, 64), torch.ones(1, 32, 16)
    _fused("GPU", l_down=ld, r_up=ru)                       # (these fit: what is refused is the CPU)
    _fused("GPU")
    _fused("GPU", l_down=ld[:, :0], r_up=ru)                # rank 0, one modality: not read
    _fused("GPU", l_down=ld, r_up=ru, inv=torch.ones(1, 64))
    _fused("l_down", l_down=ld[0], r_up=ru[0])              # without the modalities' axis
    _fused("l_down", l_down=torch.ones(2, 16, 64), r_up=torch.ones(2, 32, 16))
    _fused("l_down", l_down=torch.ones(1, 16, 48), r_up=ru)
    _fused("r_up", l_down=ld, r_up=torch.ones(1, 16, 16))
    _fused("r_up", l_down=ld, r_up=torch.ones(1, 32, 32))
    _fused("r_up", TypeError, l_down=ld, r_up=ru.bfloat16())
    _fused("together", l_down=ld)
    _fused("together", r_up=ru)


def test_a_layers_weight_fits():
    _fused("w_scale", w_scale=torch.ones(31))
    _fused("w_scale", TypeError, w_scale=torch.ones(32, dtype=torch.float64))
    _fused("wq", TypeError, wq=torch.zeros(32, 64))
    _fused("inv_smooth", TypeError, inv=torch.ones(2, 64, dtype=torch.float64))
