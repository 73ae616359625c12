"""Temperatures of a distillation whose square no float has are refused, by the call and by a stage, without a GPU."""
import pytest

from paper_2410_14312_amd import binding
from tests.test_operator_refusals import distill
from workloads.configs import distill as layer, linear

EINVAL = -1


@pytest.mark.parametrize("T", [3e-39, 4e-39, 1e-38, 1e-30, 1e-23, 1e-19, 1.9e19, 3e38])
def test_refused(T):
    assert distill(T=T) == EINVAL
    cfg = binding.StageCfg(0, 2, 2, 2, 1, 0, 0.1, 0.9)
    with pytest.raises(binding.TmpsError):
        binding.stage_bytes([linear(4, 9, False), layer(9, 1, 2, T, 0.5)], cfg)


@pytest.mark.parametrize("T", [1.2e-19, 1e-3, 1.0, 1e3, 1.8e19])
def test_accepted(T):
    """(refused for an address behind that check: nothing is launched)"""
    assert distill(T=T, z=(1 << 20) + 2) == -2
    binding.stage_bytes([linear(4, 9, False), layer(9, 1, 2, T, 0.5)], binding.StageCfg(0, 2, 2, 2, 1, 0, 0.1, 0.9))
