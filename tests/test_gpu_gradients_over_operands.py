"""Stages whose input is read by residual connections, with the gradient w.r.t. the input written over the upstream gradient or over the borrowed input, against the oracle (bounds of
tests/test_gpu_operator_layers.py)."""
import pytest

from tests.test_gpu_operator_layers import both, run
from workloads.configs import layernorm, linear, norm_join

pytestmark = pytest.mark.gpu

over = pytest.mark.parametrize("in_place", ["dy", "x"])


@both
@over
@pytest.mark.parametrize("opened", [1, 4])
def test_a_join_of_the_stage_input_among_others(dtype, in_place, opened):
    """Joins that read the first results leave their gradients open when the one of the stage input comes."""
    d, rows = 32, 3
    specs = [linear(d, d, False, rows=rows) for _ in range(6)]
    specs += [norm_join(d, rows, 6) for _ in range(opened)]
    specs += [norm_join(d, rows, len(specs) + 1), layernorm(d, rows), linear(d, d, False, rows=rows)]
    for borrow in (True, False):
        run(specs, d * rows, dtype, 3, 2, seed=opened, borrow=borrow, in_place=in_place)


@both
@over
def test_two_joins_of_the_stage_input(dtype, in_place):
    d, rows = 40, 4
    run([linear(d, d, False, rows=rows), norm_join(d, rows, 2), linear(d, d, False, rows=rows), norm_join(d, rows, 4)], d * rows, dtype, 2, 3, seed=7, borrow=True, in_place=in_place)
