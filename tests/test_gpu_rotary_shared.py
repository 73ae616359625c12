"""Rotary positions whose input other layers read too, against the oracle (bounds of tests/test_gpu_operator_layers.py): in a stage's middle, as its first layer, with the other
contribution before and behind theirs."""
import pytest

from tests.test_gpu_operator_layers import both, run
from workloads.configs import attention, linear, norm_join, resadd, rotary

pytestmark = pytest.mark.gpu


@both
@pytest.mark.parametrize("in_place", [None, "dy", "x"])
def test_shared_inputs(dtype, in_place):
    s, d, heads = 10, 16, 2
    wide, narrow, turn = linear(24, 3 * d, False, rows=s), linear(3 * d, 24, False, rows=s), rotary(s, d, heads, height=2, pairs_h=1)
    back = linear(24, 3 * d, False, rows=s)
    kw = dict(borrow=True, in_place=in_place)
    run([wide, turn, narrow, back, norm_join(3 * d, s, 4), narrow], 24 * s, dtype, 2, 2, seed=1, **kw)
    run([wide, turn, resadd(s, 1, 3 * d, 2, relu=False), narrow], 24 * s, dtype, 2, 2, seed=2, **kw)
    run([turn, narrow, back, norm_join(3 * d, s, 4)], 3 * d * s, dtype, 2, 2, seed=3, **kw)
    run([turn, turn, resadd(s, 1, 3 * d, 3, relu=False), attention(s, d, heads), linear(d, 3 * d, False, rows=s)], 3 * d * s, dtype, 2, 2, seed=4, **kw)


def test_without_an_input_gradient():
    s, d = 6, 8
    specs = [rotary(s, d, 1), linear(3 * d, 24, False, rows=s), linear(24, 3 * d, False, rows=s), norm_join(3 * d, s, 4)]
    run(specs, 3 * d * s, "f32", 2, 2, seed=5, want_dx=False)
