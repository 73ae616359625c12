"""Stages whose input is read by residual connections, with the gradient w.r.t. the input written over the upstream gradient or over the borrowed input, against the oracle (bounds of
tests/test_gpu_operator_layers.py)."""
import numpy as np
import pytest

from tests.test_gpu_operator_layers import both, run
from workloads.configs import conv, layernorm, linear, norm_join, resadd

pytestmark = pytest.mark.gpu

over = pytest.mark.parametrize("in_place", ["dy", "x"])


@both
@over
@pytest.mark.parametrize("opened", [1, 4, 8])
def test_a_join_of_the_stage_input_among_others(dtype, in_place, opened):
    """Joins that read the first results leave their gradients open when the one of the stage input comes."""
    d, rows = 32, 3
    specs = [linear(d, d, False, rows=rows) for _ in range(10)]
    specs += [norm_join(d, rows, 10) for _ in range(opened)]
    specs += [norm_join(d, rows, len(specs) + 1), layernorm(d, rows), linear(d, d, False, rows=rows)]
    for borrow in (True, False):
        run(specs, d * rows, dtype, 3, 2, seed=opened, borrow=borrow, in_place=in_place)


@both
@over
def test_two_joins_of_the_stage_input(dtype, in_place):
    d, rows = 40, 4
    run([linear(d, d, False, rows=rows), norm_join(d, rows, 2), linear(d, d, False, rows=rows), norm_join(d, rows, 4)], d * rows, dtype, 2, 3, seed=7, borrow=True, in_place=in_place)


@both
@over
def test_additions_of_the_stage_input(dtype, in_place):
    """Residual additions and dense layers that add another's input."""
    d, rows = 32, 4
    dense = linear(d, d, False, rows=rows)
    plain = lambda k: resadd(rows, 1, d, k, relu=False)   # noqa: E731
    run([dense, dense, dense, plain(4), dense], d * rows, dtype, 3, 2, seed=1, borrow=True, in_place=in_place)
    run([dense, plain(2), plain(3)], d * rows, dtype, 3, 2, seed=2, borrow=True, in_place=in_place)
    run([layernorm(d, rows), dense, linear(d, d, False, rows=rows, skip=2), layernorm(d, rows), dense], d * rows, dtype, 3, 2, seed=3, borrow=True, in_place=in_place)


@both
@over
def test_a_convolution_of_the_stage_input_beside_others(dtype, in_place):
    """Bit for bit what separate arrays give."""
    import torch
    from paper_2410_14312_amd import Stage

    h, c, M = 6, 16, 4
    specs = [conv(h, h, c, c, relu=False), conv(h, h, c, c, relu=False), conv(h, h, c, c, r=1, pad=0, relu=False, src=3), resadd(h, h, c, 2, relu=False)]
    rng = np.random.default_rng(4)
    p = [{"w": (0.1 * rng.standard_normal((c, r, r, c))).astype(np.float32), "b": rng.standard_normal(c).astype(np.float32)} for r in (3, 3, 1)] + [{}]
    x, dy = (rng.standard_normal((M, h * h * c)).astype(np.float32) for _ in range(2))
    got = []
    for place in (None, in_place):
        st = Stage(specs, dtype, M, 1, 1, 0.1, 0.9, borrow_input=True)
        st.set_params(p)
        xd, dyd = (torch.from_numpy(a).to(st.act_dtype).to(st.device) for a in (x, dy))
        dx = {None: torch.empty_like(xd), "dy": dyd, "x": xd}[place]
        st.forward_micro(0, xd)
        st.backward([0], dy=dyd, dx=dx)
        torch.cuda.synchronize()
        got.append((dx.clone(), st._flat(1, 1).clone()))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1]) and float(got[0][0].float().abs().max()) > 0


@both
@over
@pytest.mark.parametrize("kind", ["linear", "norm", "conv"])
def test_a_stage_of_one_layer(dtype, in_place, kind):
    """One kernel's workgroups read all of what the result lies over: bit for bit what separate arrays give, at a size of many workgroups."""
    import torch
    from paper_2410_14312_amd import Stage

    d, rows, M = 256, 64, 8
    specs, shapes = {"linear": ([linear(d, d, False, rows=rows)], {"w": (d, d), "b": (d,)}), "norm": ([layernorm(d, rows)], {"w": (d,), "b": (d,)}),
                     "conv": ([conv(8, 8, d, d, relu=False)], {"w": (d, 3, 3, d), "b": (d,)})}[kind]
    rng = np.random.default_rng(6)
    p = [{k: (0.05 * rng.standard_normal(v)).astype(np.float32) for k, v in shapes.items()}]
    x, dy = (rng.standard_normal((M, rows * d)).astype(np.float32) for _ in range(2))
    got = []
    for place in (None, in_place):
        st = Stage(specs, dtype, M, 1, 1, 0.1, 0.9, borrow_input=True)
        st.set_params(p)
        xd, dyd = (torch.from_numpy(a).to(st.act_dtype).to(st.device) for a in (x, dy))
        dx = {None: torch.empty_like(xd), "dy": dyd, "x": xd}[place]
        st.forward_micro(0, xd)
        st.backward([0], dy=dyd, dx=dx)
        torch.cuda.synchronize()
        got.append((dx.clone(), st._flat(1, 1).clone()))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
