"""The selective state space against its recurrence in 64 bits, position by position.

Bounds.  Beside the rounding of a result to its type, an error is counted against the sum of the sizes of what a result is a sum of.  fp32: sums of up to 128 products and of 64
positions, and exponents: delta is off by some 2^-22 of itself and an exponent E by E 2^-22, exp(-E) then by at most 2^-22 / e of one; 256 roundings of 2^-24 = 2^-16 stand above all of it.
bf16, forward: states and decayed products are operands in two terms, off by 2^-17: 2^-15 for both.  bf16, backward: decayed products are rounded once, 2^-8, in dx (of x, B and C);
what is fp32 (gradients of parameters and states) and dt's gradient before its own rounding have the fp32 bound, and three terms of states, off by 2^-25."""
import pytest
import torch

import paper_2410_14312_amd as tmps
from tests import mixers
from tests.mixers import DEV, TYPES, near

pytestmark = pytest.mark.gpu
FP32, BF16, ROUNDED = 2.0 ** -16, 2.0 ** -15, 2.0 ** -8
SIZES = [  # samples, positions, heads, dh, groups, n, from a given state
    (1, 1, 1, 1, 1, 1, False), (2, 1, 3, 64, 1, 64, True), (3, 8, 2, 20, 2, 128, True), (2, 9, 2, 16, 1, 16, True), (1, 63, 3, 32, 3, 32, False), (2, 64, 2, 64, 1, 64, True),
    (1, 65, 4, 40, 2, 24, True), (2, 130, 5, 7, 1, 5, True), (1, 200, 2, 64, 1, 128, True), (1, 100, 2, 128, 1, 33, True), (1, 70, 2, 65, 1, 127, False), (1, 1100, 2, 33, 1, 16, True),
    (9, 33, 1, 200, 1, 100, True), (3, 2, 2, 128, 1, 128, True), (2, 5, 4, 64, 2, 64, False), (2, 3, 1, 96, 1, 128, True)]


@pytest.fixture(autouse=True)
def single_precision_by_default():
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


def forward(i, size, **kw):
    samples, positions, heads, dh, groups, n, carried = size
    return tmps.selective_scan(i["x"], i["dt"], i["a_log"], i["skip"], i["dt_bias"], positions=positions, state_features=n, groups=groups, state=i["state"], **kw)


def backward(i, size, **kw):
    samples, positions, heads, dh, groups, n, carried = size
    names = ("dx", "ddt", "da_log", "dskip", "ddt_bias", "dstate")
    return dict(zip(names, tmps.selective_scan_backward(i["dy"], i["x"], i["dt"], i["a_log"], i["skip"], i["dt_bias"], positions=positions, state_features=n, groups=groups,
                                                        state=i["state"], dstate=i["dstate"], **kw)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_forward(size, dtype):
    i = mixers.scan_inputs(1, *size[:6], TYPES[dtype], size[6])
    y, state = forward(i, size, want_state=True)
    want, sizes = mixers.scan(i, *size[:6]), mixers.scan(i, *size[:6], size=True)
    near(y, want["y"], sizes["y"], FP32 if dtype == "f32" else BF16, "y")
    near(state, want["state"], sizes["state"], FP32, "state")
    assert forward(i, size)[1] is None and torch.equal(forward(i, size)[0], y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_backward(size, dtype):
    i = mixers.scan_inputs(2, *size[:6], TYPES[dtype], size[6], backward=True)
    if size[2] * size[3] * i["x"].element_size() < 16:   # (rows are read 16 bytes at a time: narrower ones are refused)
        with pytest.raises(tmps.TmpsError):
            backward(i, size)
        return
    got = backward(i, size)
    want, sizes = mixers.scan(i, *size[:6], backward=True), mixers.scan(i, *size[:6], backward=True, size=True)
    assert (got["dstate"] is None) == (not size[6])
    for name, w in want.items():
        near(got[name], w, sizes[name], ROUNDED if dtype == "bf16" and name == "dx" else FP32, name)
    again = backward(i, size)
    assert all(torch.equal(got[k], again[k]) for k in want)


def test_gradients_against_differences():
    size = (1, 70, 2, 8, 1, 6, True)
    i = mixers.scan_inputs(3, *size[:6], torch.float32, True, backward=True)
    got = backward(i, size)

    def value(j):
        out = mixers.scan(j, *size[:6])
        return float((out["y"] * i["dy"].double()).sum() + (out["state"] * i["dstate"].double()).sum())
    step = 1e-6
    gen = mixers.generator(4)
    for name, grad in (("x", "dx"), ("dt", "ddt"), ("a_log", "da_log"), ("skip", "dskip"), ("dt_bias", "ddt_bias"), ("state", "dstate")):
        way = torch.randn(i[name].shape, generator=gen).to(DEV).double()
        up, down = (value(dict(i, **{name: i[name].double() + sign * step * way})) for sign in (1, -1))
        along = float((got[grad].double() * way).sum())
        # (the difference's own error is some step^2, or 2^-53 of the value / step)
        assert abs(along - (up - down) / (2 * step)) <= 1e-4 * float((got[grad].double() * way).abs().sum()), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_wider_rows(dtype):
    size = (2, 75, 3, 24, 1, 20, True)
    i = mixers.scan_inputs(5, *size[:6], TYPES[dtype], True, backward=True)
    want, grads = forward(i, size, want_state=True), backward(i, size)
    rows, wide = i["x"].shape
    around = torch.full((rows, wide + 3 + 17), 7.0, dtype=TYPES[dtype], device=DEV)   # [1 | x | 5 | dt | 11]
    j = dict(i, x=around[:, 1:1 + wide], dt=around[:, wide + 6:wide + 9], dy=torch.cat([i["dy"], i["dy"]], 1)[:, 72:])
    j["x"].copy_(i["x"])
    j["dt"].copy_(i["dt"])
    y = torch.full((rows, 100), 3.0, dtype=TYPES[dtype], device=DEV)
    out, state = forward(j, size, want_state=True, out=y[:, 9:81])
    assert torch.equal(out, want[0]) and torch.equal(state, want[1]) and bool((y[:, :9] == 3).all()) and bool((y[:, 81:] == 3).all())
    d = torch.full_like(around, 5.0)
    got = backward(j, size, dx=d[:, 1:1 + wide], ddt=d[:, wide + 6:wide + 9])
    assert all(torch.equal(got[k], grads[k]) for k in grads)
    assert bool((d[:, 0] == 5).all()) and bool((d[:, wide + 1:wide + 6] == 5).all()) and bool((d[:, wide + 9:] == 5).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cut", [1, 8, 64, 100])
def test_a_prompt_in_parts(dtype, cut):
    """The state of the first part is where the second begins, and may be the memory of the state behind it."""
    size = (2, 150, 2, 32, 1, 48, True)
    i = mixers.scan_inputs(6, *size[:6], TYPES[dtype], True)
    want, sizes = mixers.scan(i, *size[:6]), mixers.scan(i, *size[:6], size=True)
    x, dt = i["x"].view(2, 150, -1), i["dt"].view(2, 150, -1)
    state, parts = i["state"].clone(), []
    for first, last in ((0, cut), (cut, 150)):
        j = dict(i, x=x[:, first:last].reshape(-1, x.shape[2]).contiguous(), dt=dt[:, first:last].reshape(-1, 2).contiguous(), state=state)
        y, after = forward(j, (2, last - first) + size[2:], state_out=state)
        assert after is state
        parts.append(y.view(2, last - first, -1))
    near(torch.cat(parts, 1).reshape(300, -1), want["y"], sizes["y"], FP32 if dtype == "f32" else BF16, "y")
    near(state, want["state"], sizes["state"], 2 * FP32, "state")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_numbers_that_are_not_finite_reach_later_positions_alone(dtype, bad):
    size = (2, 130, 2, 32, 1, 32, False)
    i = mixers.scan_inputs(7, *size[:6], TYPES[dtype], False)
    want, _ = forward(i, size)
    for at in (0, 37, 64, 129):
        for column in (5, 64 + 3, 96 + 3):   # of x, B, C
            j = dict(i, x=i["x"].clone())
            j["x"][at, column] = bad
            y, _ = forward(j, size)
            assert torch.equal(y[:at], want[:at]) and torch.equal(y[130:], want[130:]), (at, column)
            assert not bool(torch.isfinite(y[at]).all())
            if column == 5:   # the other features, and heads, are their own
                rest = [c for c in range(64) if c != 5]
                assert torch.equal(y[:, rest], want[:, rest])
        j = dict(i, dt=i["dt"].clone())
        j["dt"][at, 1] = bad
        y, _ = forward(j, size)
        assert torch.equal(y[:at], want[:at]) and torch.equal(y[:, :32], want[:, :32])


def test_extreme_steps():
    """Steps so large that nothing of the past is left, so small that nothing is forgotten, and none at all."""
    size = (1, 140, 3, 16, 1, 16, True)
    i = mixers.scan_inputs(8, *size[:6], torch.float32, True, backward=True)
    i["dt_bias"] = torch.tensor([60.0, -30.0, -200.0], device=DEV)
    y, state = forward(i, size, want_state=True)
    want, sizes = mixers.scan(i, *size[:6]), mixers.scan(i, *size[:6], size=True)
    near(y, want["y"], sizes["y"], FP32, "y")
    near(state, want["state"], sizes["state"], FP32, "state")
    got = backward(i, size)
    want, sizes = mixers.scan(i, *size[:6], backward=True), mixers.scan(i, *size[:6], backward=True, size=True)
    for name, w in want.items():
        near(got[name], w, sizes[name], FP32, name)


@pytest.mark.parametrize("positions", [1, 300])
def test_replays_of_a_graph(positions):
    size = (2, positions, 3, 32, 1, 32, True)
    i = mixers.scan_inputs(9, *size[:6], torch.bfloat16, True, backward=True)

    def work():
        y, state = forward(i, size, want_state=True)
        return [y, state] + [v for v in backward(i, size).values()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work()
    for seed in (10, 11, 12):
        new = mixers.scan_inputs(seed, *size[:6], torch.bfloat16, True, backward=True)
        for k in i:
            i[k].copy_(new[k])
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, work()):
            assert torch.equal(a, b)


def test_calls_on_two_streams_at_once():
    size = (2, 400, 4, 64, 1, 64, True)
    sets = [mixers.scan_inputs(20 + k, *size[:6], torch.bfloat16, True, backward=True) for k in range(2)]
    want = [(forward(i, size, want_state=True), backward(i, size)) for i in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(3):
        got = [(forward(i, size, want_state=True, stream=s), backward(i, size, stream=s)) for i, s in zip(sets, streams)]
        torch.cuda.synchronize()
        for (f, b), (wf, wb) in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(f, wf)) and all(torch.equal(b[k], wb[k]) for k in wb)


def test_no_samples():
    size = (0, 5, 2, 16, 1, 16, True)
    i = mixers.scan_inputs(1, *size[:6], torch.float32, True)
    y, state = forward(i, size, want_state=True)
    assert y.shape == (0, 32) and state.shape == (0, 2, 16, 16)


@pytest.mark.parametrize("a_log", [90.0, 200.0, 720.0])
@pytest.mark.parametrize("positions", [5, 200])
def test_rates_beyond_single_precision(positions, a_log):
    """Nothing of a state is left after a step: y = delta (C . B) x + skip x, and no gradient of the rate."""
    sizes = (2, positions, 2, 16, 1, 8, True)
    i = mixers.scan_inputs(19, *sizes[:6], torch.float32, True, True)
    i["a_log"] = torch.full_like(i["a_log"], a_log)
    y, state = forward(i, sizes, want_state=True)
    x = i["x"].double()
    xs, bs, cs = x[:, :32].view(-1, 2, 16), x[:, 32:40], x[:, 40:]
    delta = torch.nn.functional.softplus(i["dt"].double() + i["dt_bias"].double())
    terms = delta[..., None] * (cs * bs).sum(1)[:, None, None] * xs
    size = delta[..., None] * (cs * bs).abs().sum(1)[:, None, None] * xs.abs() + (i["skip"].double()[:, None] * xs).abs()
    mixers.near(y, (terms + i["skip"].double()[:, None] * xs).reshape(-1, 32), size.reshape(-1, 32), 32 * mixers.F32)
    last = (delta[..., None] * xs)[..., None] * bs[:, None, None]
    mixers.near(state, last.view(2, positions, 2, 16, 8)[:, -1], last.abs().view(2, positions, 2, 16, 8)[:, -1], 16 * mixers.F32)
    back = backward(i, sizes)
    assert all(bool(torch.isfinite(v).all()) for v in back.values()) and not bool(back["da_log"].any()) and not bool(back["dstate"].any())


@pytest.mark.parametrize("size", SIZES)
def test_backward_of_bf16_as_exact_as_forward(size):
    """Decayed products go into dx (of x, B and C) in two terms, as they do into y: the bound is the forward pass's."""
    i = mixers.scan_inputs(2, *size[:6], torch.bfloat16, size[6], backward=True)
    if size[2] * size[3] < 8:
        return   # (refused)
    want, sizes = mixers.scan(i, *size[:6], backward=True), mixers.scan(i, *size[:6], backward=True, size=True)
    near(backward(i, size)["dx"], want["dx"], sizes["dx"], BF16, "dx")


@pytest.mark.parametrize("of", ["state", "dstate"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_exponents_gradients_keep_the_states_bits(dtype, of):
    """A state, or gradient of one, of 1 + 2^-9 + 2^-17 - 2^-23 everywhere, of which two bf16 terms leave out 2^-17, and of which the sums with ones below are exact but for some 32
    roundings of 2^-24 (16 and 2 additions of a column, 6 of positions, and products) and what decays and steps are off by, 2^-22 each: 2^-18 of both terms, what a step adds and what
    it leaves of the state."""
    size = (1, 64, 1, 64, 1, 64, True)
    i = mixers.scan_inputs(30, *size[:6], TYPES[dtype], True, backward=True)
    for name in ("x", "dy", "state", "dstate"):
        i[name].zero_()
    i[of].fill_(1.0 + 2.0 ** -9 + 2.0 ** -17 - 2.0 ** -23)
    if of == "state":
        i["x"][:, 128:] = 1.0
        i["dy"].fill_(1.0)
    else:
        i["x"][:, :128] = 1.0
    i["a_log"].zero_()
    got = backward(i, size)
    want, sizes = mixers.scan(i, *size[:6], backward=True), mixers.scan(i, *size[:6], backward=True, size=True, across=True)
    for name in ("ddt", "da_log", "ddt_bias"):
        near(got[name], want[name], sizes[name], 2.0 ** -18, name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_exponents_gradients_of_what_passes_through_alone(dtype):
    """Steps that forget nearly all between steps that forget next to nothing, at a large rate: what ends before a position, or begins behind it, leaves nothing in the gradient of its
    exponent.  At the first position, from no state, that is all of it."""
    size = (2, 150, 2, 32, 1, 32, False)
    i = mixers.scan_inputs(31, *size[:6], TYPES[dtype], False, backward=True)
    i["a_log"] = torch.tensor([8.0, 10.0], device=DEV)
    i["dt_bias"].zero_()
    steps = torch.where(torch.arange(150) % 5 == 1, 300.0, 0.02)[None, :, None] * torch.exp(-i["a_log"].cpu())   # times the rate
    i["dt"] = torch.log(torch.expm1(steps.double())).expand(2, 150, 2).reshape(300, 2).to(TYPES[dtype]).to(DEV)
    x = i["x"].view(2, 150, -1)
    x[:, 0, :64] *= 2.0 ** -10
    got = backward(i, size)
    want, sizes = mixers.scan(i, *size[:6], backward=True), mixers.scan(i, *size[:6], backward=True, size=True, across=True)
    for name in ("ddt", "da_log", "ddt_bias"):
        near(got[name], want[name], sizes[name], FP32, name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_exponents_gradients_of_any_size_of_what_passes_through(size, dtype):
    i = mixers.scan_inputs(32, *size[:6], TYPES[dtype], size[6], backward=True)
    if size[2] * size[3] * i["x"].element_size() < 16:
        return   # (refused)
    got = backward(i, size)
    want, sizes = mixers.scan(i, *size[:6], backward=True), mixers.scan(i, *size[:6], backward=True, size=True, across=True)
    for name in ("ddt", "da_log", "ddt_bias"):
        near(got[name], want[name], sizes[name], FP32, name)


@pytest.mark.parametrize("positions", [1, 3])
def test_heads_of_millions_of_features(positions):
    """More slices of 64 features than a launch has in its second direction."""
    size = (1, positions, 1, 4194304 + 65, 1, 2, True)
    i = mixers.scan_inputs(33, *size[:6], torch.bfloat16, True)
    y, state = forward(i, size, want_state=True)
    want, sizes = mixers.scan(i, *size[:6]), mixers.scan(i, *size[:6], size=True)
    near(y, want["y"], sizes["y"], BF16, "y")
    near(state, want["state"], sizes["state"], FP32, "state")
