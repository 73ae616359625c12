"""The short convolution against its sums in 64 bits.  Bounds: beside the rounding to the type, 2^-18 of the sizes of a sum's terms: some 20 roundings of 2^-24 in a sum of 8 taps, SiLU
(the hardware's exponential and reciprocal, 2^-22) and its slope; parameters' gradients are sums over up to a thousand rows in chains of at most 100 additions, 2^-17."""
import pytest
import torch

import paper_2410_14312_amd as tmps
from tests import mixers
from tests.mixers import DEV, TYPES, near

pytestmark = pytest.mark.gpu
SMALL, SUMS = 2.0 ** -18, 2.0 ** -17


@pytest.fixture(autouse=True)
def single_precision_by_default():
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


def inputs(seed, samples, positions, channels, taps, t, bias=True, carried=True):
    g = mixers.generator(seed)

    def normal(*s):
        return torch.randn(*s, generator=g).to(DEV)
    rows = samples * positions
    return {"x": normal(rows, channels).to(t), "weight": normal(channels, taps), "bias": normal(channels) if bias else None,
            "tail": normal(samples, taps - 1, channels).to(t) if carried else None, "dy": normal(rows, channels).to(t),
            "dtail": normal(samples, taps - 1, channels).to(t) if carried else None}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("samples,positions,channels,taps,silu,bias,carried", [
    (1, 1, 1, 1, True, True, True), (3, 1, 64, 4, True, True, True), (1, 2, 7, 4, True, True, True), (2, 3, 40, 8, True, False, True), (2, 16, 33, 2, False, True, False),
    (1, 17, 600, 3, True, True, True), (5, 31, 8, 5, True, True, False), (2, 130, 100, 4, True, True, True), (1, 64, 2050, 4, False, False, True), (2, 5, 12, 6, True, True, True),
    (1, 9, 24, 7, True, True, True)])
def test_values_and_gradients(samples, positions, channels, taps, silu, bias, carried, dtype):
    i = inputs(1, samples, positions, channels, taps, TYPES[dtype], bias, carried)
    y, tail = tmps.short_conv(i["x"], i["weight"], i["bias"], positions=positions, tail=i["tail"], want_tail=True, silu=silu)
    want, size = mixers.conv(i["x"], i["weight"], i["bias"], positions, i["tail"], silu)
    near(y, want["y"], size["y"], SMALL, "y")
    assert torch.equal(tail.double().cpu(), want["tail"])
    got = dict(zip(("dx", "dweight", "dbias", "dtail"), tmps.short_conv_backward(i["dy"], i["x"], i["weight"], i["bias"], positions=positions, tail=i["tail"], dtail=i["dtail"], silu=silu)))
    want, size = mixers.conv(i["x"], i["weight"], i["bias"], positions, i["tail"], silu, i["dy"], i["dtail"])
    assert (got["dbias"] is None) == (not bias) and (got["dtail"] is None) == (not carried)
    for name, w in want.items():
        near(got[name], w, size[name], SUMS if name in ("dweight", "dbias") else SMALL, name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_wider_rows(dtype):
    i = inputs(2, 2, 45, 50, 4, TYPES[dtype])
    kw = dict(positions=45, tail=i["tail"])
    want, grads = tmps.short_conv(i["x"], i["weight"], i["bias"], **kw)[0], tmps.short_conv_backward(i["dy"], i["x"], i["weight"], i["bias"], dtail=i["dtail"], **kw)
    wide = torch.full((90, 171), 7.0, dtype=TYPES[dtype], device=DEV)
    x, dy, y = wide[:, 3:53], wide[:, 60:110], wide[:, 117:167]
    x.copy_(i["x"])
    dy.copy_(i["dy"])
    out, _ = tmps.short_conv(x, i["weight"], i["bias"], out=y, **kw)
    assert out is y and torch.equal(y, want)
    got = tmps.short_conv_backward(dy, x, i["weight"], i["bias"], dtail=i["dtail"], dx=y, **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, grads))
    assert all(bool((wide[:, a:b] == 7).all()) for a, b in ((0, 3), (53, 60), (110, 117), (167, 171))) and torch.equal(x, i["x"]) and torch.equal(dy, i["dy"])


@pytest.mark.parametrize("channels", [64, 50])
def test_token_by_token_in_place(channels):
    i = inputs(3, 3, 20, channels, 4, torch.bfloat16)
    want, after = tmps.short_conv(i["x"], i["weight"], i["bias"], positions=20, tail=i["tail"], want_tail=True)
    x, tail, parts = i["x"].view(3, 20, channels), i["tail"].clone(), []
    for t in range(20):
        y, out = tmps.short_conv(x[:, t], i["weight"], i["bias"], tail=tail, tail_out=tail)
        assert out is tail
        parts.append(y)
    assert torch.equal(torch.stack(parts, 1).reshape(60, channels), want) and torch.equal(tail, after)
    with pytest.raises(tmps.TmpsError):
        tmps.short_conv(i["x"], i["weight"], i["bias"], positions=20, tail=tail, tail_out=tail)


@pytest.mark.parametrize("dtype,channels", [("bf16", 513), ("bf16", 1025 + 6), ("f32", 257), ("f32", 259), ("bf16", 9)])
def test_in_place_where_a_last_piece_is_another_workgroups(dtype, channels):
    """Channels of the piece before are read again by the last, which starts within it: its results must not come from a tail that has moved on."""
    i = inputs(5, 300, 1, channels, 4, mixers.TYPES[dtype])
    want, after = tmps.short_conv(i["x"], i["weight"], i["bias"], tail=i["tail"], want_tail=True)
    for _ in range(5):
        tail = i["tail"].clone()
        y, out = tmps.short_conv(i["x"], i["weight"], i["bias"], tail=tail, tail_out=tail)
        assert out is tail and torch.equal(y, want) and torch.equal(tail, after)


def test_a_number_that_is_not_finite_stays_within_its_taps():
    i = inputs(4, 1, 60, 16, 4, torch.float32, carried=False)
    want, _ = tmps.short_conv(i["x"], i["weight"], i["bias"], positions=60)
    x = i["x"].clone()
    x[30, 3] = float("nan")
    y, _ = tmps.short_conv(x, i["weight"], i["bias"], positions=60)
    bad = torch.isnan(y)
    assert bad[30:34, 3].all() and int(bad.sum()) == 4 and torch.equal(y[~bad], want[~bad])


def test_replays_of_a_graph():
    i = inputs(5, 2, 100, 48, 4, torch.bfloat16)

    def work():
        kw = dict(positions=100, tail=i["tail"])
        return list(tmps.short_conv(i["x"], i["weight"], i["bias"], want_tail=True, **kw)) + list(tmps.short_conv_backward(i["dy"], i["x"], i["weight"], i["bias"], dtail=i["dtail"], **kw))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work()
    for seed in (6, 7, 8):
        new = inputs(seed, 2, 100, 48, 4, torch.bfloat16)
        for k in i:
            i[k].copy_(new[k])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, work()))


def alike(got, want, size, relative, name):
    """near() where both are finite; infinities and NaN in the same places."""
    got, want = got.double().cpu(), want.double().cpu()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isfinite(got), fine) and torch.equal(got[torch.isinf(want)], want[torch.isinf(want)]), name
    assert bool(((got - want).abs() <= relative * size.double().cpu() + 1e-37)[fine].all()), name


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("at", [0, 12, 13, 15, 16, 30, 31, 32, 35, 36, 37, 38])
@pytest.mark.parametrize("of", ["x", "dy", "tail"])
def test_gradients_of_numbers_that_are_not_finite(of, at, bad):
    """Without SiLU a weight's gradient is a sum of products dy x: one infinity leaves an infinity, and taps that no position of the sample reads it by are as they are without it."""
    i = inputs(6, 2, 39, 24, 4, torch.float32)
    clean = {k: v.clone() for k, v in i.items()}
    if of == "tail":
        if at > 2:
            return
        i["tail"][0, at, 5] = bad
    else:
        i[of][at, 5] = bad
    names, kw = ("dx", "dweight", "dbias", "dtail"), dict(positions=39, silu=False)
    got = dict(zip(names, tmps.short_conv_backward(i["dy"], i["x"], i["weight"], i["bias"], tail=i["tail"], dtail=i["dtail"], **kw)))
    # (from the formula: autograd's sums take zeros times what lies beside a slice)
    u = torch.cat([i["tail"], i["x"].view(2, 39, 24)], 1).double()
    dz = i["dy"].view(2, 39, 24).double()
    want = {"dweight": torch.stack([(dz * u[:, j:j + 39]).sum((0, 1)) for j in range(4)], 1), "dbias": dz.sum((0, 1))}
    du = torch.zeros_like(u)
    du[:, 39:] = i["dtail"].double()
    for j in range(4):
        du[:, j:j + 39] += dz * i["weight"][:, j].double()
    want["dx"], want["dtail"] = du[:, 3:].reshape(78, 24), du[:, :3]
    _, size = mixers.conv(clean["x"], clean["weight"], clean["bias"], 39, clean["tail"], False, clean["dy"], clean["dtail"])
    for name in names:
        alike(got[name], want[name], size[name] + want[name].abs().nan_to_num(0.0, 0.0, 0.0).cpu(), SUMS, name)
