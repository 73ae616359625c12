"""The operators of a block that mixes positions by a recurrence one after the other, as a program has them: convolution, state space, group norm, and the gradients back through all of
them to a clipped update; a prompt and its tokens, eager and replayed; streams."""
import numpy as np
import pytest
import torch

import paper_2410_14312_amd as tmps
from tests.mixers import DEV, F32, generator

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.fixture(autouse=True)
def single_precision_by_default():
    """(tests of the oracle leave their process at doubles)"""
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


class Block:
    """Rows [x B C | dt] of a product: x B C through the convolution, the state space, the norm of its groups."""

    def __init__(self, samples, positions, heads, dh, groups, n, taps=4, seed=3, dtype=torch.float32):
        g = generator(seed)
        normal = lambda *s: torch.randn(*s, generator=g)   # noqa: E731
        self.b, self.s, self.h, self.p, self.g, self.n, self.k = samples, positions, heads, dh, groups, n, taps
        self.inner, self.wide = heads * dh, heads * dh + 2 * groups * n
        rows = samples * positions
        self.host = {"rows": normal(rows, self.wide + heads).to(dtype), "weight": normal(self.wide, taps) / taps ** 0.5, "bias": 0.1 * normal(self.wide),
                     "a_log": torch.log(1.0 + 15.0 * torch.rand(heads, generator=g)), "skip": 1.0 + 0.1 * normal(heads), "dt_bias": -2.0 + torch.rand(heads, generator=g),
                     "gain": 1.0 + 0.2 * normal(self.inner), "shift": 0.1 * normal(self.inner)}
        self.dy = normal(rows, self.inner).to(dtype)
        self.dev, self.dy_dev = {k: v.to(DEV) for k, v in self.host.items()}, self.dy.to(DEV)

    def run(self, rows=None, positions=None, tail=None, state=None, keep=False, into=None):
        d, s = self.dev, positions or self.s
        rows = d["rows"] if rows is None else rows
        u, tail_out = tmps.short_conv(rows[:, :self.wide], d["weight"], d["bias"], positions=s, tail=tail, want_tail=keep, tail_out=into[0] if into else None)
        y, state_out = tmps.selective_scan(u, rows[:, self.wide:], d["a_log"], d["skip"], d["dt_bias"], s, self.n, self.g, state=state, want_state=keep, state_out=into[1] if into else None)
        out, stats = tmps.group_norm(y, d["gain"], d["shift"], groups=self.g, act="silu", rms=True)
        return out, u, y, stats, tail_out, state_out

    def gradients(self):
        d, dy = self.dev, self.dy_dev
        _, u, y, stats, _, _ = self.run()
        drows = torch.full_like(d["rows"], float("nan"))
        dyn, dgain, dshift = tmps.group_norm_backward(dy, y, stats, d["gain"], d["shift"], groups=self.g, act="silu", rms=True)[:3]
        back = tmps.selective_scan_backward(dyn, u, d["rows"][:, self.wide:], d["a_log"], d["skip"], d["dt_bias"], self.s, self.n, self.g, ddt=drows[:, self.wide:])
        du, da_log, dskip, ddt_bias = back[0], back[2], back[3], back[4]
        dweight, dbias = tmps.short_conv_backward(du, d["rows"][:, :self.wide], d["weight"], d["bias"], positions=self.s, dx=drows[:, :self.wide])[1:3]
        return {"rows": drows, "weight": dweight, "bias": dbias, "a_log": da_log, "skip": dskip, "dt_bias": ddt_bias, "gain": dgain, "shift": dshift}

    def plain(self, leaf):
        b, s, h, p, g, n, k = self.b, self.s, self.h, self.p, self.g, self.n, self.k
        rows = leaf["rows"].view(b, s, -1)
        u = torch.cat([torch.zeros(b, k - 1, self.wide, dtype=torch.float64), rows[..., :self.wide]], 1)
        u = torch.nn.functional.silu(sum(u[:, j:j + s] * leaf["weight"][:, j] for j in range(k)) + leaf["bias"])
        x = u[..., :self.inner].reshape(b, s, h, p)
        bs, cs = (v.reshape(b, s, g, 1, n).expand(b, s, g, h // g, n).reshape(b, s, h, n) for v in u[..., self.inner:].split(g * n, -1))
        delta = torch.nn.functional.softplus(rows[..., self.wide:] + leaf["dt_bias"], threshold=100)
        state, ys = torch.zeros(b, h, p, n, dtype=torch.float64), []
        for t in range(s):
            state = torch.exp(-delta[:, t] * leaf["a_log"].exp())[..., None, None] * state + (delta[:, t, :, None] * x[:, t])[..., None] * bs[:, t, :, None]
            ys.append((state * cs[:, t, :, None]).sum(-1) + leaf["skip"][:, None] * x[:, t])
        y = torch.stack(ys, 1).reshape(b * s, g, -1)
        xhat = y * (y.square().mean(2, keepdim=True) + 1e-5).rsqrt()
        return torch.nn.functional.silu(xhat.reshape(b * s, -1) * leaf["gain"] + leaf["shift"])

    def plain_loss(self, leaf):
        return (self.plain(leaf) * self.dy.double()).sum()


# Each of the three operators is sums of up to 256 terms in a row whose sizes are up to eight times the sum, and so is each of their gradients, of what the others are off by: six of them,
# 6 * 256 * 8 * 2^-24 of the largest value.
CHAIN = 6 * 256 * 8 * F32
SHAPES = [(2, 150, 4, 16, 2, 8), (3, 1, 2, 64, 1, 16), (1, 333, 6, 20, 3, 5)]


@pytest.mark.parametrize("shape", SHAPES)
def test_gradients_through_all_of_them_and_a_clipped_update(shape):
    block = Block(*shape)
    got = block.gradients()
    with torch.enable_grad():
        leaf = {k: v.double().requires_grad_(True) for k, v in block.host.items()}
        out = block.plain(leaf)
        want = dict(zip(leaf, torch.autograd.grad((out * block.dy.double()).sum(), list(leaf.values()))))
    assert float((block.run()[0].double().cpu() - out.detach()).abs().max()) <= CHAIN * float(out.detach().abs().max())
    for k in want:
        assert got[k].shape == want[k].shape
        assert float((got[k].double().cpu() - want[k]).abs().max()) <= CHAIN * float(want[k].abs().max()), k
    # clipped together to half their norm, and stepped
    norm64 = sum(v.square().sum() for v in want.values()).sqrt()
    grads = list(got.values())
    before = [g.clone() for g in grads]
    norm = tmps.clip_gradients(grads, 0.5 * float(norm64))
    assert abs(float(norm) - float(norm64)) <= CHAIN * len(grads) * float(norm64)
    for a, b in zip(grads, before):
        assert torch.allclose(a, b * (0.5 * float(norm64) / float(norm)), rtol=4 * F32, atol=1e-38)
    assert abs(float(tmps.clip_gradients(grads, INF)) - 0.5 * float(norm64)) <= 1e-5 * float(norm64)


@pytest.mark.parametrize("name", ["rows", "weight", "bias", "a_log", "skip", "dt_bias", "gain", "shift"])
def test_against_differences(name):
    """Along a direction: (L(v + h d) - L(v - h d)) / 2h in 64 bits, off by h^2 and 2^-52 / h, some 1e-9 of the loss."""
    block = Block(*SHAPES[0])
    got = block.gradients()[name].double().cpu()
    d = torch.randn(got.shape, generator=generator(7), dtype=torch.float64)
    with torch.no_grad():
        leaf = {k: v.double() for k, v in block.host.items()}
        h = 1e-5
        up, down = (float(block.plain_loss(dict(leaf, **{name: leaf[name] + e * h * d}))) for e in (1.0, -1.0))
    size = float((got.abs().max() * d.abs()).sum())
    assert abs(float((got * d).sum()) - (up - down) / (2 * h)) <= CHAIN * size + 1e-6 * size


@pytest.mark.parametrize("shape,cut", [((2, 150, 4, 16, 2, 8), 141), ((1, 90, 6, 64, 1, 128), 64), ((3, 12, 2, 20, 1, 5), 1)])
def test_a_prompt_and_its_tokens_are_the_whole(shape, cut):
    """The states of a prompt's end carried through single tokens, in place."""
    block = Block(*shape)
    b, s = shape[:2]
    want = block.run()[0].view(b, s, -1)
    rows = block.dev["rows"].view(b, s, -1)
    out, _, _, _, tail, state = block.run(rows[:, :cut].reshape(b * cut, -1), cut, keep=True)
    out = out.view(b, cut, -1)
    largest = float(want.abs().max())
    assert float((out - want[:, :cut]).abs().max()) <= CHAIN * largest
    for t in range(cut, s):
        token = block.run(rows[:, t].contiguous(), 1, tail=tail, state=state, into=(tail, state))
        assert token[4] is tail and token[5] is state
        assert float((token[0] - want[:, t]).abs().max()) <= CHAIN * largest, t


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_tokens_replayed(dtype):
    """One token's launches captured, its states in place; every replay against the eager run of its token, other work and synchronizations between them."""
    block = Block(4, 8, 4, 64, 1, 64, dtype=dtype)
    rows = block.dev["rows"].view(4, 8, -1)
    tails, states = [torch.zeros(4, 3, block.wide, dtype=dtype, device=DEV) for _ in range(2)], [torch.zeros(4, 4, 64, 64, device=DEV) for _ in range(2)]
    row = rows[:, 0].contiguous()
    block.run(row, 1, tail=tails[0], state=states[0], into=(tails[0], states[0]))
    tails[0].zero_()
    states[0].zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block.run(row, 1, tail=tails[0], state=states[0], into=(tails[0], states[0]))[0]
    for t in range(8):
        row.copy_(rows[:, t])
        graph.replay()
        torch.cuda.synchronize()
        want = block.run(rows[:, t].contiguous(), 1, tail=tails[1], state=states[1], into=(tails[1], states[1]))[0]
        assert torch.equal(out, want) and torch.equal(tails[0], tails[1]) and torch.equal(states[0], states[1]), t


def test_a_training_step_replayed():
    """The forward and backward calls and the clipping, captured, with the graph's own workspaces; inputs that change between replays."""
    block = Block(2, 700, 4, 64, 1, 64, dtype=torch.bfloat16)

    def step():
        g = block.gradients()
        grads = [g[k] for k in g]
        return grads + [tmps.clip_gradients(grads, 1.0)]
    step()
    torch.cuda.synchronize()
    graphs, results = [], []
    for _ in range(2):   # (two graphs, which have nothing in common but the inputs)
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            results.append(step())
    for k in range(4):
        block.dev["rows"].mul_(0.9)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = step()
        torch.cuda.synchronize()
        for got in results:
            assert all(torch.equal(a, b) for a, b in zip(got, want)), k


def calls():
    block = Block(3, 700, 4, 32, 2, 24)
    d, x = block.dev, block.dev["rows"][:, :block.wide]
    _, u, y, stats, _, _ = block.run()
    dt, dy = d["rows"][:, block.wide:], block.dy_dev
    du = torch.ones_like(u)
    kw = dict(positions=block.s, state_features=block.n, groups=block.g)
    return {"short_conv": lambda **k: tmps.short_conv(x, d["weight"], d["bias"], block.s, want_tail=True, **k),
            "short_conv_backward": lambda **k: tmps.short_conv_backward(du, x, d["weight"], d["bias"], block.s, **k)[:3],
            "selective_scan": lambda **k: tmps.selective_scan(u, dt, d["a_log"], d["skip"], d["dt_bias"], want_state=True, **kw, **k),
            "selective_scan_backward": lambda **k: tmps.selective_scan_backward(dy, u, dt, d["a_log"], d["skip"], d["dt_bias"], **kw, **k)[:5],
            "group_norm": lambda **k: tmps.group_norm(y, d["gain"], d["shift"], groups=4, positions=block.s, act="gelu", **k),
            "group_norm_backward": lambda **k: tmps.group_norm_backward(dy, y, tmps.group_norm(y, d["gain"], d["shift"], groups=2, positions=block.s)[1], d["gain"], d["shift"], groups=2,
                                                                        positions=block.s, **k)[:3],
            "clip_gradients": lambda **k: (lambda out: [tmps.clip_gradients([u, dy], 1.0, out=out, **k)] + out)([torch.empty_like(u), torch.empty_like(dy)])}


NAMES = ["short_conv", "short_conv_backward", "selective_scan", "selective_scan_backward", "group_norm", "group_norm_backward", "clip_gradients"]


@pytest.mark.parametrize("name", NAMES)
def test_streams(name):
    """Results belong to the stream that is given; calls that overlap have workspaces of their own."""
    call = calls()[name]
    want = call()
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [call(stream=sides[k % 2]) for k in range(12)]
    assert torch.cuda.current_stream() == torch.cuda.default_stream()
    torch.cuda.synchronize()
    segments = torch.cuda.memory_snapshot()

    def owner(t):
        return next(s["stream"] for s in segments if s["address"] <= t.data_ptr() < s["address"] + s["total_size"])
    for k, g in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(g, want))
        assert owner(g[0]) == sides[k % 2].cuda_stream


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("share", [0.25, 4.0])
def test_a_stage_clips_its_gradients(dtype, share):
    """Between a stage's backward pass and its update."""
    from paper_2410_14312_amd import Stage
    from workloads.configs import linear
    gen = generator(11)
    specs = [linear(24, 40, True), linear(40, 8, False)]
    stage = Stage(specs, dtype, 16, 1, 1, 0.5, 0.0, borrow_input=True)
    stage.set_params([{"w": torch.randn(o, i, generator=gen).numpy(), "b": torch.randn(o, generator=gen).numpy()} for i, o in ((24, 40), (40, 8))])
    x, dy = (torch.randn(16, n, generator=gen).to(DEV).to(stage.act_dtype) for n in (24, 8))
    stage.forward_micro(0, x)
    stage.backward([0], dy=dy)
    torch.cuda.synchronize()
    grads, params = stage.get_grads(), stage.get_params()
    norm64 = sum((np.asarray(v, np.float64) ** 2).sum() for p in grads for v in p.values()) ** 0.5
    norm = float(stage.clip_gradients(share * norm64))
    assert abs(norm - norm64) <= 4 * F32 * norm64
    stage.update()
    torch.cuda.synchronize()
    factor = min(1.0, share)
    for a, b, p, q in zip(grads, stage.get_grads(), params, stage.get_params()):
        for k in a:
            clipped = np.asarray(a[k], np.float64) * factor
            # (the factor has the norm's rounding, its own and the quotient's; the product one)
            assert (np.abs(b[k] - clipped) <= 8 * F32 * np.abs(clipped)).all()
            assert (np.abs(q[k] - (p[k] - 0.5 * clipped)) <= 8 * F32 * (np.abs(p[k]) + np.abs(clipped))).all()
