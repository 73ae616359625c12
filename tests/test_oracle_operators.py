"""The oracle's norms around a block, rotary positions and distillation: gradients against central differences in 64 bits (error h^2 + 2^-52 / h: 1e-6 of the largest with
h = 1e-4 is reached with room), and the definitions at points worked by hand."""
import numpy as np
import pytest

from oracle import layers as L
from oracle.stage import Stage
from workloads.configs import distill, gated_block, layernorm, linear, norm_join, rotary
from workloads.synth import param_shapes


def _stage(specs, rng, M=2):
    ps = [{k: rng.standard_normal(v) * 0.4 + (1.0 if sp["kind"] in ("norm_join", "layernorm") else 0.0) for k, v in param_shapes(sp).items()} for sp in specs]
    return Stage(specs, ps, 0.1, 0.0, M, 1), ps


@pytest.mark.parametrize("name,specs,n_in", [
    ("rms", [layernorm(6, 3, rms=True)], 18), ("join", [linear(5, 5, False, rows=2), norm_join(5, 2, 2)], 10),
    ("rms join", [linear(5, 5, False, rows=2), norm_join(5, 2, 2, rms=True), layernorm(5, 2, rms=True)], 10),
    ("gate", [linear(5, 10, False, rows=2), norm_join(5, 2, 2, gate=True), layernorm(5, 2)], 10),
    ("rotary", [rotary(6, 8, 2, height=1, width=3, pairs_w=1)], 144), ("interleaved", [rotary(6, 8, 1, height=2, width=1, pairs_h=2, own_ladders=True, interleaved=True)], 144),
    ("block", gated_block(4, 8, 2, 6), 32)])
def test_gradients(name, specs, n_in):
    rng = np.random.default_rng(len(name))
    st, ps = _stage(specs, rng)
    x = rng.standard_normal((2, n_in))
    y = st.forward_micro(0, x)
    w = rng.standard_normal(y.shape)
    dx = st.backward([0], w.reshape(2, -1))
    grads, h = st.grads, 1e-4

    def value(x_, ps_):
        return float((Stage(specs, ps_, 0.1, 0.0, 2, 1).forward_micro(0, x_) * w).sum())
    d = rng.standard_normal(x.shape)
    assert abs((value(x + h * d, ps) - value(x - h * d, ps)) / (2 * h) - (dx * d).sum()) < 1e-5 * (1 + np.abs(dx * d).sum())
    for li, g in enumerate(grads):
        for k in g or {}:
            d = rng.standard_normal(g[k].shape)
            moved = [[dict(p, **({k: p[k] + s * h * d} if i == li else {})) for i, p in enumerate(ps)] for s in (1, -1)]
            assert abs((value(x, moved[0]) - value(x, moved[1])) / (2 * h) - (g[k] * d).sum()) < 1e-5 * (1 + np.abs(g[k] * d).sum()), (li, k)


@pytest.mark.parametrize("T,alpha", [(1.0, 1.0), (2.0, 0.3), (0.5, 0.0)])
def test_distillation_gradient(T, alpha):
    rng = np.random.default_rng(4)
    z = rng.standard_normal((5, 7))
    rec = np.concatenate([np.array([[2], [-1], [0], [-1], [6]]), np.array([[1, 3, 1], [0, -1, 5], [-1, -1, -1], [-1, -1, -1], [6, 6, 6]]),
                          rng.standard_normal((5, 3)).astype(np.float32).view(np.int32)], axis=1).astype(np.int32)
    loss, cache = L.distill_forward(z, rec, 3, T, alpha)
    g, h, d = L.distill_backward(cache, 5), 1e-4, rng.standard_normal(z.shape)
    slope = (L.distill_forward(z + h * d, rec, 3, T, alpha)[0] - L.distill_forward(z - h * d, rec, 3, T, alpha)[0]) / (2 * h)
    assert abs(slope - (g * d).sum()) < 1e-6
    assert np.all(g[3] == 0) and np.allclose(g.sum(1), 0, atol=1e-15)


def test_by_hand():
    # one entry: the teacher is sure of class 1, the student gives it 1/4; with T = 2 the logits (0, 2 log 1/3 ..) are halved first
    z = np.array([[0.0, -2 * np.log(3.0)]])
    rec = np.array([[-1, 1, np.float32(0).view(np.int32)]], dtype=np.int32)
    loss, c = L.distill_forward(z, rec, 1, 2.0, 1.0)
    assert abs(loss - 4 * np.log(4.0)) < 1e-12 and np.allclose(c["g"], [[1.5, -1.5]])
    y, _ = L.norm_join_forward(np.array([[3.0, -4.0, 0.0, 0.0]]), np.array([[1.0, 2.0]]), np.ones(2), np.array([10.0, 1.0]), 2, True, True)
    n = np.array([3.0, -4.0]) / np.sqrt(12.5 + 1e-5)
    assert np.allclose(y, [[10.0, 2.0] + 0.5 * n])
    qkv = np.arange(12.0).reshape(1, 12)   # two positions of q, k, v of two features
    got = L.rotary_apply(qkv, rotary(2, 2, 1)).reshape(2, 3, 2)
    c1, s1 = np.cos(1.0), np.sin(1.0)
    assert np.allclose(got[0], qkv.reshape(2, 3, 2)[0]) and np.allclose(got[1, 0], [6 * c1 - 7 * s1, 7 * c1 + 6 * s1]) and np.allclose(got[1, 2], [10, 11])


def test_a_stage_that_distills():
    rng = np.random.default_rng(8)
    specs = [linear(3, 4, False, rows=2), distill(4, 2, 1, 1.0, 0.5)]
    st, ps = _stage(specs, rng)
    x = rng.standard_normal((2, 6))
    rec = np.array([[[0, 1, 0], [-1, -1, 0]], [[3, 3, 0], [2, -1, 0]]], dtype=np.int32)
    logits, loss = st.forward_micro(0, x, rec)
    z = logits.reshape(4, 4)
    ls = z - np.log(np.exp(z).sum(1, keepdims=True))
    assert abs(loss - (-0.5 * ls[0, 1] - 0.5 * ls[0, 0] - ls[2, 3] - 0.5 * ls[3, 2]) / 4) < 1e-12
    st.backward([0])
    assert np.isfinite(st.grads[0]["w"]).all()
