"""What the operators refuse, through the C ABI and the binding, without a GPU: every refusal comes before anything is launched."""
import ctypes as C

import pytest
import torch

import paper_2410_14312_amd as tmps
from paper_2410_14312_amd import binding

EINVAL, ESHAPE, EUNSUPPORTED, ECAP = -1, -2, -7, -8
M = 1 << 20   # addresses that nothing reads


def rotary(**kw):
    a = dict(dtype=1, heads=2, dh=64, pairs=(16, 8, 8), flags=0, base=10000.0, x=M, xs=128, y=2 * M, ys=128, pos=3 * M, n_pos=4, rows=4)
    a.update(kw)
    d = binding.RotaryDesc(a["heads"], a["dh"], (C.c_int32 * 3)(*a["pairs"]), a["flags"], a["base"])
    return binding.lib().tmps_rotary(a["dtype"], C.byref(d), a["x"], a["xs"], a["y"], a["ys"], a["pos"], a["n_pos"], a["rows"], 0, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), EINVAL), (dict(heads=0), EINVAL), (dict(dh=0), EINVAL), (dict(rows=-1), EINVAL), (dict(pairs=(-1, 8, 8)), EINVAL), (dict(pairs=(0, 0, 0)), ESHAPE),
    (dict(pairs=(16, 16, 1)), ESHAPE), (dict(pairs=(2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1)), ESHAPE), (dict(flags=4), EINVAL), (dict(base=0.0), EINVAL), (dict(base=float("nan")), EINVAL), (dict(base=float("inf")), EINVAL),
    (dict(x=None), EINVAL), (dict(y=None), EINVAL), (dict(pos=None), EINVAL), (dict(n_pos=0), EINVAL), (dict(xs=127), ESHAPE), (dict(ys=127), ESHAPE), (dict(xs=-128), ESHAPE),
    (dict(heads=2 ** 30, dh=64), EUNSUPPORTED), (dict(rows=2 ** 62), EUNSUPPORTED), (dict(xs=2 ** 60), EUNSUPPORTED), (dict(x=M + 1), ESHAPE), (dict(y=M + 1), ESHAPE), (dict(pos=M + 2), ESHAPE),
    (dict(y=M + 2), EINVAL), (dict(y=M + 256), EINVAL), (dict(y=M, ys=256), EINVAL), (dict(y=M + 256, xs=256, ys=257), EINVAL), (dict(y=M + 254, xs=256, ys=256), EINVAL), (dict(pos=2 * M + 8), EINVAL)])
def test_rotary_refuses(kw, code):
    assert rotary(**kw) == code, binding.lib().tmps_last_error()


def test_nothing_to_do():
    assert rotary(rows=0, x=None, y=None, pos=None) == 0
    assert forward(rows=0, x=None, r=None) == 0 and distill(rows=0, z=None) == 0


def forward(**kw):
    a = dict(dtype=1, flags=12, rows=8, D=64, x=M, r=2 * M, gain=3 * M, scale=4 * M, y=5 * M, pre_gain=6 * M, pre_shift=None, u=7 * M, stats=8 * M)
    a.update(kw)
    return binding.lib().tmps_norm_join_forward(*[a[k] for k in ("dtype", "flags", "rows", "D", "x", "r", "gain", "scale", "y", "pre_gain", "pre_shift", "u", "stats")], None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=-1), EINVAL), (dict(flags=16), EINVAL), (dict(flags=1), EINVAL), (dict(D=0), EINVAL), (dict(rows=-2), EINVAL), (dict(D=16385), EUNSUPPORTED), (dict(rows=2 ** 60), EUNSUPPORTED),
    (dict(u=None), EINVAL), (dict(pre_gain=None), EINVAL), (dict(pre_shift=9 * M), EINVAL), (dict(flags=8), EINVAL), (dict(u=None, pre_gain=None, pre_shift=9 * M, flags=8), EINVAL),
    (dict(x=None), EINVAL), (dict(r=None), EINVAL), (dict(gain=None), EINVAL), (dict(scale=None), EINVAL), (dict(y=None), EINVAL), (dict(stats=None), EINVAL),
    (dict(x=M + 1), ESHAPE), (dict(u=M + 1), ESHAPE), (dict(dtype=0, y=M + 2), ESHAPE), (dict(gain=M + 2), ESHAPE), (dict(stats=M + 1), ESHAPE),
    (dict(y=M), EINVAL), (dict(y=M + 1024), EINVAL), (dict(y=2 * M + 2), EINVAL), (dict(u=2 * M), EINVAL), (dict(u=5 * M), EINVAL), (dict(stats=5 * M + 512), EINVAL), (dict(u=3 * M + 128), EINVAL)])
def test_norm_join_refuses(kw, code):
    assert forward(**kw) == code, binding.lib().tmps_last_error()


def backward(**kw):
    a = dict(dtype=1, flags=12, rows=8, D=64, dy=M, du=2 * M, x=3 * M, r=4 * M, y=5 * M, stats=6 * M, gain=7 * M, scale=8 * M, pre_gain=9 * M, dx=10 * M, dr=11 * M,
             dgain_dscale=12 * M, dpre=13 * M, ws=14 * M, ws_bytes=1 << 40)
    a.update(kw)
    return binding.lib().tmps_norm_join_backward(*[a[k] for k in ("dtype", "flags", "rows", "D", "dy", "du", "x", "r", "y", "stats", "gain", "scale", "pre_gain", "dx", "dr",
                                                                  "dgain_dscale", "dpre", "ws", "ws_bytes")], None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=7), EINVAL), (dict(flags=2), EINVAL), (dict(D=-1), EINVAL), (dict(D=20000), EUNSUPPORTED), (dict(dy=None, du=None), EINVAL), (dict(y=None), EINVAL), (dict(pre_gain=None), EINVAL),
    (dict(x=None), EINVAL), (dict(r=None), EINVAL), (dict(stats=None), EINVAL), (dict(gain=None), EINVAL), (dict(scale=None), EINVAL), (dict(dgain_dscale=None), EINVAL), (dict(dpre=None), EINVAL),
    (dict(rows=0, dgain_dscale=None), EINVAL), (dict(ws=None), ECAP), (dict(ws_bytes=16), ECAP), (dict(dx=M + 1), ESHAPE), (dict(ws=M + 2), ESHAPE), (dict(dpre=M + 1), ESHAPE),
    (dict(dx=3 * M), EINVAL), (dict(dr=2 * M), EINVAL), (dict(dr=M + 2), EINVAL), (dict(dx=M), EINVAL), (dict(dx=11 * M + 64), EINVAL), (dict(dgain_dscale=7 * M), EINVAL), (dict(dpre=12 * M + 256), EINVAL),
    (dict(ws=10 * M + 4), EINVAL)])
def test_norm_join_backward_refuses(kw, code):
    assert backward(**kw) == code, binding.lib().tmps_last_error()


def test_workspaces_of_nothing():
    lib = binding.lib()
    assert lib.tmps_norm_join_workspace(0, 64) == lib.tmps_norm_join_workspace(4, 0) == lib.tmps_norm_join_workspace(4, 1 << 20) == 0
    assert lib.tmps_distill_workspace(0, 64) == lib.tmps_distill_workspace(4, 0) == 0
    assert lib.tmps_norm_join_workspace(1, 1) > 0


def distill(**kw):
    a = dict(dtype=0, classes=100, k=8, T=2.0, alpha=0.5, scale=1.0, rows=6, z=M, labels=2 * M, ls=1, ids=3 * M, teacher=4 * M, es=8, g=5 * M, loss=6 * M, ws=7 * M, ws_bytes=1 << 40)
    a.update(kw)
    d = binding.DistillDesc(a["classes"], a["k"], a["T"], a["alpha"], a["scale"])
    return binding.lib().tmps_distill(a["dtype"], C.byref(d), a["rows"], a["z"], a["labels"], a["ls"], a["ids"], a["teacher"], a["es"], a["g"], a["loss"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), EINVAL), (dict(classes=0), EINVAL), (dict(k=0), EINVAL), (dict(k=1025, es=1025), EUNSUPPORTED), (dict(classes=(1 << 23) + 1), EUNSUPPORTED), (dict(T=0.0), EINVAL), (dict(T=-1.0), EINVAL), (dict(T=float("nan")), EINVAL), (dict(T=1e-45), EINVAL), (dict(T=1e30), EINVAL),
    (dict(T=float("inf")), EINVAL), (dict(alpha=-0.1), EINVAL), (dict(alpha=1.5), EINVAL), (dict(alpha=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL), (dict(rows=-1), EINVAL),
    (dict(z=None), EINVAL), (dict(loss=None), EINVAL), (dict(ids=None), EINVAL), (dict(teacher=None), EINVAL), (dict(es=7), ESHAPE), (dict(ls=0), ESHAPE), (dict(rows=2 ** 60), EUNSUPPORTED),
    (dict(z=M + 2), ESHAPE), (dict(g=M + 2), ESHAPE), (dict(ids=M + 1), ESHAPE), (dict(g=M), EINVAL), (dict(g=M + 400), EINVAL), (dict(loss=3 * M + 4), EINVAL), (dict(loss=5 * M), EINVAL)])
def test_distill_refuses(kw, code):
    assert distill(**kw) == code, binding.lib().tmps_last_error()


def test_the_binding_refuses():
    """Shapes, types, layouts and places, before the library is asked."""
    def f(*shape, dtype=torch.float32):
        return torch.zeros(*shape, dtype=dtype)
    x, pos = f(4, 128), f(4, 3, dtype=torch.int32)
    for bad in (lambda: tmps.rotary(x, pos, 2, 64, (32, 0, 0)), lambda: tmps.rotary(x.double(), pos, 2, 64, (32, 0, 0)), lambda: tmps.rotary(x.t(), pos, 1, 4, (2, 0, 0)),
                lambda: tmps.rotary(x, pos.long(), 2, 64, (32, 0, 0)), lambda: tmps.rotary(x, pos[:, :2], 2, 64, (32, 0, 0)), lambda: tmps.rotary(x, pos, 3, 64, (32, 0, 0)),
                lambda: tmps.rotary(x, pos, 2, 64, (32, 0)), lambda: tmps.rotary(x, pos, 2, 64, (32, 0, 0), out=f(3, 128)), lambda: tmps.rotary(x[0], pos, 2, 64, (32, 0, 0)),
                lambda: tmps.rotary(x, pos, 2, 64, (32, 0, 0), out=x.bfloat16()), lambda: tmps.rotary(x, pos, 2, 64, (32, 0, 0), stream=0)):
        with pytest.raises(ValueError):
            bad()
    r, v, st = f(4, 8), f(8), f(4, 4)
    for bad in (lambda: tmps.norm_join(r, r, v, v), lambda: tmps.norm_join(r, r.half(), v, v), lambda: tmps.norm_join(r, r, v, v, gate=True), lambda: tmps.norm_join(r, r, v.double(), v),
                lambda: tmps.norm_join(f(8, 4).t(), r, v, v), lambda: tmps.norm_join(r, v, v, v), lambda: tmps.norm_join(r, r, v[:4], v), lambda: tmps.norm_join(r, r, v, v, y=f(4, 7)),
                lambda: tmps.norm_join_backward(r, None, r, r, r, st[:, :2], v, v), lambda: tmps.norm_join_backward(r.bfloat16(), None, r, r, r, st, v, v)):
        with pytest.raises(ValueError):
            bad()
    z, ids, t = f(4, 9), f(4, 2, dtype=torch.int32), f(4, 2)
    for bad in (lambda: tmps.distill(z, None, ids, t), lambda: tmps.distill(z.bfloat16(), None, ids, t), lambda: tmps.distill(z, None, ids.long(), t), lambda: tmps.distill(z, None, ids, t[:, :1]),
                lambda: tmps.distill(z, ids[:, 0], ids, t), lambda: tmps.distill(z, None, ids, t, dtype="f16"), lambda: tmps.distill(z[0], None, ids, t)):
        with pytest.raises(ValueError):
            bad()
