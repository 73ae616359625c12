"""What the operators of blocks that mix positions by a recurrence refuse, through the C ABI and the binding, without a GPU: every refusal comes before anything is launched."""
import ctypes as C

import pytest
import torch

import paper_2410_14312_amd as tmps
from paper_2410_14312_amd import binding

EINVAL, ESHAPE, EUNSUPPORTED, ECAP = -1, -2, -7, -8
M = 1 << 24   # addresses that nothing reads, as far apart as no operand is long
SILU, RMS, RELU, GELU = 64, 4, 1, 2
NAN, INF = float("nan"), float("inf")


def called(fn, order, a, kw):
    a.update(kw)
    return getattr(binding.lib(), fn)(*[a[k] for k in order], None)


def conv(**kw):
    return called("tmps_short_conv_forward", "dtype flags b s c k x xs w bias tail y ys tail_out".split(),
                  dict(dtype=1, flags=SILU, b=2, s=16, c=32, k=4, x=M, xs=32, w=2 * M, bias=3 * M, tail=4 * M, y=5 * M, ys=32, tail_out=6 * M), kw)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), EINVAL), (dict(flags=1), EINVAL), (dict(b=-1), EINVAL), (dict(s=0), EINVAL), (dict(s=2 ** 31), EUNSUPPORTED), (dict(b=2 ** 60), EUNSUPPORTED), (dict(c=0), EINVAL),
    (dict(k=0), EINVAL), (dict(k=9), EUNSUPPORTED), (dict(c=2 ** 25, xs=2 ** 25, ys=2 ** 25), EUNSUPPORTED), (dict(b=2 ** 35, s=16), EUNSUPPORTED), (dict(x=None), EINVAL), (dict(w=None), EINVAL),
    (dict(y=None), EINVAL), (dict(xs=31), ESHAPE), (dict(ys=31), ESHAPE), (dict(x=M + 1), ESHAPE), (dict(w=2 * M + 2), ESHAPE), (dict(tail=4 * M + 1), ESHAPE),
    (dict(y=M), EINVAL), (dict(y=M + 64), EINVAL), (dict(y=M + 2, xs=64, ys=64), EINVAL), (dict(y=M + 64, xs=64, ys=65), EINVAL), (dict(y=4 * M), EINVAL), (dict(tail_out=4 * M), EINVAL),
    (dict(tail_out=5 * M), EINVAL), (dict(tail_out=4 * M + 2, s=1), EINVAL), (dict(y=2 * M), EINVAL)])
def test_conv_refuses(kw, code):
    assert conv(**kw) == code, binding.lib().tmps_last_error()


def conv_back(**kw):
    return called("tmps_short_conv_backward", "dtype flags b s c k dy dys x xs w bias tail dtail dx dxs dtail_in dp ws wsb".split(),
                  dict(dtype=0, flags=0, b=2, s=16, c=32, k=4, dy=M, dys=32, x=2 * M, xs=32, w=3 * M, bias=4 * M, tail=5 * M, dtail=6 * M, dx=7 * M, dxs=32, dtail_in=8 * M, dp=9 * M,
                       ws=10 * M, wsb=1 << 22), kw)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=-1), EINVAL), (dict(flags=2), EINVAL), (dict(b=0), EUNSUPPORTED), (dict(s=-3), EINVAL), (dict(dy=None), EINVAL), (dict(dx=None), EINVAL), (dict(dp=None), EINVAL), (dict(ws=None), ECAP),
    (dict(wsb=100), ECAP), (dict(ws=10 * M + 8), ESHAPE), (dict(dys=30), ESHAPE), (dict(dxs=30), ESHAPE), (dict(dx=M), EINVAL), (dict(dx=2 * M + 128), EINVAL), (dict(dtail_in=6 * M), EINVAL),
    (dict(dtail_in=5 * M), EINVAL), (dict(dp=3 * M), EINVAL), (dict(ws=7 * M), EINVAL), (dict(dp=10 * M + 64), EINVAL), (dict(dx=7 * M + 2), ESHAPE), (dict(dp=9 * M + 2), ESHAPE)])
def test_conv_backward_refuses(kw, code):
    assert conv_back(**kw) == code, binding.lib().tmps_last_error()


def desc(a):
    return C.byref(binding.ScanDesc(a.pop("heads"), a.pop("dh"), a.pop("groups"), a.pop("n")))


def scan(**kw):
    a = dict(dtype=1, heads=4, dh=16, groups=2, n=8, b=2, s=100, x=M, xs=96, dt=2 * M, dts=4, a=3 * M, skip=4 * M, bias=5 * M, state=6 * M, y=7 * M, ys=64, out=8 * M, ws=9 * M, wsb=1 << 22)
    a.update(kw)
    d = desc(a)
    return called("tmps_scan_forward", "dtype d b s x xs dt dts a skip bias state y ys out ws wsb".split(), dict(a, d=None if kw.get("d", 1) is None else d), {})


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=5), EINVAL), (dict(d=None), EINVAL), (dict(heads=0), EINVAL), (dict(dh=0), EINVAL), (dict(groups=0), EINVAL), (dict(n=0), EINVAL), (dict(heads=3), ESHAPE), (dict(groups=3), ESHAPE),
    (dict(n=129, xs=600), EUNSUPPORTED), (dict(heads=2 ** 20, dh=64, xs=2 ** 27), EUNSUPPORTED), (dict(b=-2), EINVAL), (dict(s=0), EINVAL), (dict(b=2 ** 40), EUNSUPPORTED), (dict(x=None), EINVAL),
    (dict(dt=None), EINVAL), (dict(a=None), EINVAL), (dict(skip=None), EINVAL), (dict(bias=None), EINVAL), (dict(y=None), EINVAL), (dict(xs=95), ESHAPE), (dict(dts=3), ESHAPE), (dict(ys=63), ESHAPE),
    (dict(xs=2 ** 25), EUNSUPPORTED), (dict(x=M + 1), ESHAPE), (dict(state=6 * M + 2), ESHAPE), (dict(a=3 * M + 1), ESHAPE), (dict(y=M), EINVAL), (dict(y=2 * M), EINVAL), (dict(out=6 * M + 4), EINVAL),
    (dict(out=7 * M), EINVAL), (dict(y=6 * M), EINVAL), (dict(s=5000, ws=None), ECAP), (dict(s=5000, wsb=64), ECAP), (dict(s=5000, ws=9 * M + 4), ESHAPE), (dict(s=5000, ws=M), EINVAL),
    (dict(heads=1, dh=1, groups=1, n=1), EUNSUPPORTED), (dict(b=2 ** 20, s=2 ** 31 - 1), EUNSUPPORTED)])
def test_scan_refuses(kw, code):
    assert scan(**kw) == code, binding.lib().tmps_last_error()


def scan_back(**kw):
    a = dict(dtype=0, heads=4, dh=16, groups=1, n=8, b=2, s=100, dy=M, dys=64, dstate=2 * M, x=3 * M, xs=80, dt=4 * M, dts=4, a=5 * M, skip=6 * M, bias=7 * M, state=8 * M, dx=9 * M, dxs=80,
             ddt=10 * M, ddts=4, dp=11 * M, dstate_in=12 * M, ws=13 * M, wsb=1 << 23)
    a.update(kw)
    d = desc(a)
    return called("tmps_scan_backward", "dtype d b s dy dys dstate x xs dt dts a skip bias state dx dxs ddt ddts dp dstate_in ws wsb".split(), dict(a, d=d), {})


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=5), EINVAL), (dict(b=0), EUNSUPPORTED), (dict(dy=None), EINVAL), (dict(dx=None), EINVAL), (dict(ddt=None), EINVAL), (dict(dp=None), EINVAL), (dict(dys=60), ESHAPE), (dict(dxs=79), ESHAPE),
    (dict(ddts=3), ESHAPE), (dict(ws=None), ECAP), (dict(wsb=1 << 10), ECAP), (dict(dx=3 * M), EINVAL), (dict(dx=M), EINVAL), (dict(ddt=4 * M), EINVAL), (dict(ddt=9 * M), EINVAL), (dict(dstate_in=2 * M), EINVAL),
    (dict(dstate_in=8 * M), EINVAL), (dict(dp=10 * M), EINVAL), (dict(ws=12 * M), EINVAL), (dict(heads=1, dh=3, dys=3, dxs=80), EUNSUPPORTED), (dict(dx=9 * M, ddt=9 * M + 320, dxs=84, ddts=85), EINVAL)])
def test_scan_backward_refuses(kw, code):
    assert scan_back(**kw) == code, binding.lib().tmps_last_error()


def norm(**kw):
    return called("tmps_group_norm_forward", "dtype flags b s c g x gain shift y stats ws wsb".split(),
                  dict(dtype=1, flags=SILU, b=2, s=5000, c=32, g=4, x=M, gain=2 * M, shift=3 * M, y=4 * M, stats=5 * M, ws=6 * M, wsb=1 << 23), kw)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=9), EINVAL), (dict(flags=8), EINVAL), (dict(flags=RELU | SILU), EINVAL), (dict(flags=GELU | RELU | RMS), EINVAL), (dict(b=-1), EINVAL), (dict(s=0), EINVAL), (dict(c=0), EINVAL),
    (dict(g=0), EINVAL), (dict(g=5), ESHAPE), (dict(c=65537, g=1), EUNSUPPORTED), (dict(b=2 ** 40), EUNSUPPORTED), (dict(b=2 ** 24, c=64, g=64, s=2), EUNSUPPORTED), (dict(b=2 ** 28, s=1, c=65536, g=2), EUNSUPPORTED), (dict(x=None), EINVAL), (dict(gain=None), EINVAL), (dict(y=None), EINVAL),
    (dict(stats=None), EINVAL), (dict(ws=None), ECAP), (dict(wsb=16), ECAP), (dict(ws=6 * M + 4), ESHAPE), (dict(x=M + 1), ESHAPE), (dict(gain=2 * M + 2), ESHAPE), (dict(y=M), EINVAL), (dict(y=M + 4096), EINVAL),
    (dict(stats=4 * M + 64), EINVAL), (dict(y=2 * M), EINVAL), (dict(ws=4 * M), EINVAL)])
def test_group_norm_refuses(kw, code):
    assert norm(**kw) == code, binding.lib().tmps_last_error()


def norm_back(**kw):
    return called("tmps_group_norm_backward", "dtype flags b s c g dy x stats gain shift dx dp ws wsb".split(),
                  dict(dtype=0, flags=0, b=2, s=50, c=32, g=4, dy=M, x=2 * M, stats=3 * M, gain=4 * M, shift=5 * M, dx=6 * M, dp=7 * M, ws=8 * M, wsb=1 << 23), kw)


@pytest.mark.parametrize("kw,code", [
    (dict(b=0), EUNSUPPORTED), (dict(dy=None), EINVAL), (dict(stats=None), EINVAL), (dict(dx=None), EINVAL), (dict(dp=None), EINVAL), (dict(ws=None), ECAP), (dict(wsb=8), ECAP), (dict(dx=M), EINVAL),
    (dict(dx=2 * M), EINVAL), (dict(dp=4 * M), EINVAL), (dict(dp=6 * M + 32), EINVAL), (dict(ws=7 * M + 16), EINVAL), (dict(dx=6 * M + 2), ESHAPE)])
def test_group_norm_backward_refuses(kw, code):
    assert norm_back(**kw) == code, binding.lib().tmps_last_error()


def clip(arrays, limit=1.0, norm=9 * M, ws=8 * M, wsb=1 << 20, n=None):
    table = (binding.Array * max(len(arrays), 1))(*[binding.Array(*a) for a in arrays])
    return binding.lib().tmps_clip_gradients(table if arrays else None, len(arrays) if n is None else n, limit, norm, ws, wsb, None)


@pytest.mark.parametrize("arrays,kw,code", [
    ([(M, M, 8, 2)], {}, EINVAL), ([(M, M, -1, 0)], {}, EINVAL), ([(None, M, 8, 0)], {}, EINVAL), ([], dict(n=3), EINVAL), ([(M, M, 8, 0)], dict(n=-1), EINVAL), ([(M + 2, M + 2, 8, 0)], {}, ESHAPE),
    ([(M, M + 1, 8, 1)], {}, ESHAPE), ([(M, M, 8, 0)], dict(limit=-1.0), EINVAL), ([(M, M, 8, 0)], dict(limit=NAN), EINVAL), ([(M, M, 8, 0)], dict(norm=None), EINVAL), ([(M, M, 8, 0)], dict(norm=9 * M + 2), ESHAPE),
    ([(M, M, 8, 0)], dict(ws=None), ECAP), ([(M, M, 8, 0)], dict(wsb=8), ECAP), ([(M, M, 8, 0)], dict(ws=8 * M + 8), ESHAPE), ([(M, M, 8, 0)], dict(norm=M + 28), EINVAL), ([(M, M, 8, 0)], dict(ws=M + 16), EINVAL),
    ([(M, M, 8, 0)], dict(norm=8 * M), EINVAL), ([(M, M, 8, 0), (M, M, 8, 0)], {}, EINVAL), ([(M, M, 8, 0), (M + 16, M + 16, 8, 0)], {}, EINVAL), ([(M, M + 4, 8, 0)], {}, EINVAL),
    ([(M, 2 * M, 8, 0), (3 * M, 2 * M + 16, 8, 0)], {}, EINVAL), ([(M, 2 * M, 8, 0), (2 * M, 3 * M, 8, 0)], {}, EINVAL), ([(M, M, 8, 0), (2 * M, None, 8, 0)], {}, EINVAL),
    ([(M, M, 2 ** 41, 0)], {}, EUNSUPPORTED), ([(M, 5 * M, 100, 0), (2 * M, 3 * M, 8, 0), (5 * M + 40, 6 * M, 4, 1)], {}, EINVAL)])
def test_clipping_refuses(arrays, kw, code):
    assert clip(arrays, **kw) == code, binding.lib().tmps_last_error()


def test_nothing_to_do_and_workspaces_of_nothing():
    assert conv(b=0, x=None) == 0 and scan(b=0, x=None) == 0 and norm(b=0, x=None) == 0
    lib, d = binding.lib(), binding.ScanDesc(4, 16, 2, 8)
    assert lib.tmps_short_conv_workspace(0, 4, 8, 4) == lib.tmps_short_conv_workspace(1, 4, 8, 9) == 0 < lib.tmps_short_conv_workspace(1, 1, 1, 1)
    assert lib.tmps_scan_workspace(C.byref(d), 2, 100) == lib.tmps_scan_workspace(None, 2, 100) == lib.tmps_scan_backward_workspace(0, None, 2, 100) == 0
    assert lib.tmps_scan_workspace(C.byref(d), 2, 5000) > 0 and lib.tmps_scan_backward_workspace(1, C.byref(d), 1, 1) > 0
    assert lib.tmps_group_norm_workspace(0, 0, 4, 8, 2, 1) == lib.tmps_group_norm_workspace(0, 4, 4, 8, 3, 1) == lib.tmps_group_norm_workspace(0, 4, 1, 8, 2, 0) == 0


@pytest.mark.parametrize("heads,dh,groups,n", [(1, 64, 1, 64), (3, 65, 1, 33), (24, 64, 1, 128), (4, 200, 2, 16)])
def test_a_workspace_for_more_is_enough_for_fewer(heads, dh, groups, n):
    lib, d = binding.lib(), C.byref(binding.ScanDesc(heads, dh, groups, n))
    for fixed in (1, 7, 700, 5000):
        for sizes in ([lib.tmps_scan_workspace(d, b, fixed) for b in range(1, 80)], [lib.tmps_scan_workspace(d, fixed, s) for s in range(1, 3000, 37)],
                      [lib.tmps_scan_backward_workspace(1, d, b, fixed) for b in range(1, 80)], [lib.tmps_scan_backward_workspace(1, d, fixed, s) for s in range(1, 3000, 37)]):
            assert sizes == sorted(sizes)
    for fixed in (1, 100):
        assert all(lib.tmps_short_conv_workspace(b, fixed, 8, 4) <= lib.tmps_short_conv_workspace(b + 1, fixed, 8, 4) for b in range(1, 50))
        assert all(lib.tmps_short_conv_workspace(fixed, s, 8, 4) <= lib.tmps_short_conv_workspace(fixed, s + 1, 8, 4) for s in range(1, 300))


def test_the_binding_refuses():
    """Shapes, types, layouts and places, before the library is asked."""
    def f(*shape, dtype=torch.float32):
        return torch.zeros(*shape, dtype=dtype)
    x, w, b = f(8, 16), f(16, 4), f(16)
    for bad in (lambda: tmps.short_conv(x, w, b), lambda: tmps.short_conv(x.double(), w, b), lambda: tmps.short_conv(x[0], w, b), lambda: tmps.short_conv(x, w[:4], b), lambda: tmps.short_conv(x, w, b, positions=3),
                lambda: tmps.short_conv(x, w, b, positions=0), lambda: tmps.short_conv(x.t(), f(8, 4)), lambda: tmps.short_conv(x, w, b[:3]), lambda: tmps.short_conv(x, w, b, tail=f(8, 2, 16)),
                lambda: tmps.short_conv(x, w, b, out=f(8, 15)), lambda: tmps.short_conv_backward(x.bfloat16(), x, w, b), lambda: tmps.short_conv_backward(f(7, 16), x, w, b)):
        with pytest.raises(ValueError):
            bad()
    x, dt, h = f(8, 2 * 4 + 2 * 6), f(8, 2), f(2)
    kw = dict(positions=4, state_features=6)
    for bad in (lambda: tmps.selective_scan(x, dt, h, h, h, **kw), lambda: tmps.selective_scan(x.half(), dt, h, h, h, **kw), lambda: tmps.selective_scan(x, dt[:, :1], h, h, h, **kw),
                lambda: tmps.selective_scan(x, dt, h, h[:1], h, **kw), lambda: tmps.selective_scan(x, dt, h, h, h, positions=5, state_features=6), lambda: tmps.selective_scan(x, dt, h, h, h, positions=4, state_features=20),
                lambda: tmps.selective_scan(x, dt, f(3), f(3), f(3), **kw), lambda: tmps.selective_scan(x, dt, h, h, h, state=f(2, 2, 4, 5), **kw), lambda: tmps.selective_scan(x, dt, h, h, h, groups=0, **kw),
                lambda: tmps.selective_scan_backward(f(8, 7), x, dt, h, h, h, **kw), lambda: tmps.selective_scan_backward(f(8, 8), x, dt, h, h, h, dx=f(8, 19), **kw)):
        with pytest.raises(ValueError):
            bad()
    x, v, st = f(8, 12), f(12), f(2, 3, 2)
    for bad in (lambda: tmps.group_norm(x, v, v, groups=3), lambda: tmps.group_norm(x, v[:3], v, groups=3), lambda: tmps.group_norm(x, v, v, groups=3, act="tanh"), lambda: tmps.group_norm(x, v, v, groups=3, positions=3),
                lambda: tmps.group_norm(x.t(), f(8), None), lambda: tmps.group_norm_backward(x, x, st[:1], v, v, groups=3, positions=4), lambda: tmps.group_norm_backward(x.bfloat16(), x, st, v, v, groups=3, positions=4)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: tmps.clip_gradients([], 1.0), lambda: tmps.clip_gradients([x], 1.0), lambda: tmps.clip_gradients([x, v], 1.0, out=[x])):
        with pytest.raises(ValueError):
            bad()
    for make in (lambda t: tmps.short_conv(t, f(12, 4)), lambda t: tmps.group_norm(t, v)):
        with pytest.raises(ValueError, match="gradient"):
            make(f(8, 12).requires_grad_(True))
