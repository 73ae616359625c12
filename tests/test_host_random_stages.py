"""The stage executor (csrc/stage.cpp) on host launchers that compute in fp32 (tests/host/arithmetic.cpp), driven through the C ABI with random layer lists of dense layers, additions,
norms, norm joins and rotary positions, against the oracle in 64 bits: outputs, parameter gradients and the input's, in an array of its own, over the upstream gradient and over the
input.  A list is refused when the stage is made, or can be trained.

Values pass at most some 30 layers of sums of at most 24 terms: 2e-3 of the largest is 2^15 steps of 2^-24, of which rounding takes some hundreds and small variances magnify them by at
most 1 / sqrt(1e-5)."""
import ctypes as C
import random
import subprocess

import numpy as np
import pytest

from oracle.stage import Stage as OStage
from paper_2410_14312_amd import binding
from tests.test_host_sanitizers import ROOT
from workloads.configs import layernorm, linear, norm_join, resadd, rotary
from workloads.synth import param_shapes

S, D, N, MICRO = 4, 8, 2, 2


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("stage") / "stage.so")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-pthread", "tests/host/arithmetic.cpp",
                        "paper_2410_14312_amd/csrc/stage.cpp", "-o", so], capture_output=True, text=True, cwd=ROOT)
    assert r.returncode == 0, r.stderr
    lib = C.CDLL(so)
    for name, (result, arguments) in binding.EXPORTS.items():
        if hasattr(lib, name):
            getattr(lib, name).restype, getattr(lib, name).argtypes = result, arguments
    return lib


def aligned(n):
    a = np.zeros(n + 512, dtype=np.uint8)
    at = -a.ctypes.data % 256
    return a[at:at + n + 256]


def close(got, want):
    assert np.abs(got - want).max() <= 2e-3 * np.abs(want).max() + 1e-30


def train(lib, specs, seed, place, borrow):
    """Whether the list was taken; what it gives is compared."""
    rng = np.random.default_rng(seed)
    descs, cfg, M = binding.layer_descs(specs), binding.StageCfg(0, MICRO, N, N, 0, borrow, 0.1, 0.9), N * MICRO
    sizes = [C.c_size_t() for _ in range(4)]
    if lib.tmps_stage_bytes(descs, len(specs), C.byref(cfg), *[C.byref(v) for v in sizes]):
        return False
    regions = [aligned(v.value) for v in sizes]
    h = C.c_void_p()
    assert lib.tmps_stage_create(C.byref(h), descs, len(specs), C.byref(cfg), *[r.ctypes.data for r in regions]) == 0
    P = lib.tmps_stage_param_count(h)
    masters, grads = regions[0][:4 * P].view(np.float32), regions[1][4 * P:8 * P].view(np.float32)

    def part(flat, layer, key):
        at, n = C.c_int64(), C.c_int64()
        lib.tmps_stage_param_offset(h, layer, "wb".index(key), C.byref(at), C.byref(n))
        return flat[at.value:at.value + n.value]

    params = []
    for li, sp in enumerate(specs):
        p = {}
        for key, shape in param_shapes(sp).items():
            v = rng.standard_normal(shape)
            if sp["kind"] == "linear":
                v *= np.sqrt(1.0 / sp["din"]) if key == "w" else 0.1
            else:
                v = 0.2 * v + (key == "w" or sp["kind"] == "norm_join")
            p[key] = v.astype(np.float32)
            part(masters, li, key)[:] = p[key].ravel()
        params.append(p)
    x, dy = (rng.standard_normal((M, n(h))).astype(np.float32) for n in (lib.tmps_stage_input_elems, lib.tmps_stage_output_elems))
    oracle = OStage(specs, params, 0.1, 0.9, M, N)
    y = np.zeros_like(dy)
    for j in range(N):
        s = slice(j * MICRO, (j + 1) * MICRO)
        assert lib.tmps_forward_micro(h, j, x[s].ctypes.data, y[s].ctypes.data, None, None, None) == 0
        close(y[s], oracle.forward_micro(j, x[s].astype(np.float64)).reshape(MICRO, -1))
    want = oracle.backward(list(range(N)), dy.astype(np.float64)).reshape(x.shape)
    dx = np.zeros_like(x)
    if place == "x":
        dx = x
    elif place == "dy" and dy.size == x.size:
        dx = dy
    assert lib.tmps_backward(h, (C.c_int * N)(*range(N)), N, dy.ctypes.data, dx.ctypes.data, None) == 0, lib.tmps_last_error()
    close(dx.reshape(x.shape), want)
    for li, g in enumerate(oracle.grads):
        for key in g or {}:
            close(part(grads, li, key), g[key].ravel())
    lib.tmps_stage_destroy(h)
    return True


def some_layers(rnd):
    ls = []
    for _ in range(1 + rnd.randrange(9)):
        m = len(ls)
        kind = rnd.randrange(9) if m else rnd.choice([0, 0, 1, 6, 7])
        rms, thrice = rnd.random() < 0.5, [linear(D, 3 * D, False, rows=S), rotary(S, D, rnd.choice([1, 2, 4]), interleaved=rnd.random() < 0.5), linear(3 * D, D, False, rows=S)]
        if kind == 0:
            ls.append(layernorm(D, S, rms=rms))
        elif kind == 1:
            ls += [linear(D, 2 * D, False, rows=S), norm_join(D, S, rnd.choice([2, 2, 3, m + 2]), rms=rms, gate=True)]
        elif kind == 2:
            ls.append(linear(D, D, False, rows=S))
        elif kind in (3, 4):
            ls.append(norm_join(D, S, 2 + rnd.randrange(m), rms=rms))
        elif kind == 5:
            ls.append(resadd(S, 1, D, 2 + rnd.randrange(m), relu=False))
        elif kind == 6:
            ls += thrice
        elif kind == 7:
            ls += thrice + [linear(D, 3 * D, False, rows=S), norm_join(3 * D, S, rnd.choice([3, 4])), linear(3 * D, D, False, rows=S)]
        else:
            ls.append(linear(D, D, False, rows=S, skip=rnd.randrange(1, 4)))
    return ls


def test_random_layers(lib):
    rnd = random.Random(5)
    taken = 0
    for seed in range(700):
        ls = some_layers(rnd)
        for place in ("apart", "x", "dy"):
            taken += train(lib, ls, seed, place, rnd.randrange(2))
    assert taken > 600
