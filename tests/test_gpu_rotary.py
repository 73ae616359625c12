"""Rotary positions with several axes against complex products in 64 bits.

Error of an element u c - v s: the turn is rounded to fp32 (2^-25 of a turn at most, 2 pi 2^-25 < 1.9e-7 in the sine and cosine), sine and cosine are within 4 steps of
2^-24, the products and the sum within 2: 5e-7 (|u| + |v|).  A bf16 result is rounded on top: 2^-8 of its size."""
import numpy as np
import pytest
import torch

import paper_2410_14312_amd as tmps

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True)
def single_precision_by_default():
    """(tests of the oracle leave their process at doubles)"""
    import torch
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


def turned(x, pos, heads, dh, pairs, base, interleaved, own, inverse):
    """x, pos: numpy, rows of heads of dh features; 64 bits."""
    n, out = sum(pairs), x.astype(np.float64).reshape(len(x), heads, dh).copy()
    phi, first = [], 0
    for axis, m in enumerate(pairs):
        for j in range(m):
            phi.append(pos[:, axis].astype(np.float64) * float(base) ** (-(j / m if own else (first + j) / n)))
        first += m
    e = np.exp((-1j if inverse else 1j) * np.stack(phi, 1))[:, None]
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    z = (out[:, :, a] + 1j * out[:, :, b]) * e
    size = np.zeros_like(out)
    size[:, :, a] = size[:, :, b] = np.abs(out[:, :, a]) + np.abs(out[:, :, b])
    out[:, :, a], out[:, :, b] = z.real, z.imag
    return out.reshape(len(x), -1), size.reshape(len(x), -1)


def close(got, want, size, dtype):
    err = np.abs(got.double().cpu().numpy() - want)
    bound = 5e-7 * size + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0.0)
    assert np.all(err <= bound), float(np.max(err - bound))


def make(rows, width, dtype, n_pos=None, far=0, seed=0):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, width, generator=gen).to(TYPES[dtype])
    pos = torch.randint(-20, 5000, (rows if n_pos is None else n_pos, 3), generator=gen).to(torch.int32) + far
    return x, pos.to(torch.int32)


def base_of(base):
    return float(np.float32(base))   # (the library takes it in 32 bits)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,heads,dh,pairs,own", [(1, 1, 2, (1, 0, 0), False), (1, 24, 64, (32, 0, 0), False), (5, 3, 7, (1, 1, 1), True), (33, 4, 64, (8, 12, 12), False),
                                                      (130, 5, 48, (8, 8, 8), True), (17, 2, 80, (0, 16, 16), True), (9, 3, 36, (2, 0, 5), False), (64, 40, 128, (16, 24, 24), False),
                                                      (300, 1, 256, (128, 0, 0), False), (257, 2, 16, (0, 0, 8), True), (3, 130, 40, (20, 0, 0), False), (7, 2, 513, (3, 250, 1), True), (3, 2, 1024, (256, 100, 155), False), (3, 1, 1016, (200, 200, 107), True),
                                                      (40, 3, 24, (4, 3, 4), False), (11, 7, 22, (11, 0, 0), False)])
def test_turns(dtype, interleaved, rows, heads, dh, pairs, own):
    x, pos = make(rows, heads * dh, dtype, seed=rows + dh)
    for inverse in (False, True):
        got = tmps.rotary(x.to(DEV), pos.to(DEV), heads, dh, pairs, interleaved=interleaved, own_ladders=own, inverse=inverse)
        want, size = turned(x.float().numpy(), pos.numpy(), heads, dh, pairs, base_of(10000.0), interleaved, own, inverse)
        close(got, want, size, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_far_positions(dtype):
    """Positions of millions and the largest there are: the angle is reduced in 64 bits (relative error below 2^-48, 2e9 turns: 1e-5 of a turn is far from reached)."""
    x, pos = make(40, 2 * 64, dtype)
    pos[:, 0] = torch.tensor([0, 1, -1, 1000003, 16777217, 2 ** 31 - 1, -2 ** 31, 123456789] * 5, dtype=torch.int32)
    got = tmps.rotary(x.to(DEV), pos.to(DEV), 2, 64, (32, 0, 0), base=500000.0)
    want, size = turned(x.float().numpy(), pos.numpy(), 2, 64, (32, 0, 0), base_of(500000.0), False, False, False)
    # (2^31 radians: base^(-i / n) in 64 bits is off by 2^-50 here and there, 2e-6 of an angle of 2^31)
    close(got, want, 10 * size, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh,heads,offset,behind", [(64, 3, 0, 64), (64, 3, 8, 8), (32, 2, 1, 3), (24, 5, 4, 1), (128, 2, 0, 0)])
def test_strides_columns_and_in_place(dtype, dh, heads, offset, behind):
    """Heads inside wider rows, at any offset; in place; into other columns; the rest of the rows stays as it was.  One table of positions for every sequence."""
    rows, w = 50, heads * dh
    wide = offset + w + behind
    x, pos = make(rows, wide, dtype, n_pos=10, seed=dh)
    pairs = (dh // 2 - 3, 2, 1)
    want, size = turned(x.float().numpy()[:, offset:offset + w], np.tile(pos.numpy(), (5, 1)), heads, dh, pairs, base_of(10000.0), False, False, False)
    at = x.to(DEV)
    got = tmps.rotary(at[:, offset:offset + w], pos.to(DEV), heads, dh, pairs)
    close(got, want, size, dtype)
    out = torch.full((rows, wide + 5), 7.0, dtype=TYPES[dtype], device=DEV)
    tmps.rotary(at[:, offset:offset + w], pos.to(DEV), heads, dh, pairs, out=out[:, 3:3 + w])
    assert torch.equal(out[:, 3:3 + w], got) and bool((out[:, :3] == 7).all()) and bool((out[:, 3 + w:] == 7).all())
    ret = tmps.rotary(at[:, offset:], pos.to(DEV), heads, dh, pairs, out=at[:, offset:])
    assert ret.data_ptr() == at[:, offset:].data_ptr()
    assert torch.equal(at[:, offset:offset + w], got)
    assert torch.equal(at[:, :offset].cpu(), x[:, :offset]) and torch.equal(at[:, offset + w:].cpu(), x[:, offset + w:])
    both = torch.cat([x, torch.zeros_like(x)], 1).to(DEV)   # into other columns of the same rows
    tmps.rotary(both[:, offset:offset + w], pos.to(DEV), heads, dh, pairs, out=both[:, wide + offset:wide + offset + w])
    assert torch.equal(both[:, wide + offset:wide + offset + w], got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_back_and_forth_is_the_gradient(dtype, interleaved):
    """The inverse is the transpose: <turn(x), g> = <x, back(g)>, and back(turn(x)) = x, each to its roundings."""
    rows, heads, dh, pairs = 77, 6, 72, (9, 13, 10)
    x, pos = make(rows, heads * dh, dtype, seed=3)
    g, _ = make(rows, heads * dh, dtype, seed=4)
    kw = dict(interleaved=interleaved)
    y = tmps.rotary(x.to(DEV), pos.to(DEV), heads, dh, pairs, **kw)
    dx = tmps.rotary(g.to(DEV), pos.to(DEV), heads, dh, pairs, inverse=True, **kw)
    left, right = (y.double().cpu() * g.double()).sum().item(), (x.double() * dx.double().cpu()).sum().item()
    step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -21
    assert abs(left - right) <= 2 * step * (x.double().norm() * g.double().norm()).item()
    again = tmps.rotary(y, pos.to(DEV), heads, dh, pairs, inverse=True, **kw)
    assert (again.double().cpu() - x.double()).norm() <= 2 * step * x.double().norm()


def test_many_rows_and_no_rows():
    x, pos = make(70001, 2 * 16, "bf16", seed=9)
    got = tmps.rotary(x.to(DEV), pos.to(DEV), 2, 16, (4, 2, 2))
    want, size = turned(x.float().numpy(), pos.numpy(), 2, 16, (4, 2, 2), base_of(10000.0), False, False, False)
    close(got, want, size, "bf16")
    assert tmps.rotary(x[:0].to(DEV), pos.to(DEV), 2, 16, (4, 2, 2)).shape == (0, 32)


def test_rows_beyond_32_bit_offsets():
    """The last rows of an array of more than 2^31 elements."""
    rows, wide = 70000, 32768
    x = torch.zeros(rows, wide, dtype=torch.bfloat16, device=DEV)
    small, pos = make(3, 64, "bf16", n_pos=rows, seed=5)
    x[-3:, :64] = small.to(DEV)
    got = tmps.rotary(x[:, :64], pos.to(DEV), 1, 64, (16, 8, 8), out=x[:, wide - 64:])[-3:]
    want, size = turned(small.float().numpy(), pos.numpy()[-3:], 1, 64, (16, 8, 8), base_of(10000.0), False, False, False)
    close(got, want, size, "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_graph_and_another_stream(dtype):
    """Captured, replayed with new inputs and positions between eager calls; and eager on a stream of its own."""
    rows, heads, dh, pairs = 260, 4, 64, (16, 8, 8)
    x = torch.zeros(rows, heads * dh, dtype=TYPES[dtype], device=DEV)
    pos = torch.zeros(rows, 3, dtype=torch.int32, device=DEV)
    out = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        tmps.rotary(x, pos, heads, dh, pairs, out=out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tmps.rotary(x, pos, heads, dh, pairs, out=out)
    for seed in range(4):
        a, p = make(rows, heads * dh, dtype, seed=seed)
        x.copy_(a)
        pos.copy_(p)
        graph.replay()
        eager = tmps.rotary(x, pos, heads, dh, pairs)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        want, size = turned(a.float().numpy(), p.numpy(), heads, dh, pairs, base_of(10000.0), False, False, False)
        close(out, want, size, dtype)
