"""One workspace, sized for the largest batch, under calls of fewer rows: results are those of workspaces of their own, and memory behind the workspace stays."""
import ctypes as C

import pytest
import torch

import paper_2410_14312_amd as tmps
from paper_2410_14312_amd import binding

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.fixture(autouse=True)
def single_precision_by_default():
    """(tests of the oracle leave their process at doubles)"""
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


def workspace(need):
    return torch.full((need + 64,), 165, dtype=torch.uint8, device=DEV)


@pytest.mark.parametrize("most,fewer", [(1024, (1024, 1023, 700, 1)), (3000, (3000, 2999, 1535))])
def test_norm_join_backward(most, fewer):
    D = 768
    need = binding.lib().tmps_norm_join_workspace(most, D)
    ws = workspace(need)
    gen = torch.Generator().manual_seed(1)
    for rows in fewer:
        r, f, dy, du = (torch.randn(rows, D, generator=gen).to(DEV) for _ in range(4))
        v, w = (torch.randn(D, generator=gen).to(DEV) for _ in range(2))
        y, u, stats = tmps.norm_join(f, r, v, w, pre_gain=w, pre_shift=v)
        want = tmps.norm_join_backward(dy, du, f, r, y, stats, v, w, pre_gain=w)
        dx, dr, grads = torch.empty_like(f), torch.empty_like(r), torch.empty(4, D, device=DEV)
        binding._call(binding.lib().tmps_norm_join_backward, DEV, None, binding.TMPS_F32, 0, rows, D, dy.data_ptr(), du.data_ptr(), f.data_ptr(), r.data_ptr(), y.data_ptr(),
                      stats.data_ptr(), v.data_ptr(), w.data_ptr(), w.data_ptr(), dx.data_ptr(), dr.data_ptr(), grads.data_ptr(), grads.data_ptr() + 8 * D, ws.data_ptr(), need)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((dx, dr) + grads.unbind(0), want))
        assert bool((ws[need:] == 165).all())


@pytest.mark.parametrize("classes,most,fewer", [(50257, 80, (80, 65, 64, 33, 1)), (131071, 70, (70, 64, 48, 5))])
def test_distill(classes, most, fewer):
    need = binding.lib().tmps_distill_workspace(most, classes)
    ws = workspace(need)
    gen = torch.Generator().manual_seed(2)
    k = 7
    for rows in fewer:
        z, t = torch.randn(rows, classes, generator=gen).to(DEV), torch.randn(rows, k, generator=gen).to(DEV)
        ids = torch.randint(0, classes, (rows, k), generator=gen).to(torch.int32).to(DEV)
        want = tmps.distill(z, None, ids, t, temperature=2.0)
        loss, g = torch.empty(rows, device=DEV), torch.empty_like(z)
        d = binding.DistillDesc(classes, k, 2.0, 1.0, 1.0 / rows)
        binding._call(binding.lib().tmps_distill, DEV, None, binding.TMPS_F32, C.byref(d), rows, z.data_ptr(), None, 1, ids.data_ptr(), t.data_ptr(), k, g.data_ptr(), loss.data_ptr(),
                      ws.data_ptr(), need)
        torch.cuda.synchronize()
        assert torch.equal(loss, want[0]) and torch.equal(g, want[1]) and bool((ws[need:] == 165).all())
