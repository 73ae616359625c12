"""Distillation of wide rows with remainders behind their whole pieces, and of the widest, against 64 bits, with bounds that do not grow with the number of classes.

In steps of 2^-24: an exponential is off by |z - m| max(1, 1 / T) (its argument's rounding, 2.5 steps of it with those of 1 / T and its product with log2 e) + 4 of its own size.  A sum of
positive terms is off by its longest chain: at most 129 terms in a lane, 6 steps through a wave, 16 through a workgroup's waves, and as many again where slices are joined: 129 + 44;
the teacher's by its entries, k / 64 + 22.  So probabilities are off by c = 129 + 44 + k / 64 + 22 + 20 + 6 max|z - m| max(1, 1 / T), and the loss by c times sum p (1 + |log p| + |log q|).

The largest logits of most rows stand in their last classes, which neither an entry nor the label names: a sum that leaves one of them out is off by its own size."""
import numpy as np
import pytest
import torch

import paper_2410_14312_amd as tmps

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
STEP = 2.0 ** -24


@pytest.fixture(autouse=True)
def single_precision_by_default():
    """(tests of the oracle leave their process at doubles)"""
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


def check(z, labels, ids, teacher, T, alpha, dtype):
    rows, C = z.shape
    k = ids.shape[1]
    loss, g = (v.cpu() for v in tmps.distill(z.to(DEV), labels.to(DEV), ids.to(DEV), teacher.to(DEV), temperature=T, alpha=alpha, dtype=dtype, grad_scale=1.0))
    T, alpha = float(np.float32(T)), float(np.float32(alpha))
    for r in range(rows):   # (a row at a time: 64-bit copies of the widest are 64 MB)
        v = z[r].double()
        v = v - v.max()
        at, t = ids[r].long(), teacher[r].double() / T
        c = 129 + 44 + k / 64 + 22 + 20 + 6 * float(v.abs().max()) * max(1.0, 1.0 / T) + 2 * float((t - t.max()).abs().max())
        lq, ls = v / T - torch.logsumexp(v / T, 0), v - torch.logsumexp(v, 0)
        p = torch.softmax(t, 0)
        lp = torch.log_softmax(t, 0)
        want = alpha * T * T * (p * (lp - lq[at])).sum() - (1 - alpha) * ls[labels[r]]
        size = alpha * T * T * (p * (1 + lp.abs() + lq[at].abs())).sum() + (1 - alpha) * (1 + ls[labels[r]].abs())
        assert abs(float(loss[r].double() - want)) <= STEP * c * float(size), (r, float(loss[r]), float(want))
        q = alpha * T * torch.exp(lq) + (1 - alpha) * torch.exp(ls)
        grad, sizes = q.clone(), q.clone()
        grad.index_add_(0, at, -alpha * T * p)
        sizes.index_add_(0, at, alpha * T * p)
        grad[labels[r]] -= 1 - alpha
        sizes[labels[r]] += 1 - alpha
        err = (g[r].double() - grad).abs()
        bound = STEP * c * sizes + (2.0 ** -8 * grad.abs() if dtype == "bf16" else 0.0) + 1e-30
        assert bool((err <= bound).all()), (r, int((err - bound).argmax()), float((err - bound).max()))


def problem(rows, C, k, seed):
    gen = torch.Generator().manual_seed(seed)
    z = 2.0 * torch.randn(rows, C, generator=gen)
    for r in range(rows):   # (every fourth row as it is)
        if r % 4 < 3:
            z[r, C - 1 - r % 4] = 16.0 + r % 5
    ids = torch.stack([torch.randint(0, C - 4 - k, (1,), generator=gen) + torch.randperm(k, generator=gen) for _ in range(rows)]).to(torch.int32)
    return z, torch.randint(0, C - 4, (rows,), generator=gen).to(torch.int32), ids, 2.0 * torch.randn(rows, k, generator=gen)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C,k", [(5, 1021, 20), (5, 2047, 64), (5, 4093, 100), (5, 8191, 30), (5, 16383, 64), (66, 32766, 20), (66, 32769, 20), (66, 51199, 64), (66, 51203, 64),
                                      (66, 65535, 100), (66, 65537, 100), (66, 65538, 8), (66, 65539, 100), (66, 98301, 64), (66, 98303, 5), (66, 98305, 64), (66, 131071, 100),
                                      (66, 131069, 5), (3, 32769, 10), (7, 50257, 64), (5, 98307, 100), (48, 131071, 100), (5, 70001, 100)])
def test_remainders(dtype, rows, C, k):
    check(*problem(rows, C, k, seed=C), 2.0, 0.7, dtype)
    check(*problem(rows, C, k, seed=C + 1), 1.0, 0.4, dtype)


@pytest.mark.parametrize("rows,C", [(2, (1 << 23) - 1), (1, 1 << 23), (3, 5000001)])
def test_the_widest_rows(rows, C):
    """As many slices as a row may have."""
    check(*problem(rows, C, 40, seed=1), 1.5, 0.6, "f32")
    check(*problem(rows, C, 40, seed=2), 1.0, 1.0, "bf16")
