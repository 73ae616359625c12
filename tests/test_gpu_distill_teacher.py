"""Distillation against teachers whose logits have a large common part: a softmax is the same without it.  The logits are sums of the part and multiples of 1/16, exact in fp32, so what
a call gives with the part and without it is the same bit for bit."""
import pytest
import torch

import paper_2410_14312_amd as tmps

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(autouse=True)
def single_precision_by_default():
    """(tests of the oracle leave their process at doubles)"""
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


@pytest.mark.parametrize("rows,C,k", [(5, 100, 12), (70, 5000, 100), (3, 50000, 300), (66, 33000, 70)])
@pytest.mark.parametrize("T", [0.3, 1.0, 1.7])
def test_a_common_part_takes_no_places(rows, C, k, T):
    gen = torch.Generator().manual_seed(C)
    z = torch.randn(rows, C, generator=gen).to(DEV)
    ids = torch.stack([torch.randperm(C, generator=gen)[:k] for _ in range(rows)]).to(torch.int32).to(DEV)
    labels = torch.randint(0, C, (rows,), generator=gen).to(torch.int32).to(DEV)
    teacher = (torch.randint(-100, 100, (rows, k), generator=gen) / 16.0).to(DEV)
    want = tmps.distill(z, labels, ids, teacher, temperature=T, alpha=0.8)
    for part in (1000.0, -30000.0, 500000.0):
        got = tmps.distill(z, labels, ids, teacher + part, temperature=T, alpha=0.8)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    p = torch.softmax(teacher.double() / T, dim=1)
    lq = torch.log_softmax(z.double() / T, dim=1)
    at = ids.long()
    loss = 0.8 * T * T * (p * (p.log() - lq.gather(1, at))).sum(1) + 0.2 * -torch.log_softmax(z.double(), dim=1).gather(1, labels.long()[:, None])[:, 0]
    # (some 200 steps of 2^-24 of terms below 0.8 T^2 (|log p| + |log q|) <= 100)
    assert float((want[0].double() - loss).abs().max()) < 200 * 2.0 ** -24 * 100


@pytest.mark.parametrize("rows,C,k", [(5, 300, 12), (9, 6001, 100), (6, 60000, 40), (70, 40001, 40)])
@pytest.mark.parametrize("T", [0.5, 2.0])
def test_masks_of_the_lowest_value(rows, C, k, T):
    """The student's classes and the teacher's entries masked with the type's lowest value are those masked with minus infinity, bit for bit; a row of masked classes alone is
    uniform."""
    gen = torch.Generator().manual_seed(k)
    low = torch.finfo(torch.float32).min
    z, teacher = torch.randn(rows, C, generator=gen), torch.randn(rows, k, generator=gen)
    ids = torch.stack([torch.randperm(C // 2, generator=gen)[:k] for _ in range(rows)]).to(torch.int32).to(DEV)
    labels = torch.randint(0, C // 2, (rows,), generator=gen).to(torch.int32).to(DEV)
    hidden, absent = torch.rand(rows, C, generator=gen) < 0.3, torch.rand(rows, k, generator=gen) < 0.3
    hidden[:, :C // 2] = False
    absent[:, 0] = False
    for dtype in ("f32", "bf16"):
        got, want = (tmps.distill(z.masked_fill(hidden, v).to(DEV), labels, ids, teacher.masked_fill(absent, v).to(DEV), temperature=T, alpha=0.6, dtype=dtype) for v in (low, -float("inf")))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and bool(torch.isfinite(got[0]).all())
    loss, g = tmps.distill(torch.full((rows, C), low, device=DEV), labels, ids, torch.full((rows, k), low, device=DEV), temperature=T, alpha=0.6, grad_scale=1.0)
    same, h = tmps.distill(torch.zeros(rows, C, device=DEV), labels, ids, torch.zeros(rows, k, device=DEV), temperature=T, alpha=0.6, grad_scale=1.0)
    assert torch.equal(loss, same) and torch.equal(g, h)
