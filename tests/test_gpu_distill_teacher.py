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
