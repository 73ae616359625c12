"""What the Python binding of the direct calls keeps to, without a GPU: no library call is made."""
import pytest
import torch

from paper_2410_14312_amd import binding


def never(*args):
    raise AssertionError("the library was called")


def test_a_call_takes_no_stream_beside_the_current_one():
    """What it was given is allocated on the current stream already."""
    for stream in (0, 1 << 20):
        with pytest.raises(ValueError, match="current stream"):
            binding._call(never, torch.device("cuda:0"), stream)


def asking(*tensors):
    return [[t.clone().requires_grad_(i == k) if t.is_floating_point() else t for i, t in enumerate(tensors)] for k in range(len(tensors)) if tensors[k].is_floating_point()]


def test_tensors_that_ask_for_a_gradient_are_refused_while_gradients_are_recorded():
    """Every operand of every call; under torch.no_grad() such tensors are taken (and then refused for being on the host)."""
    import paper_2410_14312_amd as tmps

    def zeros(*shape):
        return torch.zeros(*shape, dtype=torch.float32)
    f, v, pos = zeros(4, 8), zeros(8), torch.zeros(4, 3, dtype=torch.int32)
    st, ids = zeros(4, 4), torch.zeros(4, 2, dtype=torch.int32)
    calls = [(lambda x: tmps.rotary(x, pos, 1, 8, (4, 0, 0)), (f,)), (lambda out: tmps.rotary(f, pos, 1, 8, (4, 0, 0), out=out), (f,)),
             (lambda x, r, g, s, p, q: tmps.norm_join(x, r, g, s, pre_gain=p, pre_shift=q), (f, f, v, v, v, v)), (lambda y: tmps.norm_join(f, f, v, v, y=y), (f,)),
             (lambda dy, du, x, r, y, stats, g, s, p: tmps.norm_join_backward(dy, du, x, r, y, stats, g, s, pre_gain=p), (f, f, f, f, f, st, v, v, v)),
             (lambda z, t: tmps.distill(z, None, ids, t), (f, zeros(4, 2)))]
    for call, operands in calls:
        for given in asking(*operands):
            with pytest.raises(ValueError, match="asks for a gradient"):
                call(*given)
            with torch.no_grad(), pytest.raises(ValueError, match="on a GPU"):
                call(*given)


def test_streams_are_found_without_private_names(monkeypatch):
    class Stream:
        cuda_stream = 77
    monkeypatch.setattr(torch.cuda, "current_stream", lambda index: Stream if index == 3 else None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    stream, device = binding._short_ways(torch, object())
    assert stream(3) == 77 and device() == 3
    binding._torch()
    monkeypatch.setattr(binding, "_raw_stream", stream)
    monkeypatch.setattr(binding, "_current_device", device)
    seen = []
    binding._call(lambda *a: seen.append(a) or 0, torch.device("cuda:3"), None, 5)
    assert seen == [(5, 77)]
