"""The direct calls on a stream that is given to them: what they allocate belongs to it, and results are those of the current stream."""
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


def calls():
    gen = torch.Generator().manual_seed(5)
    n = lambda *s: torch.randn(*s, generator=gen).to(DEV)   # noqa: E731
    x, pos = n(70, 128), torch.randint(0, 99, (70, 3), generator=gen).to(torch.int32).to(DEV)
    f, r, dy, du, v, w = n(70, 256), n(70, 128), n(70, 128), n(70, 128), n(128), n(128)
    y, u, stats = tmps.norm_join(f, r, v, w, pre_gain=w, pre_shift=v, gate=True)
    z, t = n(3, 70000), n(3, 5)
    ids, labels = torch.randint(0, 70000, (3, 5), generator=gen).to(torch.int32).to(DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    return {"rotary": lambda **k: (tmps.rotary(x, pos, 2, 64, (16, 8, 8), **k),),
            "norm_join": lambda **k: tmps.norm_join(f, r, v, w, pre_gain=w, pre_shift=v, gate=True, **k),
            "norm_join_backward": lambda **k: tmps.norm_join_backward(dy, du, f, r, y, stats, v, w, pre_gain=w, gate=True, **k),
            "distill": lambda **k: tmps.distill(z, labels, ids, t, temperature=2.0, alpha=0.5, **k)}


def owner(t):
    """the stream whose memory a tensor lies in"""
    for segment in torch.cuda.memory_snapshot():
        if segment["address"] <= t.data_ptr() < segment["address"] + segment["total_size"]:
            return segment["stream"]


@pytest.mark.parametrize("name", ["rotary", "norm_join", "norm_join_backward", "distill"])
def test_results_belong_to_the_stream_that_makes_them(name):
    call = calls()[name]
    want = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for given, handle in ((side, side.cuda_stream), (side.cuda_stream, side.cuda_stream), (0, 0)):
        got = call(stream=given)
        assert torch.cuda.current_stream() == torch.cuda.default_stream()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b) and owner(a) == handle
        del got


def test_a_stream_for_tensors_on_the_host_is_refused():
    z = torch.zeros(4, 4)
    with pytest.raises(ValueError):
        tmps.norm_join(z, z, z[0], z[0], stream=torch.cuda.Stream())


@pytest.mark.parametrize("name", ["norm_join_backward", "distill"])
def test_calls_on_two_streams_at_once(name):
    """Calls whose kernels may overlap, each with a workspace of its own."""
    call = calls()[name]
    want = call()
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [call(stream=sides[k % 2]) for k in range(20)]
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))
