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
