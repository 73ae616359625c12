"""What the direct calls ask for as workspace, without a GPU: a workspace of the bytes for some rows is enough for any fewer."""
import pytest

from tests.test_operator_refusals import backward, distill
from paper_2410_14312_amd import binding

ECAP = -8
ROWS = sorted(set(range(1, 140)) | {2 ** e + o for e in range(7, 21) for o in (-1, 0, 1)} | set(range(500, 9000, 37)))


@pytest.mark.parametrize("D", [1, 16, 128, 130, 256, 260, 512, 768, 1001, 2048, 4096, 4100, 8192, 16384])
def test_norm_join_workspaces_never_shrink(D):
    sizes = [binding.lib().tmps_norm_join_workspace(r, D) for r in ROWS]
    assert sizes == sorted(sizes) and sizes[0] > 0


@pytest.mark.parametrize("classes", [1, 1000, 32768, 32769, 50257, 65536, 98304, 98305, 131071, 200000, 1 << 23])
def test_distill_workspaces_never_shrink(classes):
    sizes = [binding.lib().tmps_distill_workspace(r, classes) for r in ROWS]
    assert sizes == sorted(sizes) and (sizes[0] > 0) == (classes > 32768)


def test_what_is_too_small_is_refused():
    """Less than a call's own need; the addresses are refused otherwise only behind that check."""
    assert backward(rows=1023, D=768, ws_bytes=1023 * 2 * 2 * 768 * 4 - 4) == ECAP
    assert distill(rows=48, classes=131071, ws_bytes=48 * 32 * 3 * 4 - 4) == ECAP
    assert distill(rows=48, classes=131071, ws=None) == ECAP
