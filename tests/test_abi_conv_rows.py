"""The most rows of the short convolution (no GPU needed: refused before any HIP call)."""
import ctypes

import pytest

from paper_2606_27229_amd import carve
from test_abi_ssm_host import UNSUPPORTED, cdims, conv

RUN = 24   # rows of a thread in the backward, the most of any kernel


def size(**kw):
    return carve.load_library().carve_short_conv_workspace_size(ctypes.byref(cdims(**kw)))


@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("T", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 4, 2 ** 31 - 27, 2 ** 31 - 63])
def test_rows_that_ints_cannot_count(T, W):
    """Row numbers reach a run and W - 1 rows behind the last one."""
    kw = dict(B=1, T=T, C=8, W=W)
    assert size(**kw) == 0
    for which in ("fwd", "bwd", "step"):
        assert conv(cdims(**kw), which) == UNSUPPORTED


def test_the_most_rows():
    assert 2 ** 31 - 64 + RUN + 3 < 2 ** 31
    assert size(B=1, T=2 ** 31 - 64, C=8) > 0
