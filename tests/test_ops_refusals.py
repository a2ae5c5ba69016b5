"""More refusals of the single-token step's operators, on the host: arguments
that are in range one by one but not in what the kernels make of them.  CPU
only."""
import ctypes as C

import pytest

from paper_2111_05426_amd import dsim
from test_ops import FAKE, L, cache, rows  # noqa: F401



@pytest.mark.parametrize("scale", [3e38, -3e38, 2.0 ** 127, float("inf"), -float("inf"), float("nan")])
def test_attention_scale_that_overflows(L, scale):   # noqa: F811
    """Times log2 e it would be infinite, and products of 0 then NaN."""
    rc = L.dsim_paged_attention(C.byref(cache()), 2, C.byref(rows()), C.byref(rows()), 4, FAKE, scale, 0, None, None,
                                None, 0, None)
    assert rc == -1 and "scale" in dsim.dsim_last_error(), (rc, dsim.dsim_last_error())


def test_attention_largest_scale(L):   # noqa: F811
    """2^126 is taken (and the next thing, the workspace, refused)."""
    for scale in (2.0 ** 126, -2.0 ** 126):
        rc = L.dsim_paged_attention(C.byref(cache()), 2, C.byref(rows()), C.byref(rows()), 4, FAKE, scale, 0, None, None,
                                    None, 0, None)
        assert rc == -3 and "workspace" in dsim.dsim_last_error()
