"""More refusals of the operators of a step of several tokens, on the host:
arguments that are in range one by one but not in what the kernels make of them.
CPU only."""
import pytest

from test_multi_ops import FAKE, L, cache, expect, queries, ref  # noqa: F401


@pytest.mark.parametrize("scale,cap", [(2.0 ** 126, 2.0 ** -60), (-2.0 ** 67, 2.0 ** -60), (2.0 ** 126, 0.5),
                                       (2.0 ** -126, 2.0 ** 60), (-2.0 ** -100, 2.0 ** 27), (1e-38, 50.0), (1e-45, 2.0 ** 60)])
def test_scale_and_cap_apart(L, scale, cap):   # noqa: F811
    """|scale| / cap is what a capped score is taken times: infinite it makes NaN
    of a score of 0, without fp32's bits 0 of any."""
    for n_seq in (3, 0):
        c, q = cache(n_seq=n_seq), queries(scale=scale, cap=cap, ws_bytes=0)
        expect("scale / cap", L.dsim_prompt_attention(ref(c), ref(q), None, None, None))
        expect("scale / cap", L.dsim_tree_attention(ref(c), ref(q), FAKE, 2, 2, FAKE, None))


@pytest.mark.parametrize("scale,cap", [(2.0 ** 66, 2.0 ** -60), (-2.0 ** 126, 1.0), (2.0 ** -66, 2.0 ** 60), (2.0 ** -126, 1.0),
                                       (0.0, 2.0 ** 60), (-0.0, 2.0 ** -60), (2.0 ** 126, 0.0), (2.0 ** -126, 0.0), (0.125, 50.0)])
def test_scale_and_cap(L, scale, cap):   # noqa: F811
    """Taken (and the next thing, the workspace, refused)."""
    c, q = cache(), queries(scale=scale, cap=cap, ws_bytes=0)
    expect("workspace", L.dsim_prompt_attention(ref(c), ref(q), None, None, None))
    expect("workspace", L.dsim_tree_attention(ref(c), ref(q), FAKE, 2, 2, FAKE, None))
