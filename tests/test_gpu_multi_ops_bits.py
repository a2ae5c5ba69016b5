"""Prompt and tree attention of 16 bits on the GPU to the bits that the header
states: scores, weights, statistics and sums of fp32, one rounding of the
result, however many rows a call has."""
import pytest
import torch

import multi_ops_plain as plain
from test_gpu_multi_ops import HALF
from test_gpu_multi_ops_edges import Call
from test_gpu_ops import gpu  # noqa: F401

pytestmark = pytest.mark.gpu

F16, BF16, E4M3 = torch.float16, torch.bfloat16, torch.float8_e4m3fn
MASKS = [dict(), dict(window=150), dict(cap=20.0), dict(slopes=True), dict(cap=200.0, slopes=True, scale=0.2)]


@pytest.mark.parametrize("dtype,cache", [(F16, F16), (BF16, BF16), (F16, E4M3), (BF16, E4M3)])
@pytest.mark.parametrize("group,n", [(1, 8), (1, 40), (1, 150), (8, 330)])
@pytest.mark.parametrize("mask", range(len(MASKS)))
@pytest.mark.parametrize("d,width", [(64, None), (128, 100)])
@pytest.mark.parametrize("tree", [False, True])
def test_one_rounding(dtype, cache, group, n, mask, d, width, tree):
    """A weight enters the second product as two numbers of its type: off by the
    square of a half step.  A tanh is off by 2^-20 of itself or 2^-21 of the cap,
    and a weight by that of the score.  The sum that lse is the logarithm of has
    no rounding of weights."""
    more = dict(MASKS[mask])
    if more.get("slopes"):
        more["slopes"] = 2.0 ** (-8.0 * torch.arange(1, 2 * group + 1, device="cuda") / (2 * group))
    lens = [500, 350]
    c = Call(dtype, cache, 2 * group, 2, d, 16, [n, n], [x - n if tree else x for x in lens], tree=tree, width=width, seed=mask, **more)
    out, lse, status = c.results()
    args = dict(window=more.get("window", 0), cap=more.get("cap", 0.0), exact=False)
    if tree:
        args.update(tree_mask=c.mask.cpu(), depth=c.depth.cpu())
    if "slopes" in more:
        args["slopes"] = more["slopes"].cpu()
    inputs = [x.cpu() for x in (c.q, c.k, c.v)] + [c.table_cpu.clamp(min=0), c.start.cpu(), c.len.cpu(), more.get("scale", d ** -0.5)]
    capped = 2 * args["cap"] * 2.0 ** -21
    ref, _, bound, _, _ = plain.attention(*inputs, **args, weight=HALF[dtype] ** 2 + capped,
                                          least=2.0 ** -36 if dtype == F16 else 2.0 ** -126)
    _, ref_lse, _, lse_bound, _ = plain.attention(*inputs, **args, weight=capped)
    room = bound + (ref.abs() + bound) * HALF[dtype] + (2.0 ** -25 if dtype == F16 else 0)
    off, lse_off = (out.double() - ref).abs(), (lse.double() - ref_lse).abs()
    assert status.tolist() == [0, 0]
    assert torch.all(off <= room), float((off - room).max())
    assert torch.all(lse_off <= lse_bound), float((lse_off - lse_bound).max())
