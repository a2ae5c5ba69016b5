"""Prompt and tree attention on the GPU where scores are so large that fp32's
own steps show between them."""
import math

import pytest
import torch

from test_gpu_multi_ops import HALF, weights_off
from test_gpu_multi_ops_edges import Call
from test_gpu_ops import gen, gpu  # noqa: F401

pytestmark = pytest.mark.gpu

F32, F16, BF16, E4M3 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn
TYPES = [(F32, F32), (F16, F16), (BF16, BF16), (F16, E4M3), (BF16, E4M3)]
# query heads of a cache head and tokens: blocks of 32, 64, 128 and, of two
# bytes, 256 rows
ROWS = [(1, 8), (1, 40), (1, 150), (8, 500)]
LENGTH = 700


def reference(c, scale):
    """Allowed keys, weights of the formula and outputs, in fp64."""
    n, length = c.new[0], c.lens[0]
    total = length + n if c.tree else length
    page = c.table_cpu[0].long()[torch.arange(total) // c.slots]
    k, v = (x.cpu().float().double()[page, torch.arange(total) % c.slots] for x in (c.k, c.v))
    allowed = torch.stack([c.attends(0, j) for j in range(total)], 1)
    q = c.q.cpu().double()[:n]
    heads, kv = q.shape[1], k.shape[1]
    k, v = (x.repeat_interleave(heads // kv, 1).transpose(0, 1) for x in (k, v))
    score = (q.transpose(0, 1) @ k.transpose(1, 2)) * scale
    score = torch.where(allowed, score, -math.inf)
    w = torch.softmax(score, -1)
    return w, v, (w @ v).transpose(0, 1), torch.logsumexp(score, -1).transpose(0, 1)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("group,n", ROWS)
@pytest.mark.parametrize("width", [None, 100])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("power", [22, 24, 25, 26])
def test_scores_a_step_apart(dtype, cache, group, n, width, tree, power):
    """Scores of 2^power and one to three of fp32's steps above it, the larger
    ones behind the first tiles.  All of them are exact, so a weight is off by
    what its exponent loses, t log2(e) scale (2^-23 for the factor, 2^-24 for the
    product) for a difference t, by the exponential's 2^-21, by its rounding before
    the second product and by n 2^-23 of the sums."""
    if cache == E4M3 and power > 25:
        pytest.skip("beyond the type")
    c = Call(dtype, cache, 2 * group, 2, 64, 16, [n], [LENGTH - n if tree else LENGTH], tree=tree, width=width, seed=power)
    g, step = gen(power + n), 2.0 ** (power - 23)
    c.q.zero_()
    # 2^power as a sum of four products of which each is in every type's range
    c.q[..., :4] = 2.0 ** 15
    c.q[..., 4] = 1.0
    key = torch.arange(LENGTH)
    page, slot = c.table_cpu[0].long()[key // 16], key % 16
    late = (key >= LENGTH // 2) & (key % 5 == 0)
    for most in (1, 2, 3):
        keys = torch.zeros(c.k.shape)
        keys[page, slot, :, :4] = 2.0 ** (power - 17)
        keys[page, slot, :, 4] = (torch.randint(0, most + 1, (LENGTH,), generator=g) * late * step)[:, None]
        c.k.copy_(keys.to(cache))
        for scale in (1.0, 1.379, -1.0):
            c.more["scale"] = scale
            if scale < 0:
                c.q.neg_()
            w, v, want, want_lse = reference(c, scale)
            out, lse, status = c.results()
            if scale < 0:
                c.q.neg_()
            weight, least = weights_off(dtype, n, 1, group)
            exponent = 3 * step * math.log2(math.e) * abs(scale) * (2.0 ** -23 + 2.0 ** -24)
            off = torch.where(w > 0, w * (exponent + 2.0 ** -21 + weight + LENGTH * 2.0 ** -23), 0.0) + least * w.amax(-1, keepdim=True)
            bound = (off @ v.abs() + off.sum(-1, keepdim=True) * (w @ v.abs())).transpose(0, 1)
            room = bound + (want.abs() + bound) * HALF[dtype] + (2.0 ** -25 if dtype == F16 else 0)
            assert status.tolist() == [0]
            assert torch.all((out.double() - want).abs() <= room), (most, scale)
            # the scaled maximum and the logarithm of the count, at most 10, rounded
            # to fp32, scaled by ln 2 and added: 2^-24 of each four times
            assert torch.all((lse.double() - want_lse).abs() <= (want_lse.abs() + 2 * 10) * 2.0 ** -22)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("group,n", ROWS)
@pytest.mark.parametrize("power", [10, 15, 40])
@pytest.mark.parametrize("tree", [False, True])
def test_scores_of_any_size(dtype, group, n, power, tree):
    """Scores of up to 2^80: those at the maximum share the whole weight (the
    others lie 2^12 and more below it), however coarse the maximum itself is."""
    if dtype == F16 and power > 15:
        pytest.skip("beyond the type")
    c = Call(dtype, dtype, 2 * group, 2, 64, 16, [n], [LENGTH - n if tree else LENGTH], tree=tree, seed=power, scale=0.1)
    g = gen(n + power)
    c.q.zero_()
    c.k.zero_()
    c.k[..., 0] = (torch.randint(-4, 5, c.k.shape[:3], generator=g) * 2.0 ** (power - 3)).to(dtype).cuda()
    c.q[..., 0] = torch.tensor([1.0, -0.75] * group).to(dtype).cuda() * 2.0 ** power
    w, v, want, want_lse = reference(c, 0.1)
    out, lse, status = c.results()
    # a mean of the values at the maximum, whose weights are one power of two:
    # roundings of sums of LENGTH of them, and of the result
    bound = LENGTH * 2.0 ** -23 * v.abs().max()
    assert status.tolist() == [0]
    assert torch.all((out.double() - want).abs() <= bound + (want.abs() + bound) * HALF[dtype] + (2.0 ** -25 if dtype == F16 else 0))
    assert torch.all((lse.double() - want_lse).abs() <= (want_lse.abs() + 2 * 10) * 2.0 ** -22)
