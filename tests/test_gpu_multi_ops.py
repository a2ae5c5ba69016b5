"""The operators of a step of several tokens on the GPU against plain
implementations (tests/multi_ops_plain.py): types, head layouts, lengths from
none to thousands, masks that leave rows empty, page sizes that end inside a
tile, strides, errors in device data, cut blocks of rows."""
import math

import pytest
import torch

import multi_ops_plain as plain
import step_ops
from paper_2111_05426_amd import ops
from test_gpu_ops import cache_like, deal, gen, randn, to_gpu

pytestmark = pytest.mark.gpu

F32, F16, BF16, E4M3 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn
TYPES = [(F32, F32), (F16, F16), (BF16, BF16), (F16, E4M3), (BF16, E4M3)]
HALF = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"


def ints(x):
    return torch.tensor(x, dtype=torch.int32)


def weights_off(dtype, tokens, n_seq, group):
    """What a weight may be off before the second product: fp32's bits, two
    numbers of the type for few rows, one for many; and below what part of the
    largest weight it is lost.  fp16 rounds to multiples of 2^-24, off by 2^-25,
    and the weight of the score that others are held against is 2^11.  Else
    exponentials end at 2^-126, where fp32's numbers of full precision do: the
    score that others are held against is not above the largest, whose weight is
    1 or more, so what is lost is less than 2^-126 of it."""
    if dtype == F32:
        return 0.0, 2.0 ** -126
    few = tokens * group <= 64 * n_seq
    return (HALF[dtype] ** 2 if few else HALF[dtype]), (2.0 ** -36 if dtype == F16 else 2.0 ** -126)


def random_tree(g, n):
    """Depths and mask words of n drafted tokens, a node's parent one of the
    four before it or none."""
    depth, sees = torch.zeros(n, dtype=torch.int32), torch.zeros(n, n, dtype=torch.bool)
    for i in range(n):
        parent = i - int(torch.randint(1, 6, (1,), generator=g)) if i else -1
        if parent >= 0:
            depth[i] = depth[parent] + 1
            sees[i] = sees[parent]
        sees[i, i] = True
    return depth, sees


def words(sees, n_words):
    out = torch.zeros(sees.shape[0], n_words * 32, dtype=torch.int64)
    out[:, :sees.shape[1]] = sees
    x = (out.view(sees.shape[0], n_words, 32) << torch.arange(32)).sum(-1)
    return torch.where(x >= 2 ** 31, x - 2 ** 32, x).to(torch.int32)


def check(dtype, cache, heads, kv, d, slots, new, lens, tree=False, window=0, cap=0.0, slopes=False, prefix=None,
          docs=None, scales=False, order="head", scale=None, seed=0, edit=None, width=None, spread=2.0, in_place=False,
          pad=0, expect=None):
    """new: tokens of each sequence; lens: keys of a prompt with them, or a
    tree's context; docs: the first key of every token; pad: rows of q behind
    the last sequence."""
    g = gen(seed)
    total = [max(n, 0) + (m if tree else 0) for n, m in zip(lens, new)]
    table, pages = deal(g, total, slots, width)
    keys, values = cache_like(g, pages, slots, kv, d, F32 if cache == E4M3 else cache, order)
    if cache == E4M3:
        keys, values = keys.to(E4M3), values.to(E4M3)
    tokens = sum(new)
    q = (spread * randn(g, tokens + pad, heads, d)).to(dtype)
    ks, vs = ((0.25 + torch.rand(kv, generator=g)) if scales else None for _ in range(2))
    start = ints([sum(new[:i]) for i in range(len(new) + 1)])
    slope = 2.0 ** (-8.0 * torch.arange(1, heads + 1) / heads) if slopes else None
    depth = mask = None
    if tree:
        n_words = (max(new + [1]) + 31) // 32
        trees = [random_tree(g, n) for n in new]
        depth = torch.cat([t[0] for t in trees] + [torch.zeros(pad, dtype=torch.int32)])
        mask = torch.cat([words(t[1], n_words) for t in trees] + [torch.zeros(pad, n_words, dtype=torch.int32)])
    first = None if docs is None else ints(docs + [0] * pad)
    pre = None if prefix is None else ints(prefix)
    length = ints(lens)
    ref_keys, ref_values = keys.clone(), values.clone()
    if edit:
        edit(locals())
    out = torch.full((tokens + pad, heads, d), 123.0, dtype=dtype, device="cuda")
    lse = torch.full((tokens + pad, heads), 123.0, device="cuda")
    status = torch.full((len(new),), -7, dtype=torch.int32, device="cuda")
    ws = ops.alloc_prompt_attention_workspace(tokens + pad, len(new), heads, kv, d)
    ws.fill_(255)   # nothing may depend on what it holds
    dq = q.cuda()
    if in_place:
        out = dq
    dev = dict(k=to_gpu(keys), v=to_gpu(values), k_scale=to_gpu(ks), v_scale=to_gpu(vs))
    more = dict(scale=scale, window=window, cap=cap, slopes=to_gpu(slope), workspace=ws, lse=lse, status=status)
    if tree:
        ops.dsim_tree_attention(dq, dev, table.cuda(), start.cuda(), length.cuda(), mask.cuda(), out, depth=depth.cuda(), **more)
    else:
        ops.dsim_prompt_attention(dq, dev, table.cuda(), start.cuda(), length.cuda(), out, prefix_len=to_gpu(pre),
                                  first_key=to_gpu(first), **more)
    torch.cuda.synchronize()
    used = d ** -0.5 if scale is None else scale
    weight, least = weights_off(dtype, tokens + pad, len(new), heads // kv)
    ref, ref_lse, bound, lse_bound, seen = plain.attention(
        q, ref_keys, ref_values, table.clamp(min=0), start, length, used, mask, depth, pre, first, window, cap, slope, ks,
        vs, weight, least, exact=dtype == F32)
    out, lse, status = out.cpu(), lse.cpu(), status.cpu()
    for s, n in enumerate(lens):
        assert int(status[s]) == (-7 if n < 0 else 0), s
    assert torch.equal(out[~seen], q[~seen] if in_place else torch.full_like(out[~seen], 123.0))
    assert torch.all(lse[~seen] == 123.0)
    room = bound + (ref.abs() + bound) * HALF[dtype] + (2.0 ** -25 if dtype == F16 else 0)
    off = (out.double() - ref).abs() - room
    assert torch.all(off[seen] <= 0), float(off[seen].max())
    lse_off = torch.where(ref_lse == lse.double(), torch.zeros_like(ref_lse), (lse.double() - ref_lse).abs() - lse_bound)
    assert torch.all(lse_off[seen] <= 0), float(lse_off[seen].max())
    return out


LAYOUTS = [(12, 12, 64), (8, 2, 128), (16, 1, 96), (5, 5, 80), (2, 1, 256), (3, 3, 16), (4, 4, 112), (40, 2, 64),
           (6, 2, 208), (17, 1, 144), (4, 4, 32)]


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("heads,kv,d", LAYOUTS)
def test_prompt(dtype, cache, heads, kv, d):
    scales = cache == E4M3 and heads > 4
    check(dtype, cache, heads, kv, d, 16, [1, 16, 33, 0, 100], [1, 20, 33, 7, 250], scales=scales)
    check(dtype, cache, heads, kv, d, 16, [1, 16, 33, 0, 100], [1, 20, 33, 7, 250], scales=scales, width=200)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("heads,kv,d", LAYOUTS)
def test_tree(dtype, cache, heads, kv, d):
    scales = cache == E4M3 and heads > 4
    for width in (None, 200):
        check(dtype, cache, heads, kv, d, 16, [1, 8, 33, 0, 70], [0, 20, 31, 7, 250], tree=True, scales=scales, width=width)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("slots", [1, 3, 16, 48, 64, 256])
def test_page_sizes(dtype, cache, slots):
    for width in (None, 2000 // slots + 1):
        check(dtype, cache, 4, 2, 64, slots, [1, 31, 65, 130], [40, 31, 300, 129 + 1], seed=slots, width=width)
        check(dtype, cache, 4, 2, 64, slots, [1, 5, 33], [40, 300, 63], tree=True, seed=slots, width=width)


@pytest.mark.parametrize("order", ["head", "slot", "gaps"])
@pytest.mark.parametrize("cache", [BF16, E4M3])
def test_layouts(order, cache):
    check(BF16, cache, 8, 2, 128, 16, [77, 5, 60], [77, 9, 200], order=order)
    check(BF16, cache, 8, 2, 128, 16, [7, 5, 20], [77, 9, 200], order=order, tree=True)


MASKS = [dict(window=1), dict(window=40), dict(cap=20.0), dict(slopes=True), dict(prefix=[5, 40, 0, 900]),
         dict(window=17, cap=50.0, slopes=True, prefix=[3, 0, 30, 100])]


@pytest.mark.parametrize("dtype,cache", [(F32, F32), (F16, F16), (BF16, E4M3)])
@pytest.mark.parametrize("mask", range(len(MASKS)))
@pytest.mark.parametrize("width", [None, 90])
def test_prompt_masks(dtype, cache, mask, width):
    check(dtype, cache, 4, 2, 64, 16, [20, 41, 1, 200], [20, 64, 33, 230], width=width, **MASKS[mask])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("mask", [0, 1, 2, 3])
@pytest.mark.parametrize("width", [None, 90])
def test_tree_masks(dtype, mask, width):
    check(dtype, dtype, 4, 2, 64, 16, [20, 41, 1, 3], [20, 64, 33, 0], tree=True, width=width, **MASKS[mask])


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("width", [None, 90])
def test_documents(dtype, width):
    """Documents of a sequence; first keys behind the token itself leave rows
    without keys."""
    g = gen(5)
    new, lens = [64, 150, 9], [64, 190, 9]
    docs = []
    for n, length in zip(new, lens):
        p = torch.arange(length - n, length)
        docs += (p // 37 * 37).tolist()
    for i in torch.randint(0, sum(new), (20,), generator=g).tolist():
        docs[i] = 10 ** 9
    docs[3] = -5
    check(dtype, dtype, 4, 2, 64, 16, new, lens, docs=docs, width=width)
    check(dtype, dtype, 4, 1, 64, 16, new, lens, docs=docs, width=width, window=20, prefix=[0, 150, 4])
    out = check(dtype, dtype, 4, 2, 64, 16, new, lens, docs=[10 ** 9] * sum(new), width=width)
    assert torch.all(out == 0)


@pytest.mark.parametrize("dtype,cache", TYPES)
def test_long(dtype, cache):
    """Blocks of rows that the work's cuts go through, among short ones,
    sequences that are left alone and padding."""
    new, lens = [300, 1, 0, 2, 40, 100], [3000, 3, 5, 5001, -1, 700]
    check(dtype, cache, 4, 2, 64, 16, new, lens, seed=3, pad=9)
    check(dtype, cache, 4, 1, 128, 32, new, lens, seed=4, window=1500)
    check(dtype, cache, 2, 2, 256, 16, [60, 1, 0, 2, 4, 10], lens, seed=5)
    check(dtype, cache, 20, 1, 80, 48, [20, 1, 0, 2, 4, 10], lens, seed=6)
    check(dtype, cache, 2, 1, 64, 5, [9, 1, 0, 2, 4, 10], lens, seed=7)
    check(dtype, cache, 8, 2, 128, 16, [30, 1, 0, 8, 16, 1], lens, seed=8, tree=True, pad=5)
    check(dtype, cache, 4, 4, 96, 16, [3, 1, 0, 70, 16, 1], lens, seed=9, tree=True, window=700)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("width", [None, 600])
def test_in_place(dtype, cache, width):
    lens = [5, 60, 300, -1, 77] + ([] if width is None else [4000])
    new = [5, 1, 100, 2, 77] + ([] if width is None else [80])
    check(dtype, cache, 4, 2, 64, 16, new, lens, width=width, in_place=True, pad=3)
    check(dtype, cache, 4, 2, 128, 16, new, lens, width=width, in_place=True, tree=True)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("heads,kv,d,slots", [(4, 1, 128, 16), (4, 1, 64, 48), (4, 1, 80, 7), (5, 5, 256, 16), (3, 1, 112, 32)])
def test_many_rows(dtype, cache, heads, kv, d, slots):
    """Prompts of the largest blocks of rows."""
    new, lens = [700, 3, 560, 1], [700, 900, 561, 1]
    check(dtype, cache, heads, kv, d, slots, new, lens, seed=2)
    check(dtype, cache, heads, kv, d, slots, new, lens, seed=3, window=333, cap=30.0, prefix=[40, 0, 500, 0])
    check(dtype, cache, heads, kv, d, slots, [300, 1, 800], [40, 900, 0], seed=4, tree=True, width=2000 // slots)


@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-30, 5.0])
def test_scales(scale):
    check(BF16, BF16, 4, 2, 64, 16, [20, 60], [50, 60], scale=scale)
    check(F32, F32, 4, 2, 64, 16, [2, 6], [50, 60], scale=scale, tree=True)
    if scale != 1e-30:
        check(F16, F16, 4, 2, 64, 16, [20, 60], [50, 60], scale=scale, cap=10.0)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("heads,kv,d,slots", [(8, 1, 128, 16), (16, 2, 64, 48), (8, 1, 80, 7), (10, 1, 112, 32), (8, 1, 32, 16)])
def test_largest_blocks(dtype, cache, heads, kv, d, slots):
    """More than 1,536 rows a sequence on average, in blocks of their own and
    cut ones."""
    new, lens = [330, 100], [330, 500]
    for width in (None, 2000 // slots):
        check(dtype, cache, heads, kv, d, slots, new, lens, seed=2, width=width)
        check(dtype, cache, heads, kv, d, slots, new, lens, seed=3, window=133, cap=30.0, prefix=[40, 300], width=width)
        check(dtype, cache, heads, kv, d, slots, new, lens, seed=4, slopes=True, cap=200.0, width=width)
        check(dtype, cache, heads, kv, d, slots, new, [40, 300], seed=5, tree=True, width=width)
    check(dtype, cache, heads, kv, d, slots, new, lens, seed=6, docs=[i // 97 * 97 for i in range(330)] + [350] * 100, scale=2.0)
