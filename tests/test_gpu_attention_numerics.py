"""What the paged attention's numbers are good for: weights with fp32's bits
and range whatever the cache's type, infinities and NaN as in the formula,
and errors of the size that fp32 arithmetic has (attention_bounds.py)."""
import math

import pytest
import torch

import attention_bounds as bounds
from paper_2111_05426_amd import ops
from test_gpu_ops import BF16, E4M3, F16, F32, TYPES, cache_like, deal, gen, gpu, randn, to_gpu  # noqa: F401

pytestmark = pytest.mark.gpu

WIDTHS = [None, 200]   # a workgroup per context; a block table with room for 3,200 tokens: cut and joined


def attend(q, keys, values, table, lens, scale, window=0, **scales):
    """(out, lse) of the operator for tensors on the host."""
    out = torch.full(q.shape, 9.0, dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:2], 9.0, device="cuda")
    cache = dict(k=to_gpu(keys), v=to_gpu(values), **{n: to_gpu(x) for n, x in scales.items()})
    ws = ops.alloc_paged_attention_workspace(q.shape[1], keys.shape[2], q.shape[2])
    ws.fill_(255)
    ops.dsim_paged_attention(q.cuda(), cache, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), out,
                             scale=scale, window=window, workspace=ws, lse=lse)
    return out.cpu(), lse.cpu()


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("heads,kv,d", [(4, 4, 64), (8, 2, 128), (6, 2, 80), (4, 1, 256), (3, 3, 16)])
@pytest.mark.parametrize("window", [0, 700])
def test_errors_are_those_of_fp32(dtype, cache, heads, kv, d, window):
    g = gen(d + heads)
    lens = [1, 30, 250, 0, 1500]
    table, pages = deal(g, lens, 16)
    keys, values = (x.to(cache) for x in cache_like(g, pages, 16, kv, d, F32 if cache == E4M3 else cache))
    q = (2 * randn(g, len(lens), heads, d)).to(dtype)
    scales = {n + "_scale": 0.25 + torch.rand(kv, generator=g) for n in "kv"} if cache == E4M3 else {}
    ref, ref_lse, room, lse_room = bounds.attend(q, keys, values, table.clamp(min=0), lens, d ** -0.5, window, **scales)
    out, lse = attend(q, keys, values, table, lens, d ** -0.5, window, **scales)
    print("of the room: %.2f" % bounds.off(out, ref, room) if dtype == F32 else "")
    assert bounds.within(out, ref, room)
    some = torch.tensor(lens) > 0
    assert torch.all((lse.double() - ref_lse)[some].abs() <= lse_room[some]) and torch.all(lse[3] == -math.inf)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("kv", [1, 4])   # four query heads
@pytest.mark.parametrize("width", WIDTHS)
def test_weights_keep_their_bits(dtype, cache, kv, width):
    """Two keys of values 1 and -1 whose weights nearly cancel: out = tanh(a /
    2), a the difference of their scores, one product of powers of two and a
    query's element.  The second weight exp(-a) is off by at most 2^-23 (an exponential next to 1,
    its argument exact but for 2^-24 of a), the sums 1 +- w by 2^-24 each, so
    out by 2^-22.  A weight of 16 bits is off by up to 2^-17."""
    n, d = 64, 16
    g = gen(1)
    q = torch.zeros(n, 4, d)
    q[..., 0] = (64 + torch.arange(n * 4)).view(n, 4) * 2.0 ** -9
    keys, values = torch.zeros(n, 16, kv, d), torch.zeros(n, 16, kv, d)
    keys[:, 1, :, 0], values[:, 0], values[:, 1] = -2.0 ** -5, 1.0, -1.0
    q, keys, values = q.to(dtype), keys.to(cache), values.to(cache)
    table = torch.full((n, width or 2), -1, dtype=torch.int32)
    table[:, 0] = torch.randperm(n, generator=g)
    scale = 2.0 ** -4
    out, _ = attend(q, keys, values, table, [2] * n, scale)
    ref = torch.tanh(q[..., :1].double() * 2.0 ** -5 * scale / 2).expand(n, 4, d)
    assert bool(torch.all((out.double() - ref).abs() <= 2.0 ** -22 + ref.abs() * bounds.HALF_STEP[dtype] + bounds.LEAST[dtype]))


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("n", [20, 900, 3000])
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("kv", [1, 2])   # two query heads
def test_far_keys_add_what_they_weigh(dtype, cache, n, width, kv):
    """One key with small values far above many with large ones, which weigh
    2^-50 to 2^-60 of it: nothing, and no more, comes from them."""
    g, d = gen(n), 64
    table, pages = deal(g, [n], 16, width)
    keys, values = (torch.zeros(pages, 16, kv, d) for _ in range(2))
    spot = table[0, 0].long(), 3
    keys[..., 0] = -torch.randint(50, 61, (pages, 16, kv), generator=g).float()
    values[:] = 256.0
    keys[spot], values[spot] = 0.0, 2.0 ** -9
    q = torch.zeros(1, 2, d)
    q[..., 0] = 1.0
    q, keys, values = q.to(dtype), keys.to(cache), values.to(cache)
    ref, _, room, _ = bounds.attend(q, keys, values, table.clamp(min=0), [n], math.log(2.0))
    out, _ = attend(q, keys, values, table, [n], math.log(2.0))
    assert room.max() < 2.0 ** -23 and bounds.within(out, ref, room)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("below", [0, 12, 30, 60])
@pytest.mark.parametrize("n,where", [(200, 0), (200, 70), (200, 199), (3000, 1717)])
@pytest.mark.parametrize("kv", [1, 2])
def test_infinite_values_of_small_weights(dtype, below, n, where, kv):
    """An infinite value whose key's score lies far below the others' is
    infinite in the output as long as fp32 has the weight."""
    g, d = gen(n + where), 64
    table, pages = deal(g, [n], 16, 200 if n > 1000 else None)
    keys, values = torch.zeros(pages, 16, kv, d), randn(g, pages, 16, kv, d)
    spot = table[0, where // 16].long(), where % 16
    keys[spot[0], spot[1], :, 0] = -float(below)
    values[spot[0], spot[1], :, 5], values[spot[0], spot[1], :, 9] = math.inf, -math.inf
    q = torch.zeros(1, 2, d)
    q[..., 0] = 1.0
    out, _ = attend(q.to(dtype), keys.to(dtype), values.to(dtype), table, [n], 1.0)
    assert torch.all(out[..., 5] == math.inf) and torch.all(out[..., 9] == -math.inf)
    rest = [i for i in range(d) if i not in (5, 9)]
    assert torch.all(out[..., rest].isfinite())

@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n", [1, 40, 3000])
@pytest.mark.parametrize("kv", [1, 2])
def test_scores_of_minus_infinity(dtype, n, kv):
    """Keys of score -inf weigh nothing; where there are no others the
    fraction is 0 / 0."""
    g, d = gen(n), 64
    table, pages = deal(g, [n, n + 1], 16, 200 if n > 1000 else None)
    keys, values = torch.zeros(pages, 16, kv, d), randn(g, pages, 16, kv, d)
    keys[..., 0] = -math.inf
    keys[table[1, 0].long(), 0, :, 0] = 1.0
    q = torch.zeros(2, 2, d)
    q[..., 0] = 1.0
    q, keys, values = q.to(dtype), keys.to(dtype), values.to(dtype)
    out, lse = attend(q, keys, values, table, [n, n + 1], 1.0)
    assert torch.all(out[0].isnan()) and torch.all(lse[0] == -math.inf)
    first = values[table[1, 0].long(), 0].expand(2, d) if kv == 1 else values[table[1, 0].long(), 0]
    assert torch.equal(out[1], first) and torch.all((lse[1] - 1.0).abs() <= 2.0 ** -21)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,window", [(1, 0), (33, 0), (65, 0), (65, 49), (3001, 0), (3009, 2993)])
@pytest.mark.parametrize("kv", [1, 2])
def test_keys_outside_add_nothing(dtype, n, window, kv):
    """The keys of a tile behind a sequence's end and before its window are not
    the nearest attended key again, not even a little: its value is 2^60, its
    weight 2^-110, every other value 0.  The weight's argument of 110 is off by
    2^-24 of itself for its product with the scale and 2^-24 for the scale, the
    weight by 2 ln 2 of that, 110 times 2^-22.5 in all."""
    g, d = gen(n), 64
    table, pages = deal(g, [n], 16, 200 if n > 1000 else None)
    keys, values = (torch.zeros(pages, 16, kv, d) for _ in range(2))
    last = (n - 1) if window == 0 else n - window   # next to the keys that do not count
    if n > 1:
        keys[table[0, last // 16].long(), last % 16, :, 0] = -110.0
    values[table[0, last // 16].long(), last % 16] = 2.0 ** 60
    q = torch.zeros(1, 2, d)
    q[..., 0] = 1.0
    q, keys, values = q.to(dtype), keys.to(dtype), values.to(dtype)
    ref, _, _, _ = bounds.attend(q, keys, values, table.clamp(min=0), [n], math.log(2.0), window)
    out, _ = attend(q, keys, values, table, [n], math.log(2.0), window)
    assert torch.all((out.double() / ref - 1).abs() <= 110 * 2.0 ** -22.5 + 2.0 ** -22 + bounds.HALF_STEP[dtype])


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n,window", [(1, 0), (33, 0), (65, 49), (3001, 2985)])
@pytest.mark.parametrize("kv", [1, 2])
def test_infinite_values_next_to_keys_outside(dtype, n, window, kv):
    """The first and last attended keys, infinite ones: infinite, not NaN."""
    g, d = gen(n), 64
    table, pages = deal(g, [n], 16, 200 if n > 1000 else None)
    keys, values = randn(g, pages, 16, kv, d), randn(g, pages, 16, kv, d)
    for at, sign in ((n - 1, 1.0), (max(0, n - window) if window else 0, 1.0)):
        values[table[0, at // 16].long(), at % 16, :, 7] = sign * math.inf
    out, _ = attend(randn(g, 1, 2, d).to(dtype), keys.to(dtype), values.to(dtype), table, [n], 0.125, window)
    assert torch.all(out[..., 7] == math.inf) and torch.all(out[..., :7].isfinite())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale", [0.0, -0.0, 2.0 ** -126])
@pytest.mark.parametrize("n", [5, 40, 3001])
@pytest.mark.parametrize("kv", [1, 2])
def test_tiny_scales_of_large_products(dtype, scale, n, kv):
    """Products of up to 2^126: with a scale of 0 every key weighs the same."""
    g, d = gen(n), 64
    table, pages = deal(g, [n], 16, 200 if n > 1000 else None)
    keys, values = torch.zeros(pages, 16, kv, d), randn(g, pages, 16, kv, d)
    keys[..., 0] = torch.randint(-1, 2, (pages, 16, kv), generator=g) * 2.0 ** 63
    q = torch.zeros(1, 2, d)
    q[..., 0] = 2.0 ** 63
    q, keys, values = q.to(dtype), keys.to(dtype), values.to(dtype)
    ref, ref_lse, room, lse_room = bounds.attend(q, keys, values, table.clamp(min=0), [n], scale)
    out, lse = attend(q, keys, values, table, [n], scale)
    assert bounds.within(out, ref, room) and torch.all((lse.double() - ref_lse).abs() <= lse_room)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("group", [1, 2])
def test_streamed_cache(dtype, cache, d, group):
    """A few sequences in a cache larger than the last-level cache under block
    tables with room for all of it: keys and values are read past the caches."""
    kv, slots, lens = 4, 16, [1, 50, 3000, 0, 700]
    size = torch.tensor([], dtype=cache).element_size()
    pages = 320_000_000 // (2 * slots * kv * d * size)
    g = gen(d + group)
    big = ops.alloc_kv_cache(pages, slots, kv, d, cache)
    near, count = deal(g, lens, slots)   # the same pages numbered from 0
    used = torch.randperm(pages, generator=g)[:count]
    keys, values = (x.to(cache) for x in cache_like(g, count, slots, kv, d, F32 if cache == E4M3 else cache, "slot"))
    for c, x in ((big["k"], keys), (big["v"], values)):
        if cache == E4M3:
            c.view(torch.uint8)[used.cuda()] = x.view(torch.uint8).cuda()
        else:
            c[used.cuda()] = x.cuda()
    table = torch.zeros(len(lens), pages, dtype=torch.int32)
    table[:, :near.shape[1]] = torch.where(near < 0, -1, used[near.clamp(min=0).long()]).to(torch.int32)
    q = (2 * randn(g, len(lens), kv * group, d)).to(dtype)
    out = torch.empty(q.shape, dtype=dtype, device="cuda")
    ops.dsim_paged_attention(q.cuda(), big, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), out)
    ref, _, room, _ = bounds.attend(q, keys, values, near.clamp(min=0), lens, d ** -0.5)
    assert bounds.within(out.cpu(), ref, room)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
@pytest.mark.parametrize("kv", [2, 4])
def test_scales_of_cut_contexts(dtype, scale, kv):
    g, d, lens = gen(kv), 64, [40, 2500, 0, 300]
    table, pages = deal(g, lens, 16, 200)
    keys, values = cache_like(g, pages, 16, kv, d, dtype)
    q = randn(g, len(lens), 4, d).to(dtype)
    ref, ref_lse, room, lse_room = bounds.attend(q, keys, values, table.clamp(min=0), lens, scale)
    out, lse = attend(q, keys, values, table, lens, scale)
    some = torch.tensor(lens) > 0
    assert bounds.within(out, ref, room) and torch.all((lse.double() - ref_lse)[some].abs() <= lse_room[some])


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n_seq", [3, 300])   # joined by context, by workgroup
def test_strided_rows_of_cut_contexts(dtype, n_seq):
    """q and out as parts of wider tensors, written by the join."""
    g, d, kv = gen(n_seq), 64, 2
    lens = [2500, 9, 1700] + [3] * (n_seq - 3)
    table, pages = deal(g, lens, 16, 200)
    keys, values = cache_like(g, pages, 16, kv, d, dtype)
    wide = randn(g, n_seq, 9, 96).to(dtype)
    q = wide[:, 1:5, 16:80]
    big = torch.zeros(n_seq, 8, 128, dtype=dtype, device="cuda")
    ops.dsim_paged_attention(wide.cuda()[:, 1:5, 16:80], dict(k=to_gpu(keys), v=to_gpu(values)), table.cuda(),
                             torch.tensor(lens, dtype=torch.int32, device="cuda"), big[:, 2:6, 32:96])
    ref, _, room, _ = bounds.attend(q, keys, values, table.clamp(min=0), lens, 0.125)
    assert bounds.within(big[:, 2:6, 32:96].cpu(), ref, room)
    big[:, 2:6, 32:96] = 0
    assert torch.all(big == 0)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("power", [10, 15, 40])
@pytest.mark.parametrize("n", [5, 100, 3000])
@pytest.mark.parametrize("kv", [1, 2])
def test_large_scores(dtype, power, n, kv):
    """Scores of up to 2^80: those at the maximum share the whole weight (the
    others lie 2^6 and more below it), however coarse the maximum itself is."""
    if dtype == F16 and power > 15:
        pytest.skip("beyond the type")
    g, d = gen(n + power), 64
    table, pages = deal(g, [n], 16, 200 if n > 1000 else None)
    keys, values = torch.zeros(pages, 16, kv, d), randn(g, pages, 16, kv, d)
    keys[..., 0] = torch.randint(-4, 5, (pages, 16, kv), generator=g) * 2.0 ** (power - 3)
    q = torch.zeros(1, 2, d)
    q[0, :, 0] = torch.tensor([1.0, -0.75]) * 2.0 ** power
    q, keys, values = q.to(dtype), keys.to(dtype), values.to(dtype)
    scale = 0.1
    ref, ref_lse, _, _ = bounds.attend(q, keys, values, table.clamp(min=0), [n], scale)
    out, lse = attend(q, keys, values, table, [n], scale)
    # a mean of n values at most: n roundings of sums of them and of the weights'
    assert bounds.within(out, ref, n * 2.0 ** -23 * values.double().abs().max())
    # the scaled maximum and the logarithm of the count, at most 12, rounded to
    # fp32, scaled by ln 2 and added: 2^-24 of each four times
    assert torch.all((lse.double() - ref_lse).abs() <= (ref_lse.abs() + 2 * 12) * 2.0 ** -22)


@pytest.mark.parametrize("dtype,cache", [(F32, F32), (BF16, BF16), (F16, E4M3)])
@pytest.mark.parametrize("slots,lens", [(16, [160, 3]), (16, [3200, 3199, 1]), (7, [70, 69]), (1000, [3000, 999, 1001]),
                                        (4096, [4096, 17])])
def test_contexts_that_fill_the_table(dtype, cache, slots, lens):
    """Lengths up to the table's last slot, windows as long as contexts, and a
    table that is a part of a wider one."""
    g, d, kv = gen(slots + len(lens)), 64, 2
    width = -(-lens[0] // slots)
    table, pages = deal(g, lens, slots, width)
    keys, values = (x.to(cache) for x in cache_like(g, pages, slots, kv, d, F32 if cache == E4M3 else cache))
    q = (2 * randn(g, len(lens), 4, d)).to(dtype)
    wide = torch.full((len(lens), width + 4), -9, dtype=torch.int32)
    wide[:, 1:width + 1] = table
    dev = dict(k=to_gpu(keys), v=to_gpu(values))
    for window in (0, lens[0], lens[0] - 1, 2 ** 31 - 1):
        out = torch.zeros(q.shape, dtype=dtype, device="cuda")
        status = torch.full((len(lens),), -7, dtype=torch.int32, device="cuda")
        ops.dsim_paged_attention(q.cuda(), dev, wide.cuda()[:, 1:width + 1],
                                 torch.tensor(lens, dtype=torch.int32, device="cuda"), out, window=window, status=status)
        ref, _, room, _ = bounds.attend(q, keys, values, table.clamp(min=0), lens, 0.125, window)
        assert bounds.within(out.cpu(), ref, room) and not status.any()


@pytest.mark.parametrize("heads,kv", [(1024, 1024), (1024, 4), (1000, 8)])
@pytest.mark.parametrize("width", WIDTHS)
def test_as_many_heads_as_are_taken(heads, kv, width):
    g, d, lens = gen(heads), 16, [33, 300]
    table, pages = deal(g, lens, 16, width)
    keys, values = cache_like(g, pages, 16, kv, d, BF16)
    q = (2 * randn(g, 2, heads, d)).bfloat16()
    ref, ref_lse, room, lse_room = bounds.attend(q, keys, values, table.clamp(min=0), lens, 0.25)
    out, lse = attend(q, keys, values, table, lens, 0.25)
    assert bounds.within(out, ref, room) and torch.all((lse.double() - ref_lse).abs() <= lse_room)


def test_more_sequences_than_threads():
    """Most of them left alone, some empty, a few long."""
    g, d, n = gen(5), 64, 3000
    lens = [-1] * n
    for i in range(0, n, 7):
        lens[i] = 0
    for i, x in ((0, 900), (13, 2500), (1499, 1), (1500, 3000), (2999, 77)):
        lens[i] = x
    table, pages = deal(g, lens, 16, 190)
    keys, values = cache_like(g, pages, 16, 2, d, BF16)
    q = (2 * randn(g, n, 4, d)).bfloat16()
    ref, ref_lse, room, lse_room = bounds.attend(q, keys, values, table.clamp(min=0), lens, 0.125)
    out, lse = attend(q, keys, values, table, lens, 0.125)
    lens = torch.tensor(lens)
    assert torch.all(out[lens < 0] == 9.0) and torch.all(lse[lens < 0] == 9.0)
    assert torch.all(out[lens == 0] == 0.0) and torch.all(lse[lens == 0] == -math.inf)
    some = lens > 0
    assert bounds.within(out[some], ref[some], room[some])
    assert torch.all((lse.double() - ref_lse)[some].abs() <= lse_room[some])
