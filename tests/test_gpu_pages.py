"""The append on several axes and the pages of a cache on the GPU against plain
implementations (tests/multi_ops_plain.py): equal words."""
import pytest
import torch

import multi_ops_plain as plain
import step_ops
from paper_2111_05426_amd import ops
from test_gpu_ops import cache_like, deal, gen, randn, to_gpu

pytestmark = pytest.mark.gpu

F32, F16, BF16, E4M3 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"


def ints(x):
    return torch.tensor(x, dtype=torch.int32)


# ---------------------------------------------------------------------------
# dsim_kv_append_axes
# ---------------------------------------------------------------------------
def check_axes(dtype, cache, heads, kv, d, slots, lens, sections, interleaved=False, scales=False, order="head",
               with_q=True, in_place=False, seed=0, edit=None):
    g = gen(seed)
    table, pages = deal(g, lens, slots)
    keys, values = cache_like(g, pages, slots, kv, d, F32 if cache == E4M3 else cache, order)
    if cache == E4M3:
        keys, values = keys.to(E4M3), values.to(E4M3)
    seq = torch.cat([torch.full((n,), i, dtype=torch.int32) for i, n in enumerate(lens)])
    slot = torch.cat([torch.arange(n, dtype=torch.int32) for n in lens])
    mix = torch.randperm(len(seq), generator=g)
    seq, slot = seq[mix].contiguous(), slot[mix].contiguous()
    pos = torch.randint(0, 50, (len(seq), len(sections)), generator=g, dtype=torch.int32)
    rope = ops.rope_table(50, 2 * sum(sections), device="cpu")
    qkv = (3 * randn(g, len(seq), heads + 2 * kv, d)).to(dtype)
    q, k, v = qkv.split([heads, kv, kv], dim=1)
    q_out = randn(g, len(seq), heads, d).to(dtype)
    ks, vs = ((0.01 + torch.rand(kv, generator=g)) if scales else None for _ in range(2))
    if edit:
        edit(locals())
    dev = dict(k=to_gpu(keys), v=to_gpu(values), k_scale=to_gpu(ks), v_scale=to_gpu(vs))
    dq = qkv.cuda().split([heads, kv, kv], dim=1)
    dq_out = None if not with_q else dq[0] if in_place else q_out.cuda()
    status = torch.full((len(seq),), -7, dtype=torch.int32, device="cuda")
    ops.dsim_kv_append_axes(dev, table.cuda(), dq[1], dq[2], seq.cuda(), slot.cuda(), pos.cuda(), rope.cuda(),
                            sections=sections, interleaved=interleaved, q=dq[0] if with_q else None, q_out=dq_out,
                            status=status)
    torch.cuda.synchronize()
    want = plain.append_axes(keys, values, table, k, v, seq, slot, pos, rope, sections, interleaved,
                             q if with_q else None, q if in_place else q_out, ks, vs)
    assert torch.equal(status.cpu(), want[3])
    if with_q:
        assert step_ops.same(dq_out.cpu(), want[2])
    for got, ref in ((dev["k"], want[0]), (dev["v"], want[1])):
        assert step_ops.same(got.cpu(), ref)
    return want[3]


@pytest.mark.parametrize("dtype,cache", [(F32, F32), (F16, F16), (BF16, BF16), (F16, E4M3), (BF16, E4M3)])
@pytest.mark.parametrize("heads,kv,d,sections,interleaved", [
    (12, 12, 64, [32], False), (8, 2, 128, [16, 24, 24], False), (8, 2, 128, [16, 24, 24], True), (4, 4, 64, [3, 5, 16], True),
    (4, 4, 64, [3, 5, 16], False), (5, 1, 80, [1, 0, 18, 1], False), (2, 2, 16, [1, 1, 1, 1], True),
    (2, 2, 16, [1, 1, 1, 1], False), (3, 3, 256, [0, 128], False), (7, 7, 96, [0, 0, 0, 48], True),
    (33, 3, 112, [27, 1], False), (5, 3, 16, [7, 1], False), (4, 2, 128, [2, 1, 60, 1], True),
    (4, 2, 128, [62, 1, 0, 1], False)])
def test_axes(dtype, cache, heads, kv, d, sections, interleaved):
    check_axes(dtype, cache, heads, kv, d, 16, [1, 5, 33, 16], sections, interleaved,
               scales=cache == E4M3 and heads % 2 == 0)


@pytest.mark.parametrize("order", ["head", "slot", "gaps"])
def test_axes_layouts(order):
    check_axes(BF16, BF16, 4, 2, 64, 7, [9, 1, 70], [8, 4, 20], order=order)
    check_axes(F16, F16, 6, 2, 64, 16, [20], [20, 12], with_q=False)
    check_axes(F16, F16, 6, 2, 64, 16, [20], [20, 12], in_place=True)
    check_axes(BF16, E4M3, 6, 2, 64, 16, [700, 800], [20, 12])


def test_axes_of_one_position_are_the_append():
    g = gen(2)
    n, d = 40, 128
    table, pages = deal(g, [n], 16)
    rope = ops.rope_table(n, d)
    k, v, q = (randn(g, n, h, d).bfloat16().cuda() for h in (2, 2, 6))
    seq, pos = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.arange(n, dtype=torch.int32, device="cuda")
    got = []
    for axes in (False, True):
        cache = {x: torch.zeros(pages, 16, 2, d, dtype=BF16, device="cuda") for x in "kv"}
        out = torch.empty_like(q)
        if axes:
            ops.dsim_kv_append_axes(cache, table.cuda(), k, v, seq, pos, pos[:, None].repeat(1, 3), rope,
                                    sections=[10, 50, 4], q=q, q_out=out)
        else:
            ops.dsim_kv_append(cache, table.cuda(), k, v, seq, pos, rope=rope, q=q, q_out=out)
        got.append((cache["k"], cache["v"], out))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    # without a rotation too
    cache = {x: torch.zeros(pages, 16, 2, d, dtype=BF16, device="cuda") for x in "kv"}
    ops.dsim_kv_append_axes(cache, table.cuda(), k, v, seq, pos, None, None)
    assert torch.equal(cache["k"][table[0, (pos // 16).long().cpu()].long().cuda(), (pos % 16).long()], k)


def test_axes_padding_and_errors():
    def edit(at):
        at["seq"][3], at["slot"][3] = -1, 10 ** 9
        at["seq"][5] = 2
        at["slot"][8] = -1
        at["slot"][9] = at["table"].shape[1] * 8
        at["pos"][10, 0] = 50
        at["pos"][11, 1] = -1
        at["pos"][12, 2] = 2 ** 31 - 1   # an axis of no pairs
        at["seq"][13], at["slot"][13] = 0, 24
        at["table"][0, 3] = -3
    status = check_axes(BF16, BF16, 4, 2, 64, 8, [40, 12], [20, 12, 0], edit=edit, order="slot")
    assert [int(status[i]) for i in (3, 5, 8, 9, 10, 11, 12, 13)] == [0, 512, 256, 256, 256, 256, 256, 128]


# ---------------------------------------------------------------------------
# The pool
# ---------------------------------------------------------------------------
class Both:
    """A pool, a table and layers on the GPU and in plain form."""

    def __init__(self, n_pages, rows, width, page, layers=2, heads=2, d=32, dtype=BF16, seed=0, order="slot"):
        g = gen(seed)
        self.page, self.plain = page, plain.Pool(n_pages, rows, width, page)
        self.pool = ops.alloc_page_pool(n_pages, rows)
        self.table = torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
        self.len = [0] * rows
        self.layers, self.ref = [], []
        for _ in range(layers):
            k, v = cache_like(g, n_pages, page, heads, d, F32 if dtype == E4M3 else dtype, order)
            k, v = k.to(dtype), v.to(dtype)
            self.layers.append(dict(k=to_gpu(k), v=to_gpu(v)))
            self.ref += [k.view(torch.uint8).clone() if dtype == E4M3 else k.clone(),
                         v.view(torch.uint8).clone() if dtype == E4M3 else v.clone()]
        self.d_len = torch.zeros(rows, dtype=torch.int32, device="cuda")

    def set_len(self, length):
        self.len = list(length)
        self.d_len.copy_(ints(length))

    def reserve(self, want):
        status = torch.full((len(want),), -7, dtype=torch.int32, device="cuda")
        ops.dsim_kv_reserve(self.pool, self.table, self.page, self.d_len, ints(want).cuda(), status)
        ref = [-7] * len(want)
        self.plain.reserve(self.len, want, ref)
        assert status.tolist() == ref
        return self.same(ref)

    def release(self, rows, keep):
        status = torch.full((len(rows),), -7, dtype=torch.int32, device="cuda")
        ops.dsim_kv_release(self.pool, self.table, self.page, ints(rows).cuda(), ints(keep).cuda(), status)
        self.plain.release(rows, keep)
        return self.same(status.tolist())

    def fork(self, src, dst):
        status = torch.full((len(src),), -7, dtype=torch.int32, device="cuda")
        ops.dsim_kv_fork(self.layers, self.pool, self.table, self.d_len, ints(src).cuda(), ints(dst).cuda(), status)
        ref = [-7] * len(src)
        self.plain.fork(self.len, src, dst, ref, self.ref)
        assert status.tolist() == ref
        return self.same(ref)

    def same(self, status):
        assert self.table.tolist() == self.plain.table
        assert self.pool["refs"].tolist() == self.plain.refs
        assert self.pool["held"].tolist() == self.plain.held
        assert [x % 2 ** 32 for x in self.pool["free"].tolist()] == self.plain.words()
        assert self.d_len.tolist() == self.len
        got = [x for layer in self.layers for x in (layer["k"], layer["v"])]
        for x, y in zip(got, self.ref):
            x = x.cpu()
            assert torch.equal(x.view(torch.uint8) if x.dtype == E4M3 else x, y)
        return status


def test_reserve():
    b = Both(70, 5, 20, 16)
    b.reserve([40, 0, -1, 16, 17])
    assert b.plain.table[0][:3] == [0, 1, 2] and b.plain.table[4][:2] == [4, 5]
    b.set_len([40, 0, 0, 16, 17])
    b.reserve([41, 5, 300, 17, 10])   # enough already, new, more, a page, fewer
    b.release([2, 0], [0, 17])
    b.set_len([17, 0, 0, 17, 10])
    b.reserve([100, 40, 64, 20, 20])   # the freed ones first, in order
    # 18 pages are held, 48 more leave four: not enough for the second row,
    # and so for nobody behind that needs some
    b.set_len([100, 40, 64, 20, 20])
    assert b.reserve([320, 41, 16 * 20, 20 * 16, 48]) == [0, 0, 0, 0, 0]
    b.set_len([320, 40, 320, 320, 20])
    assert b.reserve([320, 320, 320, 0, 64]) == [0, 1024, 0, 0, 1024]
    assert b.reserve([-1, 16 * 20 + 1, 0, 2 ** 31 - 1, -2 ** 31]) == [-7, 256, 0, 256, -7]
    b.set_len([100, 49, 400, -1, 20])
    assert b.reserve([100, 49, 64, 20, 20]) == [0, 256, 256, 256, 0]


@pytest.mark.parametrize("n_pages", [0, 1, 31, 32, 33, 1000, 40000])
def test_reserve_many(n_pages):
    """More pages than are dealt at once, more words than threads, more rows
    than threads."""
    g = gen(n_pages)
    rows = 1500 if n_pages == 40000 else 40
    b = Both(n_pages, rows, 100, 3, layers=1, heads=1, d=16)
    for _ in range(3):
        want = torch.randint(-3, 100, (rows,), generator=g).tolist()
        b.reserve(want)
        rows_ = torch.randint(-1, rows, (rows // 2,), generator=g).tolist()
        b.release(rows_, torch.randint(-2, 80, (rows // 2,), generator=g).tolist())


def test_release():
    b = Both(50, 6, 12, 4)
    b.reserve([17, 4, 48, 0, 3, 9])
    assert b.release([1, -1, 2, 2, 9, 5], [4, 0, 30, 5, 0, 100]) == [0, 0, 0, 0, 512, 0]
    b.release([0, 2, 5], [-5, 0, 0])
    # entries outside the cache or without a count are told of and left out
    b.reserve([20, 4, 20, 0, 3, 0])
    b.table[0, 1] = 50
    b.plain.table[0][1] = 50
    assert b.release([0], [0]) == [128]
    b.plain.refs[b.plain.table[2][2]] = 0
    b.pool["refs"].copy_(ints(b.plain.refs))
    free = b.plain.words()
    b.pool["free"].copy_(torch.tensor([x - 2 ** 32 if x >= 2 ** 31 else x for x in free], dtype=torch.int32))
    assert b.release([2], [0]) == [128]


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("order", ["head", "slot", "gaps"])
@pytest.mark.parametrize("page", [1, 5, 16])
def test_fork(dtype, order, page):
    b = Both(120, 8, 40, page, layers=3, heads=3, d=48, dtype=dtype, order=order)
    length = [37, 16, 0, 0, 0, 0, 33, 0]
    want = length[:]
    b.set_len([0] * 8)
    b.reserve(want)
    b.set_len(length)
    assert b.fork([0, 0, 1, 6], [2, 3, 4, 5]) == [0, 0, 0, 0]
    b.fork([2], [7])
    # a shared page is not written on; the last holder's own is
    b.set_len([max(n - 2, 0) for n in b.len])
    status = b.reserve([n + 3 if n else 0 for n in b.len])
    if page == 16:
        assert 2048 in status
    b.release([0, 2, 7], [0, 20, 0])
    b.release(list(range(8)), [0] * 8)
    assert b.plain.free() == list(range(120))


def test_fork_refusals():
    b = Both(12, 9, 6, 8)
    b.reserve([20, 8, 5, 0, 0, 0, 0, 0, 0])
    b.set_len([20, 8, 5, 0, 0, 0, 0, 0, 0])
    # out of the table; padding; in use; twice; a dst that is a src; nothing to copy; an empty one
    assert b.fork([0, 9, 0, 1, 0, 0, 3, 1, 5], [-1, 4, 9, 2, 3, 3, 6, 7, 8]) == [0, 512, 512, 4096, 0, 4096, 512, 0, 0]
    b.release([3, 7], [0, 0])
    b.set_len([20, 8, 60, 0, 0, 0, 0, 0, -1])
    assert b.fork([2, 8], [3, 4]) == [256, 256]
    b.set_len([20, 8, 5, 0, 0, 0, 0, 0, 0])
    # 7 pages are left: the rest is refused, whole pages need none
    assert b.fork([0, 2, 0, 2, 0], [3, 4, 5, 6, 7]) == [0] * 5
    b.release([3, 4, 5, 6, 7], [0] * 5)
    b.reserve([20, 40, 5, 0, 0, 0, 0, 0, 0])
    b.set_len([20, 40, 5, 0, 0, 0, 0, 0, 0])
    b.fork([0, 0, 0], [3, 4, 5])
    assert b.fork([2, 1, 0], [6, 7, 8]) == [1024, 0, 1024]
    b.table[1, 2] = 12
    b.plain.table[1][2] = 12
    b.release([7], [0])
    assert b.fork([1], [7]) == [128]
    # many entries for one row: the first has it
    assert b.fork([1] * 3000, [8] * 3000)[:2] == [128, 4096]


@pytest.mark.parametrize("order", ["head", "slot", "gaps"])
def test_copy_pages(order):
    for dtype, page, d in ((F32, 3, 32), (E4M3, 16, 16), (BF16, 300, 80)):
        b = Both(40, 1, 1, page, layers=70, heads=2, d=d, dtype=dtype, order=order)
        src, dst = [3, 4, 3, -1, 5, 40, 7, 9], [10, 11, 12, 13, -2, 14, 40, 9]
        ops.dsim_kv_copy_pages(b.layers, ints(src).cuda(), ints(dst).cuda())
        for x in b.ref:
            x[10], x[11], x[12] = x[3], x[4], x[3]
        b.same(None)


# ---------------------------------------------------------------------------
# dsim_kv_compact
# ---------------------------------------------------------------------------
def check_compact(start, keep, n_keep, total, slots=16, heads=2, d=64, dtype=BF16, order="head", layers=2, seed=0, edit=None):
    g = gen(seed)
    table, pages = deal(g, total, slots)
    raw = [x for _ in range(layers) for x in cache_like(g, pages, slots, heads, d, F32 if dtype == E4M3 else dtype, order)]
    raw = [x.to(dtype) for x in raw]
    dev = [dict(k=to_gpu(raw[2 * i]), v=to_gpu(raw[2 * i + 1])) for i in range(layers)]
    width = max([len(k) for k in keep] + [1])
    lists = ints([k + [0] * (width - len(k)) for k in keep])
    if edit:
        edit(locals())
    status = torch.full((len(start),), -7, dtype=torch.int32, device="cuda")
    ops.dsim_kv_compact(dev, table.cuda(), ints(start).cuda(), lists.cuda(), ints(n_keep).cuda(), status)
    ref = [(x.view(torch.uint8) if dtype == E4M3 else x).clone() for x in raw]
    want = plain.compact(ref, table, start, lists, n_keep)
    assert torch.equal(status.cpu(), want)
    for x, y in zip([t for layer in dev for t in (layer["k"], layer["v"])], ref):
        x = x.cpu()
        assert torch.equal(x.view(torch.uint8) if dtype == E4M3 else x, y)
    return want.tolist()


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("order", ["head", "slot", "gaps"])
@pytest.mark.parametrize("slots,d", [(1, 16), (5, 80), (16, 128), (64, 256)])
def test_compact(dtype, order, slots, d):
    g = gen(slots)
    total, start, keep = [300, 64, 17, 900, 1], [100, 0, 16, 0, 0], []
    for n, a in zip(total, start):
        room = n - a
        keep.append(torch.randperm(room, generator=g)[:(room + 1) // 2].sort().values.tolist())
    check_compact(start, keep, [len(k) for k in keep], total, slots, 3, d, dtype, order)


def test_compact_paths():
    """Accepted paths of drafts, some empty, and lists that nothing moves for."""
    assert check_compact([5, 20, 0, 7], [[0, 2, 5], [], [0, 1, 2], [3]], [3, 0, 3, 1], [16, 30, 9, 15], layers=70) == [0] * 4
    # n_keep beyond the width and below 0
    assert check_compact([5, 20], [[0, 2, 5], [1, 2, 3]], [9, -4], [16, 30]) == [0, 0]


def test_compact_errors():
    keep = [[1, 4, 4, 7], [0, 3, 2], [-1, 2], [2, 5, 10 ** 9], [1, 2], [3, 20, 40], [2 ** 31 - 1]]

    def edit(at):
        at["table"][5, 1] = at["pages"]
        at["table"][4, :] = -1
    got = check_compact([0, 5, 0, 0, -3, 0, 2 ** 31 - 1], keep, [4, 3, 2, 3, 2, 3, 1], [64] * 7, edit=edit)
    assert got == [256, 256, 256, 256, 256, 128, 256]


def test_beyond_32_bits():
    """Pages whose elements lie behind 2^31 of them: copied, forked, compacted."""
    heads, d, page = 8, 128, 16
    n = (1 << 31) // (heads * d * page) + 70
    cache = {x: torch.zeros(n, page, heads, d, dtype=BF16, device="cuda") for x in "kv"}
    cache["k"][n - 3].normal_()
    cache["v"][n - 3].normal_()
    ops.dsim_kv_copy_pages(cache, ints([n - 3]).cuda(), ints([n - 9]).cuda())
    assert torch.equal(cache["k"][n - 9], cache["k"][n - 3]) and torch.equal(cache["v"][n - 9], cache["v"][n - 3])
    table = ints([[n - 3, n - 9], [-1, -1]]).cuda()
    pool = ops.alloc_page_pool(n, 2)
    pool["refs"][:] = 1
    pool["free"].zero_()
    pool["refs"][n - 50] = 0
    pool["free"][(n - 50) // 32] = (1 << (n - 50) % 32) - (2 ** 32 if (n - 50) % 32 == 31 else 0)
    pool["held"][0] = 2
    length, status = ints([20, 0]).cuda(), ints([7]).cuda()
    ops.dsim_kv_fork(cache, pool, table, length, ints([0]).cuda(), ints([1]).cuda(), status)
    assert status.tolist() == [0] and table.tolist()[1] == [n - 3, n - 50] and length.tolist() == [20, 20]
    assert torch.equal(cache["k"][n - 50, :4], cache["k"][n - 9, :4]) and not cache["k"][n - 50, 4:].any()
    want = cache["v"][n - 3, 5].clone()
    ops.dsim_kv_compact(cache, table, ints([0, 0]).cuda(), ints([[5], [0]]).cuda(), ints([1, 0]).cuda())
    assert torch.equal(cache["v"][n - 3, 0], want)
