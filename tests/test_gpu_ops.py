"""The single-token step's operators on the GPU against plain
implementations (tests/step_ops.py): types, head layouts, lengths from none
to thousands, page sizes that end inside a tile, strides, masks, errors in
device data, other streams and captured graphs."""
import math

import pytest
import torch

import step_ops as plain
from paper_2111_05426_amd import ops

pytestmark = pytest.mark.gpu

F32, F16, BF16, E4M3 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape):
    return torch.randn(*shape, generator=g)


def deal(g, lens, slots, width=None, spare=2):
    """A block table that deals pages out in random order."""
    counts = [-(-max(n, 0) // slots) for n in lens]
    order = torch.randperm(sum(counts) + spare, generator=g).to(torch.int32)
    table = torch.full((len(lens), width or max(counts + [1]) + 1), -1, dtype=torch.int32)
    at = 0
    for b, c in enumerate(counts):
        table[b, :c] = order[at:at + c]
        at += c
    return table, len(order)


def cache_like(g, pages, slots, heads, d, dtype, order="head"):
    """Keys and values (pages, slots, heads, d): a head's slots of a page
    together ("head"), a slot's heads together ("slot"), or as the two parts
    of one tensor with gaps between rows ("gaps")."""
    if order == "gaps":
        both = randn(g, pages, slots, 2, heads, d + 16).to(dtype)
        return both[:, :, 0, :, :d], both[:, :, 1, :, :d]
    shape = (pages, heads, slots, d) if order == "head" else (pages, slots, heads, d)
    k, v = randn(g, *shape).to(dtype), randn(g, *shape).to(dtype)
    return (k.transpose(1, 2), v.transpose(1, 2)) if order == "head" else (k, v)


def to_gpu(t):
    """The same values, strides and gaps on the GPU."""
    if t is None:
        return None
    span = sum((n - 1) * s for n, s in zip(t.shape, t.stride())) + 1 if t.numel() else 0
    base = torch.as_strided(t, (span,), (1,), t.storage_offset()).cuda()
    return torch.as_strided(base, t.shape, t.stride())


# ---------------------------------------------------------------------------
# dsim_kv_append
# ---------------------------------------------------------------------------
def check_append(dtype, cache, heads, kv, d, slots, lens, past=0, rot=0, interleaved=False, scales=False, order="head",
                 with_q=True, in_place=False, seed=0, edit=None):
    g = gen(seed)
    table, pages = deal(g, [past + n for n in lens], slots)
    keys, values = cache_like(g, pages, slots, kv, d, F32 if cache == E4M3 else cache, order)
    if cache == E4M3:
        keys, values = keys.to(E4M3), values.to(E4M3)
    seq = torch.cat([torch.full((n,), i, dtype=torch.int32) for i, n in enumerate(lens)])
    pos = torch.cat([past + torch.arange(n, dtype=torch.int32) for n in lens])
    mix = torch.randperm(len(seq), generator=g)   # tokens in any order
    seq, pos = seq[mix].contiguous(), pos[mix].contiguous()
    qkv = (3 * randn(g, len(seq), heads + 2 * kv, d)).to(dtype)
    q, k, v = qkv.split([heads, kv, kv], dim=1)
    q_out = randn(g, len(seq), heads, d).to(dtype)
    rope = ops.rope_table(past + max(lens) + 3, rot, device="cpu") if rot else None
    ks, vs = ((0.01 + torch.rand(kv, generator=g)) if scales else None for _ in range(2))
    if edit:
        edit(locals())
    dev = dict(k=to_gpu(keys), v=to_gpu(values), k_scale=to_gpu(ks), v_scale=to_gpu(vs))
    dq = qkv.cuda().split([heads, kv, kv], dim=1)
    dq_out = None if not with_q else dq[0] if in_place else q_out.cuda()
    status = torch.full((len(seq),), -7, dtype=torch.int32, device="cuda")
    ops.dsim_kv_append(dev, table.cuda(), dq[1], dq[2], seq.cuda(), pos.cuda(), rope=to_gpu(rope),
                       interleaved=interleaved, q=dq[0] if with_q else None, q_out=dq_out, status=status)
    torch.cuda.synchronize()
    want = plain.append(keys, values, table, k, v, seq, pos, rope, interleaved, q if with_q else None,
                        q if in_place else q_out, ks, vs)
    assert torch.equal(status.cpu(), want[3])
    if with_q:
        assert plain.same(dq_out.cpu(), want[2])
    for got, ref in ((dev["k"], want[0]), (dev["v"], want[1])):
        assert plain.same(got.cpu(), ref)
    return want[3]


@pytest.mark.parametrize("dtype,cache", [(F32, F32), (F16, F16), (BF16, BF16), (F16, E4M3), (BF16, E4M3)])
@pytest.mark.parametrize("heads,kv,d,rot,interleaved", [
    (12, 12, 64, 64, False), (8, 2, 128, 128, False), (4, 4, 64, 48, True), (5, 1, 80, 40, False), (2, 2, 16, 8, True),
    (3, 3, 256, 0, False), (7, 7, 96, 96, True), (33, 3, 112, 56, False), (5, 3, 16, 16, False), (4, 2, 16, 16, True),
    (300, 100, 32, 32, False)])
def test_append(dtype, cache, heads, kv, d, rot, interleaved):
    check_append(dtype, cache, heads, kv, d, 16, [1, 5, 33, 16], rot=rot, interleaved=interleaved,
                 scales=cache == E4M3 and heads % 2 == 0)


@pytest.mark.parametrize("order", ["head", "slot", "gaps"])
@pytest.mark.parametrize("slots,past", [(1, 0), (7, 3), (64, 100)])
def test_append_layouts(order, slots, past):
    check_append(BF16, BF16, 4, 2, 64, slots, [9, 1, 70], past=past, rot=64, order=order)


def test_append_without_queries_and_in_place():
    check_append(F16, F16, 2, 2, 64, 16, [20], rot=64, with_q=False)
    check_append(F16, F16, 6, 2, 64, 16, [20], rot=64, in_place=True)
    check_append(F16, F16, 6, 2, 64, 16, [20], rot=32, interleaved=True, in_place=True)


def test_append_many_tokens():
    check_append(F16, F16, 1, 1, 16, 16, [3000, 1, 2000], rot=16)


@pytest.mark.parametrize("dtype,cache", [(F32, F32), (BF16, BF16), (F16, E4M3)])
@pytest.mark.parametrize("heads,kv,d,rot,interleaved", [(12, 12, 64, 48, True), (12, 2, 64, 64, False), (32, 8, 128, 128, False)])
def test_append_prompts(dtype, cache, heads, kv, d, rot, interleaved):
    """A wave a token and two."""
    check_append(dtype, cache, heads, kv, d, 32, [700, 1, 500], rot=rot, interleaved=interleaved, scales=cache == E4M3)


def test_append_more_tokens_than_workgroups():
    n = (1 << 20) + 5
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(n, 1, 16, device="cuda", generator=g).half() for _ in range(2))
    cache = ops.alloc_kv_cache(-(-n // 64) + 1, 64, 1, 16, F16)
    table = torch.randperm(-(-n // 64) + 1, device="cuda", generator=g).to(torch.int32)[None]
    pos = torch.arange(n, device="cuda", dtype=torch.int32)
    ops.dsim_kv_append(cache, table, k, v, torch.zeros_like(pos), pos)
    at = table[0, pos.long() // 64].long(), pos.long() % 64
    assert torch.equal(cache["k"][at], k) and torch.equal(cache["v"][at], v)


def test_append_two_tokens_of_one_place():
    """Not a call to make: each element is one of theirs, and nothing else
    changes."""
    g = gen(3)
    cache = {n: torch.zeros(2, 16, 2, 64, dtype=F16, device="cuda") for n in ("k", "v")}
    k, v = (randn(g, 3, 2, 64).half() for _ in range(2))
    one = torch.tensor([0, 0, 0], dtype=torch.int32, device="cuda")
    ops.dsim_kv_append(cache, torch.tensor([[1]], dtype=torch.int32, device="cuda"), k.cuda(), v.cuda(), one,
                       torch.tensor([4, 4, 9], dtype=torch.int32, device="cuda"))
    for c, x in ((cache["k"].cpu(), k), (cache["v"].cpu(), v)):
        assert torch.all((c[1, 4] == x[0]) | (c[1, 4] == x[1])) and torch.equal(c[1, 9], x[2])
        c[1, 4], c[1, 9] = 0, 0
        assert not c.any()


def test_cache_beyond_32_bits():
    """Pages whose elements lie behind 2^31 of them: appended, then attended to."""
    heads, d, slots = 8, 128, 16
    pages = (1 << 31) // (heads * d * slots) + 70
    cache = ops.alloc_kv_cache(pages, slots, heads, d, BF16)
    table = torch.tensor([[pages - 1, 3, pages - 2, pages - 60]], dtype=torch.int32)
    n = 60
    g = gen(7)
    k, v, q = randn(g, n, heads, d).bfloat16(), randn(g, n, heads, d).bfloat16(), randn(g, 1, 16, d).bfloat16()
    pos = torch.arange(n, dtype=torch.int32)
    ops.dsim_kv_append(cache, table.cuda(), k.cuda(), v.cuda(), torch.zeros_like(pos).cuda(), pos.cuda())
    for c, x in ((cache["k"], k), (cache["v"], v)):
        assert torch.equal(c[table[0, pos.long() // slots].long().cuda(), (pos.long() % slots).cuda()].cpu(), x)
    out = torch.empty(1, 16, d, dtype=BF16, device="cuda")
    ops.dsim_paged_attention(q.cuda(), cache, table.cuda(), torch.tensor([n], dtype=torch.int32, device="cuda"), out)
    near = torch.arange(4, dtype=torch.int32)[None]
    pad = lambda x: torch.cat([x, x[:4]]).view(4, slots, heads, d)   # noqa: E731
    ref, _, bound = plain.attend(q, pad(k), pad(v), near, torch.tensor([n]), d ** -0.5)
    assert torch.all((out.cpu().double() - ref).abs() <= bound + (ref.abs() + bound) * 2.0 ** -8)


def test_append_special_values():
    """Infinities, NaN, the largest and smallest numbers, in 16 bits and into
    an 8-bit cache (where what lies beyond its range becomes its largest)."""
    special = torch.tensor([math.inf, -math.inf, math.nan, 65504.0, -65504.0, 1e-7, 0.0, -0.0, 448.0, 464.0, 479.0,
                            2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9, 17.0, 19.0])

    def edit(at):
        for x in (at["k"], at["v"], at["q"]):
            x[:, :, :16] = special.to(x.dtype)
    for dtype, cache in ((F16, F16), (F32, F32), (BF16, BF16), (F16, E4M3)):
        check_append(dtype, cache, 2, 2, 64, 16, [9], rot=0, edit=edit)
        check_append(dtype, cache, 2, 2, 64, 16, [9], rot=16, edit=edit)


def test_append_padding_and_errors():
    """Padding leaves everything as it was; a sequence, position or page that
    does not exist is flagged, and its token writes nothing but NaN queries."""
    def edit(at):
        at["seq"][3] = -1
        at["pos"][3] = 10 ** 9
        at["seq"][5] = 2
        at["seq"][6] = 2 ** 31 - 1
        at["pos"][8] = -1
        at["pos"][9] = at["table"].shape[1] * 8
        at["pos"][10] = 2 ** 31 - 1
        at["seq"][11], at["pos"][11] = 0, 39
        at["table"][0, 4] = at["pages"]
        at["seq"][12], at["pos"][12] = 0, 24
        at["table"][0, 3] = -3
    status = check_append(BF16, BF16, 4, 2, 64, 8, [40, 12], rot=64, edit=edit, order="slot")
    assert [int(status[i]) for i in (3, 5, 6, 8, 9, 10, 11, 12)] == [0, 512, 512, 256, 256, 256, 128, 128]

    def beyond(at):   # positions behind the rotation table's end
        at["pos"][4] = at["rope"].shape[0]
    check_append(F16, F16, 2, 2, 64, 64, [20], rot=32, edit=beyond)


def test_append_nothing():
    cache = ops.alloc_kv_cache(2, 16, 2, 64, F16)
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    rows = torch.zeros(0, 2, 64, dtype=F16, device="cuda")
    ops.dsim_kv_append(cache, table, rows, rows, none, none)
    empty = ops.alloc_kv_cache(0, 16, 2, 64, F16)   # no page: every token flagged
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    rows = torch.ones(1, 2, 64, dtype=F16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ops.dsim_kv_append(empty, table, rows, rows, one, one, status=status)
    assert int(status) == ops.ST_BAD_PAGE


# ---------------------------------------------------------------------------
# dsim_paged_attention
# ---------------------------------------------------------------------------
def check_attend(dtype, cache, heads, kv, d, slots, lens, window=0, scales=False, order="head", scale=None, seed=0,
                 edit=None, spread=2.0, width=None):
    g = gen(seed)
    table, pages = deal(g, lens, slots, width)
    keys, values = cache_like(g, pages, slots, kv, d, F32 if cache == E4M3 else cache, order)
    if cache == E4M3:
        keys, values = keys.to(E4M3), values.to(E4M3)
    q = (spread * randn(g, len(lens), heads, d)).to(dtype)
    ks, vs = ((0.25 + torch.rand(kv, generator=g)) if scales else None for _ in range(2))
    seq_len = torch.tensor(lens, dtype=torch.int32)
    ref_keys, ref_values = keys.clone(), values.clone()
    if edit:   # what lies outside the attended keys
        edit(locals())
    out = torch.full((len(lens), heads, d), 123.0, dtype=dtype, device="cuda")
    lse = torch.full((len(lens), heads), 123.0, device="cuda")
    status = torch.full((len(lens),), -7, dtype=torch.int32, device="cuda")
    ws = ops.alloc_paged_attention_workspace(heads, kv, d)
    ws.fill_(255)   # NaN: nothing may depend on what it holds
    ops.dsim_paged_attention(q.cuda(), dict(k=to_gpu(keys), v=to_gpu(values), k_scale=to_gpu(ks), v_scale=to_gpu(vs)),
                             table.cuda(), seq_len.cuda(), out, scale=scale, window=window, workspace=ws, lse=lse,
                             status=status)
    torch.cuda.synchronize()
    used = d ** -0.5 if scale is None else scale
    ref, ref_lse, bound = plain.attend(q, ref_keys, ref_values, table.clamp(min=0), seq_len.clamp(min=0), used, window,
                                       ks, vs)
    out, lse, status = out.cpu().double(), lse.cpu().double(), status.cpu()
    for b, n in enumerate(lens):
        if n < 0:
            assert torch.all(out[b] == 123.0) and torch.all(lse[b] == 123.0) and int(status[b]) == -7
            continue
        assert int(status[b]) == 0
        # the type's half step relative to the value (below fp16's normal numbers: 2^-25)
        room = bound[b] + (ref[b].abs() + bound[b]) * plain.HALF_STEP[dtype] + (2.0 ** -25 if dtype == F16 else 0)
        assert torch.all((out[b] - ref[b]).abs() <= room), (b, n, float(((out[b] - ref[b]).abs() - room).max()))
        if n == 0:
            assert torch.all(lse[b] == -math.inf) and torch.all(out[b] == 0)
        else:   # off by a score's error and the sum's, and the result's own rounding
            off = 4 * (d + 2) * 2.0 ** -24 * abs(used) * 10 * spread * d + n * 2.0 ** -23 + 1e-5
            assert torch.all((lse[b] - ref_lse[b]).abs() <= off + ref_lse[b].abs() * 2.0 ** -21), (b, n)
    return out, status


TYPES = [(F32, F32), (F16, F16), (BF16, BF16), (F16, E4M3), (BF16, E4M3)]


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("heads,kv,d", [(12, 12, 64), (8, 2, 128), (16, 1, 96), (5, 5, 80), (2, 1, 256), (3, 3, 16),
                                        (4, 4, 112), (40, 2, 64), (6, 2, 208), (64, 1, 48), (17, 1, 144)])
def test_attend(dtype, cache, heads, kv, d):
    lens = [1, 16, 17, 100, 0, 33, 250]
    check_attend(dtype, cache, heads, kv, d, 16, lens, scales=cache == E4M3 and heads > 4)
    check_attend(dtype, cache, heads, kv, d, 16, lens, scales=cache == E4M3 and heads > 4, width=200)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("slots", [1, 3, 16, 48, 64, 256])
def test_attend_page_sizes(dtype, cache, slots):
    check_attend(dtype, cache, 4, 2, 64, slots, [1, 31, 32, 65, 129, 300], seed=slots)
    check_attend(dtype, cache, 4, 2, 64, slots, [1, 31, 32, 65, 129, 300], seed=slots, width=2000 // slots + 1)


@pytest.mark.parametrize("order", ["head", "slot", "gaps"])
@pytest.mark.parametrize("cache", [BF16, E4M3])
def test_attend_layouts(order, cache):
    check_attend(BF16, cache, 8, 2, 128, 16, [77, 5, 200], order=order)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("window", [1, 15, 16, 40, 1000])
def test_attend_window(dtype, window):
    """The keys before the window may be anywhere: their pages are not read."""
    def edit(at):
        for b, n in enumerate(at["lens"]):
            at["table"][b, :max(0, n - window) // 16] = -1
    check_attend(dtype, dtype, 4, 2, 64, 16, [1, 14, 41, 64, 500, 0], window=window, edit=edit)
    check_attend(dtype, dtype, 4, 2, 64, 16, [1, 14, 41, 64, 500, 0], window=window, edit=edit, width=90)


@pytest.mark.parametrize("dtype,cache", TYPES)
def test_attend_long(dtype, cache):
    """Contexts that the work's cuts go through, among short ones and empty rows."""
    lens = [5000, 3, 0, 9001, -1, 700, 1]
    check_attend(dtype, cache, 4, 2, 64, 16, lens, seed=3)
    check_attend(dtype, cache, 4, 1, 128, 32, lens, seed=4, window=4000)
    check_attend(dtype, cache, 2, 2, 256, 16, lens, seed=5)
    check_attend(dtype, cache, 20, 1, 80, 48, lens, seed=6)
    check_attend(dtype, cache, 2, 1, 64, 5, lens, seed=7)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("width", [None, 600])   # a workgroup per context; cut contexts
def test_attend_in_place(dtype, cache, width):
    lens = [5, 0, 300, -1, 77] + ([] if width is None else [9000, 2000])
    g = gen(8)
    table, pages = deal(g, lens, 16, width)
    keys, values = cache_like(g, pages, 16, 2, 64, F32 if cache == E4M3 else cache, "head")
    dev = dict(k=to_gpu(keys.to(cache)), v=to_gpu(values.to(cache)))
    q = randn(g, len(lens), 34, 64).to(dtype).cuda()
    seq_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ws = ops.alloc_paged_attention_workspace(34, 2, 64)
    out = q.clone()
    ops.dsim_paged_attention(q, dev, table.cuda(), seq_len, out, workspace=ws)
    ops.dsim_paged_attention(q, dev, table.cuda(), seq_len, q, workspace=ws)
    assert plain.same(q.cpu(), out.cpu()) and torch.all(out[1] == 0)


def test_attend_many_sequences():
    g = gen(5)
    lens = torch.randint(-1, 60, (700,), generator=g).tolist()
    check_attend(BF16, BF16, 2, 1, 64, 16, lens)
    check_attend(BF16, BF16, 2, 1, 64, 16, lens, width=100)


def test_attend_many_contexts_and_cuts():
    """More contexts than runs, some of them cut."""
    g = gen(6)
    lens = torch.randint(1, 400, (90,), generator=g).tolist() + [7000, 2500]
    check_attend(BF16, BF16, 8, 8, 64, 16, lens)
    check_attend(BF16, E4M3, 36, 9, 64, 16, lens, window=3000)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("slots", [16, 7])
def test_attend_large_cache(dtype, cache, slots):
    """A few sequences in a cache that is larger than the last-level cache,
    with block tables that have room for much of it (keys and values are then
    read past the caches)."""
    heads, d, lens = 4, 128, [1, 50, 3000, 0, 700]
    e = torch.tensor([], dtype=cache).element_size()
    pages = 320_000_000 // (2 * slots * heads * d * e)
    g = gen(slots)
    big = ops.alloc_kv_cache(pages, slots, heads, d, cache)
    counts = [-(-n // slots) for n in lens]
    used = torch.randperm(pages, generator=g)[:sum(counts)]
    table = torch.zeros(len(lens), pages, dtype=torch.int32)
    near = torch.zeros(len(lens), max(counts), dtype=torch.int32)   # the same pages numbered from 0
    at = 0
    for b, c in enumerate(counts):
        table[b, :c] = used[at:at + c].to(torch.int32)
        near[b, :c] = torch.arange(at, at + c)
        at += c
    keys, values = cache_like(g, len(used), slots, heads, d, F32 if cache == E4M3 else cache, "slot")
    keys, values = keys.to(cache), values.to(cache)
    for c, x in ((big["k"], keys), (big["v"], values)):
        if cache == E4M3:
            c.view(torch.uint8)[used.cuda()] = x.view(torch.uint8).cuda()
        else:
            c[used.cuda()] = x.cuda()
    q = (2 * randn(g, len(lens), 8, d)).to(dtype)
    out = torch.empty(q.shape, dtype=dtype, device="cuda")
    ops.dsim_paged_attention(q.cuda(), big, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), out)
    ref, _, bound = plain.attend(q, keys, values, near, torch.tensor(lens), d ** -0.5)
    room = bound + (ref.abs() + bound) * plain.HALF_STEP[dtype] + (2.0 ** -25 if dtype == F16 else 0)
    assert torch.all((out.cpu().double() - ref).abs() <= room)


def test_attend_shared_pages():
    """Sequences that share their first pages."""
    g = gen(12)
    table, pages = deal(g, [100, 130], 16)
    table[1, :5] = table[0, :5]
    keys, values = cache_like(g, pages, 16, 2, 64, F16)
    q, lens = randn(g, 2, 4, 64).half(), torch.tensor([100, 130], dtype=torch.int32)
    out = torch.empty(2, 4, 64, dtype=F16, device="cuda")
    ops.dsim_paged_attention(q.cuda(), dict(k=to_gpu(keys), v=to_gpu(values)), table.cuda(), lens.cuda(), out)
    ref, _, bound = plain.attend(q, keys, values, table.clamp(min=0), lens, 0.125)
    assert torch.all((out.cpu().double() - ref).abs() <= bound + (ref.abs() + bound) * 2.0 ** -11 + 2.0 ** -25)


def test_attend_one_context():
    check_attend(F16, F16, 16, 1, 128, 64, [20011], seed=9)


@pytest.mark.parametrize("dtype,cache", TYPES)
def test_attend_garbage_behind_the_end(dtype, cache):
    """NaN and infinities behind a sequence's end, in its last page and in
    unused pages, and page numbers that do not exist behind its last page."""
    def edit(at):
        keys, values, table, lens = (at[n] for n in ("keys", "values", "table", "lens"))
        free = torch.ones(keys.shape[:2], dtype=torch.bool)
        for b, n in enumerate(lens):
            for j in range(n):
                free[table[b, j // 16], j % 16] = False
            table[b, -(-n // 16):] = 10 ** 6 if b % 2 else -5
        spots = free.nonzero()
        for i, (pg, sl) in enumerate(spots.tolist()):
            for x, value in ((keys, (math.nan, math.inf)[i % 2]), (values, (math.nan, -math.inf, math.inf)[i % 3])):
                if x.dtype == E4M3:
                    x.view(torch.uint8)[pg, sl] = 0x7f
                else:
                    x[pg, sl] = value
    check_attend(dtype, cache, 4, 2, 64, 16, [1, 17, 31, 100, 250, 0], edit=edit)
    check_attend(dtype, cache, 4, 2, 64, 16, [1, 17, 31, 100, 250, 0], edit=edit, window=20)
    check_attend(dtype, cache, 4, 2, 64, 16, [1, 17, 31, 100, 250, 0], edit=edit, width=200)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_attend_scales(dtype):
    """A scale of none, a negative one and one that makes a single key count."""
    for scale in (0.0, -0.2, 3.0):
        check_attend(dtype, dtype, 4, 4, 64, 16, [40, 300], scale=scale)


def test_attend_long_tail_of_small_weights():
    """One key far above the others, whose weights are small each and together
    as large as it: none may be lost."""
    n, d = 8192, 64
    g = gen(11)
    for dtype in (F16, BF16, F32):
        q = torch.zeros(1, 1, d)
        q[..., 0] = 1.0
        keys = torch.zeros(n // 16, 16, 1, d)
        keys[100, 3, 0, 0] = math.log(2.0) * 18
        values = torch.ones(n // 16, 16, 1, d) + 0.25 * randn(g, n // 16, 16, 1, d)
        values[100, 3] = -1.0
        q, keys, values = q.to(dtype), keys.to(dtype), values.to(dtype)
        table = torch.arange(n // 16, dtype=torch.int32)[None]
        out = torch.empty_like(q, device="cuda")
        ops.dsim_paged_attention(q.cuda(), dict(k=keys.cuda(), v=values.cuda()), table.cuda(),
                                 torch.tensor([n], dtype=torch.int32, device="cuda"), out, scale=1.0)
        ref, _, bound = plain.attend(q, keys, values, table, torch.tensor([n]), 1.0)
        room = bound + (ref.abs() + bound) * plain.HALF_STEP[dtype]
        assert torch.all((out.cpu().double() - ref).abs() <= room)


def test_attend_not_a_number():
    """NaN and infinities among the attended keys and values reach the output
    as in the formula, whichever tile they lie in."""
    for n, where in ((200, 0), (200, 70), (200, 199), (6000, 3333)):
        for what in ("nan key", "inf value", "nan value", "all nan"):
            g = gen(n + where)
            table, pages = deal(g, [n], 16)
            keys, values = cache_like(g, pages, 16, 1, 64, F32)
            spot = (table[0, where // 16].long(), where % 16, 0)
            if what == "nan key":
                keys[spot][5] = math.nan
            elif what == "all nan":
                for j in range(where // 32 * 32, min(n, where // 32 * 32 + 32)):
                    keys[table[0, j // 16].long(), j % 16, 0] = math.nan
            else:
                values[spot][5] = math.inf if what == "inf value" else math.nan
            q = randn(g, 1, 2, 64)
            for dtype in (F32, BF16):
                out = torch.empty(1, 2, 64, dtype=dtype, device="cuda")
                ops.dsim_paged_attention(q.to(dtype).cuda(), dict(k=keys.to(dtype).cuda(), v=values.to(dtype).cuda()),
                                         table.cuda(), torch.tensor([n], dtype=torch.int32, device="cuda"), out)
                out = out.cpu()
                if what in ("nan key", "all nan"):
                    assert torch.all(out.isnan())
                elif what == "inf value":
                    assert torch.all(out[..., 5] == math.inf) and torch.all(out[..., :5].isfinite())
                else:
                    assert torch.all(out[..., 5].isnan()) and torch.all(out[..., :5].isfinite())


@pytest.mark.parametrize("longest", [9000, 600])
def test_attend_errors_in_device_data(longest):
    """A length beyond the block table and a page outside the cache are
    flagged, give NaN, and leave the other sequences right."""
    g = gen(2)
    lens = [50, 400, longest, 33, 10]
    table, pages = deal(g, lens, 16)
    keys, values = cache_like(g, pages, 16, 2, 64, F16)
    q = randn(g, 5, 4, 64).half()
    ref, _, bound = plain.attend(q, keys, values, table.clamp(min=0), torch.tensor(lens), 0.125)
    seq_len = torch.tensor(lens, dtype=torch.int32)
    seq_len[0] = table.shape[1] * 16 + 1
    table[1, 3] = pages
    table[2, longest // 16 - 10] = -1
    out = torch.zeros(5, 4, 64, dtype=F16, device="cuda")
    lse, status = torch.zeros(5, 4, device="cuda"), torch.full((5,), -7, dtype=torch.int32, device="cuda")
    ops.dsim_paged_attention(q.cuda(), dict(k=to_gpu(keys), v=to_gpu(values)), table.cuda(), seq_len.cuda(), out,
                             lse=lse, status=status)
    assert status.tolist() == [ops.ST_BAD_POSITION, ops.ST_BAD_PAGE, ops.ST_BAD_PAGE, 0, 0]
    out, lse = out.cpu(), lse.cpu()
    assert torch.all(out[:3].isnan()) and torch.all(lse[:3].isnan())
    room = bound[3:] + (ref[3:].abs() + bound[3:]) * 2.0 ** -11 + 2.0 ** -25
    assert torch.all((out[3:].double() - ref[3:]).abs() <= room)


def test_attend_no_pages():
    cache = ops.alloc_kv_cache(0, 16, 2, 64, F16)
    q = torch.ones(2, 2, 64, dtype=F16, device="cuda")
    out, status = torch.ones_like(q), torch.zeros(2, dtype=torch.int32, device="cuda")
    ops.dsim_paged_attention(q, cache, torch.zeros(2, 3, dtype=torch.int32, device="cuda"),
                             torch.tensor([0, 5], dtype=torch.int32, device="cuda"), out, status=status)
    assert torch.all(out[0] == 0) and torch.all(out[1].isnan()) and status.tolist() == [0, ops.ST_BAD_PAGE]
    ops.dsim_paged_attention(q[:0], cache, torch.zeros(0, 3, dtype=torch.int32, device="cuda"),
                             torch.zeros(0, dtype=torch.int32, device="cuda"), out[:0])


def test_attend_expanded_cache():
    """Cache heads that are one head's rows, read again (a stride of 0)."""
    g = gen(14)
    table, pages = deal(g, [70, 9], 16)
    keys, values = cache_like(g, pages, 16, 1, 64, BF16)
    q, lens = randn(g, 2, 8, 64).bfloat16(), torch.tensor([70, 9], dtype=torch.int32)
    cache = dict(k=to_gpu(keys).expand(-1, -1, 4, -1), v=to_gpu(values).expand(-1, -1, 4, -1))
    out = torch.empty(2, 8, 64, dtype=BF16, device="cuda")
    ops.dsim_paged_attention(q.cuda(), cache, table.cuda(), lens.cuda(), out)
    ref, _, bound = plain.attend(q, keys.expand(-1, -1, 4, -1), values.expand(-1, -1, 4, -1), table.clamp(min=0), lens,
                                 0.125)
    assert torch.all((out.cpu().double() - ref).abs() <= bound + (ref.abs() + bound) * 2.0 ** -8)
    rows = torch.zeros(1, 4, 64, dtype=BF16, device="cuda")
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    with pytest.raises(ops.DsimError):   # but not written
        ops.dsim_kv_append(cache, table.cuda(), rows, rows, one, one)


def test_attend_strided_rows():
    """q and out as parts of wider tensors."""
    g = gen(4)
    table, pages = deal(g, [60, 9], 16)
    keys, values = cache_like(g, pages, 16, 2, 64, BF16)
    wide = randn(g, 2, 9, 80).bfloat16()
    q = wide[:, 1:5, 16:]
    big = torch.zeros(2, 8, 128, dtype=BF16, device="cuda")
    ops.dsim_paged_attention(wide.cuda()[:, 1:5, 16:], dict(k=to_gpu(keys), v=to_gpu(values)), table.cuda(),
                             torch.tensor([60, 9], dtype=torch.int32, device="cuda"), big[:, 2:6, 32:96])
    ref, _, bound = plain.attend(q, keys, values, table.clamp(min=0), torch.tensor([60, 9]), 0.125)
    room = bound + (ref.abs() + bound) * 2.0 ** -8
    assert torch.all((big[:, 2:6, 32:96].cpu().double() - ref).abs() <= room)
    big[:, 2:6, 32:96] = 0
    assert torch.all(big == 0)


# ---------------------------------------------------------------------------
# dsim_logit_adjust
# ---------------------------------------------------------------------------
def logits_case(seed, n, vocab, dtype, width, biases=0, mask=False, bad_ids=True):
    g = gen(seed)
    x = (4 * randn(g, n, vocab)).to(dtype)
    a = {}
    if width:
        a["history"] = (vocab * torch.rand(n, width, generator=g) ** 4).to(torch.int32)
        if bad_ids:
            a["history"][:, ::7] = torch.tensor(vocab + 3, dtype=torch.int32)
            a["history"][:, 1::11] = -2
        a["history_len"] = torch.randint(-1, width + 3, (n,), generator=g, dtype=torch.int32)
        a["prompt_len"] = torch.randint(-1, width + 3, (n,), generator=g, dtype=torch.int32)
        for name in ("repetition", "frequency", "presence"):
            a[name] = 0.5 + torch.rand(n, generator=g)
    if biases:
        a["bias_id"] = torch.randint(-2, vocab + 2, (n, biases), generator=g, dtype=torch.int32)
        a["bias_id"][:, -1] = a["bias_id"][:, 0]   # the last of two counts
        a["bias"] = 6 * randn(g, n, biases)
    if mask:
        a["mask"] = torch.randint(-2 ** 31, 2 ** 31, (n, (vocab + 31) // 32), generator=g, dtype=torch.int64).to(
            torch.int32)
        a["mask"][0] = 0   # nothing allowed
        a["mask"][-1] = -1
    return x, a


def check_logits(x, a, out=None):
    d = {k: v.cuda() for k, v in a.items()}
    dx = x.cuda()
    got = torch.full_like(dx, 5.0) if out is None else out
    ops.dsim_logit_adjust(dx, got, **d)
    want = plain.logits(x, **a)
    assert plain.same(got.cpu(), want)
    assert plain.same(dx.cpu(), x)
    ops.dsim_logit_adjust(dx, dx, **d)   # in place
    assert plain.same(dx.cpu(), want)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n,vocab", [(1, 1), (3, 31), (2, 50257), (5, 8192), (4, 8193), (1, 70001)])
def test_logits(dtype, n, vocab):
    check_logits(*logits_case(vocab, n, vocab, dtype, 100, 9, True))


@pytest.mark.parametrize("parts", ["history", "bias", "mask", "none", "long"])
def test_logits_parts(parts):
    x, a = logits_case(3, 4, 20011, F16, {"history": 60, "long": 5000}.get(parts, 0), 40 if parts == "bias" else 0,
                       parts == "mask")
    check_logits(x, a)
    if parts == "history":
        for drop in ("repetition", "frequency", "presence", "prompt_len"):
            check_logits(x, {k: v for k, v in a.items() if k != drop})


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n,vocab,width", [(21, 9000, 60), (16, 8192, 5000), (70, 33000, 30), (40, 12345, 4096), (3, 40, 9000)])
def test_logits_rows_and_histories(dtype, n, vocab, width):
    """Slices of every size, rows dealt over the XCDs with some left over."""
    check_logits(*logits_case(n, n, vocab, dtype, width, 9, True))


def test_logits_special_values():
    x, a = logits_case(5, 3, 1000, F32, 400, 20, True)
    x[:, ::5] = -math.inf
    x[:, 1::9] = math.nan
    x[:, 2::9] = math.inf
    x[:, 3::9] = 0.0
    x[:, 4::9] = -0.0
    check_logits(x, a)
    check_logits(x.half(), a)


def test_logits_many_biases_of_one_token():
    x, a = logits_case(6, 2, 5000, F32, 0, 4096)
    a["bias_id"][:] = torch.randint(0, 7, a["bias_id"].shape, generator=gen(1), dtype=torch.int32)
    check_logits(x, a)


def test_logits_strided_rows():
    """Rows of wider tensors, at any element."""
    x, a = logits_case(7, 3, 3001, F16, 50, 5, True)
    wide = torch.zeros(3, 3100, dtype=F16)
    wide[:, 51:3052] = x
    dwide, dout = wide.cuda(), torch.full((3, 3333), 9.0, dtype=F16, device="cuda")
    d = {k: v.cuda() for k, v in a.items()}
    hist = torch.full((3, 64), 5, dtype=torch.int32, device="cuda")
    hist[:, :50] = d["history"]
    d["history"] = hist[:, :50]
    words = torch.zeros(3, 200, dtype=torch.int32, device="cuda")
    words[:, 1:95] = d["mask"]
    d["mask"] = words[:, 1:95]
    ops.dsim_logit_adjust(dwide[:, 51:3052], dout[:, 17:3018], **d)
    assert plain.same(dout[:, 17:3018].cpu(), plain.logits(x, **a))
    dout[:, 17:3018] = 9.0
    assert torch.all(dout == 9.0)


def test_logits_nothing():
    x = torch.zeros(0, 100, device="cuda")
    ops.dsim_logit_adjust(x, x)
    x = torch.ones(2, 100, device="cuda")
    none = torch.zeros(2, 0, dtype=torch.int32, device="cuda")
    ops.dsim_logit_adjust(x, x, history=none, history_len=torch.ones(2, dtype=torch.int32, device="cuda"),
                          repetition=torch.full((2,), 2.0, device="cuda"), bias_id=none,
                          bias=torch.zeros(2, 0, device="cuda"))
    assert torch.all(x == 1)


def test_logits_beyond_32_bits():
    """Rows behind 2^31 elements, in place."""
    vocab = 50257
    n = (1 << 31) // vocab + 9
    x = torch.zeros(n, vocab, dtype=F16, device="cuda")
    check = [0, 1, n // 2, n - 2, n - 1]
    small, a = logits_case(9, len(check), vocab, F16, 40, 3, True)
    x[check] = small.cuda()

    def spread(t):
        big = torch.zeros(n, *t.shape[1:], dtype=t.dtype, device="cuda")
        big[check] = t.cuda()
        return big
    ops.dsim_logit_adjust(x, x, **{k: spread(v) for k, v in a.items()})
    assert plain.same(x[check].cpu(), plain.logits(small, **a))


# ---------------------------------------------------------------------------
# Together
# ---------------------------------------------------------------------------
class Step:
    """A single-token step of a small model with fixed buffers: projections,
    append, attention, logits, as a serving loop holds them."""

    def __init__(self, seed=0, dtype=BF16, n=5, heads=8, kv=2, d=64, vocab=1003, slots=16, most=200):
        g = gen(seed)
        self.n, self.heads, self.kv, self.d, self.vocab = n, heads, kv, d, vocab
        dev = lambda t: t.to(dtype).cuda()   # noqa: E731
        width = heads * d
        self.embed, self.w_in = dev(randn(g, vocab, width)), dev(randn(g, width, (heads + 2 * kv) * d) * width ** -0.5)
        self.w_out = dev(randn(g, width, vocab) * width ** -0.5)
        pages = -(-most // slots)
        self.table = torch.randperm(n * pages, generator=g).to(torch.int32).view(n, pages).cuda()
        self.cache = ops.alloc_kv_cache(n * pages, slots, kv, d, dtype)
        self.rope = ops.rope_table(most, d)
        self.ws = ops.alloc_paged_attention_workspace(heads, kv, d)
        self.seq = torch.arange(n, dtype=torch.int32, device="cuda")
        self.len = torch.ones(n, dtype=torch.int32, device="cuda")
        self.tokens = torch.randint(0, vocab, (n, most), generator=g, dtype=torch.int32).cuda()
        self.penalty = torch.full((n,), 1.3, device="cuda")
        self.out = torch.zeros(n, heads, d, dtype=dtype, device="cuda")
        self.mask = torch.full((n, (vocab + 31) // 32), -2, dtype=torch.int32, device="cuda")
        self.logits = None
        self.rows = torch.arange(n, device="cuda")

    def step(self, stream=None):
        last = self.tokens[self.rows, self.len.long() - 1]
        x = self.embed[last.long()]
        qkv = (x @ self.w_in).view(self.n, self.heads + 2 * self.kv, self.d)
        q, k, v = qkv.split([self.heads, self.kv, self.kv], dim=1)
        ops.dsim_kv_append(self.cache, self.table, k, v, self.seq, self.len - 1, rope=self.rope, q=q, q_out=q,
                           stream=stream)
        ops.dsim_paged_attention(q, self.cache, self.table, self.len, self.out, workspace=self.ws, stream=stream)
        self.logits = self.out.view(self.n, -1) @ self.w_out
        ops.dsim_logit_adjust(self.logits, self.logits, history=self.tokens, history_len=self.len,
                              repetition=self.penalty, frequency=self.penalty, mask=self.mask, stream=stream)
        self.tokens[self.rows, self.len.long()] = self.logits.argmax(-1).to(torch.int32)
        self.len += 1


def test_step_against_whole_sequences():
    """Twenty steps' logits against the same model computed over the whole
    sequence each time in 64 bits from the same rounded parts."""
    m = Step(dtype=F32)
    for _ in range(20):
        m.step()
    got = m.logits.double().cpu()
    n, heads, kv, d = m.n, m.heads, m.kv, m.d
    length = int(m.len[0]) - 1
    ids = m.tokens[:, :length].long()
    qkv = (m.embed[ids] @ m.w_in).view(n, length, heads + 2 * kv, d).double().cpu()
    rope = m.rope[:length].double().cpu()
    z = torch.complex(*qkv[..., :heads + kv, :].chunk(2, dim=-1)) * torch.complex(*rope.chunk(2, dim=1))[None, :, None]
    turned = torch.cat([z.real, z.imag], dim=-1)
    q, k, v = turned[:, -1, :heads], turned[:, :, heads:], qkv[:, :, heads + kv:]
    k, v = (t.repeat_interleave(heads // kv, dim=2) for t in (k, v))
    p = torch.softmax((k * q[:, None]).sum(-1) * d ** -0.5, dim=1)
    out = (p[..., None] * v).sum(1).reshape(n, -1)
    ref = (out @ m.w_out.double().cpu())
    ref = plain.logits(ref, m.tokens.cpu(), None, torch.full((n,), length), m.penalty.double().cpu(),
                       m.penalty.double().cpu(), None, None, None, m.mask.cpu())
    fine = ref.isfinite()
    assert torch.equal(fine, got.isfinite()) and not fine[:, ::32].any()
    # sums of 512 products of numbers of size 1, in fp32, and the attention's
    assert (got[fine] - ref[fine].double()).abs().max() < 512 * 2.0 ** -23 * 4


def test_step_is_deterministic():
    a, b = Step(seed=3), Step(seed=3)
    for _ in range(5):
        a.step()
        b.step()
    assert torch.equal(a.logits, b.logits) and torch.equal(a.tokens, b.tokens)


def test_step_on_another_stream():
    a, b = Step(seed=1), Step(seed=1)
    side = torch.cuda.Stream()
    a.step()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):   # its stream is the current one
        b.step()
    side.synchronize()
    assert torch.equal(a.logits, b.logits)
    a.step()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        b.step(stream=side)         # named as well, then by its handle
        b.step(stream=side.cuda_stream)
    a.step()
    torch.cuda.synchronize()
    assert torch.equal(a.logits, b.logits)


def test_workspace_of_the_call_on_another_stream():
    """A call that allocates its own workspace, on a stream that is not the
    current one."""
    g = gen(8)
    table, pages = deal(g, [3000], 16)
    keys, values = cache_like(g, pages, 16, 1, 64, F16)
    q = randn(g, 1, 2, 64).half()
    cache, out = dict(k=to_gpu(keys), v=to_gpu(values)), torch.zeros(1, 2, 64, dtype=F16, device="cuda")
    args = q.cuda(), cache, table.cuda(), torch.tensor([3000], dtype=torch.int32, device="cuda"), out
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    ops.dsim_paged_attention(*args, stream=side)
    torch.empty(1 << 22, dtype=torch.uint8, device="cuda").fill_(255)
    torch.cuda.synchronize()
    first = out.clone()
    ops.dsim_paged_attention(*args, stream=side.cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(first, out)
    ref, _, bound = plain.attend(q, keys, values, table.clamp(min=0), torch.tensor([3000]), 0.125)
    assert torch.all((out.cpu().double() - ref).abs() <= bound + (ref.abs() + bound) * 2.0 ** -11 + 2.0 ** -25)


def test_two_calls_at_once():
    """Attention over one cache on two streams, each with its own workspace."""
    g = gen(10)
    lens = [4000, 17, 900, 2500]
    table, pages = deal(g, lens, 16)
    keys, values = cache_like(g, pages, 16, 2, 128, BF16)
    cache, table = dict(k=to_gpu(keys), v=to_gpu(values)), table.cuda()
    lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    qs = [randn(g, 4, 8, 128).bfloat16().cuda() for _ in range(2)]
    alone = [torch.empty_like(q) for q in qs]
    for q, out in zip(qs, alone):
        ops.dsim_paged_attention(q, cache, table, lens, out)
    streams, outs = [torch.cuda.Stream() for _ in qs], [torch.zeros_like(q) for q in qs]
    spaces = [ops.alloc_paged_attention_workspace(8, 2, 128) for _ in qs]
    torch.cuda.synchronize()
    for _ in range(20):
        for q, out, ws, s in zip(qs, outs, spaces, streams):
            ops.dsim_paged_attention(q, cache, table, lens, out, workspace=ws, stream=s)
    torch.cuda.synchronize()
    for a, b in zip(alone, outs):
        assert torch.equal(a, b)


def test_step_in_captured_graphs():
    """The step captured, replayed as its state goes on, with eager work
    between; two graphs share one workspace."""
    eager, m = Step(seed=2), Step(seed=2)
    other = Step(seed=2, n=5)
    other.ws = m.ws
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):   # before capture: libraries set themselves up
        Step(seed=9).step()
    torch.cuda.synchronize()
    graphs = []
    for s in (m, other):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.step()
        graphs.append(graph)
    for _ in range(6):
        eager.step()
        torch.cuda.synchronize()
        for graph, s in zip(graphs, (m, other)):
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(s.logits, eager.logits) and torch.equal(s.tokens, eager.tokens)
