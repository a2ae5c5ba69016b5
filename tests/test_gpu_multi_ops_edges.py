"""Prompt and tree attention on the GPU where it can go wrong: infinities and
NaN in masked and in attended places, pages outside the cache, starts and
lengths that do not fit, caches beyond 32 bits, more sequences than the plan's
threads, streams, captured graphs and repeated calls."""
import math

import pytest
import torch

from paper_2111_05426_amd import ops
from test_gpu_multi_ops import check, ints, random_tree, words
from test_gpu_ops import cache_like, deal, gen, gpu, randn, to_gpu  # noqa: F401

pytestmark = pytest.mark.gpu

F32, F16, BF16, E4M3 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn
TYPES = [(F32, F32), (F16, F16), (BF16, BF16), (BF16, E4M3)]
I32 = torch.int32
# rows of 32, 64, 128 and, for two bytes, 256 a block; `width`: the block
# table's, whose room decides whether blocks are cut
SIZES = [(8, 20), (40, 60), (150, 230), (600, 640)]


class Call:
    """A call that can be run again after its inputs are changed."""

    def __init__(self, dtype, cache, heads, kv, d, slots, new, lens, tree=False, width=None, seed=0, **more):
        g = gen(seed)
        self.new, self.lens, self.slots, self.tree = new, lens, slots, tree
        total = [max(n, 0) + (m if tree else 0) for n, m in zip(lens, new)]
        self.table_cpu, pages = deal(g, total, slots, width)
        k, v = cache_like(g, pages, slots, kv, d, F32 if cache == E4M3 else cache)
        self.k, self.v = to_gpu(k.to(cache)), to_gpu(v.to(cache))
        n = sum(new)
        self.q = randn(g, n, heads, d).to(dtype).cuda()
        self.start = ints([sum(new[:i]) for i in range(len(new) + 1)]).cuda()
        self.len, self.table = ints(lens).cuda(), self.table_cpu.cuda()
        self.more = more
        if tree:
            n_words = (max(new + [1]) + 31) // 32
            trees = [random_tree(g, m) for m in new]
            self.sees = [t[1] for t in trees]
            self.mask = torch.cat([words(s, n_words) for s in self.sees]).cuda()
            self.depth = torch.cat([t[0] for t in trees]).cuda()
        self.ws = ops.alloc_prompt_attention_workspace(n, len(new), heads, kv, d)
        self.out = torch.empty(n, heads, d, dtype=dtype, device="cuda")
        self.lse = torch.empty(n, heads, device="cuda")
        self.status = torch.empty(len(new), dtype=I32, device="cuda")

    def run(self, stream=None, clear=True):
        if clear:
            self.ws.fill_(255)
            self.out.fill_(123.0)
            self.lse.fill_(123.0)
            self.status.fill_(-7)
        args = dict(workspace=self.ws, lse=self.lse, status=self.status, stream=stream, **self.more)
        cache = dict(k=self.k, v=self.v)
        if self.tree:
            ops.dsim_tree_attention(self.q, cache, self.table, self.start, self.len, self.mask, self.out, depth=self.depth, **args)
        else:
            ops.dsim_prompt_attention(self.q, cache, self.table, self.start, self.len, self.out, **args)

    def results(self):
        self.run()
        torch.cuda.synchronize()
        return self.out.cpu(), self.lse.cpu(), self.status.cpu()

    def place(self, s, key):
        return int(self.table_cpu[s, key // self.slots]), key % self.slots

    def attends(self, s, key):
        """Which of a sequence's tokens attend to a key (no prefix or documents)."""
        n, length = self.new[s], self.lens[s]
        if self.tree:
            return self.sees[s][:, key - length] if key >= length else torch.ones(n, dtype=torch.bool)
        p, window = torch.arange(length - n, length), self.more.get("window", 0)
        return (p >= key) & ((p - key < window) | (window == 0))


def rows_of(c, s):
    return slice(int(c.start[s]), int(c.start[s + 1]))


def bad_value(dtype, cache):
    """Infinities where the cache's type has them."""
    return [math.nan] if cache == E4M3 else [math.inf, -math.inf, math.nan]


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("n,length", SIZES)
@pytest.mark.parametrize("width", [None, 100])
@pytest.mark.parametrize("tree", [False, True])
def test_values_that_are_not_finite(dtype, cache, n, length, width, tree):
    """Rows that do not attend to them are the same to the bit; of those that
    do, that element alone is not finite."""
    if tree:
        new, lens = [n, 3], [length - n, 9]
    else:
        new, lens = [n, 3], [length, 9]
    c = Call(dtype, cache, 2, 2, 64, 16, new, lens, tree=tree, width=width)
    want, want_lse, _ = c.results()
    odd = torch.zeros(want.shape, dtype=torch.bool)
    last = length - 1
    for i, value in enumerate(bad_value(dtype, cache)):
        for at, (key, element) in enumerate([(last, 5), (last - n // 2, 17), (length - n, 63)]):
            head = (i + at) % 2
            page, slot = c.place(0, key)
            c.v[page, slot, head, element] = value
            odd[rows_of(c, 0), head, element] |= c.attends(0, key)
    page, slot = c.place(0, last)
    if slot + 1 < 16:   # behind the last key
        c.v[page, slot + 1:] = math.nan
        c.k[page, slot + 1:] = math.nan
    out, lse, status = c.results()
    assert torch.equal(status, torch.zeros(2, dtype=I32))
    assert torch.equal(lse, want_lse)
    assert torch.equal(out[~odd], want[~odd])
    assert not out[odd].isfinite().any()


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("n,length", SIZES)
@pytest.mark.parametrize("width", [None, 100])
@pytest.mark.parametrize("tree", [False, True])
def test_special_values_with_a_bias(dtype, cache, n, length, width, tree):
    """The same where a bias by distance turns the order of the tiles."""
    slopes = torch.tensor([0.0, 0.7], device="cuda")
    c = Call(dtype, cache, 2, 2, 64, 16, [n, 3], [length - n, 9] if tree else [length, 9], tree=tree, width=width, slopes=slopes)
    want, want_lse, _ = c.results()
    odd = torch.zeros(want.shape, dtype=torch.bool)
    bad = torch.zeros(want.shape[0], dtype=torch.bool)
    for head, key, element in ((0, length - 1, 5), (1, length - n // 2 - 1, 17)):
        page, slot = c.place(0, key)
        c.v[page, slot, head, element] = math.nan
        odd[rows_of(c, 0), head, element] |= c.attends(0, key)
    first = (length - n) // 16
    for key in range(first * 16, min((first + 1) * 16, length)):
        bad[rows_of(c, 0)] |= c.attends(0, key)
    out, lse, _ = c.results()
    assert torch.equal(lse, want_lse) and torch.equal(out[~odd], want[~odd]) and not out[odd].isfinite().any()
    c.table[0, first] = -1
    out, lse, status = c.results()
    assert status.tolist() == [128, 0] and out[bad].isnan().all() and lse[bad].isnan().all()
    assert torch.equal(lse[~bad], want_lse[~bad]) and torch.equal(out[~bad][~odd[~bad]], want[~bad][~odd[~bad]])


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("n,length", SIZES)
@pytest.mark.parametrize("width", [None, 100])
@pytest.mark.parametrize("tree", [False, True])
def test_keys_that_are_nan(dtype, cache, n, length, width, tree):
    c = Call(dtype, cache, 2, 1, 64, 16, [n, 3], [length - n, 9] if tree else [length, 9], tree=tree, width=width)
    want, want_lse, _ = c.results()
    odd = torch.zeros(want.shape[0], dtype=torch.bool)
    for key in (length - 1, length - n // 2 - 1):
        page, slot = c.place(0, key)
        c.k[page, slot, 0, 7] = math.nan
        odd[rows_of(c, 0)] |= c.attends(0, key)
    out, lse, _ = c.results()
    assert torch.equal(out[~odd], want[~odd]) and torch.equal(lse[~odd], want_lse[~odd])
    assert out[odd].isnan().all() and lse[odd].isnan().all()


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("slots", [16, 48, 5])
@pytest.mark.parametrize("n,length", SIZES)
@pytest.mark.parametrize("width", [None, 300])
def test_pages_outside_the_cache(dtype, cache, slots, n, length, width):
    """Tokens that attend to one are NaN and their sequence's status says so;
    the others are the same to the bit.  Pages before the window may be gone."""
    c = Call(dtype, cache, 4, 2, 64, slots, [n, 3, 9], [length, 50, 80], width=width, window=40)
    want, want_lse, _ = c.results()
    first = (length - n) // slots   # the first new token's page
    c.table[0, first] = c.k.shape[0] + 3
    gone = (80 - 9 - 39) // slots   # pages before the last sequence's windows
    c.table[2, :gone] = -1
    odd = torch.zeros(want.shape[0], dtype=torch.bool)
    for key in range(first * slots, min((first + 1) * slots, length)):
        odd[rows_of(c, 0)] |= c.attends(0, key)
    out, lse, status = c.results()
    assert status.tolist() == [128, 0, 0]
    assert torch.equal(out[~odd], want[~odd]) and torch.equal(lse[~odd], want_lse[~odd])
    assert out[odd].isnan().all() and lse[odd].isnan().all()
    c.table[:] = -1
    out, lse, status = c.results()
    assert status.tolist() == [128, 128, 128] and out.isnan().all() and lse.isnan().all()


@pytest.mark.parametrize("width", [None, 100])
@pytest.mark.parametrize("tree", [False, True])
def test_tree_pages_outside_the_cache(width, tree):
    c = Call(BF16, BF16, 4, 2, 64, 16, [20, 40], [33, 50], tree=True, width=width)
    want, want_lse, _ = c.results()
    c.table[1, 5] = -5      # keys 80 to 95: nodes 30 to 39
    odd = torch.zeros(60, dtype=torch.bool)
    odd[20:] = c.sees[1][:, 30:].any(1)
    out, lse, status = c.results()
    assert status.tolist() == [0, 128]
    assert torch.equal(out[~odd], want[~odd]) and out[odd].isnan().all() and lse[odd].isnan().all()


@pytest.mark.parametrize("width", [None, 100])
@pytest.mark.parametrize("tree", [False, True])
def test_starts_and_lengths_that_do_not_fit(width, tree):
    c = Call(F16, F16, 4, 2, 64, 16, [20, 7, 30], [20, 40, 33], tree=tree, width=width)
    want, want_lse, _ = c.results()

    def run(start, length):
        c.start.copy_(ints(start))
        c.len.copy_(ints(length))
        return c.results()
    # tokens outside q, starts that descend: nothing is written for them
    for start, first in (([20, 20, 27, 58], 20), ([0, 20, 27, 10 ** 9], 0)):
        out, lse, status = run(start, [20, 40, 33])
        assert status.tolist() == [0, 0, 256]
        assert torch.all(out[27:] == 123) and torch.all(lse[27:] == 123)
        assert torch.equal(out[20:27], want[20:27])
    out, lse, status = run([-1, 20, 27, 57], [20, 40, 33])
    assert status.tolist() == [256, 0, 0] and torch.all(out[:20] == 123) and torch.equal(out[20:], want[20:])
    out, lse, status = run([0, 27, 20, 20], [27, 40, 33])
    assert status[1] == 256 and torch.all(out[27:] == 123)
    run([57, 0, 57, 0], [57, 57, 57])   # (more rows in all than there are tokens)
    # more keys than the table has places for, or fewer than tokens
    for bad in ([20, 10 ** 9, 33], [20, 2 ** 31 - 1, 33]) + (() if tree else ([20, 6, 33],)):
        out, lse, status = run([0, 20, 27, 57], bad)
        assert status.tolist() == [0, 256, 0]
        assert out[20:27].isnan().all() and lse[20:27].isnan().all()
        assert torch.equal(out[:20], want[:20]) and torch.equal(out[27:], want[27:])
    out, lse, status = run([0, 20, 27, 57], [20, -3, 33])
    assert status.tolist() == [0, -7, 0] and torch.all(out[20:27] == 123) and torch.equal(out[27:], want[27:])


def test_more_nodes_than_the_mask_has_bits():
    c = Call(F16, F16, 4, 2, 64, 16, [40, 7], [20, 40], tree=True)
    want, _, _ = c.results()
    c.mask = c.mask[:, :1]   # (a stride of two words)
    out, lse, status = c.results()
    assert status.tolist() == [256, 0] and out[:40].isnan().all() and torch.equal(out[40:], want[40:])


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("tree", [False, True])
def test_no_tokens(dtype, cache, tree):
    c = Call(dtype, cache, 4, 2, 64, 16, [0, 0], [5, 0], tree=tree)
    assert c.results()[2].tolist() == [0, 0]
    c = Call(dtype, cache, 4, 2, 64, 16, [0, 0], [5000, 3], tree=tree)
    assert c.results()[2].tolist() == [0, 0]
    c = Call(dtype, cache, 4, 2, 64, 16, [2, 1], [0, 0], tree=True)   # (nodes alone)
    assert c.results()[2].tolist() == [0, 0] and c.out.isfinite().all()


@pytest.mark.parametrize("dtype,cache", [(F32, F32), (BF16, BF16), (F16, E4M3)])
@pytest.mark.parametrize("width", [None, 100])
def test_large_scores(dtype, cache, width):
    """Scores of thousands, of both signs, where a row's largest comes late."""
    for scale in (3.0, -3.0):
        check(dtype, cache, 4, 2, 64, 16, [150, 3], [400, 9], scale=scale, spread=8.0, width=width)
        check(dtype, cache, 4, 2, 64, 16, [15, 3], [400, 9], scale=scale, spread=8.0, width=width, tree=True)


@pytest.mark.parametrize("dtype,cache", [(F32, F32), (F16, F16), (BF16, BF16), (F16, E4M3)])
@pytest.mark.parametrize("n", [20, 300])
def test_steep_biases_over_cut_blocks(dtype, cache, n):
    """A bias that grows by more than the weights' room from tile to tile."""
    def edit(x):
        x["slope"].copy_(torch.tensor([3.0, 0.5, -0.6, 0.001]))
    for tree in (False, True):
        check(dtype, cache, 4, 2, 64, 16, [n, 3], [1500, 900], slopes=True, width=200, edit=edit, tree=tree)


@pytest.mark.parametrize("n,cap", [(20, 0.0), (300, 0.0), (300, 20.0)])
def test_scales_below_zero(n, cap):
    """A cache head's scales of either sign, and a scale too."""
    def edit(x):
        x["ks"][0] *= -1
        x["vs"][1] *= -1
    for scale in (0.2, -0.2):
        check(BF16, E4M3, 4, 2, 64, 16, [n, 60], [n + 9, 60], scales=True, scale=scale, edit=edit, cap=cap)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tree", [False, True])
def test_more_sequences_than_threads(dtype, tree):
    g = gen(4)
    new = torch.randint(0, 4, (1500,), generator=g).tolist()
    lens = [n + int(x) for n, x in zip(new, torch.randint(0, 40, (1500,), generator=g))]
    check(dtype, dtype, 2, 1, 16, 16, new, lens, tree=tree)
    check(dtype, dtype, 2, 1, 16, 16, new, lens, tree=tree, width=100)


@pytest.mark.parametrize("n_seq", [63, 64, 65, 200, 256, 257])
@pytest.mark.parametrize("tree", [False, True])
def test_sequences_among_many(n_seq, tree):
    """Blocks find theirs among many, of which some have none."""
    g = gen(n_seq)
    new = (torch.randint(-20, 40, (n_seq,), generator=g).clamp(min=0)).tolist()
    lens = [n + int(x) for n, x in zip(new, torch.randint(0, 40, (n_seq,), generator=g))]
    for i in range(3, n_seq, 17):
        lens[i] = -1
    check(BF16, BF16, 4, 2, 32, 16, new, lens, tree=tree)
    check(F32, F32, 4, 1, 16, 16, new, lens, tree=tree)


@pytest.mark.parametrize("cache,order", [(BF16, "head"), (E4M3, "head"), (F32, "slot")])
def test_a_cache_beyond_32_bits(cache, order):
    """Pages whose first element is number 2^32 and more (2^31 and 2^32 bytes
    further on with one byte an element)."""
    slots, kv, d, n, length = 16, 4, 128, 70, 300
    each = slots * kv * d
    pages = (1 << (32 if cache == E4M3 else 31)) // each + 40
    dtype = BF16 if cache == E4M3 else cache
    c = Call(dtype, cache, 8, kv, d, slots, [n, 2], [length, 40], seed=3)
    want = c.results()
    small, first = c.k.shape[0], pages - c.k.shape[0]
    shape = (pages, kv, slots, d) if order == "head" else (pages, slots, kv, d)
    for name in ("k", "v"):
        big = torch.empty(shape, dtype=cache, device="cuda")
        big = big.transpose(1, 2) if order == "head" else big
        big[first:].copy_(getattr(c, name))
        setattr(c, name, big)
    c.table = torch.where(c.table >= 0, c.table + first, c.table)
    got = c.results()
    assert small < 40 and all(torch.equal(a, b) for a, b in zip(got, want))


class OtherDevice:
    """As a stream of another device has them."""
    cuda_stream, device_index = 0, 1


CUT = [dict(new=[150, 1, 40], lens=[900, 300, 40], width=200), dict(new=[15, 1, 40], lens=[90, 30, 40])]


@pytest.mark.parametrize("at", range(len(CUT)))
@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("tree", [False, True])
def test_streams_and_repeats(dtype, cache, at, tree):
    c = Call(dtype, cache, 8, 2, 64, 16, tree=tree, **CUT[at])
    want = c.results()
    side = torch.cuda.Stream()
    for stream in (None, side, side.cuda_stream):
        with torch.cuda.stream(side):
            c.run(stream)
        side.synchronize()
        assert all(torch.equal(a.cpu(), b) for a, b in zip((c.out, c.lse, c.status), want))
    with pytest.raises(ValueError, match="stream must be on cuda:0"):
        c.run(OtherDevice())
    c.ws = None   # one of the call's own
    with torch.cuda.stream(side):
        c.run(clear=False)
    side.synchronize()
    assert torch.equal(c.out.cpu(), want[0])


@pytest.mark.parametrize("at", range(len(CUT)))
@pytest.mark.parametrize("dtype,cache", TYPES)
def test_captured_graphs(dtype, cache, at):
    """Two graphs that share a workspace, replayed with eager work between
    them, on inputs that change."""
    a = Call(dtype, cache, 8, 2, 64, 16, seed=1, **CUT[at])
    b = Call(dtype, cache, 8, 2, 64, 16, seed=2, tree=True, **CUT[at])
    b.ws = a.ws = max(a.ws, b.ws, key=len)
    graphs = []
    for c in (a, b):
        c.run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.run(clear=False)
        graphs.append(graph)
    for turn in range(4):
        want = []
        for c in (a, b):
            c.q.mul_(0.75)
            c.len.sub_(1 if c.tree else 0)
            want.append(c.results())
        for c, graph, w in zip((a, b), graphs, want):
            for x in (c.ws, c.out, c.lse, c.status):
                x.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x.cpu(), y) for x, y in zip((c.out, c.lse, c.status), w)), turn


def test_versions():
    """What the calls write counts as changed in place, what they read does not."""
    c = Call(F32, F32, 4, 2, 64, 16, [3, 2], [9, 5])
    t = Call(F32, F32, 4, 2, 64, 16, [3, 2], [9, 5], tree=True)
    for x in (c, t):
        written, read = [x.out, x.lse, x.status, x.ws], [x.q, x.k, x.v, x.table, x.start, x.len]
        before = [[y._version for y in z] for z in (written, read)]
        x.run(clear=False)
        assert all(y._version > n for y, n in zip(written, before[0])) and [y._version for y in read] == before[1]
        w = torch.ones((), device="cuda", requires_grad=True)
        y = (w * x.out).sum()
        x.run(clear=False)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()


@pytest.mark.parametrize("dtype,cache", [(F16, F16), (BF16, BF16), (F16, E4M3), (BF16, E4M3)])
@pytest.mark.parametrize("slots", [16, 48, 5])
@pytest.mark.parametrize("width", [None, 400])
@pytest.mark.parametrize("tree", [False, True])
def test_special_values_in_the_largest_blocks(dtype, cache, slots, width, tree):
    """More than 1,536 rows a sequence on average: blocks of 256."""
    n, length = 500, 620
    c = Call(dtype, cache, 16, 2, 64, slots, [n, 3], [length - n, 9] if tree else [length, 9], tree=tree, width=width)
    want, want_lse, _ = c.results()
    odd, nan = torch.zeros(want.shape, dtype=torch.bool), torch.zeros(want.shape[:2], dtype=torch.bool)
    for head, key, element in ((0, length - 1, 5), (1, length - n // 2 - 1, 17), (1, length - n, 63)):
        page, slot = c.place(0, key)
        c.v[page, slot, head, element] = math.nan
        odd[rows_of(c, 0), 8 * head:8 * head + 8, element] |= c.attends(0, key)[:, None]
    out, lse, _ = c.results()
    assert torch.equal(lse, want_lse) and torch.equal(out[~odd], want[~odd]) and not out[odd].isfinite().any()
    page, slot = c.place(0, length - 40)
    c.k[page, slot, 0, 3] = math.nan
    nan[rows_of(c, 0), :8] |= c.attends(0, length - 40)[:, None]
    at = (length - 90) // slots
    c.table[0, at] = c.k.shape[0]
    for key in range(at * slots, (at + 1) * slots):
        nan[rows_of(c, 0)] |= c.attends(0, key)[:, None]
    out, lse, status = c.results()
    assert status.tolist() == [128, 0]
    assert out[nan].isnan().all() and lse[nan].isnan().all() and torch.equal(lse[~nan], want_lse[~nan])
    rest = ~(odd | nan[:, :, None])
    assert torch.equal(out[rest], want[rest])
