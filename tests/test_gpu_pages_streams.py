"""The cache's pages on streams and in captured graphs: what a replay deals
out, forks, copies, moves and takes back is what calls one by one do."""
import pytest
import torch

from paper_2111_05426_amd import ops
from test_gpu_ops import gen, gpu  # noqa: F401

pytestmark = pytest.mark.gpu

I32, BF16 = torch.int32, torch.bfloat16
PAGE, ROWS, PAGES = 16, 12, 64


class OtherDevice:
    """As a stream of another device has them."""
    cuda_stream, device_index = 0, 1


class State:
    def __init__(self):
        self.cache = ops.alloc_kv_cache(PAGES, PAGE, 2, 32, BF16)
        g = torch.Generator(device="cuda").manual_seed(1)
        for t in self.cache.values():
            t.copy_(torch.randn(t.shape, device="cuda", generator=g))
        self.pool = ops.alloc_page_pool(PAGES, ROWS)
        self.table = torch.full((ROWS, 8), -1, dtype=I32, device="cuda")
        self.len, self.want, self.status, self.none = (torch.zeros(ROWS, dtype=I32, device="cuda") for _ in range(4))
        self.want[:4] = torch.tensor([20, 40, 1, 100], dtype=I32)
        self.src, self.dst = (torch.tensor(x, dtype=I32, device="cuda") for x in ([0, 1, 3, 3], [4, 5, 6, 7]))
        self.gone = torch.tensor([5, 1], dtype=I32, device="cuda")
        self.fork_status, self.two = (torch.zeros(n, dtype=I32, device="cuda") for n in (4, 2))
        self.keep = torch.arange(1, 30, 2, dtype=I32, device="cuda").repeat(ROWS, 1)
        self.count = torch.zeros(ROWS, dtype=I32, device="cuda")
        self.count[6] = 15
        self.from_, self.to = (torch.tensor(x, dtype=I32, device="cuda") for x in ([0, -1, 2], [60, 5, 61]))

    def step(self, stream=None):
        """Rows 0 to 3 grow (3 into row 2's fork's room), are forked, and all
        of the forks end again."""
        ops.dsim_kv_reserve(self.pool, self.table, PAGE, self.len, self.want, self.status, stream=stream)
        torch.maximum(self.len, self.want, out=self.len)
        ops.dsim_kv_fork(self.cache, self.pool, self.table, self.len, self.src, self.dst, self.fork_status, stream=stream)
        ops.dsim_kv_compact(self.cache, self.table, self.none, self.keep, self.count, stream=stream)
        ops.dsim_kv_copy_pages(self.cache, self.from_, self.to, stream=stream)

    def back(self, stream=None):
        ops.dsim_kv_release(self.pool, self.table, PAGE, self.dst, self.none[:4], stream=stream)
        ops.dsim_kv_release(self.pool, self.table, PAGE, self.gone, self.two, stream=stream)
        self.len[4:8].zero_()   # (filled by a kernel)
        self.len[1:2].zero_()
        self.want[:4] += 5

    def seen(self):
        torch.cuda.synchronize()
        return [x.clone() for x in (*self.cache.values(), *self.pool.values(), self.table, self.len, self.status, self.fork_status)]


def test_on_another_stream():
    a, b = State(), State()
    side = torch.cuda.Stream()
    for stream in (None, side, side.cuda_stream):
        a.step()
        want = a.seen()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            b.step(stream)
        side.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(b.seen(), want))
        a.back()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            b.back(stream)
        side.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(b.seen(), a.seen()))
    assert torch.all(a.fork_status == 0)


def test_captured():
    a, b = State(), State()
    State().step()
    State().back()
    torch.cuda.synchronize()
    graphs = []
    for what in ("step", "back"):
        keep = b.len.clone(), b.want.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            getattr(b, what)()
        graphs.append(graph)
        assert torch.equal(b.len, keep[0]) and torch.equal(b.want, keep[1])   # (captured, not run)
    for _ in range(4):
        a.step()
        want = a.seen()
        graphs[0].replay()
        assert all(torch.equal(x, y) for x, y in zip(b.seen(), want))
        a.back()
        want = a.seen()
        graphs[1].replay()
        assert all(torch.equal(x, y) for x, y in zip(b.seen(), want))


def test_stream_of_another_device():
    s = State()
    with pytest.raises(ValueError, match="stream must be on cuda:0"):
        s.step(OtherDevice())
    with pytest.raises(ValueError, match="stream must be on cuda:0"):
        s.back(OtherDevice())
    with pytest.raises(ValueError, match="stream must be on cuda:0"):
        ops.dsim_kv_copy_pages(s.cache, s.from_, s.to, stream=OtherDevice())
    rows = torch.zeros(3, 2, 32, dtype=BF16, device="cuda")
    with pytest.raises(ValueError, match="stream must be on cuda:0"):
        ops.dsim_kv_append_axes(s.cache, s.table, rows, rows, s.none[:3], s.none[:3], None, None, stream=OtherDevice())


def test_versions():
    s = State()
    written = [*s.cache.values(), *s.pool.values(), s.table, s.status, s.fork_status]
    before = [t._version for t in written]
    s.step()
    assert all(t._version > n for t, n in zip(written, before))
    assert all(t._version == 0 for t in (s.src, s.dst, s.none, s.keep))
