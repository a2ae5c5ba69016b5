"""The single-token step's operators on streams and in captured graphs where
the block table has room for long contexts, so that the attention is cut,
goes through its workspace and is joined."""
import pytest
import torch

from paper_2111_05426_amd import ops
from test_gpu_ops import F16, Step, cache_like, deal, gen, gpu, randn, to_gpu  # noqa: F401

pytestmark = pytest.mark.gpu

I32 = torch.int32


class OtherStream:
    """As a stream of another device has them."""
    cuda_stream, device_index = 0, 1


@pytest.mark.parametrize("name", ["append", "attention", "logits"])
def test_stream_of_another_device(name):
    call = {"append": lambda **kw: ops.dsim_kv_append(cache, table, rows, rows, seq, seq, **kw),
            "attention": lambda **kw: ops.dsim_paged_attention(q, cache, table, seq, torch.empty_like(q), workspace=ws, **kw),
            "logits": lambda **kw: ops.dsim_logit_adjust(x, x, **kw)}[name]
    cache = {n: torch.zeros(4, 16, 2, 64, device="cuda") for n in ("k", "v")}
    table, rows = torch.zeros(3, 2, dtype=I32, device="cuda"), torch.zeros(3, 2, 64, device="cuda")
    q, seq = torch.zeros(3, 4, 64, device="cuda"), torch.arange(3, dtype=I32, device="cuda")
    ws, x = ops.alloc_paged_attention_workspace(4, 2, 64), torch.zeros(2, 100, device="cuda")
    with pytest.raises(ValueError, match="stream must be on cuda:0"):
        call(stream=OtherStream())
    call(stream=torch.cuda.current_stream())
    call(stream=torch.cuda.Stream())
    torch.cuda.synchronize()


class LongStep(Step):
    """Contexts of many lengths under a block table for 3,000 tokens; with more
    than 512 contexts the cuts are kept by workgroup, with fewer by context."""

    def __init__(self, n, seed=0):
        super().__init__(seed=seed, n=n, most=3000)
        g = torch.Generator(device="cuda").manual_seed(seed)
        for x in self.cache.values():
            x.copy_(torch.randn(x.shape, device="cuda", generator=g))
        lens = torch.randint(1, 60, (n,), generator=gen(seed), dtype=torch.int32)
        lens[:5] = torch.tensor([2900, 1, 1500, 40, 2000])
        self.len.copy_(lens)


@pytest.mark.parametrize("n", [5, 300])
def test_long_contexts_in_captured_graphs(n):
    """Captured, replayed as the state goes on, with eager work between; two
    graphs share one workspace, which each replay finds full of NaN."""
    eager, m, other = (LongStep(n, seed=2) for _ in range(3))
    other.ws = m.ws
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):   # before capture: libraries set themselves up
        LongStep(n, seed=9).step()
    torch.cuda.synchronize()
    graphs = []
    for s in (m, other):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.step()
        graphs.append(graph)
    for _ in range(4):
        eager.step()
        torch.cuda.synchronize()
        for graph, s in zip(graphs, (m, other)):
            m.ws.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(s.out, eager.out) and torch.equal(s.logits, eager.logits)
            assert torch.equal(s.tokens, eager.tokens)
    assert eager.logits[:, 1].isfinite().all()


@pytest.mark.parametrize("n", [5, 300])
def test_long_contexts_are_deterministic(n):
    a, b = LongStep(n, seed=3), LongStep(n, seed=3)
    for _ in range(3):
        a.step()
        b.step()
        assert torch.equal(a.out, b.out) and torch.equal(a.logits, b.logits) and torch.equal(a.tokens, b.tokens)


@pytest.mark.parametrize("n", [5, 300])
def test_long_contexts_on_another_stream(n):
    a, b = LongStep(n, seed=1), LongStep(n, seed=1)
    side = torch.cuda.Stream()
    for stream in (None, side, side.cuda_stream):
        a.step()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            b.step(stream=stream)
        side.synchronize()
        assert torch.equal(a.out, b.out) and torch.equal(a.logits, b.logits)


@pytest.mark.parametrize("by_handle", [False, True])
def test_a_calls_own_workspace_is_not_handed_out_again(monkeypatch, by_handle):
    """While a call on another stream is still to run, its workspace's memory
    is nobody else's."""
    g = gen(8)
    table, pages = deal(g, [3000], 16)
    keys, values = cache_like(g, pages, 16, 1, 64, F16)
    q, out = randn(g, 1, 2, 64).half().cuda(), torch.zeros(1, 2, 64, dtype=F16, device="cuda")
    args = q, dict(k=to_gpu(keys), v=to_gpu(values)), table.cuda(), torch.tensor([3000], dtype=I32, device="cuda"), out
    need = ops.dsim_paged_attention_workspace(2, 1, 64)
    ops.dsim_paged_attention(*args)
    want = out.clone()
    # memory of that size that is free is handed out again at once
    first = torch.empty(need, dtype=torch.uint8, device="cuda")
    address = first.data_ptr()
    del first
    assert torch.empty(need, dtype=torch.uint8, device="cuda").data_ptr() == address
    made, make = [], ops._workspace

    def workspace(*a):
        w = make(*a)
        made.append(w.data_ptr())
        return w
    monkeypatch.setattr(ops, "_workspace", workspace)
    side, big = torch.cuda.Stream(), torch.ones(8192, 8192, device="cuda")
    busy = torch.empty_like(big)
    torch.matmul(big, big, out=busy)   # (the library sets itself up)
    out.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            torch.matmul(big, big, out=busy)
    ops.dsim_paged_attention(*args, stream=side.cuda_stream if by_handle else side)
    others = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(8)]
    pending = not side.query()
    for x in others:
        x.fill_(255)
    torch.cuda.synchronize()
    assert pending and made and all(x.data_ptr() != made[0] for x in others)
    assert torch.equal(out, want)
