"""The operators of steps of several tokens together, as a program that serves
a model runs them: pages reserved, prompts appended and attended, trees of
drafts appended, attended, their accepted path moved to the context's end and
the rest given back, sequences forked and released.  A record on the host
holds what every sequence's cache should hold."""
import pytest
import torch

import multi_ops_plain as plain
import step_ops
from paper_2111_05426_amd import ops
from test_gpu_multi_ops import HALF, ints, random_tree, weights_off, words
from test_gpu_ops import gen, gpu, randn  # noqa: F401

pytestmark = pytest.mark.gpu

F32, F16, BF16, E4M3 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn
I32 = torch.int32
HEADS, KV, D, PAGE, ROWS, WIDTH = 4, 2, 64, 16, 4, 40


class Server:
    """Two layers, four rows of a block table and the pages they hold."""

    def __init__(self, dtype, cache, seed):
        self.g, self.dtype, self.cache_type = gen(seed), dtype, cache
        self.pages = 150
        self.layers = [ops.alloc_kv_cache(self.pages, PAGE, KV, D, cache) for _ in range(2)]
        for x in self.layers:
            for t in x.values():   # (what nobody wrote may be anything)
                t.view(torch.uint8).fill_(0xff)
        self.pool = ops.alloc_page_pool(self.pages, ROWS)
        self.table = torch.full((ROWS, WIDTH), -1, dtype=I32, device="cuda")
        self.len = torch.zeros(ROWS, dtype=I32, device="cuda")
        self.status = torch.zeros(ROWS, dtype=I32, device="cuda")
        self.rope_cpu = ops.rope_table(WIDTH * PAGE, D, device="cpu")
        self.rope = self.rope_cpu.cuda()
        self.record = [[] for _ in range(ROWS)]   # of (layer 0's key, value, layer 1's key, value)

    def told(self, want=(0,) * ROWS):
        assert self.status.tolist() == list(want)

    def reserve(self, new_len):
        ops.dsim_kv_reserve(self.pool, self.table, PAGE, self.len, ints(new_len).cuda(), self.status)
        self.told()

    def append(self, seq, slot, pos):
        """New tokens of every layer; returns the queries and what the cache
        holds of them."""
        n = len(seq)
        kept = []
        for layer in self.layers:
            k, v, q = (randn(self.g, n, h, D).to(self.dtype) for h in (KV, KV, HEADS))
            turned = torch.empty_like(q, device="cuda")
            status = torch.full((n,), -7, dtype=I32, device="cuda")
            ops.dsim_kv_append_axes(layer, self.table, k.cuda(), v.cuda(), ints(seq).cuda(), ints(slot).cuda(),
                                    torch.tensor(pos, dtype=I32).view(n, -1).cuda(), self.rope, sections=[20, 12], q=q.cuda(),
                                    q_out=turned, status=status)
            assert torch.all(status == 0)
            for i in range(n):
                row = torch.cat([self.rope_cpu[pos[i][0], :20], self.rope_cpu[pos[i][1], 20:32],
                                 self.rope_cpu[pos[i][0], 32:52], self.rope_cpu[pos[i][1], 52:]])
                both = (step_ops.rotate(k[i].float(), row, False), v[i].float())
                both = [step_ops.to_e4m3(x) if self.cache_type == E4M3 else x.to(self.cache_type) for x in both]
                kept.append(both) if layer is self.layers[0] else kept[i].extend(both)
            queries = turned.cpu() if layer is self.layers[0] else queries
        return queries, kept

    def dense(self, records):
        """A cache of its own for records, one page each."""
        most = max(len(r) for r in records)
        keys, values = (torch.zeros(len(records), most, KV, D, dtype=self.cache_type) for _ in range(2))
        for s, r in enumerate(records):
            for j, x in enumerate(r):
                keys[s, j], values[s, j] = x[0], x[1]
        return keys, values, torch.arange(len(records), dtype=I32)[:, None]

    def right(self, q, out, records, start, length, **masks):
        weight, least = weights_off(self.dtype, q.shape[0], ROWS, HEADS // KV)
        want, _, bound, _, seen = plain.attention(q, *self.dense(records), start, length, D ** -0.5, weight=weight, least=least,
                                                  exact=self.dtype == F32, **masks)
        room = bound + (want.abs() + bound) * HALF[self.dtype] + (2.0 ** -25 if self.dtype == F16 else 0)
        assert seen.all() and torch.all((out.cpu().double() - want).abs() <= room)

    def prompts(self, n):
        """n new tokens for each row, at its end."""
        have = [len(r) for r in self.record]
        self.reserve([h + m for h, m in zip(have, n)])
        places = [(s, have[s] + i) for s in range(ROWS) for i in range(n[s])]
        q, kept = self.append([s for s, _ in places], [p for _, p in places], [(p, p // 3) for _, p in places])
        for (s, _), x in zip(places, kept):
            self.record[s].append(x)
        self.len += ints(n).cuda()
        start = ints([sum(n[:s]) for s in range(ROWS + 1)])
        out = torch.empty_like(q, device="cuda")
        ops.dsim_prompt_attention(q.cuda(), self.layers[0], self.table, start.cuda(), self.len, out, status=self.status)
        self.told()
        self.right(q, out, self.record, start, self.len.cpu())

    def drafts(self, n, rows, captured=False):
        """A tree of n[s] nodes for each row; a path of it is accepted."""
        have = [len(r) for r in self.record]
        self.reserve([h + m for h, m in zip(have, n)])
        trees = [random_tree(self.g, m) for m in n]
        depth = torch.cat([t[0] for t in trees])
        mask = torch.cat([words(t[1], 1) for t in trees])
        places = [(s, i) for s in range(ROWS) for i in range(n[s])]
        at = [have[s] + int(trees[s][0][i]) for s, i in places]
        q, kept = self.append([s for s, _ in places], [have[s] + i for s, i in places], [(p, p // 3) for p in at])
        start = ints([sum(n[:s]) for s in range(ROWS + 1)])
        out = torch.empty_like(q, device="cuda")
        path = []
        for s in range(ROWS):
            leaf = int(torch.randint(0, max(n[s], 1), (1,), generator=self.g))
            path.append(trees[s][1][leaf].nonzero().flatten().tolist() if n[s] and s in rows else [])
        keep = torch.full((ROWS, 8), -1, dtype=I32)
        for s, p in enumerate(path):
            keep[s, :min(len(p), 8)] = ints(p[:8])
        count = ints([min(len(p), 8) for p in path]).cuda()
        args = [x.cuda() for x in (q, start, mask, depth, keep, torch.arange(ROWS, dtype=I32))]
        ws = ops.alloc_prompt_attention_workspace(q.shape[0], ROWS, HEADS, KV, D)
        more = torch.zeros_like(self.len)

        def step():
            ops.dsim_tree_attention(args[0], self.layers[0], self.table, args[1], self.len, args[2], out, depth=args[3],
                                    status=self.status, workspace=ws)
            ops.dsim_kv_compact(self.layers, self.table, self.len, args[4], count)
            torch.add(self.len, count, out=more)
            ops.dsim_kv_release(self.pool, self.table, PAGE, args[5], more)
        if captured:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
            graph.replay()
        else:
            step()
        torch.cuda.synchronize()
        self.told()
        self.len.copy_(more)
        by_row = [[kept[i] for i, (t, _) in enumerate(places) if t == s] for s in range(ROWS)]
        self.right(q, out, [r + x for r, x in zip(self.record, by_row)], start, ints(have), tree_mask=mask, depth=depth)
        for s, p in enumerate(path):
            self.record[s] = self.record[s] + [by_row[s][i] for i in p[:8]]

    def fork(self, src, dst):
        status = torch.full((len(src),), -7, dtype=I32, device="cuda")
        ops.dsim_kv_fork(self.layers, self.pool, self.table, self.len, ints(src).cuda(), ints(dst).cuda(), status)
        assert torch.all(status == 0)
        for a, b in zip(src, dst):
            self.record[b] = list(self.record[a])

    def release(self, rows):
        ops.dsim_kv_release(self.pool, self.table, PAGE, ints(rows).cuda(), torch.zeros(len(rows), dtype=I32, device="cuda"))
        for s in rows:
            self.record[s] = []
            self.len[s] = 0

    def consistent(self):
        table, held, refs = self.table.cpu(), self.pool["held"].cpu(), self.pool["refs"].cpu()
        free = self.pool["free"].cpu()
        counts = torch.zeros(self.pages, dtype=I32)
        assert self.len.tolist() == [len(r) for r in self.record]
        for s, r in enumerate(self.record):
            assert held[s] == -(-len(r) // PAGE) and torch.all(table[s, held[s]:] == -1)
            for j, x in enumerate(r):
                page = int(table[s, j // PAGE])
                for i, t in enumerate((self.layers[0]["k"], self.layers[0]["v"], self.layers[1]["k"], self.layers[1]["v"])):
                    if j % 7 == 0 or j > len(r) - 20:
                        assert torch.equal(t[page, j % PAGE].cpu().view(torch.uint8), x[i].view(torch.uint8)), (s, j, i)
            for page in table[s, :held[s]].tolist():
                counts[page] += 1
        assert torch.equal(refs, counts)
        bits = [(int(free[p // 32]) >> p % 32 & 1) for p in range(self.pages)]
        assert bits == [int(c == 0) for c in counts]


@pytest.mark.parametrize("dtype,cache", [(F32, F32), (F16, F16), (BF16, BF16), (BF16, E4M3)])
@pytest.mark.parametrize("captured", [False, True])
def test_a_run(dtype, cache, captured):
    m = Server(dtype, cache, seed=5)
    m.prompts([37, 64, 0, 0])
    m.consistent()
    m.prompts([3, 30, 0, 200])
    m.drafts([7, 20, 0, 32], (0, 1, 3), captured)
    m.consistent()
    m.fork([0], [2])
    m.consistent()
    m.drafts([1, 9, 12, 5], (0, 1, 2), captured)   # (row 3's drafts are all refused)
    m.consistent()
    m.release([1])
    m.fork([3], [1])
    m.consistent()
    for _ in range(2):
        m.drafts([6, 6, 6, 6], (0, 1, 2, 3), captured)
        m.consistent()
    m.prompts([100, 1, 0, 17])
    m.consistent()
    m.release([2, 0, 1, 3])
    m.consistent()
    assert torch.all(m.pool["refs"] == 0)
