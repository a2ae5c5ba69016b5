"""Prompt and tree attention on the GPU where keys end at the last places that
a block table may have, 2^31 - 1: the same to the bit as at places a multiple
of the tiles before."""
import pytest
import torch

from test_gpu_multi_ops_edges import Call, I32
from test_gpu_ops import gpu  # noqa: F401

pytestmark = pytest.mark.gpu

F32, F16, BF16, E4M3 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn


@pytest.mark.parametrize("dtype,cache", [(F32, F32), (BF16, BF16), (F16, E4M3)])
@pytest.mark.parametrize("slots", [16, 15])
@pytest.mark.parametrize("group,n", [(1, 8), (1, 40), (1, 150), (8, 250)])
@pytest.mark.parametrize("what", ["window", "first_key", "slopes", "tree", "tree_slopes"])
def test_keys_at_the_tables_end(dtype, cache, slots, group, n, what):
    tree = what.startswith("tree")
    places = (2 ** 31 - 1) // slots * slots
    period = slots * 256                       # of pages and tiles
    for behind in (0, 3):                      # places that are left
        total = places - behind
        short = total % period + 2 * period
        window = 300
        more = dict(window=window) if what != "first_key" else {}
        if "slopes" in what:
            more["slopes"] = torch.tensor([0.5, 0.003] * group, device="cuda")
        if what == "first_key":
            more["first_key"] = torch.full((n,), short - window, dtype=I32, device="cuda")
        c = Call(dtype, cache, 2 * group, 2, 64, slots, [n], [short - n if tree else short], tree=tree,
                 width=(short + period) // slots, **more)
        pages = -(-short // slots)
        gone = (short - n - window) // slots   # nobody attends to these
        c.table[0, :gone] = -1
        want = c.results()
        assert want[2].tolist() == [0] and want[0].isfinite().all()
        far = torch.full((1, places // slots), -1, dtype=I32, device="cuda")
        last = -(-total // slots)
        far[0, last - (pages - gone):last] = c.table[0, gone:pages]
        c.table = far
        c.len.fill_(total - n if tree else total)
        if what == "first_key":
            c.more["first_key"].fill_(total - window)
        got = c.results()
        assert got[2].tolist() == [0]
        assert all(torch.equal(x, y) for x, y in zip(got, want)), behind
