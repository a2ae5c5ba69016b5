"""dsim_kv_reserve on rows that went back behind pages which others hold too,
against a plain implementation that looks at every page that would be written
to; and forks from rows that the call has as a dst."""
import pytest
import torch

import multi_ops_plain as plain
from test_gpu_ops import gen, gpu  # noqa: F401
from test_gpu_pages import BF16, E4M3, F32, Both, ints

pytestmark = pytest.mark.gpu


class Pool(plain.Pool):
    """What a row holds from the page of place length on is written to where it
    grows, up to its new length: no page of that may be another row's too."""

    def reserve(self, length, want, status):
        told = list(status)
        for s, n in enumerate(want):
            held = self.held[s]
            if n < 0 or self.pages(n) > len(self.table[s]) or not 0 <= length[s] <= held * self.page or n <= length[s]:
                continue
            pages = self.table[s][length[s] // self.page:min(held, self.pages(n))]
            if any(not 0 <= p < len(self.refs) for p in pages):
                told[s] = 128
            elif any(self.refs[p] > 1 for p in pages):
                told[s] = 2048
        refused = [s for s, st in enumerate(told) if st in (128, 2048)]
        super().reserve(length, [-1 if s in refused else n for s, n in enumerate(want)], status)
        for s in refused:
            status[s] = told[s]


def both(n_pages, rows, width, page):
    b = Both(n_pages, rows, width, page, layers=1, heads=1, d=16)
    b.plain = Pool(n_pages, rows, width, page)
    return b


def forked(page, length, rows=4, n_pages=400, width=120):
    """Rows 1 and 2 are forks of row 0's `length` places, row 3 has as many of
    its own."""
    b = both(n_pages, rows, width, page)
    b.set_len([0] * rows)
    b.reserve([length, 0, 0, length] + [-1] * (rows - 4))
    b.set_len([length, 0, 0, length] + [0] * (rows - 4))
    assert b.fork([0, 0], [1, 2]) == [0, 0]
    return b


@pytest.mark.parametrize("page", [1, 5, 16])
@pytest.mark.parametrize("back", [0, 1, 2, 3, 20, 37, 48])
def test_rows_that_went_back(page, back):
    """To the middle of a page and to its beginning, by a page and by many."""
    length = 48
    b = forked(page, length)
    n = length - back
    b.set_len([n, n, length, n])
    status = b.reserve([n + 3, n, length + 2, n + 60])
    # row 0 writes to pages that rows 1 and 2 hold unless those end before n
    assert status == [2048 if n < length // page * page else 0, 0, 0, 0]
    # what the row does not use it gives back, and then has its own
    if n % page == 0:
        b.release([0], [n])
        assert b.reserve([n + 3, n, -1, -1])[:2] == [0, 0]
    else:
        b.release([1, 2], [0, 0])
        b.set_len([n, 0, 0, n])
        assert b.reserve([n + 3, -1, -1, -1])[0] == 0


def test_pages_behind_the_first_that_is_written():
    """Its own page, and another's behind it; up to the new length only."""
    b = both(40, 3, 12, 4)
    b.reserve([40, 8, 0])
    b.set_len([40, 8, 0])
    shared = b.plain.table[0][5]          # places 20 to 23
    for t in (b.table, ):
        t[2, 0] = shared
    b.plain.table[2][0] = shared
    b.plain.refs[shared] = 2
    b.pool["refs"][shared] = 2
    b.plain.held[2] = 1
    b.pool["held"][2] = 1
    for n, want, told in ((13, 20, 0), (13, 21, 2048), (20, 21, 2048), (24, 30, 0), (23, 23, 0), (23, 0, 0), (0, 40, 2048),
                          (0, 44, 2048)):
        b.set_len([n, 8, 1])
        assert b.reserve([want, 8, 1]) == [told, 0, 0], (n, want)
    # a page outside the cache is told of before one that is shared
    b.table[0, 7] = 40
    b.plain.table[0][7] = 40
    for n, want, told in ((0, 28, 2048), (0, 29, 128), (28, 29, 128), (32, 33, 0)):
        b.set_len([n, 8, 1])
        assert b.reserve([want, 8, 1]) == [told, 0, 0], (n, want)


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("order", ["head", "slot", "gaps"])
@pytest.mark.parametrize("page", [1, 5, 16])
def test_forks_that_went_back(dtype, order, page):
    b = Both(120, 8, 40, page, layers=3, heads=3, d=48, dtype=dtype, order=order)
    b.plain = Pool(120, 8, 40, page)
    length = [37, 16, 0, 0, 0, 0, 33, 0]
    b.set_len([0] * 8)
    b.reserve(length[:])
    b.set_len(length)
    assert b.fork([0, 0, 1, 6], [2, 3, 4, 5]) == [0, 0, 0, 0]
    b.fork([2], [7])
    b.set_len([max(n - 2, 0) for n in b.len])
    told = b.reserve([n + 3 if n else 0 for n in b.len])
    # 35 places of 37: pages of 5 and 16 were copied there; 14 of 16; 31 of 33
    assert told == {1: [2048] * 8, 5: [0, 2048, 0, 0, 2048, 0, 0, 0], 16: [0, 2048, 0, 0, 2048, 2048, 2048, 0]}[page]
    b.release([0, 2, 7], [0, 20, 0])
    b.release(list(range(8)), [0] * 8)
    assert b.plain.free() == list(range(120))


@pytest.mark.parametrize("rows", [4, 70, 1500])
def test_long_rows(rows):
    """Hundreds of pages to look at in some rows and none in others, of more
    rows than threads."""
    g = gen(rows)
    page, width = 1, 700
    b = both(rows * 12 + 3000, rows, width, page)
    want = [700 if s % max(rows // 4, 3) == 0 else 5 for s in range(rows)]
    b.reserve(want)
    b.set_len(want)
    dst = [s for s in range(rows) if want[s] == 5][:3]
    b.release(dst, [0] * len(dst))
    b.set_len([0 if s in dst else n for s, n in enumerate(want)])
    long = [s for s in range(rows) if want[s] == 700]
    b.fork([long[0], long[-1], long[0]][:len(dst)], dst)
    for _ in range(4):
        back = [int(torch.randint(0, n + 1, (1,), generator=g)) for n in b.len]
        keep = b.len
        b.set_len(back)
        b.reserve([int(torch.randint(-1, 701, (1,), generator=g)) for _ in range(rows)])
        b.set_len([min(n, h * page) for n, h in zip(keep, b.plain.held)])


def test_forks_from_rows_that_are_dst():
    """A row that holds pages stays as it is though a fork of the call would
    have it, so another fork may copy it; one that is empty may not be copied,
    and a refused fork has its dst all the same."""
    b = Both(60, 8, 10, 8)
    b.reserve([20, 13, 5, 0, 0, 0, 0, 0])
    b.set_len([20, 13, 5, 0, 0, 0, 0, 0])
    assert b.fork([0, 1], [1, 3]) == [4096, 0]
    assert b.fork([1, 0], [5, 1]) == [0, 4096]
    b.release([3, 5], [0, 0])
    b.set_len([20, 13, 5, 0, 0, 0, 0, 0])
    assert b.fork([0, 4, 4], [4, 5, 6]) == [0, 512, 512]
    assert b.fork([9, 0], [5, 5]) == [512, 4096]
    assert b.fork([5, 0], [5, 6]) == [512, 0]


def test_a_page_that_is_shared_is_not_written():
    """What the reserve lets through is appended: the other row's tokens stay."""
    from paper_2111_05426_amd import ops
    page, d = 1, 16
    cache = {x: torch.zeros(40, page, 1, d, dtype=BF16, device="cuda") for x in "kv"}
    pool, table = ops.alloc_page_pool(40, 2), torch.full((2, 20), -1, dtype=torch.int32, device="cuda")
    length, status = ints([0, 0]).cuda(), ints([0, 0]).cuda()
    ops.dsim_kv_reserve(pool, table, page, length, ints([8, 0]).cuda(), status)
    length.copy_(ints([8, 0]))
    cache["k"].normal_()
    one = ints([7]).cuda()
    ops.dsim_kv_fork(cache, pool, table, length, ints([0]).cuda(), ints([1]).cuda(), one)
    want = cache["k"].clone()
    length.copy_(ints([6, 8]))
    ops.dsim_kv_reserve(pool, table, page, length, ints([8, 8]).cuda(), status)
    rows = torch.ones(2, 1, d, dtype=BF16, device="cuda")
    seq = torch.where(status[0] == 0, ints([0, 0]).cuda(), ints([-1, -1]).cuda())
    ops.dsim_kv_append(cache, table, rows, rows, seq, ints([6, 7]).cuda())
    at = table[1, :8].long()
    assert one.tolist() == [0] and status.tolist() == [2048, 0] and torch.equal(cache["k"][at], want[at])
