"""Page operators on pools whose requests do not fit the near paths: rows told apart in memory, sums beyond 32 bits."""
import numpy as np
import pytest
import torch

from paper_2605_21603_amd import binding as B
from pages_model import DONE, NONE_LEFT, REFUSED
from test_gpu_pages import DEV, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [8192, 8193, 20000])
def test_rows_told_apart_in_lds_and_in_memory(rows):
    """Around the most rows that are told apart in LDS: requests that name a row again, everywhere in the list, are refused."""
    rs = np.random.RandomState(rows)
    c = Case(pages=30000, rows=rows, width=2, layers=1, kv=1, hd=8, max_requests=rows)
    named = np.concatenate([rs.permutation(rows)[:5000], [0, rows - 1, rows, -1, 1 << 30]])
    named = np.concatenate([named, rs.choice(named, 1500)])
    got = c.resize(rs.permutation(named), rs.randint(0, 33, len(named)))
    assert got.count(REFUSED) >= 1500 and DONE in got
    c.resize(np.flatnonzero(c.model.lens > 0)[::2], np.zeros(len(np.flatnonzero(c.model.lens > 0)[::2]), np.int64))
    empty, full = np.flatnonzero(c.model.lens == 0), np.flatnonzero(c.model.lens > 0)
    kids = np.concatenate([empty[:2500], empty[:300], [rows, -5]])
    got = c.fork(rs.choice(full, len(kids)), rs.permutation(kids))
    assert got.count(REFUSED) == 302 and got.count(DONE) == 2500
    c.compact()


def test_the_workspace_may_hold_anything():
    """The owners of rows that are told apart in memory are set by the call itself."""
    c = Case(pages=300, rows=9000, width=2, layers=1, kv=1, hd=8, max_requests=40)
    for fill in (0xFF, 0, 0x55):
        c.pool._workspace.bytes.fill_(fill)
        c.resize([8999, 8500, 8999, 17], [20, 0, 3, 9])
        c.pool._workspace.bytes.fill_(fill)
        c.resize([8999, 17], [0, 0])


@pytest.mark.parametrize("width", [1 << 20, (1 << 20) + 1, 1 << 28])
def test_requests_for_more_pages_than_32_bits_count(width):
    """Rows of 2^20 pages, of one more, and of 2^28: what a list of requests asks for goes beyond 2^32 pages in the widest tables, with one request that can be
    served in front, and those that need none behind."""
    rows = 17
    k = torch.zeros((1, 20, 1, 1, 8), dtype=torch.bfloat16, device=DEV)
    ints = lambda a: torch.tensor(list(a), dtype=torch.int32, device=DEV)
    table = torch.zeros((rows, width), dtype=torch.int32, device=DEV)
    pool = B.PagePool(k, k.clone().view(1, 20, 1, 8, 1), table, ints([0] * rows), ints([0] * 20), rows + 1)
    got = pool.resize(ints(list(range(rows)) + [0]), ints([3] + [width] * (rows - 2) + [0, 1]))
    assert got.tolist() == [DONE] + [NONE_LEFT] * (rows - 2) + [DONE, REFUSED]
    assert pool.seq_len.tolist() == [3] + [0] * (rows - 1) and table[0, :4].tolist() == [0, 1, 2, 0] and pool.ref_count.tolist() == [1] * 3 + [0] * 17
    assert not table[1:].any()
    # a request that fits behind those that do not is not served either; the next call's are
    assert pool.resize(ints([1, 2]), ints([width, 1])).tolist() == [NONE_LEFT, NONE_LEFT]
    assert pool.fork(ints([0, 0]), ints([5, 6])).tolist() == [DONE, DONE]
    assert pool.resize(ints([0, 5, 16]), ints([2, 3 + 17, width])).tolist() == [DONE, DONE, NONE_LEFT]
    assert table[5, :21].tolist() == [0, 1, 2] + list(range(3, 20)) + [0] and pool.ref_count.tolist() == [3, 3, 2] + [1] * 17
