"""The cache calls on another stream than the current one, which is busy and still has to write to memory that it has freed: what
the calls make for themselves must be theirs."""
import pytest
import torch

import paper_2410_09687_b200 as moin
from test_gpu_kv import DEV, i32

pytestmark = pytest.mark.gpu
BUSY = 40_000_000     # clocks: about 20 ms


def belongs_to(t, stream):
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"] == stream.cuda_stream
    raise AssertionError("not the allocator's")


class busy:
    """The current stream sleeps, then fills blocks of these sizes, which it has freed long before."""

    def __init__(self, *sizes):
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        blocks = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in sizes for _ in range(2)]
        torch.cuda._sleep(BUSY)
        for b in blocks:
            b.fill_(0x7B)


def side():
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    return s


@pytest.mark.parametrize("n_rows,max_pages,n_pages", [(3, 5, 12), (300, 40, 9000), (7, 2, 700000)])
def test_tables_made_on_a_stream(n_rows, max_pages, n_pages):
    s = side()
    busy(4 * n_rows * max_pages, 4 * n_pages, 4 * n_rows, 4)
    tables = moin.KvTables.empty(n_rows, max_pages, n_pages, 16, DEV, stream=s)
    with torch.cuda.stream(s):
        batch = moin.KvBatch(2, 40, DEV)
        want = i32([17, 20])
    moin.kv_update(tables, want, batch, stream=s)
    torch.cuda.synchronize()
    assert tables.free_pages.cpu().tolist() == list(range(n_pages))[::-1] and int(tables.n_free) == n_pages - 4
    assert tables.lens.cpu().tolist() == [17, 20] + [0] * (n_rows - 2)
    assert batch.slot.cpu().tolist()[:37] == list(range(17)) + list(range(32, 52))
    for t in (tables.block_table, tables.free_pages, tables.lens, tables.n_free):
        assert belongs_to(t, s)


def test_tables_over_given_tensors():
    s = side()
    with torch.cuda.stream(s):
        table, free = (torch.zeros(n, dtype=torch.int32, device=DEV) for n in ((5, 4), (30,)))
    busy(20, 4)
    tables = moin.KvTables(table, free, 16, stream=s)
    torch.cuda.synchronize()
    assert tables.lens.cpu().tolist() == [0] * 5 and int(tables.n_free) == 30 and free.cpu().tolist() == list(range(30))[::-1]
    assert belongs_to(tables.lens, s) and belongs_to(tables.n_free, s)
