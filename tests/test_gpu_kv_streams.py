"""The cache calls on another stream than the current one, which is busy and still has to write to memory that it has freed: what
the calls make for themselves must be theirs."""
import numpy as np
import pytest
import torch

import kv_ref as ref
import paper_2410_09687_b200 as moin
from test_gpu_kv import DEV, _dev, _serve, i32

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


def bytes_of(*tensors):
    return [t.numel() * t.element_size() for t in tensors]


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


@pytest.mark.parametrize("n", [40, 20000])
def test_rope_table_on_a_stream(n):
    want = moin.rope_table(n, 64, 1e4, DEV)
    s = side()
    busy(*bytes_of(want))
    got = moin.rope_table(n, 64, 1e4, DEV, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and belongs_to(got, s)


@pytest.mark.parametrize("lens,H,G,D,new", [([30, 7], 2, 4, 64, 1), ([700, 2000, 40], 4, 8, 64, 1), ([900, 700], 4, 8, 64, 300), ([500] * 40, 2, 4, 128, 6)])
def test_append_read_and_attention_on_a_stream(lens, H, G, D, new):
    """Small outputs and large ones; whole items, shares, the kernel of long chunks."""
    rng = np.random.default_rng(len(lens))
    cache, tables, _, slot = _serve(rng, lens, H, D, 32)
    R, last = len(lens), np.concatenate([np.arange(b - min(n, new), b) for n, b in zip(lens, np.cumsum(lens))])
    T = len(last)
    cu, at = i32(np.concatenate([[0], np.cumsum([min(n, new) for n in lens])])), i32(np.asarray(slot)[last])
    k, v, q = (_dev(ref.bf16(rng.standard_normal((T, h, D)).astype(np.float32))) for h in (H, H, H * G))
    args = (q, cu, i32(lens), new, max(lens))
    start = cache.pages.clone()
    moin.kv_append(cache, at, k, v)
    want = [cache.pages.clone(), *moin.kv_read(cache, at), moin.kv_attention(cache, tables, *args)]
    cache.pages.copy_(start)
    s = side()
    busy(*bytes_of(*want[1:]))
    moin.kv_append(cache, at, k, v, stream=s)
    got = [*moin.kv_read(cache, at, stream=s), moin.kv_attention(cache, tables, *args, stream=s)]
    torch.cuda.synchronize()
    for x, y in zip([cache.pages, *got], want):
        assert torch.equal(x, y)
    assert all(belongs_to(t, s) for t in got)
    # one of two outputs given; the current stream named; the default stream by its handle
    k2 = torch.empty_like(k)
    gk, gv = moin.kv_read(cache, at, k=k2, stream=s)
    assert gk is k2 or gk.data_ptr() == k2.data_ptr()
    again = moin.kv_attention(cache, tables, *args, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert belongs_to(gv, s) and torch.equal(gv, want[2]) and torch.equal(k2, want[1]) and torch.equal(again, want[3])
    with torch.cuda.stream(s):
        first = moin.kv_attention(cache, tables, *args, stream=torch.cuda.default_stream())
    torch.cuda.synchronize()
    assert torch.equal(first, want[3]) and belongs_to(first, torch.cuda.default_stream())


def test_cached_forward_on_a_stream():
    import moin_inputs as mi
    from test_gpu_decoder import CFG, gpu_model
    gm = gpu_model(mi.decoder_model(CFG, seed=4))
    rope = moin.rope_table(64, 64, CFG.rope_base, DEV)
    tok = i32(np.random.default_rng(3).integers(0, CFG.vocab, 25))

    def run(stream):
        with torch.cuda.stream(stream or torch.cuda.current_stream()):
            caches = [moin.KvCache(torch.zeros(8, CFG.n_kv_heads, 1, 1, 1152, dtype=torch.uint8, device=DEV)) for _ in range(CFG.n_layers)]
            batch, lens, expert = moin.KvBatch(2, 25, DEV), i32([20, 5]), i32([3, -1])
        tables = moin.KvTables.empty(2, 4, 8, 16, DEV, stream=stream)
        moin.kv_update(tables, lens, batch, stream=stream)
        if stream is not None:
            busy(2 * 25 * CFG.vocab)
        return moin.decoder_forward_cached(gm, tok, moin.KvLayers(caches), tables, batch, expert, rope, logits_mode=moin.LOGITS_ALL, stream=stream)

    want = run(None)
    s = side()
    got = run(s)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and belongs_to(got, s)
