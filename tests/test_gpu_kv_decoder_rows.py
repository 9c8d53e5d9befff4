"""Rows of the cached decoder forward that no new token stands behind: requests without new tokens, batches without any."""
import ctypes

import numpy as np
import pytest
import torch

import moin_inputs as mi
import paper_2410_09687_b200 as moin
from gpu_util import DEV
from paper_2410_09687_b200.binding import lib
from test_gpu_decoder import CFG, gpu_model
from test_gpu_kv_decoder import MAX_PAGES, PAGE, ROWS, i32, server

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gm():
    return gpu_model(mi.decoder_model(CFG, seed=4, missing=(2,)))


@pytest.fixture(scope="module")
def rope():
    return moin.rope_table(MAX_PAGES * PAGE, 64, CFG.rope_base, DEV)


def full(*shape):
    return torch.full(shape, 7.0, dtype=torch.bfloat16, device=DEV)


def test_a_step_without_new_tokens(gm, rope):
    """One request ends, one stays, one is refused: nothing to run, zeros for the last tokens' logits, caches as they were; also captured."""
    tables, layers = server()
    batch = moin.kv_update(tables, i32([30, 4]), moin.KvBatch(2, 34, DEV))
    tok = i32(np.random.default_rng(0).integers(0, CFG.vocab, 34))
    moin.decoder_forward_cached(gm, tok, layers, tables, batch, None, rope)
    pages = [c.pages.clone() for c in layers.caches]
    empty = moin.kv_update(tables, i32([0, 4, 5]), moin.KvBatch(3, 0, DEV))
    assert empty.kv_len.cpu().tolist() == [0, 4, 0] and int(empty.refused) == 1
    args = (gm, tok[:0], layers, tables, empty, i32([3, 0, 1]), rope)
    given = full(3, CFG.vocab)
    assert moin.decoder_forward_cached(*args, logits=given) is given and (given == 0).all()
    new = moin.decoder_forward_cached(*args)
    assert new.shape == (3, CFG.vocab) and (new == 0).all()
    assert moin.decoder_forward_cached(*args, logits_mode=moin.LOGITS_ALL).shape == (0, CFG.vocab)
    assert moin.decoder_forward_cached(*args, logits_mode=moin.LOGITS_NONE) is None
    given.fill_(7)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        moin.decoder_forward_cached(*args, logits=given)
    given.fill_(7)
    g.replay()
    assert (given == 0).all()
    assert all(torch.equal(c.pages, p) for c, p in zip(layers.caches, pages)) and tables.lens.cpu().tolist()[:3] == [0, 4, 0]
    assert tables.lens.shape == (ROWS,)


def forward(gm, rope, fill, batch, tables, tok, expert, **kw):
    """All rows' logits and hidden states, over a workspace and caches that hold `fill` in every byte."""
    layers = moin.KvLayers([moin.KvCache(torch.full((40, CFG.n_kv_heads, 1, 1, 1152), fill, dtype=torch.uint8, device=DEV)) for _ in range(CFG.n_layers)])
    n = lib().moin_decoder_cached_workspace_bytes(ctypes.byref(gm.c), batch.R, batch.T, kw.get("max_q", 0), MAX_PAGES * PAGE)
    ws = torch.full((n,), fill, dtype=torch.uint8, device=DEV)
    hidden = torch.empty(batch.T, CFG.hidden, dtype=torch.float32, device=DEV)
    logits = moin.decoder_forward_cached(gm, tok, layers, tables, batch, expert, rope, logits_mode=moin.LOGITS_ALL, hidden_out=hidden, workspace=ws, **kw)
    return logits, hidden


@pytest.mark.parametrize("lens,pad,experts", [([9, 4], 6, True), ([70, 33], 90, True), ([5], 3, False), ([300, 200], 700, True), ([1] * 30, 2, True)])
def test_rows_behind_the_last_request(gm, rope, lens, pad, experts):
    """They are the same whatever the workspace held, finite, and those of a refused request's base-model token: attention outputs of zero."""
    lens = [min(n, MAX_PAGES * PAGE) for n in lens]
    R, T = len(lens) + 1, sum(lens) + 2 + pad
    rng = np.random.default_rng(pad)
    tok = rng.integers(0, CFG.vocab, T)
    tok[sum(lens):sum(lens) + 2] = tok[-2:]
    got = []
    for fill in (0x00, 0xFF, 0x47):
        tables = moin.KvTables.empty(R, MAX_PAGES, 40, PAGE, DEV)
        held = sum(-(-n // PAGE) for n in lens)
        tables.n_free.fill_(held)                       # the last request gets no page
        batch = moin.kv_update(tables, i32(lens + [2]), moin.KvBatch(R, T, DEV))
        assert int(batch.refused) == 1 and int(batch.cu_q[-1]) == T - pad
        expert = i32([i % 3 * 2 for i in range(R - 1)] + [-1]) if experts else None
        got.append(forward(gm, rope, fill, batch, tables, i32(tok), expert))
    for logits, hidden in got:
        assert hidden.isfinite().all() and torch.equal(logits, got[0][0]) and torch.equal(hidden, got[0][1])
    logits, hidden = got[0]
    assert torch.equal(hidden[sum(lens):sum(lens) + 2], hidden[-2:]) and torch.equal(logits[sum(lens):sum(lens) + 2], logits[-2:])


def test_more_queries_than_declared(gm, rope):
    """A request with more new tokens than max_q: what the attention does not answer is zero, not what the workspace held."""
    lens, T = [8, 3], 11
    tok = i32(np.random.default_rng(5).integers(0, CFG.vocab, T))
    got = []
    for fill in (0x00, 0xFF):
        tables = moin.KvTables.empty(2, MAX_PAGES, 40, PAGE, DEV)
        batch = moin.kv_update(tables, i32(lens), moin.KvBatch(2, T, DEV))
        got.append(forward(gm, rope, fill, batch, tables, tok, i32([0, 3]), max_q=3))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1]) and got[0][1].isfinite().all()


def test_no_request_at_all(gm, rope):
    """R = 0 with room for tokens: all rows are behind the last request."""
    T = 12
    tok = i32(np.random.default_rng(6).integers(0, CFG.vocab, T))
    tables = moin.KvTables.empty(2, MAX_PAGES, 40, PAGE, DEV)
    none = moin.kv_update(tables, i32([]), moin.KvBatch(0, T, DEV))
    one = moin.kv_update(tables, i32([0]), moin.KvBatch(1, T, DEV))
    got, same = (forward(gm, rope, 0xFF, b, tables, tok, e) for b, e in ((none, None), (one, i32([3]))))
    assert got[1].isfinite().all() and torch.equal(got[1], same[1]) and torch.equal(got[0], same[0])
    layers = moin.KvLayers([moin.KvCache.empty(40, PAGE, CFG.n_kv_heads, 64, DEV) for _ in range(CFG.n_layers)])
    assert moin.decoder_forward_cached(gm, tok, layers, tables, none, None, rope).shape == (0, CFG.vocab)
