"""Rows of the cached decoder forward that no new token stands behind: requests without new tokens, batches without any."""
import numpy as np
import pytest
import torch

import moin_inputs as mi
import paper_2410_09687_b200 as moin
from gpu_util import DEV
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
