"""Calls whose holders live on another device than the current one: refused, whatever is there.  (One GPU is enough: the holders and
the current device are named, not used.)"""
import sys

import pytest
import torch

import moin_inputs as mi
import paper_2410_09687_b200 as moin
from test_gpu_decoder import CFG, gpu_model
from test_gpu_kv import DEV, i32

pytestmark = pytest.mark.gpu


def test_tables_on_another_device():
    tables = moin.KvTables.empty(2, 3, 6, 16, DEV)
    moin.kv_update(tables, i32([20, 3]), moin.KvBatch(2, 23, DEV))
    tables.device = 1
    with pytest.raises(moin.MoinError, match="device 1"):
        tables.reset()
    with pytest.raises(moin.MoinError, match="device 1"):
        tables.reset(torch.cuda.current_stream())
    assert tables.lens.cpu().tolist() == [20, 3] and int(tables.n_free) == 3
    tables.device = 0
    tables.reset()
    assert tables.lens.cpu().tolist() == [0, 0] and int(tables.n_free) == 6


def test_tables_and_rope_table_made_beside_the_current_device(monkeypatch):
    stream, table, free = torch.cuda.current_stream(), torch.zeros(2, 3, dtype=torch.int32, device=DEV), torch.zeros(6, dtype=torch.int32, device=DEV)
    real = torch.cuda.current_device
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1 if sys._getframe(1).f_globals["__name__"].startswith("paper_2410_09687_b200") else real())
    for call in (lambda: moin.KvTables(table, free, 16, stream=stream), lambda: moin.rope_table(8, 64, 1e4, DEV, stream=stream)):
        with pytest.raises(moin.MoinError, match="device 0, the current one is 1"):
            call()
    monkeypatch.undo()
    assert moin.rope_table(8, 64, 1e4, DEV).shape == (8, 32, 2) and moin.KvTables(table, free, 16).free_pages.cpu().tolist() == [5, 4, 3, 2, 1, 0]


def test_model_on_another_device():
    gm = gpu_model(mi.decoder_model(CFG, seed=4))
    tables, batch = moin.KvTables.empty(1, 2, 2, 16, DEV), moin.KvBatch(1, 3, DEV)
    layers = moin.KvLayers([moin.KvCache.empty(2, 16, CFG.n_kv_heads, 64, DEV) for _ in range(CFG.n_layers)])
    moin.kv_update(tables, i32([3]), batch)
    args = (gm, i32([1, 2, 3]), layers, tables, batch, None, moin.rope_table(32, 64, CFG.rope_base, DEV))
    moin.decoder_forward_cached(*args)
    gm.device = torch.device("cuda:1")
    with pytest.raises(moin.MoinError, match="model is on device 1"):
        moin.decoder_forward_cached(*args)
