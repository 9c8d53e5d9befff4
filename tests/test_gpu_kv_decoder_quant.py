"""The cached decoder forward on a base of 8-bit codes: prompts (weights converted before the GEMMs) and steps of a few tokens (inside
them), block by block against the restatement of tests/test_gpu_kv_decoder.py over the converted weights."""
import types

import numpy as np
import pytest
import torch

import moin_inputs as mi
import oracle
import paper_2410_09687_b200 as moin
from gpu_util import DEV, REL_FRO
from test_gpu_decoder import CFG
from test_gpu_kv_decoder import MAX_PAGES, PAGE, block, i32, server
from test_gpu_quant import quantise

pytestmark = pytest.mark.gpu
ORDER = oracle.PROJ_ORDER


def test_blocks_of_a_quantised_base():
    model = mi.decoder_model(CFG, seed=4, missing=(2,))
    q = [{p: quantise(model.W[l][p]) for p in ORDER} for l in range(CFG.n_layers)]
    W = [{p: torch.from_numpy(oracle.dequant_fp8(c.numpy(), s.numpy()).view(np.int16)).view(torch.bfloat16) for p, (c, s) in layer.items()} for layer in q]
    pools = [{p: moin.Pool(model.pools[l][p].A.to(DEV), model.pools[l][p].B.to(DEV), model.pools[l][p].slot_of_expert.to(DEV)) for p in ORDER}
             for l in range(CFG.n_layers)]
    gm = moin.DecoderModel(CFG, model.embed.to(DEV), model.lm_head.to(DEV), model.final_norm.to(DEV), [t.to(DEV) for t in model.attn_norm],
                           [t.to(DEV) for t in model.mlp_norm], [{} for _ in range(CFG.n_layers)], pools, CFG.E, CFG.scale,
                           W8=[{p: c.to(DEV) for p, (c, s) in layer.items()} for layer in q], W_scale=[{p: s.to(DEV) for p, (c, s) in layer.items()} for layer in q])
    plain = types.SimpleNamespace(W=W, pools=model.pools, attn_norm=model.attn_norm, mlp_norm=model.mlp_norm)
    rng = np.random.default_rng(0)
    tables, layers = server()
    rope = moin.rope_table(MAX_PAGES * PAGE, 64, CFG.rope_base, DEV)
    lens = np.zeros(3, np.int64)
    for want in ([150, 60, 9], [151, 61, 10], [151, 0, 14]):
        new = np.maximum(np.array(want) - lens, 0)
        T = int(new.sum())
        batch = moin.kv_update(tables, i32(want), moin.KvBatch(3, T, DEV))
        expert = np.array([3, -1, 0])
        h = rng.standard_normal((T, CFG.hidden)).astype(np.float32)
        for l in range(CFG.n_layers):
            out = torch.empty(T, CFG.hidden, dtype=torch.float32, device=DEV)
            moin.decoder_forward_cached(gm, torch.zeros(T, dtype=torch.int32, device=DEV), layers, tables, batch, i32(expert), rope,
                                        logits_mode=moin.LOGITS_NONE, hidden_in=torch.from_numpy(h).to(DEV), hidden_out=out, layer_begin=l, layer_end=l + 1)
            want_h, _, _ = block(plain, l, h.astype(np.float64), expert[np.repeat(np.arange(3), new)], batch.pos.cpu().numpy(), batch,
                                 tables.block_table.cpu().numpy(), None, layers.caches[l].pages.cpu().numpy(), rope.cpu().numpy())
            d = out.double().cpu().numpy() - h
            assert np.linalg.norm(d - (want_h - h)) <= REL_FRO * np.linalg.norm(want_h - h), (want, l)
            h = want_h.astype(np.float32)
        lens = np.array(want)
