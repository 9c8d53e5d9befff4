"""New outputs of the router, layer and decoder calls on another stream than the current one, which is busy and still has to write to
memory that it has freed: they belong to the stream of the call."""
import numpy as np
import pytest
import torch

import moin_inputs as mi
import paper_2410_09687_b200 as moin
from gpu_util import DEV, gpu_pool
from test_gpu_decoder import CFG, gpu_model
from test_gpu_kv_streams import belongs_to, busy, side

pytestmark = pytest.mark.gpu


def beside_a_busy_stream(call):
    """call(stream) -> tensors: the same on a side stream as on the current one."""
    want = [t.clone() for t in call(None)]
    s = side()
    busy(*[t.numel() * t.element_size() for t in want])
    got = call(s)
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g, w) and belongs_to(g, s)


def bf16(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV).to(torch.bfloat16)


def test_router_calls():
    gen = torch.Generator(device=DEV).manual_seed(1)
    table, q = bf16(gen, 300, 128), bf16(gen, 77, 128)
    router = moin.Router(table)
    beside_a_busy_stream(lambda s: [moin.Router(table, stream=s).inv_norm])
    beside_a_busy_stream(lambda s: [moin.route(router, q, stream=s)])
    beside_a_busy_stream(lambda s: list(moin.route_top2(router, q, stream=s).values()))


def test_layer_and_plan():
    gen = torch.Generator(device=DEV).manual_seed(2)
    T, d_in, d_out, E = 96, 128, 192, 5
    x, W, te = bf16(gen, T, d_in), bf16(gen, d_out, d_in), torch.randint(0, E, (T,), generator=gen, device=DEV).int()
    pool = gpu_pool(mi.make_pool(E, 16, d_in, d_out, 3))
    plan, ws = moin.plan_build(te, E), torch.empty(1 << 22, dtype=torch.uint8, device=DEV)
    beside_a_busy_stream(lambda s: [moin.lora_linear(plan, x, W, pool, 0.5, workspace=ws, stream=s)])
    want = plan.read()
    s = side()
    busy(plan.buffer.numel())
    other = moin.plan_build(te, E, stream=s)
    got = other.read(s)
    torch.cuda.synchronize()
    got2 = other.read()
    assert belongs_to(other.buffer, s)
    for k in ("perm", "seg_expert", "seg_start", "tile_row0", "tile_rows", "tile_expert"):
        assert np.array_equal(got[k], want[k]) and np.array_equal(got2[k], want[k])


def test_centroids_and_weights():
    gen = torch.Generator(device=DEV).manual_seed(3)
    K, D, T = 12, 64, 400
    x, old = bf16(gen, T, D), bf16(gen, K, D)
    plan = moin.plan_build(torch.randint(0, K, (T,), generator=gen, device=DEV).int(), K)
    beside_a_busy_stream(lambda s: [moin.kmeans_update(plan, x, old, stream=s)])
    codes = torch.randint(0, 120, (160, 128), generator=gen, device=DEV).to(torch.uint8)
    scale = torch.rand(160, generator=gen, device=DEV)
    beside_a_busy_stream(lambda s: [moin.dequant_fp8(codes, scale, stream=s)])


def test_decoder():
    gm = gpu_model(mi.decoder_model(CFG, seed=4))
    gm.workspace(2, 25)
    tok = torch.from_numpy(np.random.default_rng(3).integers(0, CFG.vocab, 25).astype(np.int32)).to(DEV)
    cu, ids = (torch.tensor(v, dtype=torch.int32, device=DEV) for v in ([0, 20, 25], [3, -1]))
    for mode in (moin.LOGITS_ALL, moin.LOGITS_LAST):
        beside_a_busy_stream(lambda s: [moin.decoder_forward(gm, tok, cu, ids, 20, mode, stream=s)])


def test_selftest():
    s = side()
    busy(12)
    r = moin.selftest_bounded_wait(200, stream=s)
    moin.device_status_reset(s)
    torch.cuda.synchronize()
    assert r["first_wait_returned_ok"] in (0, 1) and r["second_wait_returned_ok"] in (0, 1) and r["waited_us"] >= 0
