"""The decoder forward on top of the 4-bit cache: block by block against a numpy restatement that attends to what the GPU has
stored (so that a code that rounds the other way is not counted as an error of everything behind it), and generation loops."""
import numpy as np
import pytest
import torch

import kv_ref as ref
import moin_inputs as mi
import paper_2410_09687_b200 as moin
from gpu_util import DEV, REL_FRO
from test_gpu_decoder import CFG, gpu_model

pytestmark = pytest.mark.gpu
PAGE, ROWS, MAX_PAGES, PAGES = 16, 7, 12, 50


def f64(t):
    return t.to(torch.float64).cpu().numpy()


def b64(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


def i32(a):
    return torch.as_tensor(np.ascontiguousarray(a, np.int32)).to(DEV)


@pytest.fixture(scope="module")
def setup():
    model = mi.decoder_model(CFG, seed=4, missing=(2,))
    return model, gpu_model(model)


def server():
    caches = [moin.KvCache(torch.full((PAGES, CFG.n_kv_heads, 1, 1, 1152), 0xFF, dtype=torch.uint8, device=DEV)) for _ in range(CFG.n_layers)]
    return moin.KvTables.empty(ROWS, MAX_PAGES, PAGES, PAGE, DEV), moin.KvLayers(caches)


def linear(model, l, name, x, expert):
    """x [T, d_in], expert per token: bf16(x W^T + s (x A^T) B^T)."""
    pool = model.pools[l][name]
    y = x @ f64(model.W[l][name]).T
    so = pool.slot_of_expert.cpu().numpy()
    for e in set(expert.tolist()):
        if e >= 0 and so[e] >= 0:
            at = expert == e
            y[at] += CFG.scale * (x[at] @ f64(pool.A[so[e]]).T) @ f64(pool.B[so[e]]).T
    return b64(y)


def norm(h, gain):
    return b64(h / np.sqrt((h * h).mean(-1, keepdims=True) + CFG.rms_eps) * f64(gain))


def block(model, l, h, expert, pos, batch, table, rows, pages, rope):
    """One block for the packed tokens; keys and values as stored in `pages`.  Returns (h after, rotated keys, values)."""
    T = h.shape[0]
    xn = norm(h, model.attn_norm[l])
    q, k, v = (linear(model, l, n, xn, expert).reshape(T, -1, 64) for n in "qkv")
    qr, kr = (ref.rotate(x.astype(np.float32), np.clip(pos, 0, None), rope) for x in (q, k))
    att, _ = ref.attention(pages, table, rows, batch.cu_q.cpu().numpy(), batch.kv_len.cpu().numpy(), qr, 0.125, PAGE)
    h = h + linear(model, l, "o", b64(np.nan_to_num(att).reshape(T, -1)), expert)
    xn = norm(h, model.mlp_norm[l])
    gate, up = linear(model, l, "gate", xn, expert), linear(model, l, "up", xn, expert)
    return h + linear(model, l, "down", b64(gate / (1 + np.exp(-gate)) * up), expert), kr, v.astype(np.float32)


# rows of the tables, wanted lengths: prompts; single tokens; a chunk, an end, a late prompt; a request too long for its row
STEPS = [([4, 0, 2], [40, 1, 17]), ([0, 2, 4], [2, 18, 41]), ([4, 6, 0, 2], [0, 33, 30, 19]), ([6, 2, 5], [34, MAX_PAGES * PAGE + 1, 5])]
EXPERTS = {0: 3, 2: -1, 4: 0, 5: 2, 6: 5}     # (expert 2 has no adapter)


def test_blocks_on_top_of_the_cache(setup):
    model, gm = setup
    rng = np.random.default_rng(0)
    tables, layers = server()
    rope = moin.rope_table(MAX_PAGES * PAGE, 64, CFG.rope_base, DEV)
    lens = np.zeros(ROWS, np.int64)
    for rows, want in STEPS:
        fits = np.array(want) <= MAX_PAGES * PAGE
        new = np.where(fits, np.maximum(np.array(want) - lens[rows], 0), 0)
        T = int(new.sum())
        batch = moin.kv_update(tables, i32(want), moin.KvBatch(len(rows), T, DEV), rows=i32(rows))
        assert int(batch.refused) == int((~fits).sum())
        req = np.repeat(np.arange(len(rows)), new)
        expert = np.array([EXPERTS[r] for r in rows])
        pos = batch.pos.cpu().numpy()
        h = rng.standard_normal((T, CFG.hidden)).astype(np.float32)
        for l in range(CFG.n_layers):
            out = torch.empty(T, CFG.hidden, dtype=torch.float32, device=DEV)
            moin.decoder_forward_cached(gm, torch.zeros(T, dtype=torch.int32, device=DEV), layers, tables, batch, i32(expert), rope, rows=i32(rows),
                                        logits_mode=moin.LOGITS_NONE, hidden_in=torch.from_numpy(h).to(DEV), hidden_out=out, layer_begin=l, layer_end=l + 1)
            pages, table = layers.caches[l].pages.cpu().numpy(), tables.block_table.cpu().numpy()
            want_h, kr, v = block(model, l, h.astype(np.float64), expert[req], pos, batch, table, np.array(rows), pages, rope.cpu().numpy())
            d = out.double().cpu().numpy() - h
            assert np.linalg.norm(d - (want_h - h)) <= REL_FRO * np.linalg.norm(want_h - h), (rows, l)
            # what was stored is the block's keys and values: half a step, what 15 steps of a bf16 scale may miss (15 x 2^-8), and a
            # bf16 step (2^-7) of the element and of the row's minimum where the two sides round differently
            for kv, x in ((0, kr), (1, v)):
                c, s, z = ref.load(pages, batch.slot.cpu().numpy(), kv)
                got = (z[..., None] + s[..., None] * c)[:, :, 0]
                assert (np.abs(got - x) <= 0.56 * s + 2.0 ** -6 * np.abs(x).max(-1, keepdims=True)).all()
            h = want_h.astype(np.float32)
        for r, w, ok in zip(rows, want, fits):
            lens[r] = w if ok else lens[r]


def test_all_blocks_at_once_and_logits(setup):
    """A whole forward is its blocks one after the other, bit for bit; the last tokens' logits are rows of all tokens' logits; without
    new tokens they are zeros; room behind the last request changes nothing of the requests."""
    model, gm = setup
    rng = np.random.default_rng(1)
    rope = moin.rope_table(MAX_PAGES * PAGE, 64, CFG.rope_base, DEV)
    for pad in (0, 9):
        tables, layers = server()
        rows, want = [1, 3, 0], [50, 0, 21]
        T = 71 + pad
        batch = moin.kv_update(tables, i32(want), moin.KvBatch(3, T, DEV), rows=i32(rows))
        tok = rng.integers(0, CFG.vocab, T)
        tok[71:] = 2 ** 31 - 1                       # behind the requests: any id
        args = (gm, i32(tok), layers, tables, batch, i32([3, 0, 1]), rope)
        full = moin.decoder_forward_cached(*args, rows=i32(rows), logits_mode=moin.LOGITS_ALL)
        last = moin.decoder_forward_cached(*args, rows=i32(rows))
        assert torch.equal(last[[0, 2]], full[[49, 70]]) and (last[1] == 0).all() and full[:71].isfinite().all()
        pages = [c.pages.clone() for c in layers.caches]
        h = None
        for l in range(CFG.n_layers):
            out = torch.empty(T, CFG.hidden, dtype=torch.float32, device=DEV)
            step = moin.decoder_forward_cached(*args, rows=i32(rows), logits_mode=moin.LOGITS_ALL if l == CFG.n_layers - 1 else moin.LOGITS_NONE,
                                               hidden_in=h, hidden_out=out, layer_begin=l, layer_end=l + 1)
            h = out
        assert torch.equal(step[:71], full[:71])
        assert all(torch.equal(c.pages, p) for c, p in zip(layers.caches, pages))


def test_captured_decode_steps(setup):
    """Greedy generation of six tokens: one captured step replayed (lengths, tokens and pages advance on the GPU) against single
    calls; the batch has room for more tokens than it has."""
    _, gm = setup
    rope = moin.rope_table(MAX_PAGES * PAGE, 64, CFG.rope_base, DEV)
    prompt = [30, 15, 47]
    tok0 = i32(np.random.default_rng(2).integers(0, CFG.vocab, sum(prompt)))
    expert = i32([3, 0, -1])

    def start():
        tables, layers = server()
        want = i32(prompt)
        batch = moin.kv_update(tables, want, moin.KvBatch(3, sum(prompt), DEV))
        logits = moin.decoder_forward_cached(gm, tok0, layers, tables, batch, expert, rope)
        tok = torch.zeros(5, dtype=torch.int32, device=DEV)
        tok[:3] = logits.argmax(-1).int()
        return tables, layers, want, moin.KvBatch(3, 5, DEV), tok, torch.empty(3, CFG.vocab, dtype=torch.bfloat16, device=DEV)

    def step(tables, layers, want, batch, tok, logits):
        want += 1
        moin.kv_update(tables, want, batch)
        moin.decoder_forward_cached(gm, tok, layers, tables, batch, expert, rope, max_q=1, logits=logits)
        tok[:3] = logits.argmax(-1).int()

    sv, plain = start(), []
    for _ in range(6):
        step(*sv)
        plain.append((sv[4].clone(), sv[5].clone()))
    sv = start()
    keep = [t.clone() for t in (sv[0].block_table, sv[0].free_pages, sv[0].lens, sv[0].n_free, sv[2], sv[4])]
    warm = torch.cuda.Stream()
    with torch.cuda.stream(warm):
        step(*sv)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(*sv)
    for t, k in zip((sv[0].block_table, sv[0].free_pages, sv[0].lens, sv[0].n_free, sv[2], sv[4]), keep):
        t.copy_(k)
    for tok, logits in plain:
        g.replay()
        assert torch.equal(sv[5], logits) and torch.equal(sv[4], tok)
    assert sv[0].lens.cpu().tolist()[:3] == [36, 21, 53]


def test_decoder_refusals(setup):
    _, gm = setup
    tables, layers = server()
    batch = moin.kv_update(tables, i32([3]), moin.KvBatch(1, 3, DEV))
    tok, rope = i32([1, 2, 3]), moin.rope_table(MAX_PAGES * PAGE, 64, CFG.rope_base, DEV)
    go = lambda **kw: moin.decoder_forward_cached(*[kw.get(n, d) for n, d in (("model", gm), ("tok", tok), ("layers", layers), ("tables", tables),  # noqa: E731
                                                                                ("batch", batch), ("expert", None), ("rope", rope))],
                                                  **{k: v for k, v in kw.items() if k in ("workspace", "hidden_in", "logits")})
    go()
    other = moin.KvLayers([moin.KvCache.empty(4, 32, CFG.n_kv_heads, 64, DEV) for _ in range(CFG.n_layers)])
    wide = moin.KvLayers([moin.KvCache.empty(4, 16, CFG.n_kv_heads, 128, DEV) for _ in range(CFG.n_layers)])
    heads = moin.KvLayers([moin.KvCache.empty(4, 16, CFG.n_kv_heads + 1, 64, DEV) for _ in range(CFG.n_layers)])
    for kw in ({"layers": other}, {"layers": wide}, {"layers": heads}, {"layers": moin.KvLayers(layers.caches[:-1])}, {"rope": rope[:100].contiguous()},
               {"workspace": torch.empty(256, dtype=torch.uint8, device=DEV)}, {"tok": tok[:2]}, {"expert": i32([0, 1])},
               {"hidden_in": torch.zeros(3, CFG.hidden, dtype=torch.bfloat16, device=DEV)}, {"logits": torch.zeros(3, CFG.vocab, dtype=torch.bfloat16, device=DEV)}):
        with pytest.raises(moin.MoinError):
            go(**kw)
    go()
