"""Calls of the key/value cache that the library refuses: found on the host before anything is launched, so no GPU is needed
(the addresses are never used).  And the reference of the GPU tests against itself: layout and tables."""
import ctypes

import numpy as np
import pytest

import kv_ref as ref

INVALID, SHAPE, MISALIGNED, WORKSPACE, NO_DEVICE, CUDA = -1, -2, -3, -4, -8, -6
A = 1 << 20     # an aligned address


@pytest.fixture(scope="module")
def lib():
    import torch
    if torch.cuda.is_available():
        pytest.skip("made-up addresses: only where nothing can be launched")
    from paper_2410_09687_b200 import binding, build
    build.build()
    return binding


def _kv(b, pages=A, n_pages=8, page_tokens=16, heads=2, dim=64):
    return ctypes.byref(b._Kv(pages, n_pages, page_tokens, heads, dim))


def _tables(b, table=A, free=A, lens=A, n_free=A, n_rows=4, max_pages=8, n_pages=8, page_tokens=16):
    return ctypes.byref(b._KvTables(table, free, lens, n_free, n_rows, max_pages, n_pages, page_tokens))


def _batch(b, R=2, T=4, cu=A, kv=A, slot=A, pos=A, refused=A):
    return ctypes.byref(b._KvBatch(R, T, cu, kv, slot, pos, refused))


KV_BAD = [({"pages": None}, INVALID), ({"n_pages": 0}, INVALID), ({"heads": 0}, INVALID), ({"dim": 32}, SHAPE), ({"dim": 96}, SHAPE),
          ({"page_tokens": 8}, SHAPE), ({"page_tokens": 48}, SHAPE), ({"n_pages": 1 << 27}, SHAPE), ({"pages": A + 8}, MISALIGNED)]


@pytest.mark.parametrize("bad,status", KV_BAD)
def test_caches_refused(lib, bad, status):
    L = lib.lib()
    kv = _kv(lib, **bad)
    assert L.moin_kv_append(kv, A, A, 128, A, 128, None, None, 0, 1, None) == status
    assert L.moin_kv_read(kv, A, A, 128, A, 128, 1, None) == status
    assert L.moin_kv_attention(kv, _tables(lib), None, A, A, 1, 1, 1, 1, A, 256, 4, 1.0, None, 0, A, 256, A, 1 << 30, None) == status


@pytest.mark.parametrize("args,status", [
    ({"T": -1}, INVALID), ({"slot": None}, INVALID), ({"k": None}, INVALID), ({"v": None}, INVALID), ({"rope": A}, INVALID),
    ({"rope_len": -1}, INVALID), ({"ks": 120}, SHAPE), ({"vs": 129}, SHAPE), ({"ks": 132}, SHAPE), ({"k": A + 2}, MISALIGNED),
    ({"v": A + 8}, MISALIGNED), ({"rope": A + 4, "pos": A}, MISALIGNED), ({"T": 0}, 0), ({}, NO_DEVICE)])
def test_append_and_read_refused(lib, args, status):
    a = {"slot": A, "k": A, "ks": 128, "v": A, "vs": 128, "pos": None, "rope": None, "rope_len": 16, "T": 3} | args
    L, kv = lib.lib(), _kv(lib)
    assert L.moin_kv_append(kv, a["slot"], a["k"], a["ks"], a["v"], a["vs"], a["pos"], a["rope"], a["rope_len"], a["T"], None) == status
    if not {"rope", "rope_len"} & set(args):
        assert L.moin_kv_read(kv, a["slot"], a["k"], a["ks"], a["v"], a["vs"], a["T"], None) == status


@pytest.mark.parametrize("tables,batch,want,status", [
    ({"table": None}, {}, A, INVALID), ({"free": None}, {}, A, INVALID), ({"lens": None}, {}, A, INVALID), ({"n_free": None}, {}, A, INVALID),
    ({"n_rows": 0}, {}, A, INVALID), ({"max_pages": 0}, {}, A, INVALID), ({"page_tokens": 24}, {}, A, SHAPE), ({"n_rows": 65537}, {}, A, SHAPE),
    ({"max_pages": (1 << 26) + 1}, {}, A, SHAPE), ({"n_pages": 1 << 27}, {}, A, SHAPE), ({}, {"R": -1}, A, INVALID), ({}, {"T": -1}, A, INVALID),
    ({}, {"cu": None}, A, INVALID), ({}, {"refused": None}, A, INVALID), ({}, {"kv": None}, A, INVALID), ({}, {"slot": None}, A, INVALID),
    ({}, {"pos": None}, A, INVALID), ({}, {}, None, INVALID), ({}, {"R": 5}, A, SHAPE),
    ({"n_rows": 64, "max_pages": 1 << 26}, {"R": 64}, A, SHAPE), ({}, {}, A, NO_DEVICE)])
def test_updates_refused(lib, tables, batch, want, status):
    assert lib.lib().moin_kv_update(_tables(lib, **tables), None, want, _batch(lib, **batch), None, None, None) == status


@pytest.mark.parametrize("args,status", [
    ({"R": -1}, INVALID), ({"T": -1}, INVALID), ({"cu": None}, INVALID), ({"kv_len": None}, INVALID), ({"q": None}, INVALID),
    ({"out": None}, INVALID), ({"heads": 0}, SHAPE), ({"heads": 5}, SHAPE), ({"R": 5}, SHAPE), ({"rope": A, "rope_len": 99}, SHAPE),
    ({"qs": 260}, SHAPE), ({"os": 248}, SHAPE), ({"q": A + 8}, MISALIGNED), ({"out": A + 4}, MISALIGNED), ({"rope": A + 8, "rope_len": 128}, MISALIGNED),
    ({"ws": None}, WORKSPACE), ({"ws": A + 8}, WORKSPACE), ({"n_ws": 15}, WORKSPACE),
    ({"R": 0}, 0), ({"T": 0}, 0), ({}, NO_DEVICE), ({"rope": A, "rope_len": 100}, NO_DEVICE)])
def test_attention_refused(lib, args, status):
    a = {"R": 2, "T": 3, "cu": A, "kv_len": A, "q": A, "qs": 256, "heads": 4, "rope": None, "rope_len": 0, "out": A, "os": 256, "ws": A,
         "n_ws": 1 << 30} | args
    got = lib.lib().moin_kv_attention(_kv(lib), _tables(lib), None, a["cu"], a["kv_len"], a["R"], a["T"], 2, 100, a["q"], a["qs"], a["heads"], 0.125,
                                      a["rope"], a["rope_len"], a["out"], a["os"], a["ws"], a["n_ws"], None)
    assert got == status


def test_tables_and_cache_must_agree(lib):
    L = lib.lib()
    for t in ({"page_tokens": 32}, {"n_rows": 0}, {"table": None}):
        assert L.moin_kv_attention(_kv(lib), _tables(lib, **t), None, A, A, 1, 1, 1, 1, A, 256, 4, 1.0, None, 0, A, 256, A, 1 << 30, None) < 0


@pytest.mark.parametrize("args,status", [
    ({"caches": None}, INVALID), ({"tables": None}, INVALID), ({"batch": None}, INVALID), ({"rope": None}, INVALID), ({"rope_len": 99}, SHAPE),
    ({"rope": A + 4}, MISALIGNED), ({"t": {"table": None}}, INVALID), ({"t": {"page_tokens": 32}}, SHAPE), ({"k": {"dim": 128}}, SHAPE),
    ({"k": {"heads": 3}}, SHAPE), ({"k": {"pages": None}}, INVALID), ({"b": {"slot": None}}, INVALID), ({"b": {"R": 5}}, SHAPE),
    ({"ws": A + 16}, WORKSPACE), ({"n_ws": 4096}, WORKSPACE), ({"b": {"T": 0}}, 0), ({}, NO_DEVICE)])
def test_cached_forward_refused(lib, args, status):
    m = lib._Model()
    m.n_layers, m.hidden, m.n_heads, m.n_kv_heads, m.head_dim, m.ffn, m.vocab, m.rms_eps, m.rope_base = 2, 128, 4, 2, 64, 128, 64, 1e-5, 1e4
    m.embed = m.lm_head = m.final_norm = A
    ptrs = (ctypes.c_void_p * 14)(*[A] * 14)
    m.attn_norm = m.mlp_norm = m.W = ctypes.cast(ptrs, ctypes.POINTER(ctypes.c_void_p))
    a = {"rope": A, "rope_len": 100, "ws": A, "n_ws": 1 << 30} | args
    one = {"pages": A, "n_pages": 8, "page_tokens": 16, "heads": 2, "dim": 64} | args.get("k", {})
    caches = (lib._Kv * 2)(*[lib._Kv(A, 8, 16, 2, 64), lib._Kv(*one.values())])
    got = lib.lib().moin_decoder_forward_cached(ctypes.byref(m), A, None if "caches" in args else caches,
                                                None if "tables" in args else _tables(lib, **args.get("t", {})), None,
                                                None if "batch" in args else _batch(lib, **args.get("b", {})), None, 2, 100, a["rope"], a["rope_len"],
                                                A, 1, None, a["ws"], a["n_ws"], None)
    assert got == status


def test_rope_table_refused(lib):
    L = lib.lib()
    for args, status in (((A, -1, 64, 1e4), INVALID), ((A, 4, 64, 0.0), INVALID), ((A, 4, 64, float("nan")), INVALID), ((A, 4, 48, 1e4), SHAPE),
                         ((None, 4, 64, 1e4), INVALID), ((A + 8, 4, 64, 1e4), MISALIGNED), ((None, 0, 64, 1e4), 0), ((A, 4, 64, 1e4), NO_DEVICE)):
        assert L.moin_rope_table(*args, None) == status


def test_cpu_tensors_are_refused(lib):
    import torch
    import paper_2410_09687_b200 as moin
    with pytest.raises(moin.MoinError):
        moin.KvCache.empty(2, 16, 1, 64, "cpu")
    with pytest.raises(moin.MoinError):
        moin.KvTables(torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 16)


def test_sizes(lib):
    L = lib.lib()
    assert L.moin_kv_bytes(1, 16, 1, 64) == 1152 and L.moin_kv_bytes(10, 128, 3, 128) == 10 * 8 * 3 * 2 * 1152
    assert L.moin_kv_bytes(1 << 20, 64, 8, 128) == (1 << 20) * 4 * 8 * 2 * 1152      # beyond 32 bits
    assert L.moin_kv_bytes(-1, 16, 1, 64) == 0


def test_reference_layout_is_a_bijection():
    for kv in range(2):
        seen = {ref.byte_of(kv, tok, ch) for tok in range(16) for ch in range(64)}
        assert len(seen) == 1024 and {b for b, _ in seen} == set(range(512 * kv, 512 * kv + 512))
        owner = {}
        for tok in range(16):
            for ch in range(64):
                assert owner.setdefault(ref.byte_of(kv, tok, ch)[0], tok) == tok     # a byte belongs to one token
    assert sorted(ref.pair_of(kv, tok) for kv in range(2) for tok in range(16)) == list(range(1024, 1152, 4))


def test_reference_quantisation():
    rng = np.random.default_rng(0)
    x = ref.bf16(rng.standard_normal((200, 64)).astype(np.float32) * 10.0 ** rng.integers(-6, 6, (200, 1)))
    c, s, z = ref.quantise(x)
    # half a step, and what 15 steps of a bf16 scale may miss of the span: 15 steps x 2^-8
    assert (np.abs(ref.values(x) - x) <= s[:, None] * (0.5 + 15 * 2.0 ** -8) * (1 + 1e-6)).all()
    assert (c.min(-1) == 0).all() and (z == x.min(-1)).all()
    const = ref.bf16(np.full((3, 64), [[7.3], [0.0], [-1e30]], np.float32))
    assert (ref.values(const) == const).all()
    bad = np.zeros((3, 64), np.float32)
    bad[0, 5], bad[1, 6], bad[2, 0], bad[2, 1] = np.inf, np.nan, 3e38, -3e38
    assert np.isnan(ref.values(bad)).all()
    pages = np.full((2, 1, 2, 1, 1152), 0xA5, np.uint8)
    ref.store(pages, [3, 40, -1], x[:3, None], 0)
    ref.store(pages, [3, 40, -1], x[3:6, None], 1)
    for kv, rows in ((0, x[:2]), (1, x[3:5])):
        c, s, z = ref.load(pages, [3, 40], kv)
        assert np.array_equal(z[..., None] + s[..., None] * c, ref.values(rows)[:, None, None])
